"""An eps that fp32 cannot hold does not switch the norm of kvcomm_place_qkv off."""
import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding

from test_wide_numbers import M, STREAM, Tensor, library  # noqa: F401

LEAST = 2.0 ** -149   # of fp32


@pytest.mark.parametrize("eps", [1e-50, 2.0 ** -151, -1e-50, -5e-324])
def test_refused(library, eps):  # noqa: F811
    t = Tensor(4)
    with pytest.raises(kv.KVCommError, match="norm_eps") as e:
        kv.kvcomm_place_qkv(M, t, None, None, 0, q_out=t, norm_eps=eps, stream=STREAM)
    assert e.value.status == binding.EINVAL and not library.calls


@pytest.mark.parametrize("eps", [0, 0.0, -0.0, LEAST, 1e-40, 1, 1e-6])
def test_others_go_through(library, eps):  # noqa: F811
    t = Tensor(4)
    kv.kvcomm_place_qkv(M, t, None, None, 0, q_out=t, norm_eps=eps, stream=STREAM)
    assert len(library.calls) == 1


@pytest.mark.gpu
def test_on_the_device():
    m = kv.Model(1, 1, 1, 64, torch.bfloat16, 1e4)
    x = 3 + torch.arange(64, device="cuda").bfloat16().view(1, 1, 1, 64).expand(1, 1, 3, 64).contiguous()
    for eps in (1e-50, -1e-50):
        with pytest.raises(kv.KVCommError):
            kv.kvcomm_place_qkv(m, x, None, None, 0, norm_eps=eps)
    # next to squares of 9 and more every eps below 2^-24 is lost, so the least one gives the bits of another small one
    assert torch.equal(kv.kvcomm_place_qkv(m, x, None, None, 0, norm_eps=LEAST)[0], kv.kvcomm_place_qkv(m, x, None, None, 0, norm_eps=1e-30)[0])
    assert not torch.equal(kv.kvcomm_place_qkv(m, x, None, None, 0, norm_eps=LEAST)[0], kv.kvcomm_place_qkv(m, x, None, None, 0)[0])

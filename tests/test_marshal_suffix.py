"""The native module against the ctypes code, for the calls around the suffix: the same bits from every form of a call, and what it declines is refused or
converted by the general path."""
import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding

from test_marshal import Counts, Declines

CALLS = {"place_qkv", "quantize_kv4", "dequantize_kv4", "suffix_attn_kv4", "suffix_attn_window", "suffix_attn_kv4_workspace", "suffix_attn_window_workspace"}
L, H, G, D = 2, 2, 3, 64


def _everything(dtype, order, dev="cuda"):
    m = kv.Model(L, H, H * G, D, dtype, 1e4)
    g = torch.Generator(device=dev)
    g.manual_seed(3)

    def make(h, n):
        x = torch.randn((L, h, n + (5 if order == "slice" else 0), D), generator=g, device=dev).to(dtype)
        return x[:, :, 2:2 + n] if order == "slice" else x.transpose(0, 1).contiguous().transpose(0, 1) if order == "heads_first" else x
    w = torch.rand((L, D), generator=g, device=dev).to(dtype)
    outs = []
    for n_ctx, tq in ((0, 1), (40, 9), (900, 3)):
        q, k, v, x = make(H * G, tq), make(H, tq), make(H, tq), make(H, n_ctx + tq)
        cache_k, cache_v = make(H, n_ctx + tq), make(H, n_ctx + tq)
        outs += [kv.kvcomm_place_qkv(m, q, k, v, n_ctx), kv.kvcomm_place_qkv(m, q, k, v, 5, norm_eps=1e-5, q_weight=w, k_weight=w[1]),
                 kv.kvcomm_place_qkv(m, None, k, None, 5, k_out=cache_k[:, :, n_ctx:], norm_eps=1)[1]]
        k4, v4 = kv.kvcomm_quantize_kv4(m, cache_k, x)
        outs += [k4, v4, kv.kvcomm_dequantize_kv4(m, k4, v4)]
        for kw in (dict(), dict(softmax_scale=0.3, want_lse=True), dict(softmax_scale=1, stream=torch.cuda.current_stream())):
            outs += [kv.kvcomm_suffix_attn_kv4(m, q, k4, list(v4), n_ctx, **kw), kv.kvcomm_suffix_attn_window(m, q, cache_k, cache_v, n_ctx, 30, 2, **kw)]
    torch.cuda.synchronize()
    return outs


def _flat(x):
    return [x] if isinstance(x, torch.Tensor) else [t for y in x for t in _flat(y)]


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["whole", "slice", "heads_first"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_same_bits_as_through_ctypes(monkeypatch, dtype, order):
    kv.load_library()
    counts = Counts(binding._native)
    monkeypatch.setattr(binding, "_native", counts)
    native = _flat(_everything(dtype, order))
    assert set(counts.took) == CALLS and not counts.declined
    monkeypatch.setattr(binding, "_native", Declines())
    general = _flat(_everything(dtype, order))
    assert len(native) == len(general)
    for i, (a, b) in enumerate(zip(native, general)):
        assert a.dtype == b.dtype and torch.equal(a, b), f"output {i}"


@pytest.mark.gpu
def test_what_is_converted():
    """Numbers of other types are converted by the general path, as everywhere."""
    m = kv.Model(1, 1, 1, 64, torch.bfloat16, 10000)
    x = torch.randn((1, 1, 4, 64), device="cuda").bfloat16()
    cache = torch.randn((1, 1, 9, 64), device="cuda").bfloat16()
    import numpy as np
    want = kv.kvcomm_place_qkv(m, x, None, None, 5)[0]
    assert torch.equal(kv.kvcomm_place_qkv(m, x, None, None, np.int64(5))[0], want)
    want = kv.kvcomm_suffix_attn_window(m, x, cache, cache, 5, 3, 1)
    assert torch.equal(kv.kvcomm_suffix_attn_window(m, x, cache, cache, np.int64(5), np.int32(3), np.int64(1)), want)


@pytest.mark.gpu
def test_another_device_is_refused(monkeypatch):
    """A stream of another device than the tensors'."""
    class Elsewhere:
        device_index = 1
        cuda_stream = 0
    m = kv.Model(1, 1, 1, 64, torch.bfloat16, 1e4)
    x = torch.randn((1, 1, 4, 64), device="cuda").bfloat16()
    cache = torch.randn((1, 1, 9, 64), device="cuda").bfloat16()
    new = lambda n, per: torch.empty((1, 1, n, 64 // per), dtype=torch.uint8, device="cuda")
    pair = lambda: (new(9, 2), new(9, 32))
    k4, v4, y = pair(), pair(), torch.empty_like(x)
    calls = [lambda: kv.kvcomm_place_qkv(m, x, None, None, 0, q_out=y, stream=Elsewhere()),
             lambda: kv.kvcomm_quantize_kv4(m, cache, cache, out_k=k4, out_v=v4, stream=Elsewhere()),
             lambda: kv.kvcomm_dequantize_kv4(m, k4, v4, out_k=torch.empty_like(cache), out_v=torch.empty_like(cache), stream=Elsewhere()),
             lambda: kv.kvcomm_suffix_attn_kv4(m, x, k4, v4, 5, out=y, stream=Elsewhere()),
             lambda: kv.kvcomm_suffix_attn_window(m, x, cache, cache, 5, 3, out=y, stream=Elsewhere())]
    for call in calls:
        with pytest.raises(kv.KVCommError):
            call()

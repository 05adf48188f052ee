"""Numbers beyond the 32 bits of the C interface: no call passes on what ctypes would wrap.  The library is replaced by one that notes what it is given (CPU
only; tensors are stand-ins that no kernel ever sees)."""
import sys
import types

import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding

from test_marshal import Declines

BF16 = torch.bfloat16
M = kv.Model(1, 1, 1, 64, BF16, 1e4)
STREAM = types.SimpleNamespace(device_index=0, cuda_stream=0)
TOO_WIDE = (2 ** 31, 2 ** 32, 2 ** 32 + 5, sys.maxsize, -2 ** 31 - 1, -2 ** 32 + 5, 2 ** 70)


class Tensor:
    """Says of itself what the binding asks of a device tensor."""
    is_cuda = True

    def __init__(self, n, D=64, dtype=BF16, h=1):
        self.shape, self.dtype, self.device = (1, h, n, D), dtype, torch.device("cpu")

    def stride(self, i=None):
        s = (self.shape[1] * self.shape[2] * self.shape[3], self.shape[2] * self.shape[3], self.shape[3], 1)
        return s if i is None else s[i]

    def data_ptr(self): return 0x1000
    def get_device(self): return 0
    def dim(self): return 4
    def is_contiguous(self): return True
    def numel(self): return self.shape[1] * self.shape[2] * self.shape[3]
    def element_size(self): return 2


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, [a for a in args if isinstance(a, int)]))
            return 0
        return call


@pytest.fixture
def library(monkeypatch):
    kv.load_library()
    lib = Library()
    monkeypatch.setattr(binding, "_lib", lib)
    monkeypatch.setattr(binding, "_native", Declines())
    return lib


def _window(n_ctx=5, window=3, n_sinks=0, cache=9):
    return kv.kvcomm_suffix_attn_window(M, Tensor(4), Tensor(cache), Tensor(cache), n_ctx, window, n_sinks, out=Tensor(4), workspace=Tensor(1), stream=STREAM)


def _refused(library, call):
    with pytest.raises(kv.KVCommError, match="32 bits") as e:
        call()
    assert e.value.status == kv.binding.EINVAL and not library.calls


@pytest.mark.parametrize("x", TOO_WIDE)
def test_positions_and_lengths_are_refused(library, x):
    t = Tensor(4)
    align = dict(base_k=t, base_v=t, anchor_dk=[], anchor_dv=[], weights=None, delta_pos=3, out_k=t, out_v=t)
    one = dict(weights=types.SimpleNamespace(dtype=torch.float32, is_contiguous=lambda: True, numel=lambda: 0, data_ptr=lambda: 0), anchor_dk=[t], anchor_dv=[t])
    q8 = lambda **kw: dict(base_k=t, base_v=t, anchor_dk8=[], anchor_dv8=[], scale_k=[], scale_v=[], weights=None, delta_pos=3, out_k=t, out_v=t) | kw
    w2 = types.SimpleNamespace(dim=lambda: 2, dtype=torch.float32, is_contiguous=lambda: True, is_cuda=True, shape=(1, 1), device="cpu", data_ptr=lambda: 0)
    for call in (lambda: kv.kvcomm_place_qkv(M, t, None, None, x, q_out=t, stream=STREAM),
                 lambda: kv.kvcomm_suffix_attn_kv4_workspace(M, x, 1), lambda: kv.kvcomm_suffix_attn_kv4_workspace(M, 5, x),
                 lambda: kv.kvcomm_suffix_attn_window_workspace(M, x, 1, 3), lambda: kv.kvcomm_suffix_attn_window_workspace(M, 5, x, 3),
                 lambda: kv.kvcomm_suffix_attn_workspace(M, x, 1), lambda: kv.kvcomm_suffix_attn_workspace(M, 5, x),
                 lambda: kv.kvcomm_suffix_attn_confined(M, t, Tensor(9), Tensor(9), 5, x, out=t, stream=STREAM),
                 lambda: kv.kvcomm_align_kv(M, **align | dict(delta_pos=x), stream=STREAM),
                 lambda: kv.kvcomm_align_kv(M, **align | one, anchor_delta_pos=[x], stream=STREAM),
                 lambda: kv.kvcomm_align_kv(M, **align | one, anchor_len=[x], stream=STREAM),
                 lambda: kv.kvcomm_align_kv_batch(M, [align | dict(delta_pos=x)], stream=STREAM),
                 lambda: kv.kvcomm_align_kv_batch(M, [align | one | dict(anchor_delta_pos=[x])], stream=STREAM),
                 lambda: kv.kvcomm_align_kv_batch_beside(M, [align], x, stream=STREAM),
                 lambda: kv.kvcomm_align_kv_q8(M, **q8(delta_pos=x), stream=STREAM),
                 lambda: kv.kvcomm_align_kv_q8_batch(M, [q8(delta_pos=x)], stream=STREAM),
                 lambda: kv.kvcomm_capture_offsets(M, t, t, t, t, x, out_dk=t, out_dv=t, stream=STREAM),
                 lambda: kv.kvcomm_anchor_predict(w2, [x], 4, 0.5, result_out=t, workspace=t, stream=STREAM),
                 lambda: kv.kvcomm_anchor_predict(w2, [4], x, 0.5, result_out=t, workspace=t, stream=STREAM)):
        _refused(library, call)


@pytest.mark.parametrize("x", TOO_WIDE)
def test_windows_beyond_every_cache(library, x):
    """More tokens than a cache can hold mean all of them; a negative number is refused as others are."""
    if x < 0:
        for call in (lambda: _window(window=x), lambda: _window(n_sinks=x), lambda: kv.kvcomm_suffix_attn_window_workspace(M, 5, 4, x),
                     lambda: kv.kvcomm_suffix_attn_window_workspace(M, 5, 4, 3, x)):
            _refused(library, call)
        return
    most = 2 ** 31 - 1
    _window(window=x)
    _window(n_sinks=x)
    kv.kvcomm_suffix_attn_window_workspace(M, 5, 4, x, x)
    at = lambda i: library.calls[i][1]
    assert at(0)[:4] == [5, 4, most, 0] and at(1)[:4] == [5, 4, 3, most] and at(2) == [5, 4, most, most]


def test_numbers_that_fit_go_through(library):
    t = Tensor(4)
    for x in (-2 ** 31, -5, 0, 2 ** 31 - 1):
        kv.kvcomm_place_qkv(M, t, None, None, x, q_out=t, stream=STREAM)
        assert library.calls[-1][1][:2] == [4, x]
    _window(5, 2 ** 31 - 1, 2 ** 31 - 1)
    assert library.calls[-1][1][:4] == [5, 4, 2 ** 31 - 1, 2 ** 31 - 1]


def test_more_tokens_than_32_bits_count(library):
    """Expanded tensors can have any number of rows."""
    wide = 2 ** 32 + 4
    t, c = Tensor(wide), (Tensor(wide, 32, torch.uint8), Tensor(wide, 2, torch.uint8))
    for call in (lambda: kv.kvcomm_place_qkv(M, t, None, None, 0, q_out=t, stream=STREAM),
                 lambda: kv.kvcomm_quantize_kv4(M, t, t, out_k=c, out_v=c, stream=STREAM),
                 lambda: kv.kvcomm_dequantize_kv4(M, c, c, out_k=t, out_v=t, stream=STREAM),
                 lambda: kv.kvcomm_suffix_attn_window(M, t, t, t, 0, 3, out=t, workspace=t, stream=STREAM),
                 lambda: kv.kvcomm_suffix_attn_kv4(M, t, c, c, 0, out=t, workspace=t, stream=STREAM)):
        _refused(library, call)


@pytest.mark.gpu
def test_on_the_device():
    m = kv.Model(1, 2, 4, 64, BF16, 1e4)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q, k, v = (torch.randn((1, h, n, 64), generator=g, device="cuda").to(BF16) for h, n in ((4, 3), (2, 700), (2, 700)))
    whole = kv.kvcomm_suffix_attn_window(m, q, k, v, 697, 700)
    for wide in (2 ** 32 + 64, sys.maxsize):
        assert torch.equal(kv.kvcomm_suffix_attn_window(m, q, k, v, 697, wide), whole)
        assert torch.equal(kv.kvcomm_suffix_attn_window(m, q, k, v, 697, 1, wide), kv.kvcomm_suffix_attn_window(m, q, k, v, 697, 1, 700))
    for first in (2 ** 32, 2 ** 31, -2 ** 31 - 1):
        with pytest.raises(kv.KVCommError):
            kv.kvcomm_place_qkv(m, q, None, None, first)

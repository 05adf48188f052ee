"""Attention through windows and over 4-bit caches at sizes near what a launch holds (fewer than 2^32 threads): refused is what its own kernel cannot take,
not what another one could not."""
import pytest
import torch

import paper_2510_12872_amd as kv

from launches import BF16, F32
from test_gpu_window_kv4_tiles import attention64, check
from test_window_kv4_launches import launches

MOST = 2 ** 31 - 1
# L, Hkv, G, D, dtype, n_ctx, tq, window (0: 4-bit cache), sinks, with scratch
PROMPTS = [(32, 8, 4, D, dt, 0, 131072, w, 4 if w else 0, ws) for D in (64, 128, 256) for dt in (BF16, F32) for w in (0, 4096) for ws in (True, False)]
PROMPTS += [(80, 8, 8, 128, BF16, 1000, 300001, 1024, 4, True), (1, 1, 16, 128, BF16, 0, 2 ** 26 + 1, 100, 0, True), (1, 1, 1, 64, BF16, 0, 2 ** 30, 1, 0, False)]
BEYOND = [(32, 8, 64, 128, BF16, 0, 2 ** 20, 4096, 4, True), (32, 8, 64, 128, BF16, 0, 2 ** 20, 0, 0, True), (1, 1, 64, 128, BF16, 0, 2 ** 25, 100, 0, True),
          (1, 1, 64, 128, BF16, 0, 2 ** 25, 0, 0, True), (32, 8, 4, 128, F32, 0, 2 ** 19, 100, 0, True), (1, 1, 1, 64, BF16, 1, 2 ** 30, 5, 0, True),
          (2 ** 24, 1, 1, 128, BF16, 0, 1, 1, 0, True), (2 ** 24, 1, 1, 128, BF16, 0, 1, 0, 0, True)]
BEYOND += [(MOST, MOST, 1, D, dt, n_ctx, 1, w, 0, ws) for D in (64, 256) for dt in (BF16, F32) for n_ctx in (0, 100000) for w in (0, 7) for ws in (True, False)]


def test_what_fits_is_launched(tmp_path):
    for c, r in zip(PROMPTS, launches(tmp_path, PROMPTS)):
        assert r["status"] == 0 and len(r["launches"]) == 1, c
        (name, (x, y, z), threads), = r["launches"]
        assert x * threads < 2 ** 32 and y == z == 1, c
        L, hkv, G, D, dt, _, tq = c[:7]
        rows = 32 if dt == F32 else threads // 2    # of a block
        assert ("attn_f32_kernel" if dt == F32 else "attn_mfma_kernel") in name
        assert x == L * hkv * -(-G * tq // rows), c


def test_what_does_not_is_refused(tmp_path):
    for c, r in zip(BEYOND, launches(tmp_path, BEYOND)):
        assert r["status"] == -2 and r["launches"] == [] and r["workspace"] == 0, c


@pytest.mark.gpu
def test_many_rows():
    """2^27 packed rows and more, the layers and heads over the same queries and keys (strides 0): each gives the bits of the first."""
    L, Hkv, G, D, n_ctx, tq, window, sinks = 8, 16, 16, 64, 0, 65601, 3, 1
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q, k, v = (torch.randn((1, 1, n, D), generator=g, device="cuda").bfloat16() for n in (tq, n_ctx + tq, n_ctx + tq))
    many = lambda t, h: t.expand(L, h, -1, -1)
    m = kv.Model(L, Hkv, Hkv * G, D, torch.bfloat16, 1e4)
    out = kv.kvcomm_suffix_attn_window(m, many(q, Hkv * G), many(k, Hkv), many(v, Hkv), n_ctx, window, sinks)
    first = out[0, :G]
    for l in range(L):
        assert bool((out[l].view(Hkv, G, tq, D) == first).all())
    tail = tq - 500   # the last queries against float64, which see keys from tail - 2 on, and the sink
    keys = torch.cat([torch.zeros(1, dtype=torch.long), torch.arange(tail - window + 1, tq)]).cuda()
    want = attention64(q[:, :, tail:].expand(1, G, -1, -1), k[:, :, keys], v[:, :, keys], len(keys) - 500, window, sinks)
    check(first[:, tail:].unsqueeze(0), want[0], want[2], "out")

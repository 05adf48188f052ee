"""Rows so far apart that a cache's offsets pass 32 bits: the bits of contiguous tensors, from every call around the suffix."""
import pytest
import torch

import paper_2510_12872_amd as kv

APART = 1 << 25   # bytes from token to token
TOKENS = 264      # 8.9 GB


@pytest.fixture(scope="module")
def memory():
    return torch.empty((TOKENS * APART,), dtype=torch.uint8, device="cuda")


def _far(memory, x, slot):
    """x [1, 1, n, D] with rows APART bytes apart, in slot `slot` of 1 MB of every row's piece."""
    row = APART // x.element_size()
    whole = memory.view(x.dtype)
    out = torch.as_strided(whole, x.shape, (0, 0, row, 1), slot * (1 << 20) // x.element_size())
    return out.copy_(x)


@pytest.mark.gpu
@pytest.mark.parametrize("tq", [1, 70])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_bits_of_near_rows(memory, dtype, tq):
    D, G, n_ctx = 128, 4, TOKENS - tq
    m = kv.Model(1, 1, G, D, dtype, 1e4)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    new = lambda h, n: torch.randn((1, h, n, D), generator=g, device="cuda").to(dtype)
    q, k, v = new(G, tq), new(1, TOKENS), new(1, TOKENS)
    far_k, far_v = _far(memory, k, 0), _far(memory, v, 1)
    want = kv.kvcomm_suffix_attn_window(m, q, k, v, n_ctx, 90, 3)
    assert torch.equal(kv.kvcomm_suffix_attn_window(m, q, far_k, far_v, n_ctx, 90, 3), want)
    k4, v4 = kv.kvcomm_quantize_kv4(m, k, v)
    far4 = [tuple(_far(memory, torch.zeros_like(t), 2 + 2 * i + j) for j, t in enumerate(pair)) for i, pair in enumerate((k4, v4))]
    kv.kvcomm_quantize_kv4(m, far_k, far_v, out_k=far4[0], out_v=far4[1])
    assert all(torch.equal(a, b) for pair, far in zip((k4, v4), far4) for a, b in zip(pair, far))
    assert torch.equal(kv.kvcomm_suffix_attn_kv4(m, q, *far4, n_ctx), kv.kvcomm_suffix_attn_kv4(m, q, k4, v4, n_ctx))
    back = kv.kvcomm_dequantize_kv4(m, *far4, out_k=_far(memory, torch.zeros_like(k), 6), out_v=_far(memory, torch.zeros_like(k), 7))
    assert all(torch.equal(a, b) for a, b in zip(back, kv.kvcomm_dequantize_kv4(m, k4, v4)))
    placed = kv.kvcomm_place_qkv(m, None, far_k, far_v, 5, k_out=_far(memory, torch.zeros_like(k), 8), v_out=_far(memory, torch.zeros_like(k), 9), norm_eps=1e-6)
    assert all(torch.equal(a, b) for a, b in zip(placed[1:], kv.kvcomm_place_qkv(m, None, k, v, 5, norm_eps=1e-6)[1:]))


@pytest.mark.gpu
def test_many_rows_and_far_rows(memory):
    """Launches of many rows over far rows (the heads share them)."""
    D, H, G, tq = 128, 8, 8, 260
    n_ctx = TOKENS - tq
    m = kv.Model(1, H, H * G, D, torch.bfloat16, 1e4)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    new = lambda n: torch.randn((1, 1, n, D), generator=g, device="cuda").bfloat16()
    q = torch.randn((1, H * G, tq, D), generator=g, device="cuda").bfloat16()
    near = [new(TOKENS) for _ in range(2)]
    far = [_far(memory, t, i) for i, t in enumerate(near)]
    heads = lambda t: t.as_strided((1, H, TOKENS, t.shape[3]), (0, 0, t.stride(2), 1), t.storage_offset())
    assert torch.equal(kv.kvcomm_suffix_attn_window(m, q, *(heads(t) for t in far), n_ctx, 100, 3),
                       kv.kvcomm_suffix_attn_window(m, q, *(heads(t) for t in near), n_ctx, 100, 3))
    one = kv.Model(1, 1, 1, D, torch.bfloat16, 1e4)
    near4 = kv.kvcomm_quantize_kv4(one, *near)
    far4 = [tuple(_far(memory, t, 2 + 2 * i + j) for j, t in enumerate(pair)) for i, pair in enumerate(near4)]
    pairs = lambda x: [tuple(heads(t) for t in pair) for pair in x]
    assert torch.equal(kv.kvcomm_suffix_attn_kv4(m, q, *pairs(far4), n_ctx), kv.kvcomm_suffix_attn_kv4(m, q, *pairs(near4), n_ctx))

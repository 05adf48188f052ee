"""The 4-bit cache format: kvcomm_quantize_kv4 and kvcomm_dequantize_kv4 against a float64 encoder and decoder, bit for bit, and their refusals."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding

from plain64 import SIZES, decode4, encode4, f64


def test_the_encoder_that_is_compared_with():
    """Hand-made codes: every tie, the limit of a scale, signs, an odd block."""
    x = np.zeros((1, 32))
    x[0, :14] = [7, 5, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, -6, -0.2, 5.0001, 0.2501, 2.4999, -7]
    codes, scales = encode4(x)
    assert scales.tolist() == [[127]]
    code = np.stack([codes & 15, codes >> 4], -1).reshape(-1)[:14]
    assert code.tolist() == [7, 6, 6, 4, 4, 2, 2, 0, 15, 8, 7, 1, 4, 15]
    x[0, 0] = 7.0001
    assert encode4(x)[1].tolist() == [[128]]
    assert decode4(codes, scales)[0, :9].tolist() == [6, 4, 4, 2, 2, 1, 1, 0, -6]
    x[0, 31] = np.nan
    assert encode4(x)[1].tolist() == [[255]] and np.isnan(decode4(*encode4(x))).all()
    assert encode4(np.zeros((2, 64)))[1].tolist() == [[2, 2], [2, 2]]


def _values(shape, dtype, seed):
    """Normal values of very different sizes from block to block, with blocks at the format's limits."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g).unflatten(-1, (-1, 32))
    x = x * torch.exp2(torch.randint(-20, 20, x.shape[:-1] + (1,), generator=g).float())
    x = x.flatten(-2)
    flat = x.view(-1, 32)
    level = torch.tensor(np.concatenate([SIZES, SIZES[:-1] + np.diff(SIZES) / 2, [7, 6.5, 7.03125]]).astype(np.float32))
    for i, scale in enumerate((1.0, 2.0 ** -125, 2.0 ** 60, 2.0 ** -126, 2.0 ** -130, 2.0 ** 125)):   # (2^-130: below the least scale)
        if i < len(flat):
            flat[i, :18] = level[:18] * scale
            flat[i, 18:26] = -level[8:16] * scale
    if len(flat) > 8:
        flat[6] = 0
        flat[7, 3] = 3e38
        flat[8] = -0.0
    return x.to(dtype)


CASES = [(1, 1, 64, torch.bfloat16, 1), (32, 8, 128, torch.bfloat16, 1), (2, 3, 128, torch.bfloat16, 77), (1, 2, 256, torch.bfloat16, 9),
         (2, 2, 64, torch.float32, 33), (1, 1, 128, torch.float32, 130), (3, 1, 256, torch.float32, 17), (1, 2, 64, torch.bfloat16, 1025)]


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["whole", "slice", "heads_first"])
@pytest.mark.parametrize("L,H,D,dtype,n", CASES)
def test_bit_for_bit(L, H, D, dtype, n, order):
    m = kv.Model(L, H, H, D, dtype, 1e4)
    k, v = _values((L, H, n, D), dtype, 1), _values((L, H, n, D), dtype, 2)

    def place(t, fill=None):   # on the device, in memory of another order
        if order == "slice":
            big = torch.zeros(t.shape[:2] + (t.shape[2] + 7,) + t.shape[3:], dtype=t.dtype, device="cuda")
            out = big[:, :, 4:4 + t.shape[2]]
        elif order == "heads_first":
            out = torch.zeros((H, L) + t.shape[2:], dtype=t.dtype, device="cuda").permute(1, 0, 2, 3)
        else:
            out = torch.zeros(t.shape, dtype=t.dtype, device="cuda")
        return out.copy_(t)
    empty = lambda per: place(torch.zeros((L, H, n, D // per), dtype=torch.uint8))
    k4, v4 = (empty(2), empty(32)), (empty(2), empty(32))
    kv.kvcomm_quantize_kv4(m, place(k), place(v), out_k=k4, out_v=v4)
    for x, (codes, scales) in ((k, k4), (v, v4)):
        want_codes, want_scales = encode4(f64(x))
        assert np.array_equal(scales.cpu().numpy(), want_scales)
        got, want = decode4(codes.cpu().numpy(), want_scales), decode4(want_codes, want_scales)
        assert np.array_equal(got, want)
        err = np.abs(want - f64(x)).reshape(want_scales.shape + (32,)).max(-1)
        fits = np.abs(f64(x)).reshape(want_scales.shape + (32,)).max(-1) <= 7 * 2.0 ** 125
        assert np.all(err[fits] <= (2.0 ** (want_scales.astype(np.float64) - 127))[fits])
    kb, vb = kv.kvcomm_dequantize_kv4(m, k4, v4, out_k=place(k), out_v=place(v))
    for got, (codes, scales) in ((kb, k4), (vb, v4)):
        assert np.array_equal(f64(got), decode4(codes.cpu().numpy(), scales.cpu().numpy()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_code_and_scale_back(dtype):
    """All 16 codes at all scales: 0 (2^-127) to 255 (NaN).  What a type cannot hold becomes infinite."""
    codes = torch.zeros((1, 1, 256, 32), dtype=torch.uint8)
    codes[..., :16] = (torch.arange(16) | (15 - torch.arange(16)) << 4).to(torch.uint8)
    scales = torch.arange(256, dtype=torch.uint8).view(1, 1, 256, 1).expand(1, 1, 256, 2).contiguous()
    m = kv.Model(1, 1, 1, 64, dtype, 1e4)
    dev = codes.cuda(), scales.cuda()
    got, _ = kv.kvcomm_dequantize_kv4(m, dev, (dev[0].clone(), dev[1].clone()))
    want = decode4(codes.numpy(), scales.numpy())
    with np.errstate(all="ignore"):
        want = np.where(np.abs(want) >= 2.0 ** 128, np.sign(want) * np.inf, want)
    assert np.array_equal(f64(got), want, equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("odd", [float("nan"), float("inf"), -float("inf")])
def test_odd_blocks(dtype, odd):
    """A block with a NaN or an infinity is NaN as a whole, its neighbours are not touched."""
    m = kv.Model(1, 1, 1, 128, dtype, 1e4)
    x = torch.ones((1, 1, 3, 128), dtype=dtype, device="cuda")
    x[0, 0, 1, 70] = odd
    x4, _ = kv.kvcomm_quantize_kv4(m, x, torch.zeros_like(x))
    back, zero = kv.kvcomm_dequantize_kv4(m, x4, kv.kvcomm_quantize_kv4(m, torch.zeros_like(x), torch.zeros_like(x))[0])
    want = torch.ones_like(x)
    want[0, 0, 1, 64:96] = float("nan")
    assert torch.equal(torch.isnan(back), torch.isnan(want)) and torch.equal(back.nan_to_num(9.0), want.nan_to_num(9.0))
    assert bool((zero == 0).all())


@pytest.mark.gpu
def test_rows_of_a_longer_cache_on_another_stream():
    """Token by token into a longer cache, on a side stream: the bits of the whole, and the other rows as they were."""
    L, H, D, n = 2, 2, 128, 9
    m = kv.Model(L, H, H, D, torch.bfloat16, 1e4)
    k, v = _values((L, H, n, D), torch.bfloat16, 5).cuda(), _values((L, H, n, D), torch.bfloat16, 6).cuda()
    want = kv.kvcomm_quantize_kv4(m, k, v)
    big = [tuple(torch.full((L, H, n + 4, D // per), 99, dtype=torch.uint8, device="cuda") for per in (2, 32)) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for i in range(n):
        at = [tuple(t[:, :, 2 + i:3 + i] for t in pair) for pair in big]
        kv.kvcomm_quantize_kv4(m, k[:, :, i:i + 1], v[:, :, i:i + 1], out_k=at[0], out_v=at[1], stream=side)
    side.synchronize()
    for pair, pair_want in zip(big, want):
        for t, tw in zip(pair, pair_want):
            assert torch.equal(t[:, :, 2:2 + n], tw)
            assert bool((t[:, :, :2] == 99).all()) and bool((t[:, :, 2 + n:] == 99).all())


@pytest.mark.gpu
@pytest.mark.parametrize("D,dtype", [(128, torch.bfloat16), (64, torch.float32)])
def test_records(D, dtype):
    """Keys and values of a token together, codes and scales of a token together: the bits of separate tensors."""
    L, H, n = 2, 3, 21
    m = kv.Model(L, H, H, D, dtype, 1e4)
    kv_rows = _values((L, n, 2, H, D), dtype, 8).cuda()
    k, v = (kv_rows[:, :, i].transpose(1, 2) for i in range(2))
    record = -(-(D // 2 + D // 32) // 16) * 16
    raw = torch.zeros((2, L, H, n, record), dtype=torch.uint8, device="cuda")
    pair = lambda i: (raw[i][..., :D // 2], raw[i][..., D // 2:D // 2 + D // 32])
    got = kv.kvcomm_quantize_kv4(m, k, v, out_k=pair(0), out_v=pair(1))
    want = kv.kvcomm_quantize_kv4(m, k.contiguous(), v.contiguous())
    assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))
    back = torch.zeros_like(kv_rows)
    kv.kvcomm_dequantize_kv4(m, pair(0), pair(1), out_k=back[:, :, 0].transpose(1, 2), out_v=back[:, :, 1].transpose(1, 2))
    assert all(torch.equal(back[:, :, i].transpose(1, 2), t) for i, t in enumerate(kv.kvcomm_dequantize_kv4(m, *want)))


@pytest.mark.gpu
def test_refusals_of_the_binding():
    m = kv.Model(2, 2, 4, 64, torch.bfloat16, 1e4)
    x = lambda n=3, h=2, d=torch.bfloat16, D=64: torch.zeros((2, h, n, D), dtype=d, device="cuda")
    c = lambda n=3, h=2, D=64: (x(n, h, torch.uint8, D // 2), x(n, h, torch.uint8, D // 32))
    bad = [(x(), x(4), c(), c()), (x(), x(d=torch.float32), c(), c()), (x(h=1), x(h=1), c(h=1), c(h=1)), (x(), x(), c(4), c()),
           (x(), x(), c(), (c()[0], c(D=128)[1])), (x().cpu(), x(), c(), c()), (x(0), x(0), c(0), c(0)), (x(), x(), c(), tuple(t.cpu() for t in c()))]
    for k, v, k4, v4 in bad:
        with pytest.raises(kv.KVCommError):
            kv.kvcomm_quantize_kv4(m, k, v, out_k=k4, out_v=v4)
        with pytest.raises(kv.KVCommError):
            kv.kvcomm_dequantize_kv4(m, k4, v4, out_k=k, out_v=v)
    same = c()
    with pytest.raises(kv.KVCommError):
        kv.kvcomm_quantize_kv4(m, x(), x(), out_k=same, out_v=same)


def test_refusals_of_the_library():
    lib = kv.load_library()
    T = lambda ptr, sl=1 << 20, sh=1 << 12, st=128: binding._CTensor(ptr, sl, sh, st)
    c4 = lambda ptr, **kw: binding._CTensor4(T(ptr, 1 << 18, 1 << 12, 64), T(ptr + (1 << 24), **{**dict(sl=1 << 16, sh=1 << 8, st=4), **kw}))

    def call(k=T(0x10000000), v=T(0x20000000), n=4, k4=c4(0x30000000), v4=c4(0x40000000), D=128, dtype=1, back=False):
        m = ctypes.byref(binding._CModel(2, 2, 4, D, dtype, 1e4))
        return lib.kvcomm_dequantize_kv4(m, k4, v4, n, k, v, None) if back else lib.kvcomm_quantize_kv4(m, k, v, n, k4, v4, None)
    codes = lambda **kw: binding._CTensor4(T(**{**dict(ptr=0x30000000, sl=1 << 18, sh=1 << 12, st=64), **kw}), c4(0x30000000).scales)
    inval = [dict(n=0), dict(n=-3), dict(k=T(None)), dict(v=T(0x20000008)), dict(k=T(0x10000000, st=4)), dict(k4=codes(ptr=None)), dict(k4=codes(ptr=0x30000008)),
             dict(k4=codes(st=72)), dict(k4=codes(sh=-64)), dict(k4=c4(0x30000002)), dict(k4=c4(0x30000000, st=2)), dict(k4=c4(0x30000000, sh=-4)),
             dict(v4=c4(0x30000000)), dict(k=T(0x30000000)), dict(v=T(0x40000000 + (1 << 24))), dict(dtype=3)]
    for change in inval:
        for back in (False, True):
            if not (back and "v4" in change):   # (two inputs may be one)
                assert call(**change, back=back) == -1, (change, back)
    # keys' codes and scales in records of 80 bytes a token: 64 and 4 bytes beside each other, and one byte too far
    record = lambda at: binding._CTensor4(T(0x30000000, 80 * 1024, 80 * 256, 80), T(0x30000000 + at, 80 * 1024, 80 * 256, 80))
    assert call(k4=record(60)) == -1 and call(k4=record(80 - 0)) == -1
    assert call(D=96) == -2
    assert call(n=1 << 30, k=T(0x10000000, sl=1 << 50, sh=1 << 45), v=T(0x10000000 + (1 << 42), sl=1 << 50, sh=1 << 45),
                k4=binding._CTensor4(T(1 << 56, 1 << 50, 1 << 45, 64), T((1 << 56) + (1 << 40), 1 << 50, 1 << 45, 4)),
                v4=binding._CTensor4(T(1 << 58, 1 << 50, 1 << 45, 64), T((1 << 58) + (1 << 40), 1 << 50, 1 << 45, 4))) == -2   # more blocks than a launch holds

"""kvcomm_suffix_attn_window and kvcomm_suffix_attn_kv4 against masked attention in float64 over the keys that a query sees, and their refusals."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding

from plain64 import attention, check, decode4, f64

BF16, F32 = torch.bfloat16, torch.float32
NAN, INF = float("nan"), float("inf")

# L, Hkv, G, D, dtype, n_ctx, tq, window, sinks
WINDOWS = [(1, 1, 1, 64, BF16, 0, 1, 1, 0), (1, 2, 4, 128, BF16, 0, 5, 2, 1), (2, 2, 2, 64, F32, 30, 7, 9, 3), (1, 1, 4, 128, BF16, 700, 1, 100, 4),
           (1, 2, 4, 128, BF16, 2000, 1, 1500, 0), (1, 2, 4, 128, BF16, 900, 33, 65, 70), (1, 1, 8, 256, BF16, 300, 40, 31, 5), (1, 1, 2, 64, BF16, 500, 90, 128, 33),
           (1, 1, 3, 128, BF16, 640, 100, 300, 4), (1, 1, 4, 64, BF16, 1100, 80, 1, 0), (1, 1, 4, 128, BF16, 1100, 70, 5000, 2), (2, 1, 1, 256, BF16, 70, 200, 50, 64),
           (1, 1, 2, 128, F32, 100, 50, 33, 1), (1, 2, 1, 256, F32, 40, 17, 16, 40), (1, 1, 4, 64, F32, 513, 1, 129, 2), (1, 1, 1, 64, F32, 0, 90, 40, 0),
           (1, 1, 4, 128, BF16, 0, 300, 64, 1), (1, 1, 4, 128, BF16, 63, 260, 191, 64), (1, 1, 2, 64, BF16, 4000, 130, 2500, 130), (1, 8, 4, 128, BF16, 1500, 2, 700, 4),
           (1, 1, 8, 128, BF16, 1000, 600, 400, 100), (1, 1, 4, 256, BF16, 900, 300, 500, 10), (1, 1, 1, 256, BF16, 900, 60, 700, 70)]
# L, Hkv, G, D, n_ctx, tq(, dtype)
COMPACT = [(1, 1, 1, 64, 0, 1, F32), (2, 2, 4, 64, 77, 5, F32), (1, 1, 2, 128, 300, 40, F32), (1, 2, 1, 256, 130, 17, F32), (1, 4, 8, 64, 500, 64, F32),
           (1, 1, 4, 256, 33, 90, F32), (1, 1, 1, 64, 0, 1), (1, 2, 4, 128, 0, 5), (2, 1, 2, 64, 31, 1), (1, 2, 4, 128, 700, 1), (1, 8, 4, 128, 3100, 1), (1, 1, 8, 256, 1200, 2), (1, 2, 4, 128, 90, 33),
           (1, 1, 2, 64, 500, 90), (1, 1, 3, 128, 640, 100), (1, 1, 1, 256, 70, 200), (1, 1, 4, 128, 0, 300), (1, 1, 4, 64, 2100, 260), (2, 2, 1, 128, 64, 64),
           (1, 1, 8, 128, 1000, 600), (1, 1, 4, 256, 900, 300), (4, 8, 1, 128, 1023, 1)]
name = lambda c: "-".join(str(x).replace("torch.", "") for x in c)


def _rand(shape, dtype, g, sigma=1.0):
    return (sigma * torch.randn(shape, generator=g)).to(dtype)


def _qkv(L, Hkv, G, D, dtype, n_ctx, tq, seed=0):
    g = torch.Generator().manual_seed(seed)
    return _rand((L, Hkv * G, tq, D), dtype, g), _rand((L, Hkv, n_ctx + tq, D), dtype, g), _rand((L, Hkv, n_ctx + tq, D), dtype, g)


def _codes(shape, g, spread=3):
    """A compact tensor with every code and scales over a few powers of two."""
    codes = torch.randint(0, 256, shape[:-1] + (shape[-1] // 2,), generator=g, dtype=torch.uint8)
    scales = torch.randint(125 - spread, 126, shape[:-1] + (shape[-1] // 32,), generator=g).to(torch.uint8)
    return codes, scales


def _window(m, q, k, v, n_ctx, window, sinks, **kw):
    return kv.kvcomm_suffix_attn_window(m, q.cuda(), k.cuda(), v.cuda(), n_ctx, window, sinks, want_lse=True, **kw)


def _no_scratch():
    return torch.empty((1,), dtype=torch.uint8, device="cuda")   # too small for any call: keys in one piece


@pytest.mark.gpu
@pytest.mark.parametrize("case", WINDOWS, ids=name)
def test_window_against_float64(case):
    L, Hkv, G, D, dtype, n_ctx, tq, window, sinks = case
    m = kv.Model(L, Hkv, Hkv * G, D, dtype, 1e4)
    q, k, v = _qkv(*case[:7])
    want, lse, tol, tol_lse = attention(f64(q), f64(k), f64(v), n_ctx, dtype, window, sinks)
    for kw in (dict(), dict(workspace=_no_scratch())):
        out, got_lse = _window(m, q, k, v, n_ctx, window, sinks, **kw)
        check(out, want, tol, "out")
        check(got_lse, lse, tol_lse, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("case", WINDOWS, ids=name)
def test_what_a_query_does_not_see_has_no_influence(case):
    """Rows that no query sees hold NaN, some that a part of them sees an infinity or a NaN among the values: each result as over its own keys."""
    L, Hkv, G, D, dtype, n_ctx, tq, window, sinks = case
    m = kv.Model(L, Hkv, Hkv * G, D, dtype, 1e4)
    q, k, v = _qkv(*case[:7], seed=1)
    N = n_ctx + tq
    unseen = torch.arange(sinks, max(sinks, n_ctx + 1 - window))
    k[:, :, unseen] = NAN
    v[:, :, unseen] = NAN
    if tq > 3:
        v[:, :, N - 2, 3] = INF              # seen by the last two queries only
        k[:, :, N - 1, 5] = NAN              # by the last one
        first = n_ctx + 1 - window           # by the first query, until it leaves the window
        if first >= sinks:
            v[:, :, first, 7] = NAN
    want, lse, tol, tol_lse = attention(f64(q), f64(k), f64(v), n_ctx, dtype, window, sinks)
    for kw in (dict(), dict(workspace=_no_scratch())):
        out, got_lse = _window(m, q, k, v, n_ctx, window, sinks, **kw)
        check(out, want, tol, "out")
        check(got_lse, lse, tol_lse, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("case", COMPACT, ids=name)
def test_compact_against_float64(case):
    L, Hkv, G, D, n_ctx, tq = case[:6]
    dtype = case[6] if len(case) > 6 else BF16
    m = kv.Model(L, Hkv, Hkv * G, D, dtype, 1e4)
    g = torch.Generator().manual_seed(2)
    q = _rand((L, Hkv * G, tq, D), dtype, g)
    k4, v4 = _codes((L, Hkv, n_ctx + tq, D), g), _codes((L, Hkv, n_ctx + tq, D), g)
    k, v = (decode4(c.numpy(), s.numpy()) for c, s in (k4, v4))
    dev = lambda pair: tuple(t.cuda() for t in pair)
    want, lse, tol, tol_lse = attention(f64(q), k, v, n_ctx, dtype)
    for kw in (dict(), dict(workspace=_no_scratch())):
        out, got_lse = kv.kvcomm_suffix_attn_kv4(m, q.cuda(), dev(k4), dev(v4), n_ctx, want_lse=True, **kw)
        check(out, want, tol, "out")
        check(got_lse, lse, tol_lse, "lse")
    if tq > 3:   # blocks of NaN that only the last queries see
        v4[1][:, :, -2, 0] = 255
        k4[1][:, :, -1, 1] = 255
        k, v = (decode4(c.numpy(), s.numpy()) for c, s in (k4, v4))
        want, lse, tol, tol_lse = attention(f64(q), k, v, n_ctx, dtype)
        for kw in (dict(), dict(workspace=_no_scratch())):
            out, got_lse = kv.kvcomm_suffix_attn_kv4(m, q.cuda(), dev(k4), dev(v4), n_ctx, want_lse=True, **kw)
            check(out, want, tol, "out with NaN")
            check(got_lse, lse, tol_lse, "lse with NaN")


@pytest.mark.gpu
@pytest.mark.parametrize("D,tq", [(64, 1), (128, 1), (128, 40), (256, 70)])
def test_large_scores_and_a_scale(D, tq):
    """Scores of hundreds that grow along the keys (the running maximum moves all the time), and one value of the type's lowest."""
    n_ctx, G = 700, 2
    g = torch.Generator().manual_seed(4)
    q, k, v = (_rand(s, BF16, g) for s in ((1, G, tq, D), (1, 1, n_ctx + tq, D), (1, 1, n_ctx + tq, D)))
    q[..., 0], k[..., 0] = 16.0, torch.linspace(-30, 30, n_ctx + tq).to(BF16)
    m = kv.Model(1, 1, G, D, BF16, 1e4)
    k[0, 0, 3, 1] = torch.finfo(BF16).min / 64
    for scale in (1.0, 0.01):
        want, lse, tol, tol_lse = attention(f64(q), f64(k), f64(v), n_ctx, BF16, 300, 4, scale)
        out, got = _window(m, q, k, v, n_ctx, 300, 4, softmax_scale=scale)
        check(out, want, tol, "window")
        check(got, lse, tol_lse, "window lse")
    k[0, 0, 3, 1] = 0
    k4, v4 = kv.kvcomm_quantize_kv4(m, k.cuda(), v.cuda())
    kd, vd = (f64(t) for t in kv.kvcomm_dequantize_kv4(m, k4, v4))
    for scale in (1.0, 0.01):
        want, lse, tol, tol_lse = attention(f64(q), kd, vd, n_ctx, BF16, scale=scale)
        out, got = kv.kvcomm_suffix_attn_kv4(m, q.cuda(), k4, v4, n_ctx, scale, want_lse=True)
        check(out, want, tol, "kv4")
        check(got, lse, tol_lse, "kv4 lse")


def _strided(t, order):
    if order == "slice":
        big = torch.full(t.shape[:2] + (t.shape[2] + 11,) + t.shape[3:], 77, dtype=t.dtype, device="cuda")
        out = big[:, :, 8:8 + t.shape[2]]
    elif order == "tokens_first":
        out = torch.zeros((t.shape[2],) + t.shape[:2] + t.shape[3:], dtype=t.dtype, device="cuda").permute(1, 2, 0, 3)
    else:
        out = torch.zeros((t.shape[1], t.shape[0]) + t.shape[2:], dtype=t.dtype, device="cuda").permute(1, 0, 2, 3)
    return out.copy_(t)


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["slice", "tokens_first", "heads_first"])
@pytest.mark.parametrize("n_ctx,tq", [(600, 1), (300, 37), (513, 280)])
def test_strides_and_streams(order, n_ctx, tq):
    """Caches, queries and outputs of any order give the bits of contiguous ones, on another stream too."""
    L, Hkv, G, D = 2, 2, 4, 128
    m = kv.Model(L, Hkv, G * Hkv, D, BF16, 1e4)
    q, k, v = (t.cuda() for t in _qkv(L, Hkv, G, D, BF16, n_ctx, tq, 9))
    k4, v4 = kv.kvcomm_quantize_kv4(m, k, v)
    place = lambda t: _strided(t, order)
    pair = lambda p: tuple(place(t) for t in p)
    side = torch.cuda.Stream()
    for call, ck, cv, moved in ((lambda *a, **kw: kv.kvcomm_suffix_attn_window(m, *a, n_ctx, 200, 5, want_lse=True, **kw), k, v, place),
                                (lambda *a, **kw: kv.kvcomm_suffix_attn_kv4(m, *a, n_ctx, want_lse=True, **kw), k4, v4, pair)):
        want, lse = call(q, ck, cv)
        out = place(torch.zeros_like(q))
        got, got_lse = call(place(q), moved(ck), moved(cv), out=out)
        assert got is out and torch.equal(got, want) and torch.equal(got_lse, lse)
        side.wait_stream(torch.cuda.current_stream())
        got, got_lse = call(q, ck, cv, stream=side)
        side.synchronize()
        assert torch.equal(got, want) and torch.equal(got_lse, lse)


@pytest.mark.gpu
def test_a_wide_window_is_the_whole_cache():
    L, Hkv, G, D, n_ctx, tq = 1, 2, 4, 128, 800, 30
    m = kv.Model(L, Hkv, G * Hkv, D, BF16, 1e4)
    q, k, v = (t.cuda() for t in _qkv(L, Hkv, G, D, BF16, n_ctx, tq, 3))
    whole = kv.kvcomm_suffix_attn(m, q, k, v, n_ctx).float()
    for window in (n_ctx + tq, 2 ** 31 - 1):
        assert (kv.kvcomm_suffix_attn_window(m, q, k, v, n_ctx, window, 7).float() - whole).abs().max() < 2e-2
    assert (kv.kvcomm_suffix_attn_window(m, q, k, v, n_ctx, 1, 2 ** 31 - 1).float() - whole).abs().max() < 2e-2   # every token is a sink


@pytest.mark.gpu
@pytest.mark.parametrize("n_ctx,tq", [(3000, 1), (300, 50)])
def test_captured_and_replayed(n_ctx, tq):
    """A graph of placement, compression and both attentions, replayed over changed inputs with eager work between, against eager calls."""
    L, Hkv, G, D = 1, 4, 4, 128
    m = kv.Model(L, Hkv, G * Hkv, D, BF16, 1e4)
    N = n_ctx + tq
    g = torch.Generator().manual_seed(6)
    new = lambda h, n: _rand((L, h, n, D), BF16, g).cuda()
    x = [new(Hkv * G, tq), new(Hkv, tq), new(Hkv, tq)]
    cache = [new(Hkv, N), new(Hkv, N)]
    k4, v4 = kv.kvcomm_quantize_kv4(m, *cache)
    last = lambda pair: tuple(t[:, :, n_ctx:] for t in pair)

    def steps():
        q, k, v = kv.kvcomm_place_qkv(m, *x, n_ctx, k_out=cache[0][:, :, n_ctx:], v_out=cache[1][:, :, n_ctx:], norm_eps=1e-6)
        kv.kvcomm_quantize_kv4(m, k, v, out_k=last(k4), out_v=last(v4))
        return (kv.kvcomm_suffix_attn_window(m, q, *cache, n_ctx, 500, 4), kv.kvcomm_suffix_attn_kv4(m, q, k4, v4, n_ctx),
                *kv.kvcomm_dequantize_kv4(m, k4, v4))
    steps()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):   # two graphs over the same buffers, each with its own scratch
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = steps()
        graphs.append((graph, outs))
    for r in range(4):
        for t in x:
            t.copy_(_rand(t.shape, BF16, g))
        graph, outs = graphs[r % 2]
        graph.replay()
        got = [t.clone() for t in outs]
        torch.cuda.synchronize()
        eager = steps()
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), r


@pytest.mark.gpu
def test_refusals_of_the_binding():
    m = kv.Model(1, 2, 4, 64, BF16, 1e4)
    t = lambda h, n, d=BF16, D=64: torch.zeros((1, h, n, D), dtype=d, device="cuda")
    q, k, v = t(4, 3), t(2, 10), t(2, 10)
    for bad in (dict(k=t(2, 9)), dict(v=t(1, 10)), dict(q=t(3, 3)), dict(k=t(2, 10, F32)), dict(window=0), dict(window=-1), dict(sinks=-1), dict(n_ctx=6),
                dict(q=t(4, 0), n_ctx=10), dict(out=t(4, 2)), dict(lse_out=torch.zeros((1, 4, 2), device="cuda")), dict(v=v.cpu()),
                dict(lse_out=torch.zeros((1, 4, 3))), dict(workspace=torch.zeros((64,)))):
        a = {**dict(q=q, k=k, v=v, n_ctx=7, window=4, sinks=0), **bad}
        with pytest.raises(kv.KVCommError):
            kv.kvcomm_suffix_attn_window(m, a.pop("q"), a.pop("k"), a.pop("v"), a.pop("n_ctx"), a.pop("window"), a.pop("sinks"), want_lse=True, **a)
    c = lambda n=10, h=2, D=64: (t(h, n, torch.uint8, D // 2), t(h, n, torch.uint8, D // 32))
    for bad in (dict(k=c(9)), dict(v=c(10, 1)), dict(k=(c()[0], c(9)[1])), dict(v=(c()[0], c(D=128)[1])), dict(q=t(4, 3, F32)), dict(n_ctx=6), dict(out=t(2, 3)),
                dict(k=tuple(x.cpu() for x in c()))):
        a = {**dict(q=q, k=c(), v=c(), n_ctx=7), **bad}
        with pytest.raises(kv.KVCommError):
            kv.kvcomm_suffix_attn_kv4(m, a.pop("q"), a.pop("k"), a.pop("v"), a.pop("n_ctx"), **a)


def test_refusals_of_the_library():
    lib = kv.load_library()
    T = lambda ptr=0x10000, sl=1 << 20, sh=1 << 16, st=128: binding._CTensor(ptr, sl, sh, st)
    none = binding._CTensor(None, 0, 0, 0)
    model = lambda D=128, dtype=1, hq=4: ctypes.byref(binding._CModel(2, 2, hq, D, dtype, 1e4))

    def window(q=T(), k=T(), v=T(), n_ctx=10, tq=4, window=3, sinks=0, out=T(), m=model()):
        return lib.kvcomm_suffix_attn_window(m, q, k, v, n_ctx, tq, window, sinks, 0.0, out, None, None, 0, None)
    for bad in (dict(tq=0), dict(n_ctx=-1), dict(window=0), dict(window=-5), dict(sinks=-1), dict(q=none), dict(k=none), dict(v=T(0x10008)), dict(out=none),
                dict(k=T(st=4)), dict(m=None), dict(m=model(dtype=5))):
        assert window(**bad) == -1, bad
    assert window(n_ctx=2 ** 30) == -2 and window(m=model(D=80)) == -2 and window(m=model(hq=5)) == -2
    c4 = lambda ptr=0x100000, st=64, ss=4: binding._CTensor4(T(ptr, st=st), T(0x200000, st=ss))

    def compact(q=T(), k=c4(), v=c4(), n_ctx=10, tq=4, out=T(), m=model()):
        return lib.kvcomm_suffix_attn_kv4(m, q, k, v, n_ctx, tq, 0.0, out, None, None, 0, None)
    for bad in (dict(tq=0), dict(n_ctx=-1), dict(q=none), dict(k=c4(None)), dict(v=c4(0x100008)), dict(k=c4(st=40)), dict(v=c4(ss=2)), dict(out=none), dict(m=None)):
        assert compact(**bad) == -1, bad
    assert compact(n_ctx=2 ** 30) == -2 and compact(m=model(D=80)) == -2 and compact(k=c4(st=1 << 26)) == -2 and compact(v=c4(ss=1 << 26)) == -2
    for need in (lib.kvcomm_suffix_attn_window_workspace(model(), 100, 0, 3, 0), lib.kvcomm_suffix_attn_window_workspace(model(), 100, 1, 0, 0),
                 lib.kvcomm_suffix_attn_kv4_workspace(model(), -1, 1), lib.kvcomm_suffix_attn_kv4_workspace(None, 5, 1)):
        assert need == 0

"""Batches of sequences in pages: placement into them and attention over them, behind a shared prefix or none, against float64."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding

from paged64 import LAYOUTS, Case, attention, place, pools
from plain64 import check, f64

BF16, F32 = torch.bfloat16, torch.float32


def _id(c):
    return "-".join(f"{k}{str(v).replace('torch.', '').replace(' ', '')}" for k, v in c.items())


# L, H, G, D, dtype and what Case() takes
SHAPES = [
    dict(L=1, H=2, G=4, D=128, dtype=BF16, rows=[1, 1, 1], lens=[1, 17, 300], page=16, one=True),
    dict(L=1, H=8, G=4, D=128, dtype=BF16, rows=[1] * 5, lens=[16, 700, 33, 2100, 64], page=64, one=True),
    dict(L=2, H=2, G=2, D=64, dtype=BF16, rows=[3, 0, 40, 1], lens=[3, 50, 100, 90], page=32, pad=2, before=1, layout="token_major"),
    dict(L=1, H=1, G=8, D=256, dtype=BF16, rows=[2, 1, 5], lens=[130, 64, 5], page=16, layout="interleaved"),
    dict(L=1, H=2, G=5, D=128, dtype=BF16, rows=[7, 1, 30], lens=[40, 65, 30], page=256, layout="heads_last"),
    dict(L=1, H=2, G=4, D=128, dtype=BF16, rows=[70, 129, 1], lens=[200, 129, 77], page=16, layout="plain"),
    dict(L=1, H=1, G=1, D=64, dtype=BF16, rows=[300, 64], lens=[450, 1000], page=64),
    dict(L=2, H=2, G=2, D=64, dtype=F32, rows=[1, 9, 0, 33], lens=[20, 9, 4, 100], page=16, pad=1, layout="token_major"),
    dict(L=1, H=1, G=8, D=128, dtype=F32, rows=[1, 1], lens=[333, 1], page=32, one=True, layout="interleaved"),
    dict(L=1, H=2, G=3, D=256, dtype=F32, rows=[4, 20], lens=[50, 41], page=16, layout="heads_last"),
]
PREFIXES = [0, 1, 45, 576]


@pytest.mark.gpu
@pytest.mark.parametrize("prefix", PREFIXES)
@pytest.mark.parametrize("shape", SHAPES, ids=_id)
def test_attention_against_float64(shape, prefix):
    c = Case(**shape, prefix=prefix)
    out, lse = torch.full_like(c.q, 7.0), torch.full(c.q.shape[:3], 7.0, device="cuda")
    c.attend(out=out, lse_out=lse, want_lse=True)
    want, want_lse, tol, tol_lse = attention(c, untouched=7.0)
    check(out, want, tol, "out")
    check(lse, want_lse, tol_lse, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("prefix", [0, 70])
def test_rows_that_see_nothing_and_entries_that_are_no_page(dtype, prefix):
    """More rows than tokens, no tokens, a negative length, entries of the table beyond the pool, a length beyond the table."""
    c = Case(1, 2, 4, 64, dtype, rows=[5, 3, 2, 1, 4, 1], lens=[2, 0, -7, 130, 200, 90], page=16, prefix=prefix,
             missing=[(3, 2, -1), (3, 8, 10 ** 6), (4, 0, -(2 ** 31)), (4, 5, 2 ** 31 - 1), (4, 12, -1), (5, 0, -1), (5, 1, -1), (5, 2, -1), (5, 3, -1), (5, 4, -1), (5, 5, -1)])
    out, lse = c.attend(want_lse=True)
    want, want_lse, tol, tol_lse = attention(c)
    check(out, want, tol, "out")
    check(lse, want_lse, tol_lse, "lse")
    c.lens = [2, 0, -7, 130, 200, 10 ** 9]
    c.batch.lens.copy_(torch.tensor(c.lens, dtype=torch.int32))
    c.pages_k.nan_to_num_(0.25)
    c.pages_v.nan_to_num_(0.5)
    out, lse = c.attend(want_lse=True)
    c.lens[5] = c.table.shape[1] * 16   # the row stands behind them all and sees what is there
    c.rows[5] = 1
    want, want_lse, tol, tol_lse = attention(c)
    check(out, want, tol, "out")
    check(lse, want_lse, tol_lse, "lse")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("prefix", [0, 33])
def test_infinities_and_nan(dtype, prefix):
    """In tokens that some rows see and others do not, in keys and in values."""
    c = Case(1, 2, 2, 128, dtype, rows=[6, 40, 1, 1], lens=[70, 40, 50, 64], page=16, prefix=prefix)
    for b, t, pool, value in ((0, 66, c.pages_v, float("nan")), (0, 68, c.pages_v, float("inf")), (1, 20, c.pages_k, float("nan")), (1, 35, c.pages_v, float("-inf")),
                              (2, 7, c.pages_v, float("inf")), (3, 9, c.pages_k, float("-inf"))):
        e, s = c.token(b, t)
        pool[:, 1, e, s, 5] = value
    out, lse = c.attend(want_lse=True)
    want, want_lse, tol, tol_lse = attention(c)
    check(out, want, tol, "out")
    check(lse, want_lse, tol_lse, "lse")
    c.q[:, :, 3] = float("inf")
    out = c.attend()
    assert bool(torch.isnan(out[:, :, 3]).any())
    check(out[:, :, 6:46], want[:, :, 6:46], tol[:, :, 6:46], "other rows")


@pytest.mark.gpu
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("shape", [dict(L=2, H=2, G=4, D=128, dtype=BF16, rows=[1, 7, 0, 20], lens=[30, 7, 5, 100], page=16, pad=3, before=2),
                                   dict(L=1, H=8, G=4, D=128, dtype=BF16, rows=[1] * 70, lens=[5 * i % 90 + 1 for i in range(70)], page=32, one=True),
                                   dict(L=1, H=3, G=2, D=64, dtype=F32, rows=[2] * 66, lens=[7 * i % 40 for i in range(66)], page=16, missing=[(3, 1, -1), (4, 0, 9999)]),
                                   dict(L=3, H=1, G=8, D=256, dtype=F32, rows=[5, 9], lens=[3, 90], page=64)], ids=_id)
def test_placement_against_float64(shape, layout):
    for eps, first in ((0.0, 0), (1e-5, 2560), (1e-6, -4)):
        c = Case(**shape, layout=layout, fill=3.0)
        m = c.model
        g = torch.Generator().manual_seed(5)
        x = torch.randn((m.n_layers, c.n, m.n_q_heads + 2 * m.n_kv_heads, m.head_dim), generator=g).to(m.dtype).cuda()
        q, k, v = (t.transpose(1, 2) for t in x.split([m.n_q_heads, m.n_kv_heads, m.n_kv_heads], 2))
        w = (1 + 0.2 * torch.randn((2, m.n_layers, m.head_dim), generator=g)).to(m.dtype).cuda()
        q_out = torch.full(q.shape, 3.0, dtype=m.dtype, device="cuda")
        want = place(c, q, k, v, q_out, first, eps, f64(w[0]), f64(w[1]))
        norm = dict(norm_eps=eps, q_weight=w[0], k_weight=w[1]) if eps else {}
        assert kv.kvcomm_place_qkv_paged(m, q, k, v, c.batch, c.pages_k, c.pages_v, first, q_out=q_out, **norm) is q_out
        check(q_out, want[0], want[3], "q_out")
        check(c.pages_k, want[1], want[4], "pages_k")
        check(c.pages_v, want[2], np.zeros_like(want[2]), "pages_v")


@pytest.mark.gpu
def test_placement_is_that_of_one_sequence():
    """Bit for bit kvcomm_place_qkv of each sequence; in place; without the queries, the keys or the values."""
    c = Case(2, 2, 4, 128, BF16, rows=[1, 50, 9], lens=[33, 50, 100], page=16, fill=0.0)
    m = c.model
    q, k, v = torch.randn_like(c.q), torch.randn_like(c.q[:, :2]), torch.randn_like(c.q[:, :2])
    norm = dict(norm_eps=1e-6, k_weight=torch.rand((128,), device="cuda").bfloat16())
    q_out = kv.kvcomm_place_qkv_paged(m, q, k, v, c.batch, c.pages_k, c.pages_v, 100, **norm)
    for b in range(3):
        rows, first = slice(int(c.starts[b]), int(c.starts[b + 1])), 100 + c.lens[b] - c.rows[b]
        one = kv.kvcomm_place_qkv(m, q[:, :, rows], k[:, :, rows], v[:, :, rows], first, **norm)
        assert torch.equal(q_out[:, :, rows], one[0])
        for i in range(c.rows[b]):
            e, s = c.token(b, c.lens[b] - c.rows[b] + i)
            assert torch.equal(c.pages_k[:, :, e, s], one[1][:, :, i]) and torch.equal(c.pages_v[:, :, e, s], one[2][:, :, i])
    c.pages_k.zero_(), c.pages_v.zero_()   # (the sequences' older tokens)
    kv.kvcomm_place_qkv_paged(m, q, k, v, c.batch, c.pages_k, c.pages_v, 100, **norm)
    before = c.pages_k.clone(), c.pages_v.clone()
    c.pages_k.zero_(), c.pages_v.zero_()
    assert kv.kvcomm_place_qkv_paged(m, None, k, None, c.batch, c.pages_k, None, 100, **norm) is None
    assert torch.equal(c.pages_k, before[0]) and not bool(c.pages_v.any())
    kv.kvcomm_place_qkv_paged(m, None, None, v, c.batch, None, c.pages_v, 100)
    assert torch.equal(c.pages_v, before[1])
    assert torch.equal(kv.kvcomm_place_qkv_paged(m, q, None, None, c.batch, None, None, 100, norm_eps=1e-6), q_out)
    kv.kvcomm_place_qkv_paged(m, q, k, v, c.batch, c.pages_k, c.pages_v, 100, q_out=q, **norm)
    assert torch.equal(q, q_out) and torch.equal(c.pages_k, before[0])


@pytest.mark.gpu
def test_starts_that_are_no_starts_stay_in_bounds():
    """Decreasing, negative and too large: which rows are written is not defined, but nothing else is."""
    c = Case(1, 2, 4, 128, BF16, rows=[4, 30, 2], lens=[40, 90, 20], page=16, prefix=40, fill=0.0)
    guard = torch.full((1, 8, c.n + 16, 128), 5.0, dtype=BF16, device="cuda")
    for starts in ([30, 4, 36, 0], [-5, 100, 7, 2 ** 31 - 1], [2 ** 31 - 1, -(2 ** 31), 0, 36], [36, 36, 36, 36]):
        c.batch.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        out = guard[:, :, 8:8 + c.n]
        c.attend(out=out)
        kv.kvcomm_place_qkv_paged(c.model, c.q, c.q[:, :2], c.q[:, 2:4], c.batch, c.pages_k, c.pages_v, q_out=out)
        torch.cuda.synchronize()
        assert bool((guard[:, :, :8] == 5).all()) and bool((guard[:, :, 8 + c.n:] == 5).all())


def _tensors():
    T = lambda ptr, sl=1 << 20, sh=1 << 12, st=128: binding._CTensor(ptr, sl, sh, st)
    P = lambda ptr, sl=1 << 20, sh=1 << 12, sp=1 << 14, st=128: binding._CPages(ptr, sl, sh, sp, st)
    B = lambda **kw: binding._CBatch(*[{**dict(table=0x1000, lens=0x2000, starts=0x3000, table_stride=8, table_width=8, n_seqs=3, n_rows=9, page_size=16,
                                                n_pages=4, max_rows=0), **kw}[f] for f, _ in binding._CBatch._fields_])
    return T, P, B


BAD_BATCHES = [dict(lens=None), dict(lens=0x2002), dict(starts=0x3001), dict(table=0x1003), dict(table=None), dict(n_seqs=0), dict(n_rows=0), dict(n_rows=-1),
               dict(table_width=-1), dict(n_pages=-1), dict(table_stride=-1), dict(max_rows=-1), dict(page_size=0), dict(page_size=-16), dict(starts=None)]
UNSUPPORTED_BATCHES = [dict(page_size=8), dict(page_size=48), dict(page_size=131072), dict(n_seqs=8193), dict(table_width=1 << 27)]


def test_refusals_of_the_library():
    """On the host, before anything is launched."""
    lib = kv.load_library()
    T, P, B = _tensors()
    none, model = T(None, 0, 0, 0), lambda D=128, dtype=1: binding._CModel(2, 2, 4, D, dtype, 1e4)

    def attend(q=T(0x10000), k=P(0x8000000), v=P(0x9000000), b=B(), out=T(0xa000000), lse=None, pk=None, pv=T(0xc000000), n_prefix=5, m=model()):
        args = (q,) if pk is None else (q, pk, pv, n_prefix)
        return (lib.kvcomm_paged_attn if pk is None else lib.kvcomm_paged_attn_prefix)(ctypes.byref(m), *args, k, v, ctypes.byref(b), 0.0, out, lse, None, 0, None)

    def put(q=T(0x10000), k=T(0x800000), v=T(0x1000000), b=B(), first=0, wq=None, wk=None, eps=0.0, out=T(0xa000000), pk=P(0x20000000), pv=P(0x40000000), m=model()):
        return lib.kvcomm_place_qkv_paged(ctypes.byref(m), q, k, v, ctypes.byref(b), first, wq, wk, 0, 0, eps, out, pk, pv, None)
    for change in BAD_BATCHES:
        assert attend(b=B(**change)) == -1 and put(b=B(**change)) == -1 and attend(b=B(**change), pk=T(0xb000000)) == -1, change
    for change in UNSUPPORTED_BATCHES:
        assert attend(b=B(**change)) == -2 and put(b=B(**change)) == -2, change
    for change in (dict(q=none), dict(out=none), dict(k=P(None)), dict(v=P(0x9000008)), dict(k=P(0x8000000, sp=4)), dict(v=P(0x9000000, sp=-128)), dict(lse=2),
                   dict(q=T(0x10000, st=4)), dict(pk=none), dict(pk=T(0xb000000), pv=none), dict(pk=T(0xb000000), n_prefix=0), dict(pk=T(0xb000000), n_prefix=-1),
                   dict(m=model(0))):
        assert attend(**change) == -1, change
    for q in (T(0x10000), T(0x10000 + 256), T(0x10000 + 16)):   # the outputs are the queries, or share some of them
        assert attend(q=q, out=T(0x10000)) == -1 and attend(q=q, out=T(0x10000), pk=T(0xb000000)) == -1
    assert attend(m=model(96)) == -2 and attend(pk=T(0xb000000), n_prefix=2 ** 30 + 1) == -2
    for change in (dict(q=none), dict(out=none), dict(k=none), dict(pv=P(None)), dict(pk=P(0x20000008)), dict(first=2 ** 31 - 100), dict(eps=-1.0), dict(eps=float("nan")),
                   dict(wq=0x1000), dict(wq=0x1004, eps=1e-5), dict(q=none, out=none, wq=0x1000, eps=1e-5), dict(pk=P(0x10000)), dict(pk=P(0x40000000)), dict(out=T(0x800000)),
                   dict(out=T(0x20000000)), dict(out=T(0x10000 + 256)), dict(b=B(lens=0x20000010)), dict(b=B(table=0x40000000)), dict(b=B(starts=0xa000000)),
                   dict(q=none, out=none, k=none, pk=P(None), v=none, pv=P(None)), dict(pv=P(0x20000000 + 2 * 128)), dict(pv=P(0x20000000 + 16)),
                   dict(pv=P(0x20000000 + 2 * 2048, st=256), pk=P(0x20000000, st=128))):
        assert put(**change) == -1, change


def test_pools_that_lie_interleaved_are_told_apart():
    """Host tensors: where there is no GPU the launch that follows the look at the pools fails, and is the only thing that does."""
    lib = kv.load_library()
    m = binding._CModel(3, 4, 8, 64, 1, 1e4)
    T, P, B = _tensors()
    dev = lambda layout: pools(3, 4, 5, 16, 64, BF16, layout, 0.0, "cpu")

    def meet(k, v):
        desc = [binding._CPages(t.data_ptr(), *t.stride()[:4]) for t in (k, v)]
        q = T(0x10000, 4096 * 4, 4096, 64)
        b = B(n_rows=3, starts=0x3000, n_pages=5)
        return lib.kvcomm_place_qkv_paged(ctypes.byref(m), T(None, 0, 0, 0), q, T(0x80000, 4096 * 4, 4096, 64), ctypes.byref(b), 0, None, None, 0, 0, 0.0,
                                          T(None, 0, 0, 0), *desc, None)
    if torch.cuda.is_available():
        pytest.skip("host pointers: only where nothing can be launched")
    for layout in LAYOUTS:
        k, v = dev(layout)
        assert meet(k, v) == -4, layout   # past every check, no GPU to launch on
        assert meet(k, k) == -1
    x = torch.zeros((5, 3, 2, 4, 16, 64), dtype=BF16)
    a, b = (x[:, :, i].permute(1, 2, 0, 3, 4) for i in range(2))
    flat = x.flatten()
    shifted = torch.as_strided(flat, b.shape, b.stride(), b.storage_offset() - 64)   # a row further down: into the other pool
    assert meet(a, b) == -4 and meet(a, shifted) == -1


@pytest.mark.gpu
def test_refusals_of_the_binding():
    c = Case(2, 2, 2, 64, BF16, rows=[1, 3], lens=[9, 20], page=16, prefix=8)
    m, b = c.model, c.batch
    batch = lambda **kw: kv.Batch(**{**dict(table=b.table, lens=b.lens, starts=b.starts), **kw})
    base = dict(q=c.q, pages_k=c.pages_k, pages_v=c.pages_v, batch=b)
    bad = [dict(q=c.q[:, :2]), dict(q=c.q.float()), dict(q=c.q.cpu()), dict(pages_k=c.pages_k[:, :, 1:]), dict(pages_v=c.pages_v.float()), dict(pages_k=c.q), dict(pages_v=c.pages_v[..., :32]),
           dict(batch=batch(table=b.table.long())), dict(batch=batch(table=b.table[:1])), dict(batch=batch(table=b.table.cpu())), dict(batch=batch(lens=b.lens.cpu())),
           dict(batch=batch(lens=b.lens[:, None])), dict(batch=batch(starts=b.starts[:2])), dict(batch=batch(starts=None)), dict(batch=batch(max_rows=-1)),
           dict(batch=batch(table=b.table.repeat(1, 2)[:, ::2])), dict(out=c.q[:, :, :2]), dict(lse_out=torch.zeros((2, 4, 3), device="cuda")),
           dict(batch=batch(max_rows=2 ** 31))]
    for change in bad:
        for prefix in ((), (c.prefix_k, c.prefix_v)):
            args = {**base, **change}
            with pytest.raises(kv.KVCommError):
                (kv.kvcomm_paged_attn_prefix if prefix else kv.kvcomm_paged_attn)(m, args.pop("q"), *prefix, args.pop("pages_k"), args.pop("pages_v"), args.pop("batch"), **args)
    for prefix in ((c.prefix_k[:, :1], c.prefix_v), (c.prefix_k, c.prefix_v[:, :, 1:]), (c.prefix_k[:, :, :0], c.prefix_v[:, :, :0]), (None, None), (c.prefix_k, None)):
        with pytest.raises(kv.KVCommError):
            kv.kvcomm_paged_attn_prefix(m, c.q, *prefix, c.pages_k, c.pages_v, b)
    k = c.q[:, :2]
    for change in (dict(k=None), dict(pages_k=None), dict(q=None, k=None, v=None, pages_k=None, pages_v=None), dict(v=c.q), dict(q=c.q[:, :, :2]), dict(pages_v=c.pages_k),
                   dict(q_weight=torch.ones((64,), device="cuda").bfloat16()), dict(norm_eps=-1.0), dict(norm_eps=1e-60), dict(first_pos=2 ** 31 - 5), dict(first_pos=2 ** 40),
                   dict(q_out=k), dict(q_out=torch.empty_like(c.q).cpu()), dict(batch=batch(starts=None))):
        args = {**dict(q=c.q, k=k, v=k.clone(), batch=b, pages_k=c.pages_k, pages_v=c.pages_v), **change}
        with pytest.raises(kv.KVCommError):
            kv.kvcomm_place_qkv_paged(m, args.pop("q"), args.pop("k"), args.pop("v"), args.pop("batch"), args.pop("pages_k"), args.pop("pages_v"), **args)

"""Batches in pages, the walk of the wavefront kernels where items follow each other inside a wavefront's run: sequences of many tokens beside sequences
without any, idle rows of a decoded batch among them, against float64."""
import pytest
import torch

import paper_2510_12872_amd as kv

from paged64 import Case, attention
from plain64 import check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _close(c, got, what=""):
    want, want_lse, tol, tol_lse = attention(c)
    check(got[0], want, tol, what + " out")
    check(got[1], want_lse, tol_lse, what + " lse")


def _idle(n, long):
    """Lengths of n sequences: the first, the last and every third of them has no token."""
    return [(0, -3)[b % 2] if b % 3 == 0 or b == n - 1 else long + 7 * b % 90 for b in range(n)]


# items * (layer, kv head) pairs are more than half of the wavefronts, so runs are not cut within items: a run holds the end of one and others behind it
@pytest.mark.parametrize("prefix", [0, 40, 300])
@pytest.mark.parametrize("case", [
    dict(L=4, H=8, G=4, D=128, dtype=BF16, rows=[1] * 40, lens=_idle(40, 260), page=16, one=True),
    dict(L=5, H=8, G=4, D=128, dtype=BF16, rows=[3, 2, 1, 0, 4] * 8, lens=_idle(40, 230), page=64, pad=1),   # tiles of 16 rows, and sequences without rows
    dict(L=4, H=8, G=5, D=128, dtype=BF16, rows=[5, 6, 4, 1] * 10, lens=_idle(40, 200), page=32),            # tiles of 32 rows
    dict(L=4, H=16, G=2, D=64, dtype=BF16, rows=[1] * 45, lens=_idle(45, 300), page=16, one=True),
    dict(L=2, H=16, G=1, D=256, dtype=BF16, rows=[1] * 40, lens=_idle(40, 210), page=16, one=True),
    dict(L=4, H=16, G=2, D=64, dtype=F32, rows=[1] * 45, lens=_idle(45, 120), page=16, one=True),
], ids=lambda c: f"D{c['D']}-G{c['G']}-{str(c['dtype'])[6:]}-rows{max(c['rows'])}")
def test_sequences_without_tokens_between_long_ones(case, prefix):
    c = Case(**case, prefix=prefix)
    outs = [c.attend(want_lse=True), c.attend(want_lse=True, workspace=torch.empty((0,), dtype=torch.uint8, device="cuda"))]
    for got, what in zip(outs, ("workspace", "no workspace")):
        _close(c, got, what)
    for got in (c.attend(want_lse=True) for _ in range(3)):
        assert all(torch.equal(a, b) for a, b in zip(got, outs[0]))


@pytest.mark.parametrize("n_pages,width", [(0, 3), (2, 0)])
@pytest.mark.parametrize("G,D", [(4, 128), (2, 64), (1, 256)])
def test_a_prefix_and_no_pages(G, D, n_pages, width):
    """Every sequence behind the prefix is without tokens: the walk goes from a prefix of many halves to items of none, head after head."""
    L, H, n, n_prefix = 4, 16, 24, 700
    g = torch.Generator().manual_seed(D)
    m = kv.Model(L, H, H * G, D, BF16, 1e4)
    rnd = lambda *shape: torch.randn(shape, generator=g).bfloat16().cuda()
    q, k, v = rnd(L, H * G, n, D), rnd(L, H, n_prefix, D), rnd(L, H, n_prefix, D)
    pool = torch.full((L, H, n_pages, 16, D), float("nan"), dtype=BF16, device="cuda")
    batch = kv.Batch(torch.zeros((n, width), dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda"))
    rows, keys = q.double().view(L, H, G * n, D), k.double().transpose(-1, -2).contiguous()
    w = torch.softmax((rows @ keys) / D ** 0.5, -1)
    want, size = ((w @ x).view(q.shape) for x in (v.double(), v.double().abs()))
    # as in paged64.attention: products of D channels, sums of 700 terms, probabilities and the result rounded
    ds = (D + 4) * 2.0 ** -24 * (rows.abs() @ keys.abs()).amax(-1).view(L, H * G, n, 1) / D ** 0.5
    tol = 1.01 * ((2 * ds + (n_prefix + 32) * 2.0 ** -24 + 2.0 ** -8) * size + 2.0 ** -8 * want.abs())
    for kw in (dict(), dict(workspace=torch.empty((0,), dtype=torch.uint8, device="cuda"))):
        got = kv.kvcomm_paged_attn_prefix(m, q, k, v, pool, pool.clone(), batch, **kw)
        assert bool(((got.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n_seqs,n_rows,entries", [(123, 54728, 11), (266, 59538, 14), (128, 46555, 13)])
def test_more_rows_together_than_the_batch_has(dtype, n_seqs, n_rows, entries):
    """starts that falls from sequence to sequence: every other one claims all rows, and their halves together leave 31 bits.  Which rows are written is not defined,
    but nothing else is, and the call ends."""
    D, page = 64, 65536
    m = kv.Model(1, 1, 1, D, dtype, 1e4)
    pool = torch.zeros((1, 1, 1, page, D), dtype=dtype, device="cuda")
    table = torch.zeros((n_seqs, entries), dtype=torch.int32, device="cuda")   # every token in the one page
    lens = torch.full((n_seqs,), entries * page, dtype=torch.int32, device="cuda")
    starts = torch.tensor([n_rows * (b % 2) for b in range(n_seqs + 1)], dtype=torch.int32, device="cuda")
    batch = kv.Batch(table, lens, starts, max_rows=1)   # (a hint: the wavefront kernels take them)
    q = torch.zeros((1, 1, n_rows, D), dtype=dtype, device="cuda")
    guard = torch.full((1, 1, n_rows + 128, D), 5.0, dtype=dtype, device="cuda")
    lse = torch.full((n_rows + 128,), 5.0, device="cuda")
    need = kv.kvcomm_paged_attn_workspace(m, n_rows, page, 1, batch)
    ws = torch.full((need + 4096,), 9, dtype=torch.uint8, device="cuda")
    for w in (ws[:need], ws[:0]):
        kv.kvcomm_paged_attn(m, q, pool, pool, batch, out=guard[:, :, 64:64 + n_rows], lse_out=lse[64:64 + n_rows].view(1, 1, n_rows), want_lse=True, workspace=w)
    torch.cuda.synchronize()
    assert bool((guard[:, :, :64] == 5).all()) and bool((guard[:, :, 64 + n_rows:] == 5).all()) and bool((ws[need:] == 9).all())
    assert bool((lse[:64] == 5).all()) and bool((lse[64 + n_rows:] == 5).all())


@pytest.mark.parametrize("case", [
    dict(L=4, H=8, G=8, D=128, dtype=BF16, rows=[1] * 40, lens=_idle(40, 100), page=16, prefix=1100, one=True),
    dict(L=4, H=8, G=8, D=64, dtype=BF16, rows=[1] * 40, lens=_idle(40, 100), page=16, prefix=1100, one=True),
    dict(L=4, H=8, G=16, D=256, dtype=BF16, rows=[1] * 30, lens=_idle(30, 100), page=32, prefix=1100, one=True),
    dict(L=4, H=8, G=3, D=128, dtype=BF16, rows=[1, 2, 9] * 10, lens=_idle(30, 100), page=32, prefix=1100),
    dict(L=4, H=8, G=8, D=128, dtype=F32, rows=[1] * 20, lens=_idle(20, 60), page=16, prefix=200, one=True),
], ids=lambda c: f"D{c['D']}-{str(c['dtype'])[6:]}-rows{max(c['rows'])}")
def test_the_same_bits_after_anything(case):
    """Sequences without tokens behind a prefix: what an earlier launch has left on the chip does not show, not in the last bit either."""
    c = Case(**case)
    n = len(c.rows)
    bad = Case(**{**case, "rows": [1] * n, "lens": [64] * n, "prefix": 0, "one": True})   # fills what the kernels keep there with NaN
    bad.pages_k.fill_(float("nan")), bad.pages_v.fill_(float("nan"))
    outs = []
    for i in range(6):
        if i % 2:
            bad.attend()
        else:
            torch.zeros((1 << 26,), device="cuda").add_(1)
            kv.kvcomm_paged_attn(c.model, c.q, torch.zeros_like(c.pages_k), torch.zeros_like(c.pages_v), c.batch)
        outs.append(c.attend(want_lse=True))
    for got in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got, outs[0]))
    _close(c, outs[0])

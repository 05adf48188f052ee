"""Batches in pages: keys whose scores are minus infinity (a channel of -inf as a mask) count as weight 0 wherever they lie; a row that sees keys but no finite score is 0 / 0 as in
the attention over a whole cache (NaN, log-sum-exp -inf), and one that sees no key 0 and -inf."""
import numpy as np
import pytest
import torch

from paged64 import Case, attention
from plain64 import check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
INF = float("inf")

CASES = [  # kernels: wavefronts (items cut or not), tiles of rows (one run, several), both, fp32
    dict(L=1, H=2, G=4, D=128, dtype=BF16, rows=[1, 1, 1], lens=[500, 40, 0], page=16, one=True),
    dict(L=1, H=2, G=4, D=128, dtype=BF16, rows=[2, 5, 3], lens=[2, 700, 1], page=32),                  # (two rows before their sequence)
    dict(L=4, H=16, G=2, D=64, dtype=BF16, rows=[1] * 40, lens=[37 * b % 200 for b in range(40)], page=16, one=True),
    dict(L=1, H=2, G=1, D=256, dtype=BF16, rows=[4, 9], lens=[300, 5], page=16),
    dict(L=1, H=2, G=4, D=128, dtype=BF16, rows=[90, 1, 70], lens=[200, 77, 40], page=16, pad=1),
    dict(L=1, H=2, G=2, D=128, dtype=BF16, rows=[200], lens=[2500], page=64),
    dict(L=1, H=2, G=1, D=64, dtype=BF16, rows=[300, 40], lens=[320, 1500], page=256),
    dict(L=1, H=2, G=2, D=256, dtype=BF16, rows=[100], lens=[1300], page=64),
    dict(L=2, H=2, G=2, D=64, dtype=F32, rows=[1, 33, 4], lens=[300, 100, 2], page=16),
    dict(L=1, H=2, G=3, D=128, dtype=F32, rows=[1, 1], lens=[333, 1], page=32, one=True),
]


def _id(c):
    return f"D{c['D']}-{str(c['dtype'])[6:]}-rows{max(c['rows'])}of{len(c['rows'])}-lens{max(c['lens'])}"


def _case(case, prefix, **kw):
    c = Case(**{**case, **kw}, prefix=prefix)
    c.q[..., 5] = 1.0   # the masking channel: a key with -inf there scores -inf with every query
    return c


def _calls(c):
    yield "workspace", c.attend(want_lse=True)
    yield "no workspace", c.attend(want_lse=True, workspace=torch.empty((0,), dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("prefix", [0, 33, 900])
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_rows_without_a_finite_score(case, prefix):
    """All keys of one kv head hidden so, in pages and prefix."""
    c = _case(case, prefix)
    G = c.model.n_q_heads // c.model.n_kv_heads
    good = {what: got for what, got in _calls(c)}
    c.pages_k[:, 1, ..., 5] = -INF
    if prefix:
        c.prefix_k[:, 1, :, 5] = -INF
    sees = np.zeros(c.n, dtype=bool)
    rows = np.zeros(c.n, dtype=bool)
    for b, n in enumerate(c.rows):
        for i in range(n):
            rows[c.starts[b] + i] = True
            sees[c.starts[b] + i] = prefix > 0 or len(c.seen(b, i)[0]) > 0
    sees, blind = (torch.from_numpy(x).cuda() for x in (sees & rows, rows & ~sees))
    head = slice(G, 2 * G)
    for what, (out, lse) in _calls(c):
        assert bool((lse[:, head][:, :, sees | blind] == -INF).all()), what
        assert bool(torch.isnan(out[:, head][:, :, sees]).all()), what
        assert not bool(out[:, head][:, :, blind].any()), what
        for h in range(c.model.n_q_heads):
            if not G <= h < 2 * G:
                assert torch.equal(out[:, h], good[what][0][:, h]) and torch.equal(lse[:, h], good[what][1][:, h]), (what, h)


@pytest.mark.parametrize("prefix", [0, 33, 900])
@pytest.mark.parametrize("case", [CASES[0], CASES[4], CASES[5], CASES[8]], ids=_id)
def test_the_same_where_entries_are_no_page(case, prefix):
    """What the formula computes again, key by key."""
    c = _case(case, prefix, missing=[(0, 1, -1), (0, 3, 10 ** 6)])
    c.pages_k[..., 5] = -INF
    if prefix:
        c.prefix_k[..., 5] = -INF
    row = int(c.starts[1]) - 1
    for what, (out, lse) in _calls(c):
        assert bool(torch.isnan(out[:, :, row]).all()) and bool((lse[:, :, row] == -INF).all()), what


@pytest.mark.parametrize("hide", ["pages", "prefix", "first pages", "last pages"])
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_hidden_keys_beside_others(case, hide):
    """Against float64 without the hidden keys."""
    prefix = 0 if hide == "first pages" else 300
    c = _case(case, prefix)
    page = c.page
    some = lambda b: c.lens[b] // page // 2 if hide == "first pages" else 0   # entries that stay as they are begin here ...
    until = lambda b: c.lens[b] // page // 2 if hide == "last pages" else -(-max(c.lens[b], 0) // page) if hide in ("prefix", "first pages") else 0   # ... and end here
    hidden = [(b, e) for b in range(len(c.rows)) for e in range(-(-max(c.lens[b], 0) // page)) if not some(b) <= e < until(b)]
    for b, e in hidden:
        c.pages_k[:, :, int(c.table[b, e]), :, 5] = -INF
    if hide == "prefix":
        c.prefix_k[..., 5] = -INF
    got = list(_calls(c))
    seen = [[len(c.seen(b, i)[0]) > 0 for i in range(n)] for b, n in enumerate(c.rows)]
    for b, e in hidden:
        c.table[b, e] = -1
    if hide == "prefix":
        c.prefix = 0
    want, want_lse, tol, tol_lse = attention(c)
    for b, n in enumerate(c.rows):   # rows of which every key is hidden
        for i in range(n):
            if not c.prefix and not c.seen(b, i)[0] and (seen[b][i] or hide == "prefix"):
                want[:, :, c.starts[b] + i] = np.nan
    for what, (out, lse) in got:
        check(out, want, tol, what + " out")
        check(lse, want_lse, tol_lse, what + " lse")

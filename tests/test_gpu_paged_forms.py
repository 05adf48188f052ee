"""Batches in pages: every kernel that a call reaches, the forms of a call, and what the documentation allows around it."""
import numpy as np
import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import binding

from paged64 import Case, attention, place
from plain64 import check, f64
from test_marshal import Counts, Declines

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def _close(c, got, untouched=0.0, what=""):
    want, want_lse, tol, tol_lse = attention(c, untouched=untouched)
    check(got[0], want, tol, what + " out")
    check(got[1], want_lse, tol_lse, what + " lse")


def _id(c):
    return "-".join(f"{k}{str(v).replace('torch.', '').replace(' ', '')[:40]}" for k, v in c.items())


CASES = [
    # more sequences than a wavefront has lanes, with and without starts; some empty
    dict(L=1, H=2, G=2, D=64, dtype=BF16, rows=[1] * 150, lens=[7 * i % 120 + 1 for i in range(150)], page=16, one=True),
    dict(L=1, H=1, G=4, D=64, dtype=BF16, rows=[i % 3 for i in range(131)], lens=[i % 3 + 5 * i % 70 for i in range(131)], page=32, pad=1),
    dict(L=1, H=1, G=2, D=64, dtype=F32, rows=[i % 3 for i in range(131)], lens=[i % 3 + 5 * i % 70 for i in range(131)], page=16),
    # a token's heads over several tiles of rows
    dict(L=1, H=1, G=20, D=128, dtype=BF16, rows=[1, 1, 1], lens=[40, 300, 1], page=16, one=True),
    dict(L=1, H=2, G=40, D=64, dtype=BF16, rows=[1, 2, 1], lens=[40, 300, 1], page=16),
    dict(L=1, H=3, G=17, D=64, dtype=F32, rows=[1, 1], lens=[40, 300], page=16, one=True),
    # few and many rows in one batch: all kernels of a call
    dict(L=1, H=2, G=4, D=128, dtype=BF16, rows=[1, 90, 2, 8, 9, 1], lens=[500, 200, 2, 300, 9, 1], page=16, pad=2),
    dict(L=2, H=1, G=2, D=256, dtype=BF16, rows=[1, 90, 16, 17], lens=[300, 90, 100, 17], page=32),
    # keys of many rows cut into runs, the last of which some rows do not reach
    dict(L=1, H=1, G=2, D=128, dtype=BF16, rows=[200], lens=[2500], page=64),
    dict(L=1, H=1, G=1, D=64, dtype=BF16, rows=[300, 40], lens=[320, 1500], page=256),
    dict(L=1, H=1, G=2, D=256, dtype=BF16, rows=[100], lens=[1300], page=64),
    # 256 rows a block
    dict(L=1, H=1, G=8, D=64, dtype=BF16, rows=[150], lens=[400], page=16),
    dict(L=1, H=1, G=8, D=128, dtype=BF16, rows=[70, 80], lens=[100, 333], page=16),
]


@pytest.mark.parametrize("prefix", [0, 33, 1000])
@pytest.mark.parametrize("case", CASES, ids=_id)
def test_kernels_against_float64(case, prefix):
    c = Case(**case, prefix=prefix)
    _close(c, c.attend(want_lse=True))


@pytest.mark.parametrize("case", [
    # a prefix for some tiles of rows, on the wavefronts' axis: with and without starts, a last tile that is not full, sequences that end within one
    dict(L=1, H=2, G=4, D=128, dtype=BF16, rows=[1] * 21, lens=[11 * i % 90 + 1 for i in range(21)], page=16, prefix=500, one=True),
    dict(L=2, H=1, G=3, D=64, dtype=BF16, rows=[i % 4 for i in range(30)], lens=[i % 4 + 3 * i % 40 for i in range(30)], page=16, pad=2, before=1, prefix=257),
    dict(L=1, H=1, G=8, D=256, dtype=BF16, rows=[1] * 9, lens=[40, 1, 0, 70, 33, 32, 31, 64, 5], page=32, prefix=300, one=True),
    # so many that its tiles are of 128 and 256 rows, and so few of them that keys are cut
    dict(L=4, H=8, G=8, D=64, dtype=BF16, rows=[1] * 64, lens=[7 * i % 60 + 1 for i in range(64)], page=16, prefix=700, one=True),
    dict(L=4, H=8, G=4, D=128, dtype=BF16, rows=[1] * 30, lens=[7 * i % 60 + 1 for i in range(30)], page=16, prefix=2100, one=True),
    dict(L=4, H=4, G=4, D=256, dtype=BF16, rows=[1] * 40, lens=[7 * i % 60 + 1 for i in range(40)], page=16, prefix=1100, one=True),
], ids=_id)
def test_tokens_of_many_sequences_behind_a_prefix(case):
    c = Case(**case)
    _close(c, c.attend(want_lse=True))


@pytest.mark.parametrize("prefix", [0, 70])
@pytest.mark.parametrize("case", [CASES[1], CASES[2], CASES[4], CASES[6], CASES[7]], ids=_id)
def test_without_a_workspace(case, prefix):
    """None, one that is too small, one that is misaligned: every item is one wavefront's work."""
    c = Case(**case, prefix=prefix)
    need = c.workspace()
    big = torch.empty((need + 64,), dtype=torch.uint8, device="cuda")
    outs = []
    for ws in (big[:0], big[:max(need - 16, 0)], big[8:8 + need]):
        ws.fill_(7)
        outs.append(c.attend(want_lse=True, workspace=ws))
        assert bool((ws == 7).all())
    _close(c, outs[0])
    assert all(torch.equal(a, b) for x in outs[1:] for a, b in zip(outs[0], x))
    big.fill_(255)   # NaN: what it holds does not matter
    _close(c, c.attend(want_lse=True, workspace=big[:need]))


@pytest.mark.parametrize("case", [CASES[6], CASES[2], CASES[8], dict(CASES[8], G=1, rows=[300]), CASES[0]], ids=_id)
@pytest.mark.parametrize("prefix", [0, 300])
def test_the_same_bits_again(case, prefix):
    c = Case(**case, prefix=prefix)
    a = c.attend(want_lse=True)
    for stream in (None, torch.cuda.Stream(), torch.cuda.Stream()):
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        b = c.attend(want_lse=True, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_hints_that_are_wrong():
    """max_rows says how many rows a sequence has about: any value gives the result."""
    c = Case(1, 2, 4, 128, BF16, rows=[1, 90, 9], lens=[500, 200, 300], page=16, prefix=50)
    for most in (0, 1, 3, 10 ** 9):
        c.batch = kv.Batch(c.batch.table, c.batch.lens, c.batch.starts, max_rows=most)
        _close(c, c.attend(want_lse=True), what=str(most))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_pages_that_are_shared(dtype):
    """By sequences, and twice within one."""
    c = Case(1, 2, 2, 64, dtype, rows=[1, 1, 3], lens=[50, 64, 40], page=16)
    c.table[1, 0] = c.table[0, 0]
    c.table[1, 2] = c.table[1, 1]
    c.batch.table.copy_(torch.from_numpy(c.table))
    _close(c, c.attend(want_lse=True))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [[1, 1], [5, 40]])
def test_far_pages(dtype, rows):
    """Pages and rows more than 2^32 bytes apart."""
    c = Case(1, 2, 2, 64, dtype, rows=rows, lens=[30, 70], page=16, prefix=40)
    far = 1 << 29   # elements from page to page

    def spread(t):
        x = torch.empty((c.n_pages * far,), dtype=dtype, device="cuda")
        y = torch.as_strided(x, t.shape, (0, 16 * 64, far, 64, 1))   # [page, head, slot], one layer
        y.copy_(t)
        return y
    near = c.attend(want_lse=True)
    c.pages_k, c.pages_v = spread(c.pages_k), spread(c.pages_v)
    got = c.attend(want_lse=True)
    assert all(torch.equal(a, b) for a, b in zip(got, near))
    m = c.model
    q, k, v = torch.randn_like(c.q), torch.randn_like(c.q[:, :2]), torch.randn_like(c.q[:, :2])
    want = place(c, q, k, v, torch.zeros_like(q), 0, 0.0, None, None)
    q_out = kv.kvcomm_place_qkv_paged(m, q, k, v, c.batch, c.pages_k, c.pages_v)
    check(q_out, want[0], want[3], "q_out")
    check(c.pages_k, want[1], want[4], "pages_k")
    check(c.pages_v, want[2], np.zeros_like(want[2]), "pages_v")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_beyond_the_exponent(dtype):
    """References so large that their rounding reaches the exponent: the rows are computed by the formula."""
    c = Case(1, 1, 2, 64, dtype, rows=[1, 40], lens=[100, 60], page=16, prefix=80, sigma=2000.0)
    _close(c, c.attend(want_lse=True))


def test_a_graph_follows_its_batch():
    """A captured step of place and attention: tokens, tables and starts change between replays, an eager step works with the same tensors in between, and two graphs
    share a workspace."""
    L, H, G, D, B = 2, 2, 4, 128, 5
    m = kv.Model(L, H, H * G, D, BF16, 1e4)
    c = Case(L, H, G, D, BF16, rows=[1] * B, lens=[40, 17, 16, 200, 90], page=16, prefix=150, fill=0.0)
    table = torch.full((B, 20), -1, dtype=torch.int32, device="cuda")
    lens = c.batch.lens
    pool = torch.randperm(64, generator=torch.Generator().manual_seed(2)).int().cuda()
    pk, pv = (torch.randn((L, 64, H, 16, D), device="cuda").bfloat16().transpose(1, 2) for _ in range(2))
    for b in range(B):
        table[b, :12] = pool[12 * b:12 * b + 12] if b < 5 else -1
    table[3] = -1
    table[3, :4] = pool[60:64]
    one, two = kv.Batch(table, lens), kv.Batch(table, lens, torch.arange(0, 2 * B + 1, 2, dtype=torch.int32, device="cuda"), max_rows=2)
    need = max(kv.kvcomm_paged_attn_prefix_workspace(m, 150, b.lens.shape[0] * r, 16, 64, b) for b, r in ((one, 1), (two, 2)))
    ws = torch.empty((need,), dtype=torch.uint8, device="cuda")

    def tensors(n):
        return [torch.randn((L, h, n, D), device="cuda").bfloat16() for h in (H * G, H, H)] + [torch.zeros((L, H * G, n, D), dtype=BF16, device="cuda") for _ in range(2)]

    def step(batch, q, k, v, placed, out):
        kv.kvcomm_place_qkv_paged(m, q, k, v, batch, pk, pv, 150, q_out=placed)
        kv.kvcomm_paged_attn_prefix(m, placed, c.prefix_k, c.prefix_v, pk, pv, batch, out=out, workspace=ws)
    sets = [(one, *tensors(B)), (two, *tensors(2 * B))]
    graphs = []
    for s in sets:
        step(*s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(*s)
        graphs.append(g)
    start = pk.clone(), pv.clone()
    for i in range(6):
        lens += 1 + i
        if i == 2:
            table[0, :6] = table[0, :6].flip(0)
        if i == 4:
            two.starts.copy_(torch.tensor([0, 0, 5, 6, 10, 10], dtype=torch.int32))
        for s, g in zip(sets, graphs):
            s[1].normal_()
            s[5].zero_()
            pk.copy_(start[0]), pv.copy_(start[1])
            g.replay()
            torch.cuda.synchronize()
            got = s[5].clone(), pk.clone(), pv.clone()
            pk.copy_(start[0]), pv.copy_(start[1])
            s[5].zero_()
            step(*s)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (s[5], pk, pv))), i


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_native_module_makes_the_same_calls(monkeypatch, dtype):
    kv.load_library()

    def everything():
        outs = []
        for one in (True, False):
            c = Case(2, 2, 3, 64, dtype, rows=[1, 1, 1], lens=[20, 1, 90], page=16, prefix=20, one=one, layout="token_major", pad=0 if one else 2, fill=0.0)
            w = torch.ones((2, 64), dtype=dtype, device="cuda")
            for kw in (dict(), dict(norm_eps=1e-5, q_weight=w, k_weight=w[1]), dict(norm_eps=1)):
                outs += [kv.kvcomm_place_qkv_paged(c.model, c.q, c.q[:, :2], c.q[:, 2:4], c.batch, c.pages_k, c.pages_v, 7, **kw), c.pages_k.clone(), c.pages_v.clone()]
            kv.kvcomm_place_qkv_paged(c.model, None, c.q[:, :2], None, c.batch, c.pages_k, None)
            outs += [kv.kvcomm_place_qkv_paged(c.model, c.q, None, None, c.batch, None, None), c.pages_k.clone()]
            for kw in (dict(), dict(softmax_scale=0.3, want_lse=True), dict(softmax_scale=1, stream=torch.cuda.current_stream())):
                outs += [kv.kvcomm_paged_attn(c.model, c.q, c.pages_k, c.pages_v, c.batch, **kw), c.attend(**kw)]
        torch.cuda.synchronize()
        return [t for x in outs for t in (x if isinstance(x, tuple) else (x,))]
    counts = Counts(binding._native)
    monkeypatch.setattr(binding, "_native", counts)
    native = everything()
    assert set(counts.took) == {"place_qkv_paged", "paged_attn_workspace", "paged_attn"} and not counts.declined
    monkeypatch.setattr(binding, "_native", Declines())
    general = everything()
    assert len(native) == len(general) and all(torch.equal(a, b) for a, b in zip(native, general))


def test_another_device_is_refused():
    class Elsewhere:
        device_index = 1
        cuda_stream = 0
    c = Case(1, 1, 1, 64, BF16, rows=[1, 2], lens=[5, 20], page=16, prefix=8, fill=0.0)
    out = torch.empty_like(c.q)
    ws = torch.empty((c.workspace(),), dtype=torch.uint8, device="cuda")
    for call in (lambda: c.attend(out=out, workspace=ws, stream=Elsewhere()),
                 lambda: kv.kvcomm_place_qkv_paged(c.model, c.q, c.q.clone(), c.q.clone(), c.batch, c.pages_k, c.pages_v, q_out=out, stream=Elsewhere())):
        with pytest.raises(kv.KVCommError):
            call()


def test_no_pages_at_all():
    """A table without entries or a pool without pages: the prefix alone, or nothing."""
    for n_pages, width in ((0, 3), (2, 0)):
        for dtype in (BF16, F32):
            m = kv.Model(1, 2, 8, 64, dtype, 1e4)
            q, k = torch.randn((1, 8, 3, 64), device="cuda").to(dtype), torch.randn((1, 2, 40, 64), device="cuda").to(dtype)
            pool = torch.full((1, 2, n_pages, 16, 64), float("nan"), dtype=dtype, device="cuda")
            batch = kv.Batch(torch.zeros((3, width), dtype=torch.int32, device="cuda"), torch.tensor([5, 0, 1], dtype=torch.int32, device="cuda"))
            out, lse = kv.kvcomm_paged_attn(m, q, pool, pool.clone(), batch, want_lse=True)
            assert not bool(out.any()) and bool((lse == -float("inf")).all())
            got = kv.kvcomm_paged_attn_prefix(m, q, k, k, pool, pool.clone(), batch)
            want = torch.softmax((q.double().view(1, 2, 4, 3, 64) @ k.double()[:, :, None].transpose(-1, -2)) / 8, -1) @ k.double()[:, :, None]
            # probabilities and the result rounded to the type, half a step each
            half = {BF16: 2.0 ** -8, F32: 2.0 ** -24 * 70}[dtype]
            assert (got.double() - want.reshape(got.shape)).abs().max() <= 2.1 * half * k.double().abs().max()
            placed = kv.kvcomm_place_qkv_paged(m, q, k[:, :, :3], k[:, :, 3:6], batch, pool, pool.clone(), 3)
            assert torch.equal(placed[:, :, 2], kv.kvcomm_place_qkv(m, q[:, :, 2:], None, None, 3)[0][:, :, 0])
            assert torch.equal(placed[:, :, 0], kv.kvcomm_place_qkv(m, q[:, :, :1], None, None, 7)[0][:, :, 0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("prefix", [0, 40, 300])
def test_sequences_that_claim_the_same_rows(dtype, prefix):
    """starts that goes up and down between 130 sequences, each with up to all rows: which rows are written, and with what, is not defined, but nothing else is."""
    n = 60
    c = Case(1, 2, 4, 64, dtype, rows=[n] + [0] * 129, lens=[3 * i % 50 for i in range(130)], page=16, prefix=prefix, fill=0.0)
    need = c.workspace()
    for starts in ([n * (i % 2) for i in range(131)], [(37 * i) % (n + 5) - 2 for i in range(131)], [-(2 ** 31) if i % 3 else 2 ** 31 - 1 for i in range(131)]):
        c.batch.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        for most in (0, 1):
            c.batch = kv.Batch(c.batch.table, c.batch.lens, c.batch.starts, max_rows=most)
            ws = torch.full((max(need, c.workspace()) + 4096,), 9, dtype=torch.uint8, device="cuda")
            guard = torch.full((1, 8, n + 16, 64), 5.0, dtype=dtype, device="cuda")
            lse = torch.full((8 * n + 64,), 5.0, device="cuda")
            use = c.workspace()
            for w in (ws[:use], None):
                c.attend(out=guard[:, :, 8:8 + n], lse_out=lse[32:32 + 8 * n].view(1, 8, n), want_lse=True, workspace=w)
            kv.kvcomm_place_qkv_paged(c.model, c.q, c.q[:, :2], c.q[:, 2:4], c.batch, c.pages_k, c.pages_v, q_out=guard[:, :, 8:8 + n])
            torch.cuda.synchronize()
            assert bool((guard[:, :, :8] == 5).all()) and bool((guard[:, :, 8 + n:] == 5).all()) and bool((ws[use:] == 9).all())
            assert bool((lse[:32] == 5).all()) and bool((lse[32 + 8 * n:] == 5).all())

"""The run of a batch's operators as a program uses them: sequences of a PagedCache behind an agent's cache, placed and attended to step by step."""
import numpy as np
import pytest
import torch

import paper_2510_12872_amd as kv
from paper_2510_12872_amd import hotpath

from plain64 import HALF_STEP, attention, check, f64, placed


def _cpu(n_pages=6, page=16):
    return hotpath.PagedCache(kv.Model(1, 1, 1, 64, torch.float32, 1e4), n_pages, page, "cpu")


def test_pages_are_handed_out_and_taken_back():
    c = _cpu()
    a, b = c.open(), c.open()
    batch = c.extend([a, b], [20, 1])
    assert batch.lens.tolist() == [20, 1] and batch.starts.tolist() == [0, 20, 21] and batch.max_rows == 20
    assert len(c.pages[a]) == 2 and len(c.pages[b]) == 1 and len(set(c.pages[a] + c.pages[b])) == 3
    assert batch.table.tolist() == [c.pages[a], c.pages[b] + [-1]]
    batch = c.extend([b, a], [1, 1])
    assert batch.lens.tolist() == [2, 21] and batch.starts is None
    with pytest.raises(kv.KVCommError):
        c.extend([a], [16 * 6])                       # no room: nothing has changed
    assert c.lens == {a: 21, b: 2} and len(c._free) == 3
    for seqs, rows in (([a, a], [1, 1]), ([7], [1]), ([a], [1, 2]), ([a], [-1]), ([], [])):
        with pytest.raises(kv.KVCommError):
            c.extend(seqs, rows)
    c.extend([a], [30])
    c.retract([a], [30])
    assert c.lens[a] == 21 and len(c.pages[a]) == 2 and len(c._free) == 3
    c.close(a)
    assert sorted(c._free + c.pages[b]) == list(range(6)) and a not in c.lens
    assert c.extend([b], [0]).starts.tolist() == [0, 0]


def test_a_batch_that_cannot_be_made_takes_no_pages(monkeypatch):
    c = _cpu()
    a = c.open()
    c.extend([a], [20])

    def no_memory(*args, **kw):
        raise MemoryError
    with monkeypatch.context() as m:
        m.setattr(hotpath.kv, "Batch", no_memory)
        with pytest.raises(MemoryError):
            c.extend([a], [40])
    assert c.lens[a] == 20 and len(c.pages[a]) == 2 and len(c._free) == 4
    for seqs, rows in (([a], [21]), ([a], [-1]), ([a, a], [1, 1]), ([9], [0]), ([a], [])):
        with pytest.raises(kv.KVCommError):
            c.retract(seqs, rows)
        assert c.lens[a] == 20 and len(c.pages[a]) == 2 and len(c._free) == 4


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n_prefix", [0, 100])
def test_steps_against_float64(dtype, n_prefix):
    """Questions of several lengths behind one cache, then tokens of some of them, one sequence closed and another opened in between.  Each sequence's keys and
    values are kept beside, as placed by the formula, and attended to by it: what the kernels read is their own rounding of those."""
    L, H, G, D, eps = 2, 2, 2, 64, 1e-5
    m = kv.Model(L, H, H * G, D, dtype, 1e4)
    g = torch.Generator().manual_seed(1)
    rnd = lambda *shape: torch.randn(shape, generator=g).to(dtype).cuda()
    prefix = (rnd(L, H, n_prefix, D), rnd(L, H, n_prefix, D)) if n_prefix else None
    pre = [f64(t) for t in prefix] if n_prefix else [np.zeros((L, H, 0, D))] * 2
    w = (1 + 0.1 * torch.randn((L, D), generator=g)).to(dtype).cuda()
    cache = hotpath.PagedCache(m, 20, 16, "cuda")
    kept = {}
    a, b, c = cache.open(), cache.open(), cache.open()
    plan = [([a, b, c], [5, 40, 1]), ([a, b, c], [1, 1, 1]), ([c, a], [17, 1]), "close b", ([a, "d"], [1, 70]), ([a, "d", c], [1, 1, 1])]
    half = HALF_STEP[dtype]
    for step in plan:
        if step == "close b":
            cache.close(b)
            d = cache.open()
            continue
        seqs, rows = [d if s == "d" else s for s in step[0]], step[1]
        n = sum(rows)
        q, k, v = rnd(L, H * G, n, D), rnd(L, H, n, D), rnd(L, H, n, D)
        out = hotpath.batch_step(m, q, k, v, cache, seqs, rows, prefix, q_weight=w, k_weight=w, norm_eps=eps)
        at = 0
        for s, r in zip(seqs, rows):
            rows_, t0 = slice(at, at + r), cache.lens[s] - r
            at += r
            qs, _ = placed(f64(q[:, :, rows_]), n_prefix + t0, m.rope_theta, eps, f64(w))
            ks, koff = placed(f64(k[:, :, rows_]), n_prefix + t0, m.rope_theta, eps, f64(w))
            old = kept.get(s, [np.zeros((L, H, 0, D))] * 2)
            kept[s] = [np.concatenate([old[0], ks], 2), np.concatenate([old[1], f64(v[:, :, rows_])], 2)]
            # the cache's rows: each within its rounding of the formula's
            for t in range(t0, t0 + r):
                e, slot = cache.pages[s][t // 16], t % 16
                check(cache.k[:, :, e, slot], ks[:, :, t - t0], koff[:, :, t - t0] * (1 + half) + half * np.abs(ks[:, :, t - t0]), "key")
            keys, vals = (np.concatenate([p, x], 2) for p, x in zip(pre, kept[s]))
            want, _, tol, _ = attention(qs, keys, vals, n_prefix + t0, dtype)
            # queries and keys are rounded to the type before their product, half a step each (and the fp32 error before it, below another): a score is off by
            # 4 half steps of the sum of its magnitudes, a probability by twice that
            ds = 4 * half * (np.abs(keys) @ np.ones(D)).max() * np.abs(qs).max() / np.sqrt(D)
            tol = tol + 2 * ds * np.abs(vals).max()
            check(out[:, :, rows_], want, tol, f"sequence {s}")


@pytest.mark.gpu
def test_a_step_is_the_suffix_of_every_sequence():
    """The same as suffix_step of each sequence on a cache of its own, up to rounding of sums in another order."""
    L, H, G, D, P = 2, 2, 4, 128, 200
    m = kv.Model(L, H, H * G, D, torch.bfloat16, 5e5)
    prefix = tuple(torch.randn((L, H, P, D), device="cuda").bfloat16() for _ in range(2))
    cache, rows = hotpath.PagedCache(m, 30, 32, "cuda"), [33, 1, 8]
    seqs = [cache.open() for _ in rows]
    q, k, v = (torch.randn((L, h, sum(rows), D), device="cuda").bfloat16() for h in (H * G, H, H))
    out = hotpath.batch_step(m, q, k, v, cache, seqs, rows, prefix)
    at = 0
    for n in rows:
        one = tuple(torch.cat([p, torch.zeros((L, H, n, D), device="cuda").bfloat16()], 2) for p in prefix)
        part = [t[:, :, at:at + n] for t in (q, k, v)]
        want = hotpath.suffix_step(m, *part, one, P)
        # both round probabilities to bf16 (half a step of the sum of magnitudes each, at most the largest value) and the result
        tol = 4 * 2.0 ** -8 * torch.stack([p.float().abs().max() for p in (*prefix, v)]).max()
        assert (out[:, :, at:at + n].float() - want.float()).abs().max() <= tol
        at += n


@pytest.mark.gpu
def test_a_step_that_fails_leaves_the_cache():
    m = kv.Model(1, 2, 2, 64, torch.bfloat16, 1e4)
    cache = hotpath.PagedCache(m, 4, 16, "cuda")
    s = cache.open()
    q = torch.randn((1, 2, 20, 64), device="cuda").bfloat16()
    for bad in (dict(k=q[:, :1]), dict(prefix=(q, q[:, :, :3])), dict(out=q.float()), dict(rows=[19]), dict(rows=[80])):
        args = {**dict(q=q, k=q.clone(), v=q.clone(), rows=[20]), **bad}
        with pytest.raises(kv.KVCommError):
            hotpath.batch_step(m, args.pop("q"), args.pop("k"), args.pop("v"), cache, [s], args.pop("rows"), **args)
        assert cache.lens[s] == 0 and cache.pages[s] == [] and len(cache._free) == 4
    hotpath.batch_step(m, q, q.clone(), q.clone(), cache, [s], [20])
    assert cache.lens[s] == 20 and len(cache.pages[s]) == 2

"""Batches of sequences in pages: makers of them, and placement and attention over them in float64 numpy, written from their definitions."""
import numpy as np
import torch

import paper_2510_12872_amd as kv

from plain64 import HALF_STEP, f64, placed

LAYOUTS = ("pages_first", "token_major", "plain", "interleaved", "heads_last")


def pools(L, H, n_pages, page, D, dtype, layout, fill=float("nan"), device="cuda"):
    """(pages_k, pages_v) [L, H, pages, slots, D] in one of several orders of memory."""
    new = lambda *shape: torch.full(shape, fill, dtype=dtype, device=device)
    if layout == "pages_first":    # [layer, page, head, slot]
        return tuple(new(L, n_pages, H, page, D).transpose(1, 2) for _ in range(2))
    if layout == "token_major":    # [layer, page, slot, head]
        return tuple(new(L, n_pages, page, H, D).permute(0, 3, 1, 2, 4) for _ in range(2))
    if layout == "heads_last":     # [page, slot, layer, head], rows further apart than they are long
        return tuple(new(n_pages, page, L, H, D + 32)[..., :D].permute(2, 3, 0, 1, 4) for _ in range(2))
    if layout == "interleaved":    # [page, layer, keys and values, head, slot]
        x = new(n_pages, L, 2, H, page, D)
        return tuple(x[:, :, i].permute(1, 2, 0, 3, 4) for i in range(2))
    return tuple(new(L, H, n_pages, page, D) for _ in range(2))


class Case:
    """Sequences of rows[b] new tokens, the last of lens[b] (more rows than tokens: the first of them lie before their sequence), in pages of a pool in
    random order; missing: (sequence, entry) of the table that are no page.  What no token lies in holds `fill`."""

    def __init__(self, L, H, G, D, dtype, rows, lens, page, prefix=0, layout="pages_first", pad=0, before=0, missing=(), seed=0, fill=float("nan"),
                 one=False, sigma=1.0):
        g = torch.Generator().manual_seed(seed)
        rnd = lambda *shape: (sigma * torch.randn(shape, generator=g)).to(dtype)
        self.model = kv.Model(L, H, H * G, D, dtype, 1e4)
        self.page, self.rows, self.lens, self.prefix = page, rows, lens, prefix
        of = [-(-max(n, 0) // page) for n in lens]
        self.n_pages, width = sum(of) + 2, max(of) + 1
        order = torch.randperm(self.n_pages, generator=g).tolist()
        table = np.full((len(rows), width), -1, dtype=np.int32)
        for b, m in enumerate(of):
            table[b, :m] = [order.pop() for _ in range(m)]
        for b, e, value in missing:
            table[b, e] = value
        self.table = table
        self.starts = np.concatenate([[before], before + np.cumsum(rows)]).astype(np.int32)
        self.n = int(self.starts[-1]) + pad
        self.pages_k, self.pages_v = pools(L, H, self.n_pages, page, D, dtype, layout, fill)
        for pool in (self.pages_k, self.pages_v):
            for b, n in enumerate(lens):
                for e in range(of[b]):
                    if 0 <= table[b, e] < self.n_pages:
                        m = min(page, n - e * page)
                        pool[:, :, int(table[b, e]), :m] = rnd(L, H, m, D).cuda()
        self.q = rnd(L, H * G, self.n, D).cuda()
        self.prefix_k = self.prefix_v = None
        if prefix:   # rows of a longer cache
            x = torch.full((2, L, H, prefix + 40, D), fill, dtype=dtype)
            x[:, :, :, 3:3 + prefix] = rnd(2, L, H, prefix, D)
            x = x.cuda()
            self.prefix_k, self.prefix_v = x[0, :, :, 3:3 + prefix], x[1, :, :, 3:3 + prefix]
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        self.batch = kv.Batch(dev(table), dev(np.array(lens, dtype=np.int32)), None if one else dev(self.starts), max_rows=max(rows))

    def attend(self, **kw):
        if self.prefix:
            return kv.kvcomm_paged_attn_prefix(self.model, self.q, self.prefix_k, self.prefix_v, self.pages_k, self.pages_v, self.batch, **kw)
        return kv.kvcomm_paged_attn(self.model, self.q, self.pages_k, self.pages_v, self.batch, **kw)

    def workspace(self):
        if self.prefix:
            return kv.kvcomm_paged_attn_prefix_workspace(self.model, self.prefix, self.n, self.page, self.n_pages, self.batch)
        return kv.kvcomm_paged_attn_workspace(self.model, self.n, self.page, self.n_pages, self.batch)

    def token(self, b, t):
        """(page, slot) of a token, None: it is not there."""
        if t < 0 or t >= max(self.lens[b], 0) or t // self.page >= self.table.shape[1]:
            return None
        e = int(self.table[b, t // self.page])
        return (e, t % self.page) if 0 <= e < self.n_pages else None

    def seen(self, b, i):
        """Tokens that row i of sequence b sees: lists of pages and slots."""
        at = [self.token(b, t) for t in range(max(0, self.lens[b] - self.rows[b] + i + 1))]
        at = [x for x in at if x is not None]
        return [e for e, _ in at], [s for _, s in at]


def attention(c, scale=None, untouched=0.0):
    """(out, lse, bound of out's error, bound of lse's) of a case."""
    m = c.model
    L, H, G, D = m.n_layers, m.n_kv_heads, m.n_q_heads // m.n_kv_heads, m.head_dim
    q, pk, pv = f64(c.q), f64(c.pages_k), f64(c.pages_v)
    fk, fv = (f64(c.prefix_k), f64(c.prefix_v)) if c.prefix else (np.zeros((L, H, 0, D)),) * 2
    scale = 1 / np.sqrt(D) if scale is None else scale
    half = HALF_STEP[m.dtype]
    out, lse = np.full(q.shape, untouched), np.full(q.shape[:3], untouched)
    tol, tol_lse = np.zeros(q.shape), np.zeros(q.shape[:3])
    for b in range(len(c.rows)):
        for i in range(c.rows[b]):
            row = int(c.starts[b]) + i
            e, s = c.seen(b, i)
            for l in range(L):
                for h in range(H):
                    k, v = np.concatenate([fk[l, h], pk[l, h, e, s]]), np.concatenate([fv[l, h], pv[l, h, e, s]])
                    for hq in range(h * G, h * G + G):
                        if len(k) == 0:
                            out[l, hq, row], lse[l, hq, row] = 0, -np.inf
                            continue
                        with np.errstate(all="ignore"):
                            x = k @ q[l, hq, row] * scale
                            top = x.max()
                            w = np.exp(x - top)
                            out[l, hq, row] = (w / w.sum()) @ v
                            lse[l, hq, row] = top + np.log(w.sum())
                            size = np.abs(w / w.sum()) @ np.abs(v)
                            # as in plain64.attention: a score is off by the roundings of D products, their sum and the scale; probabilities by two of those,
                            # the exponential and sums of N terms (joining runs of keys: an exponential, a product and a sum each, within the 32), bf16 by the
                            # rounding before the second product; then the result's own rounding
                            ds = (D + 4) * 2.0 ** -24 * (np.abs(k) @ np.abs(q[l, hq, row])).max() * scale
                            rel = 2 * ds + (len(x) + 32) * 2.0 ** -24 + (half if m.dtype == torch.bfloat16 else 0)
                            least = 2.0 ** -126 * (1 + np.nan_to_num(np.abs(v), posinf=0).sum(0))
                            tol[l, hq, row] = 1.01 * (rel * size + half * np.abs(out[l, hq, row])) + least
                            tol_lse[l, hq, row] = ds + (len(x) + 32) * 2.0 ** -24 * max(1.0, abs(lse[l, hq, row]))
    return out, lse, tol, tol_lse


def place(c, q, k, v, q_out, first, eps, wq, wk):
    """(q_out, pages_k, pages_v, and the bounds of q_out's and pages_k's errors) after the call, from what they held before."""
    m, half = c.model, HALF_STEP[c.model.dtype]
    x, y, z = f64(q), f64(k), f64(v)
    out, pk, pv = f64(q_out), f64(c.pages_k), f64(c.pages_v)
    tol, tol_k = np.zeros(out.shape), np.zeros(pk.shape)
    for b in range(len(c.rows)):
        t0, r0, n = c.lens[b] - c.rows[b] if c.lens[b] > 0 else -c.rows[b], int(c.starts[b]), c.rows[b]
        rows = slice(r0, r0 + n)
        if n == 0:
            continue
        want, off = placed(x[:, :, rows], first + t0, m.rope_theta, eps, wq)
        out[:, :, rows], tol[:, :, rows] = want, off * (1 + half) + half * np.abs(want)
        want, off = placed(y[:, :, rows], first + t0, m.rope_theta, eps, wk)
        for i in range(n):
            at = c.token(b, t0 + i)
            if at is not None:
                pk[:, :, at[0], at[1]], pv[:, :, at[0], at[1]] = want[:, :, i], z[:, :, r0 + i]
                tol_k[:, :, at[0], at[1]] = off[:, :, i] * (1 + half) + half * np.abs(want[:, :, i])
    return out, pk, pv, tol, tol_k

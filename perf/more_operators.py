"""Timed cases of serving a batch of sequences whose keys and values lie in the pages of one pool: appending to the pages, the attention
over them, and the attention of a batch whose sequences all continue one cache (the assembled cache of an agent).

A case is a dict of plain values; `op` says which operator one pass runs:

  append   projections of the batch's new tokens: RMS norm of every head's query and key (eps > 0), rotation to the tokens' positions, keys and
           values into their slots of the pages
  paged    causal attention of every sequence's new tokens over its own pages
  prefix   the same where every sequence stands behind one cache of `prefix` tokens, which all rows see

A batch has `B` sequences of `rows0` to `rows` new tokens each, behind `ctx0` to `ctx` tokens that the pages hold already.  The rows of all
sequences lie behind each other, those of sequence b from starts[b] on; its pages hold lens[b] tokens, the new ones last, token t
in slot t % page of page table[b, t // page].  Rows behind the last sequence (`pad` of them) belong to none and stay as they were.
Queries and outputs are [layers, heads, rows, channels], pools [layers, kv heads, pages, slots, channels].
"""
import math

import torch

own = False   # True: run() calls the framework, False: it computes the plain forms

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LLAMA8B = dict(L=32, hkv=8, hq=32, D=128, dtype="bf16", theta=5e5)
LLAMA8B_LAYER = {**LLAMA8B, "L": 1}
TINY = dict(L=2, hkv=4, hq=8, D=64, dtype="f32", theta=1e4)


def listed():
    return [
        # One decoded token of eight sequences, one layer of a model without head norms: the smallest call.
        dict(name="append_token", op="append", **LLAMA8B_LAYER, B=8, rows0=1, rows=1, ctx0=600, ctx=3100, page=16, pad=0, eps=0.0),
        # Ragged rows of the tiny fp32 configuration, with norms, in a padded batch.
        dict(name="append_tiny_f32", op="append", **TINY, B=5, rows0=1, rows=17, ctx0=0, ctx=301, page=16, pad=3, eps=1e-5),
        # Prompts of six agents, all layers, with norms.
        dict(name="append_prompts", op="append", **LLAMA8B, B=6, rows0=100, rows=1200, ctx0=0, ctx=4000, page=64, pad=0, eps=1e-6),
        # One decoded token of eight sequences, one layer: latency.
        dict(name="paged_token", op="paged", **LLAMA8B_LAYER, B=8, rows0=1, rows=1, ctx0=600, ctx=3100, page=16, pad=0),
        # One decoded token of sixteen sequences of very different lengths, all layers: memory's rate.
        dict(name="paged_token_long", op="paged", **LLAMA8B, B=16, rows0=1, rows=1, ctx0=500, ctx=16000, page=64, pad=0),
        # Ragged rows of the tiny fp32 configuration in a padded batch.
        dict(name="paged_tiny_f32", op="paged", **TINY, B=5, rows0=1, rows=33, ctx0=0, ctx=301, page=16, pad=2),
        # Pieces of prompts of six agents, four layers, on what the pages hold of them.
        dict(name="paged_prompts", op="paged", **{**LLAMA8B, "L": 4}, B=6, rows0=100, rows=2000, ctx0=0, ctx=6000, page=64, pad=0),
        # One decoded token of eight answers to the same cache (llama8b_5agents: 512 + 4 * 512 tokens), one layer.
        dict(name="prefix_token", op="prefix", **LLAMA8B_LAYER, prefix=2560, B=8, rows0=1, rows=1, ctx0=0, ctx=200, page=16, pad=0),
        # One decoded token of 64 answers to a long cache, all layers.
        dict(name="prefix_tokens", op="prefix", **LLAMA8B, prefix=8192, B=64, rows0=1, rows=1, ctx0=0, ctx=500, page=32, pad=0),
        # One decoded token of four answers to a very long cache, all layers: memory's rate.
        dict(name="prefix_few_long", op="prefix", **LLAMA8B, prefix=32768, B=4, rows0=1, rows=1, ctx0=10, ctx=100, page=16, pad=0),
        # Questions of 20 to 100 tokens to the same cache, eight layers.
        dict(name="prefix_suffix", op="prefix", **{**LLAMA8B, "L": 8}, prefix=4096, B=16, rows0=20, rows=100, ctx0=0, ctx=0, page=16, pad=5),
        # Odd sizes of the tiny fp32 configuration (64 + 128 tokens and one more).
        dict(name="prefix_tiny_f32", op="prefix", **TINY, prefix=193, B=6, rows0=1, rows=5, ctx0=0, ctx=40, page=16, pad=1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def _draw(rng):
    op = rng.choice(["append", "append", "paged", "paged", "paged", "prefix", "prefix", "prefix"])
    hkv, f32 = rng.choice([1, 2, 4, 8, 8, 8]), rng.random() < 0.2
    c = dict(op=op, L=rng.choice([1, _log_int(rng, 1, 4 if f32 else 32)]), hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 4, 5, 8]),
             D=rng.choice([64, 128, 128, 128, 256]), dtype="f32" if f32 else "bf16", theta=rng.choice([1e4, 5e5]))
    most = rng.choice([1, 1, _log_int(rng, 1, 64 if f32 else 2000)])
    longest = _log_int(rng, 1, 2000 if f32 else 16000)
    c.update(B=_log_int(rng, 1, 64), rows0=rng.randint(0 if most > 1 else 1, most), rows=most, ctx0=rng.randint(0, longest), ctx=longest,
             page=rng.choice([16, 16, 32, 64, 128, 256]), pad=rng.choice([0, 0, 1, 5]) if most > 1 else 0)
    if op == "append":
        c.update(eps=rng.choice([0.0, 1e-6, 1e-5]))
    if op == "prefix":
        c.update(prefix=_log_int(rng, 1, 2000 if f32 else 32768))
    return c


def _cost(c):
    """Seconds of a plain pass, roughly: its scores in fp32, the values it reads, the calls it makes."""
    starts, lens = batch(c)
    rows, L = starts[-1], c["L"]
    if c["op"] == "append":
        return rows * L * (c["hq"] + 2 * c["hkv"]) * c["D"] * 100 / 4e12 + _pool_bytes(c) / 2e12
    pairs = sum((b - a) * n for a, b, n in zip(starts, starts[1:], lens)) + rows * c.get("prefix", 0)
    tokens = sum(lens) + c.get("prefix", 0)
    return L * c["hq"] * pairs * (4 * c["D"] / 60e12 + 40 / 4e12) + L * c["hkv"] * tokens * c["D"] * 80 / 4e12 + c["B"] * 2e-4


def _pool_bytes(c):
    pages = sum(-(-n // c["page"]) for n in batch(c)[1])
    return 2 * c["L"] * c["hkv"] * pages * c["page"] * c["D"] * (2 if c["dtype"] == "bf16" else 4)


def draw(rng):
    cost, room = max(_cost(c) for c in listed()) * 0.7, max(_pool_bytes(c) for c in listed())
    while True:
        c = _draw(rng)
        if batch(c)[0][-1] > 0 and _cost(c) <= cost and _pool_bytes(c) <= room:
            return c


# ------------------------------------------------------------------------------------------ inputs
def _spread(lo, hi, n, turn):
    """n whole numbers from lo to hi, the last one hi, in no order: more of them short than long."""
    at = [((i + 1) * turn) % 1.0 for i in range(n - 1)] + [1.0]
    return [round(lo + (hi - lo) * x * x) for x in at]


def batch(c):
    """(starts [B + 1], lens [B]) of a case: rows and tokens of its sequences."""
    rows = _spread(c["rows0"], c["rows"], c["B"], 0.6180339887498949)
    ctx = _spread(c["ctx0"], c["ctx"], c["B"], 0.41421356237309515)
    starts = [0]
    for n in rows:
        starts.append(starts[-1] + n)
    return starts, [n + m for n, m in zip(rows, ctx)]


def _random(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000033 * (int(seed) + 1) % (2 ** 62))

    def normal(shape, dtype):
        if dtype == torch.float32 or math.prod(shape) < 1 << 28:
            return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)
        return torch.stack([normal(shape[1:], dtype) for _ in range(shape[0])])   # a layer at a time
    return normal, g


def prepare(case, seed):
    c, dt = case, DTYPES[case["dtype"]]
    r, g = _random(seed)
    L, hkv, hq, D, B, page = c["L"], c["hkv"], c["hq"], c["D"], c["B"], c["page"]
    starts, lens = batch(c)
    n = starts[-1] + c["pad"]
    of = [-(-x // page) for x in lens]                     # pages of each sequence
    n_pages, width = sum(of) + 3, max(of) + 1              # (some pages are nobody's)
    order = torch.randperm(n_pages, generator=g, device=DEV).int()
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, m in enumerate(of):
        table[b, :m] = order[at:at + m]
        at += m
    s = dict(case=dict(c), table=table, lens=torch.tensor(lens, dtype=torch.int32, device=DEV), starts=torch.tensor(starts, dtype=torch.int32, device=DEV),
             host=(starts, lens))
    # a page holds the slots of one head behind each other: [layer, page, head, slot, channel]
    s["pages_k"], s["pages_v"] = (r((L, n_pages, hkv, page, D), dt).transpose(1, 2) for _ in range(2))
    if own:   # the framework's description of the model and of the batch, which a program makes once
        import paper_2510_12872_amd as kv
        s["model"] = kv.Model(L, hkv, hq, D, dt, c["theta"])
        one = c["rows0"] == c["rows"] == 1 and c["pad"] == 0
        s["batch"] = kv.Batch(table, s["lens"], None if one else s["starts"], max_rows=c["rows"])
    if c["op"] == "append":
        # a layer's projections lie token by token, all heads of a token together: [layer, token, head, channel]
        x = r((L, n, hq + 2 * hkv, D), dt)
        s["q"], s["k"], s["v"] = (t.transpose(1, 2) for t in x.split([hq, hkv, hkv], 2))
        s["q_weight"], s["k_weight"] = (1.0 + 0.1 * r((2, L, D), torch.float32)).to(dt).unbind(0)
        s["q_out"] = torch.zeros((L, hq, n, D), dtype=dt, device=DEV)
        return s
    s["q"] = r((L, hq, n, D), dt)
    s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros((L, hq, n), dtype=torch.float32, device=DEV)
    if c["op"] == "prefix":
        s["prefix_k"], s["prefix_v"] = r((L, hkv, c["prefix"], D), dt), r((L, hkv, c["prefix"], D), dt)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _append(s):
    c, n = s["case"], s["host"][0][-1]
    half, page = c["D"] // 2, c["page"]
    row = torch.arange(n, device=DEV)
    seq = torch.searchsorted(s["starts"][1:], row.int(), right=True)
    t = s["lens"][seq] - s["starts"][seq + 1] + row        # token of its sequence
    at = s["table"][seq, t // page].long(), t % page
    angle = t.double()[:, None] * c["theta"] ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
    cos, sin = angle.cos().float(), angle.sin().float()

    def head(x, weight):
        x = x[:, :, :n].float()
        if c["eps"] > 0:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + c["eps"]) * weight.float()[:, None, None, :]
        a, b = x[..., :half], x[..., half:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    s["q_out"][:, :, :n] = head(s["q"], s["q_weight"]).to(s["q_out"].dtype)
    s["pages_k"][:, :, at[0], at[1]] = head(s["k"], s["k_weight"]).to(s["q_out"].dtype)
    s["pages_v"][:, :, at[0], at[1]] = s["v"][:, :, :n]
    return s["q_out"], s["pages_k"], s["pages_v"]


def _part(rows, k, v, hidden=None):
    """(unnormalised output, maximum, sum) of rows [heads, n, D] over keys and values [heads, N, D], all fp32; hidden: [n, N]."""
    scores = torch.bmm(rows, k.transpose(1, 2).contiguous()).mul_(rows.shape[-1] ** -0.5)
    if hidden is not None:
        scores.masked_fill_(hidden, -math.inf)
    most = scores.amax(-1, keepdim=True)
    p = scores.sub_(most).exp_()
    return torch.bmm(p, v), most, p.sum(-1, keepdim=True)


def _attention(s):
    c, (starts, lens) = s["case"], s["host"]
    L, hkv, G, D, page = c["L"], c["hkv"], c["hq"] // c["hkv"], c["D"], c["page"]
    q = s["q"].float().view(L * hkv, G, -1, D)
    if c["op"] == "prefix":   # once for the rows of all sequences
        before = [x.view(L * hkv, G, starts[-1], -1) for x in _part(
            q[:, :, :starts[-1]].reshape(L * hkv, -1, D), s["prefix_k"].float().view(L * hkv, -1, D), s["prefix_v"].float().view(L * hkv, -1, D))]
    for b, N in enumerate(lens):
        first, end = starts[b], starts[b + 1]
        n = end - first
        if n == 0:
            continue
        pages = s["table"][b, :-(-N // page)].long()
        k, v = (s[x][:, :, pages].flatten(2, 3)[:, :, :N].float().view(L * hkv, N, D) for x in ("pages_k", "pages_v"))
        hidden = None
        if n > 1:
            hidden = (torch.arange(N, device=DEV) > torch.arange(N - n, N, device=DEV)[:, None]).repeat(G, 1)
        o, most, total = _part(q[:, :, first:end].reshape(L * hkv, -1, D), k, v, hidden)
        if c["op"] == "prefix":
            o0, most0, total0 = (x[:, :, first:end].reshape(L * hkv, G * n, -1) for x in before)
            top = torch.maximum(most, most0)
            f, f0 = (most - top).exp(), (most0 - top).exp()
            o, most, total = o * f + o0 * f0, top, total * f + total0 * f0
        s["out"][:, :, first:end] = (o / total).view(L, hkv * G, n, D).to(s["out"].dtype)
        s["lse"][:, :, first:end] = (most + total.log()).view(L, hkv * G, n)
    return s["out"], s["lse"]


def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2510_12872_amd as kv
        m, b = s["model"], s["batch"]
        if c["op"] == "append":
            norm = dict(q_weight=s["q_weight"], k_weight=s["k_weight"], norm_eps=c["eps"]) if c["eps"] > 0 else {}
            kv.kvcomm_place_qkv_paged(m, s["q"], s["k"], s["v"], b, s["pages_k"], s["pages_v"], q_out=s["q_out"], **norm)
            return s["q_out"], s["pages_k"], s["pages_v"]
        if c["op"] == "paged":
            return kv.kvcomm_paged_attn(m, s["q"], s["pages_k"], s["pages_v"], b, out=s["out"], lse_out=s["lse"], want_lse=True)
        return kv.kvcomm_paged_attn_prefix(m, s["q"], s["prefix_k"], s["prefix_v"], s["pages_k"], s["pages_v"], b, out=s["out"], lse_out=s["lse"],
                                           want_lse=True)
    return _append(s) if c["op"] == "append" else _attention(s)


# ------------------------------------------------------------------------------------------ what it cannot do without
def work(case):
    c = case
    L, hkv, hq, D, es = c["L"], c["hkv"], c["hq"], c["D"], 2 if c["dtype"] == "bf16" else 4
    starts, lens = batch(c)
    n = starts[-1]
    if c["op"] == "append":
        return {"bytes": 2 * L * (hq + 2 * hkv) * n * D * es + (2 * L * D * es if c["eps"] > 0 else 0),
                "flops": L * (hq + hkv) * n * D * (7 if c["eps"] > 0 else 3)}
    pairs, tokens = n * c.get("prefix", 0), c.get("prefix", 0)
    for a, b, N in zip(starts, starts[1:], lens):
        m = b - a
        pairs += m * (N - m) + m * (m + 1) // 2
        tokens += N if m else 0
    return {"bytes": 2 * L * hkv * tokens * D * es + 2 * L * hq * n * D * es + 4 * L * hq * n, "flops": 4 * D * L * hq * pairs}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s, c = prepare(case, seed), case
    D, L, hkv, hq, page = c["D"], c["L"], c["hkv"], c["hq"], c["page"]
    starts, lens = batch(c)
    table = s["table"].tolist()
    if c["op"] == "append":
        i = torch.arange(D // 2, device=DEV, dtype=torch.float64)
        outs = [torch.zeros(s["q_out"].shape, dtype=torch.float64, device=DEV), s["pages_k"].double(), s["pages_v"].double()]

        def moved(x, w, first):
            x = x.double()
            if c["eps"] > 0:
                x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / D + c["eps"]) * w.double().view(L, 1, 1, D)
            turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV),
                               (first + torch.arange(x.shape[2], device=DEV, dtype=torch.float64))[:, None] / c["theta"] ** (2 * i / D))
            z = torch.complex(x[..., :D // 2], x[..., D // 2:]) * turn
            return torch.cat((z.real, z.imag), -1)
        for b, N in enumerate(lens):
            rows = slice(starts[b], starts[b + 1])
            first = N - (starts[b + 1] - starts[b])
            outs[0][:, :, rows] = moved(s["q"][:, :, rows], s["q_weight"], first)
            k, v = moved(s["k"][:, :, rows], s["k_weight"], first), s["v"][:, :, rows].double()
            t = first
            while t < N:   # page by page
                end = min(N, t - t % page + page)
                slots = slice(t % page, t % page + end - t)
                outs[1][:, :, table[b][t // page], slots] = k[:, :, t - first:end - first]
                outs[2][:, :, table[b][t // page], slots] = v[:, :, t - first:end - first]
                t = end
        return tuple(outs)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    P = c.get("prefix", 0)
    for l in range(L):
        for b, N in enumerate(lens):
            first, end = starts[b], starts[b + 1]
            pages = torch.tensor(table[b][:-(-N // page)], device=DEV, dtype=torch.long)
            k, v = (s["pages_" + x][l][:, pages].reshape(hkv, -1, D)[:, :N].double() for x in "kv")
            if P:
                k, v = torch.cat((s["prefix_k"][l].double(), k), 1), torch.cat((s["prefix_v"][l].double(), v), 1)
            key = torch.arange(P + N, device=DEV)
            for a in range(first, end, 256):
                z = min(a + 256, end)
                seen = key <= (P + N - end + torch.arange(a, z, device=DEV))[:, None]
                x = torch.matmul(s["q"][l, :, a:z].double().view(hkv, hq // hkv, z - a, D), k.transpose(1, 2).contiguous()[:, None]) / math.sqrt(D)
                x = torch.where(seen, x, -math.inf)
                lse[l, :, a:z] = torch.logsumexp(x, -1).view(hq, z - a)
                out[l, :, a:z] = torch.matmul(torch.softmax(x, -1), v[:, None]).view(hq, z - a, D)
    return out, lse

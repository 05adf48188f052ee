"""Placement, the 4-bit format and masked attention in float64 numpy, written from their definitions, with bounds on how far a kernel's result may
be off by its roundings alone (half a step each: bf16 2^-8, fp32 2^-24, relative)."""
import numpy as np
import torch

SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def placed(x, first, theta, eps, weight=None):
    """(values, bound of the fp32 error before the last rounding) of queries or keys [L, H, n, D]; weight [L, D]."""
    D = x.shape[-1]
    if eps > 0:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * weight[:, None, None, :]
    a, b = x[..., :D // 2], x[..., D // 2:]
    angle = (first + np.arange(x.shape[2]))[:, None] * theta ** (-2.0 * np.arange(D // 2) / D)
    want = np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], -1)
    # sum of up to 16 squares per lane and 5 joins (21), mean and eps (2), root, quotient, weight (3), cos or sin (1), product and sum (2): < 32 half steps
    off = 32 * 2.0 ** -24 * (np.abs(a) + np.abs(b))
    return want, np.concatenate([off, off], -1)


def encode4(x):
    """[..., D] -> (codes [..., D/2], scale bytes [..., D/32])."""
    x = x.reshape(x.shape[:-1] + (-1, 32))
    odd = ~np.isfinite(x).all(-1)
    most = np.where(np.isfinite(x), np.abs(x), 0).max(-1)
    e = np.full(most.shape, -125)
    while (more := (most > 7 * 2.0 ** e) & (e < 125)).any():
        e = e + more
    y = np.abs(np.where(np.isfinite(x), x, 0)) / 2.0 ** e[..., None]
    off = np.abs(y[..., None] - SIZES)
    best = off.min(-1, keepdims=True)
    code = np.argmax((off == best) * np.array([2, 1, 2, 1, 2, 1, 2, 1]), -1)   # ties to the even code
    code = (code + 8 * np.signbit(x)).reshape(x.shape[:-2] + (-1,)).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(odd, 255, e + 127).astype(np.uint8)


def decode4(codes, scales):
    code = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (-1,))
    size = np.where(code >= 8, -1.0, 1.0) * SIZES[code & 7]
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return size * scale.repeat(32, -1)


def attention(q, k, v, n_ctx, dtype, window=None, sinks=0, scale=None):
    """(out, lse, bound of out's error, bound of lse's).  Keys that a query does not see are left out, whatever they hold."""
    L, Hq, tq, D = q.shape
    Hkv, N = k.shape[1], k.shape[2]
    assert N == n_ctx + tq
    scale = 1 / np.sqrt(D) if scale is None else scale
    out, lse = np.empty_like(q), np.empty(q.shape[:3])
    tol, tol_lse = np.empty_like(q), np.empty(q.shape[:3])
    j = np.arange(N)
    for l in range(L):
        for h in range(Hq):
            kk, vv = k[l, h * Hkv // Hq], v[l, h * Hkv // Hq]
            for i in range(tq):
                p = n_ctx + i
                seen = j <= p if window is None else (j <= p) & ((j > p - window) | (j < sinks))
                with np.errstate(all="ignore"):
                    s = kk[seen] @ q[l, h, i] * scale
                    m = s.max()
                    e = np.exp(s - m)
                    w = e / e.sum()
                    out[l, h, i] = w @ vv[seen]
                    lse[l, h, i] = m + np.log(e.sum())
                    size = np.abs(w) @ np.abs(vv[seen])
                    # a score: products of D channels summed in fp32 and scaled; D + 4 half steps of the sum of magnitudes
                    ds = (D + 4) * 2.0 ** -24 * (np.abs(kk[seen]) @ np.abs(q[l, h, i])).max() * scale
                    # probabilities: a wrong score changes them and their sum (2 ds), the exponential and sums of N terms, for bf16 the
                    # rounding before the second product; then the result's own rounding
                    rel = 2 * ds + (len(s) + 32) * 2.0 ** -24 + (HALF_STEP[dtype] if dtype == torch.bfloat16 else 0)
                    # below 2^-126, the least normal number of both types, a step is no longer relative: probabilities and results there are
                    # off by up to 2^-126 (subnormal or zero), each of the probabilities times a value
                    least = 2.0 ** -126 * (1 + np.nan_to_num(np.abs(vv[seen]), posinf=0).sum(0))
                    tol[l, h, i] = 1.01 * (rel * size + HALF_STEP[dtype] * np.abs(out[l, h, i])) + least
                    tol_lse[l, h, i] = ds + (len(s) + 32) * 2.0 ** -24 * max(1.0, abs(lse[l, h, i]))
    return out, lse, tol, tol_lse


def check(got, want, tol, what):
    """Within tol where want is a number; infinities and NaN in the same places."""
    got = f64(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), f"{what}: NaN in other places"
    assert np.array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)]), f"{what}: infinities"
    off = np.abs(got[fine] - want[fine]) - tol[fine]
    assert off.size == 0 or off.max() <= 0, f"{what}: {(off > 0).sum()} of {off.size} values, worst by {off.max():.3e} beyond its bound {tol[fine][off.argmax()]:.3e}"

"""The bounded cache and the windowed attention in fp64 with numpy, one function
per definition, with no fusion (test infrastructure only).

A 4-bit block of 32 values: the smallest e with max |x| <= 7 * 2^e, kept in
[-100, 125], stored as e + 127; the code (sign, two exponent bits, one mantissa
bit) nearest to x / 2^e, ties to the even code.
"""
from __future__ import annotations

import numpy as np

FP4_STEPS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ------------------------------------------------------------- 4-bit rows
def fp4_encode(x):
    """Codes [..., D / 2] and scale bytes [..., D / 32] (uint8) of rows [..., D]."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = np.abs(blocks).max(-1)
    bad = ~np.isfinite(blocks).all(-1)
    e = np.full(top.shape, -100)
    fits = lambda k: top <= 7.0 * np.ldexp(1.0, k)  # noqa: E731
    for k in range(-100, 126):                       # the smallest that fits
        e = np.where(fits(k) & (e == -100) & ~fits(-100), np.where(fits(k - 1), e, k), e)
    e = np.where(~bad & ~fits(125), 125, e)
    y = np.abs(np.where(bad[..., None], 0.0, blocks)) / np.ldexp(1.0, e)[..., None]
    far = np.abs(y[..., None] - FP4_STEPS)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])       # even codes first: they win ties
    code = order[far[..., order].argmin(-1)]
    code = np.where(bad[..., None], 0, code | (np.signbit(blocks) << 3)).reshape(x.shape)
    packed = (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)
    return packed, np.where(bad, 255, e + 127).astype(np.uint8)


def fp4_decode(codes, scales):
    """fp64 values [..., D]."""
    codes = np.asarray(codes)
    code = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(code & 8, -1.0, 1.0) * FP4_STEPS[code & 7]
    scale = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return v * np.repeat(scale, 32, -1)


# ------------------------------------------------------------- attention
def _softmax_rows(z, sees):
    """Softmax of z over the last axis where `sees`; rows that see nothing are 0."""
    p = np.zeros(z.shape)
    for r in np.ndindex(z.shape[:-1]):
        s = sees[r]
        if s.any():
            e = np.exp(z[r][s] - z[r][s].max())
            p[r][s] = e / e.sum()
    return p


def _weighted(p, sees, v):
    """Rows of p . v over the seen keys only (the others may hold anything)."""
    out = np.zeros(p.shape[:-1] + v.shape[-1:])
    for r in np.ndindex(p.shape[:-1]):
        out[r] = p[r][sees[r]] @ v[sees[r]]
    return out


def attend(q, k, v, pos, seen, scale=None):
    """One (sequence, group): q [n_q, G, D] over its live slots k, v [n, D], pos [n].
    Returns (out [n_q, G, D], what every slot received [n], p [n_q, G, n], sees)."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n_q, g, d = q.shape
    c = 1.0 / np.sqrt(d) if scale is None else scale
    sees = np.ones((n_q, g, len(k)), dtype=bool)
    if n_q > 1:
        sees &= (np.asarray(pos)[None, :] <= (seen - n_q + np.arange(n_q))[:, None])[:, None, :]
    with np.errstate(invalid="ignore"):
        z = c * np.einsum("igd,sd->igs", q, k) if len(k) else np.zeros((n_q, g, 0))
        p = _softmax_rows(z, sees)
        return _weighted(p, sees, v), np.where(sees, p, 0.0).sum((0, 1)), p, sees


def window_attention(q, k, v, window, n_sinks, scale=None):
    """One sequence: q [Lq, Hq, D], the last Lq tokens, over k, v [Lk, Hkv, D]."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    lq, hq, d = q.shape
    lk, hkv, _ = k.shape
    c = 1.0 / np.sqrt(d) if scale is None else scale
    out = np.zeros(q.shape)
    t = lk - lq + np.arange(lq)[:, None]
    j = np.arange(lk)[None, :]
    sees = (j <= t) & ((j > t - window) | (j < n_sinks))
    for h in range(hq):
        g = h // (hq // hkv)
        with np.errstate(invalid="ignore"):
            z = c * (q[:, h] @ k[:, g].T) if lk else np.zeros((lq, 0))
            out[:, h] = _weighted(_softmax_rows(z, sees), sees, v[:, g])
    return out


# -------------------------------------------------------------- eviction
def evict(weight, pos, n, seen, budget, n_sinks, n_recent):
    """One (sequence, group) with n live slots: [(to, from), ...] moves, new length."""
    if n <= budget:
        return [], n

    def rank(s):        # the first to go first
        held = pos[s] < n_sinks or pos[s] >= seen - n_recent
        w = -np.inf if np.isnan(weight[s]) else float(weight[s])
        return (held, not np.isnan(weight[s]) if not held else True, 0.0 if held else w, -s)

    gone = set(sorted(range(n), key=rank)[:n - budget])
    holes = [s for s in range(budget) if s in gone]
    tails = [s for s in range(budget, n) if s not in gone]
    assert len(holes) == len(tails)
    return list(zip(holes, tails)), budget

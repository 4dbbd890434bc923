"""Shared by the tests of the bounded cache and the windowed attention: caches
with given lengths on the GPU, and how far an output may be from the oracle's.

Tolerance of an attention output o = sum p v / sum p, with everything counted
that the kernels round (u = 2^-24, fp32; a rounding to bf16 is off by 2^-8 of
the value at most, one to fp32 by u):
  logits   a dot product of D terms in fp32: (D + 2) u sum |q| |k|, times the
           scale; the product with the scale, the subtraction of the reference
           (itself up to 2^8 away) and the exponential: 4 u |z| + 8 u.  That is
           the relative error dz of a p.
  p        rounded to bf16 twice (16 bits): 2^-16; once: 2^-8; fp32 paths: u.
  sums     n terms each, in fp32: n u, of p |v| and of p.
  output   rounded to its type once.
So |error| <= half_step |o| + (2 dz + part + 2 n u) sum p |v|.
A slot's weight adds rows of p: (2 dz + 2 n u + rows u) of what it received,
and one rounding of the new weight per addition.
"""
import numpy as np
import torch

from oracle import cache_oracle as CO

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def p_part(dtype, bits=16):
    """How far one probability is rounded before the product with V."""
    return 2.0 ** -bits if dtype == torch.bfloat16 else 2.0 ** -23


def logit_error(q, k, scale):
    """dz for every row against every key: q [..., D], k [n, D]."""
    d = q.shape[-1]
    size = np.abs(q) @ np.abs(k).T * scale
    return (d + 2) * U * size + 4 * U * size + 8 * U


def attention_tolerance(o, p, sees, dz, v, dtype, part):
    """o [..., D] of rows p [..., n] over v [n, D]."""
    n = p.shape[-1]
    worst = np.where(sees, dz, 0.0).max(-1, initial=0.0)[..., None]
    va = np.where(np.isfinite(v), np.abs(v), 0.0)
    return half_step(dtype) * np.abs(o) + (2 * worst + part + 2 * n * U) * (p @ va) + 1e-30


def bits(t):
    """Raw bits of a device tensor on the host."""
    t = t.contiguous()
    view = {2: torch.int16, 4: torch.int32, 1: torch.uint8}[t.element_size()]
    return t.view(view).cpu().numpy()


def values(t):
    return t.float().cpu().numpy().astype(np.float64)


def state(cache):
    """Everything a cache holds, on the host: rows as raw bits."""
    got = {n: bits(getattr(cache, n)) for n in ("k", "v", "pos", "weight", "length", "seen")}
    if cache.k_scale is not None:
        got.update(k_scale=bits(cache.k_scale), v_scale=bits(cache.v_scale))
    return got


def rows_of(cache, name):
    """fp64 values of a cache's rows [batch, Hkv, capacity, D] (the oracle's decoding)."""
    t = getattr(cache, name)
    s = getattr(cache, name + "_scale")
    if s is None:
        return values(t)
    return CO.fp4_decode(t.cpu().numpy(), s.cpu().numpy())


def make_cache(C, dtype, lengths, capacity, head_dim, gpu, seed, shuffled=True, past=0):
    """A cache whose group (b, g) has lengths[b][g] live slots; `dtype`: a torch dtype or
    C.FP4.  Dead slots hold what a row must never see: NaN rows, scales and weights."""
    g = np.random.default_rng(seed)
    lengths = np.asarray(lengths, dtype=np.int32)
    b, h = lengths.shape
    cache = C.Cache.empty(b, h, capacity, head_dim, dtype, gpu)
    cap = cache.capacity
    pos = np.full((b, h, cap), -7, dtype=np.int32)
    weight = np.full((b, h, cap), np.nan, dtype=np.float32)
    for i in range(b):
        for j in range(h):
            n = lengths[i, j]
            order = g.permutation(n) if shuffled else np.arange(n)
            pos[i, j, :n] = order + np.where(order < n // 2, 0, past)
            weight[i, j, :n] = g.random(n) ** 2
    dead = np.arange(cap)[None, None, :] >= lengths[..., None]
    for name in ("k", "v"):
        x = g.standard_normal((b, h, cap, head_dim)).astype(np.float32)
        x[..., :2] *= 4.0
        t = torch.from_numpy(x).to(gpu)
        if dtype == C.FP4:
            codes, scales = CO.fp4_encode(x)
            codes[dead], scales[dead] = 0xFF, 0xFF
            getattr(cache, name).copy_(torch.from_numpy(codes))
            getattr(cache, name + "_scale").copy_(torch.from_numpy(scales))
        else:
            getattr(cache, name).copy_(t)
            getattr(cache, name)[torch.from_numpy(dead).to(gpu)] = float("nan")
    cache.pos.copy_(torch.from_numpy(pos))
    cache.weight.copy_(torch.from_numpy(weight))
    cache.length.copy_(torch.from_numpy(lengths))
    cache.seen.copy_(torch.from_numpy(lengths + past))
    return cache

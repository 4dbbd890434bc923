"""Attention over long splits of a paged cache on the GPU: page numbers over many windows of them,
pages that are missing in the middle of the walk, and infinite values of V.

The reference is the definition in fp64 on the GPU; tolerances as tests/cache_helpers.py derives them.
A bf16 sequence of more than 32 query rows per group goes to the kernel for many rows, in blocks of
256 rows where the call has a sequence of more than 128, else of 128."""
import sys

import numpy as np
import pytest
import torch

from oracle import paged_oracle as PO
from paper_2606_24467_amd import compresskv as C
from tests import cache_helpers as H
from tests import paged_helpers as PH
from tests.test_gpu_paged import BF16, F32, KIND_IDS, KINDS

pytestmark = pytest.mark.gpu


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


def _randn(shape, dtype, gpu, seed):
    return torch.randn(shape, generator=torch.Generator(device=gpu).manual_seed(seed), device=gpu).to(dtype)


def _pool(cache_dtype, n_pages, hkv, d, gpu, seed, page=16):
    """k, v, k_scale, v_scale of a pool of random rows."""
    x = [_randn((n_pages, hkv, page, d), F32, gpu, seed + i) for i in range(2)]
    if cache_dtype != C.FP8:
        return [t.to(cache_dtype) for t in x] + [None, None]
    codes = [t.to(torch.float8_e4m3fn).view(torch.uint8) for t in x]
    g = torch.Generator(device=gpu).manual_seed(seed + 2)
    return codes + [torch.randint(126, 128, (n_pages, hkv, page, d // 32), generator=g, device=gpu,
                                  dtype=torch.uint8) for _ in x]


def _cache(cache_dtype, lengths, hkv, d, gpu, seed, spare=3):
    """A cache of sequences of these lengths, their pages of 16 tokens in no order.  Slots past the last
    token, and pages that nobody has, hold NaN."""
    need = [-(-n // 16) for n in lengths]
    n_pages = sum(need) + spare
    order = np.random.default_rng(seed).permutation(n_pages).astype(np.int32)
    table = np.full((len(lengths), max(need)), -1, dtype=np.int32)
    live = torch.zeros((n_pages, 16), dtype=torch.bool)
    for b, (m, n) in enumerate(zip(need, lengths)):
        table[b, :m], order = order[:m], order[m:]
        j = torch.arange(n)
        live[torch.from_numpy(table[b]).long()[j // 16], j % 16] = True
    rows = _pool(cache_dtype, n_pages, hkv, d, gpu, seed)
    dead = (~live).to(gpu)[:, None].expand(n_pages, hkv, 16)
    for x in rows:
        if x is not None:
            x[dead] = 0xFF if cache_dtype == C.FP8 else float("nan")
    return C.PagedCache(*rows, torch.from_numpy(table).to(gpu),
                        torch.tensor(lengths, dtype=torch.int32, device=gpu))


def _rows(cache, name, table, n):
    """fp64 rows [n, Hkv, D] of a sequence, and which are there."""
    page = table.long()[torch.arange(n, device=table.device) // cache.page_size]
    there = (page >= 0) & (page < cache.n_pages)
    slot = torch.arange(n, device=table.device) % cache.page_size
    page = torch.where(there, page, 0)
    x = getattr(cache, name)[page, :, slot]
    if cache.k_scale is not None:
        codes = torch.tensor(np.append(PO.FP8_STEPS, np.nan), device=x.device)
        s = getattr(cache, name + "_scale")[page, :, slot]
        size = torch.where(s == 255, torch.nan, torch.exp2(s.double() - 127)).repeat_interleave(32, -1)
        x = torch.where(x >= 128, -1.0, 1.0).double() * codes[(x & 127).long()] * size
    return x.double(), there


def _reference(cache, table, n, q, scale):
    """(o, how far an output may be from it) [m, Hq, D] of q, the last m of a sequence's n tokens."""
    m, hq, d = q.shape
    group = hq // cache.n_kv_heads
    k, there = _rows(cache, "k", table, n)
    v, _ = _rows(cache, "v", table, n)
    t = n - m + torch.arange(m, device=q.device)
    sees = (torch.arange(n, device=q.device)[None] <= t[:, None]) & there[None]       # [m, n]
    sees = sees.repeat_interleave(group, 0)                                           # rows of a group
    o, tol = torch.zeros((m, hq, d), device=q.device).double(), torch.zeros((m, hq, d), device=q.device).double()
    bits = 8 if q.dtype == BF16 and m * group > 32 else 16
    for g in range(cache.n_kv_heads):
        at = slice(g * group, (g + 1) * group)
        rows = q[:, at].double().reshape(m * group, d)
        kg = torch.where(there[:, None], k[:, g], 0.0)
        z = scale * (rows @ kg.T.contiguous())
        size = scale * (rows.abs() @ kg.abs().T.contiguous())
        dz = torch.where(sees, (d + 6) * H.U * size + 8 * H.U, 0.0).amax(1, keepdim=True)
        p = torch.softmax(z.masked_fill(~sees, -1e30), 1) * sees
        fine = torch.isfinite(v[:, g])
        vg = torch.where(fine & there[:, None], v[:, g], 0.0)
        one = p @ vg
        seen = (sees & (p > 0)).double()
        for wild, value in ((v[:, g] == torch.inf, torch.inf), (v[:, g] == -torch.inf, -torch.inf),
                            (v[:, g].isnan(), torch.nan)):
            hit = seen @ (wild & there[:, None]).double()
            one = one + torch.where(hit > 0, value, 0.0)
        off = (H.half_step(q.dtype) * torch.where(torch.isfinite(one), one.abs(), 0.0)
               + (2 * dz + H.p_part(q.dtype, bits) + 2 * n * H.U) * (p @ vg.abs()) + 1e-30)
        o[:, at], tol[:, at] = one.reshape(m, group, d), off.reshape(m, group, d)
    return o, tol


def _check(cache, n_new, q, out, scale, only=None):
    """Outputs against the reference, of the sequences `only`."""
    at = np.cumsum([0] + list(n_new))
    lengths = cache.length.cpu().tolist()
    for b in range(len(n_new)) if only is None else only:
        if n_new[b] == 0:
            continue
        want, tol = _reference(cache, cache.page_table[b], lengths[b], q[at[b]:at[b + 1]], scale)
        got = out[at[b]:at[b + 1]].double()
        fine = torch.isfinite(want)
        assert (got.isnan() == want.isnan()).all(), b
        assert (got[~fine & ~want.isnan()] == want[~fine & ~want.isnan()]).all(), b
        off = torch.where(fine, (got - want).abs(), 0.0)
        assert (off <= tol).all(), (b, (off / tol).max().item())


# ------------------------------------------------------------------ windows of pages
FORMS = [   # name, sequences, new tokens, Hq, Hkv: keys of a split about 10000
    ("few", 64, (1,), 32, 8),
    ("masks", 66, (1, 8, 3), 32, 8),           # two row tiles; more than 64 sequences are summed up before
    ("128", 32, (4, 6), 128, 8),               # 64 to 96 rows per group
    ("256", 16, (64, 50), 32, 2),              # 800 to 1024
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("form", FORMS, ids=lambda f: f[0])
@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
def test_page_numbers_over_many_windows(gpu, kind, form, d):
    """20000 tokens in pages of 16, each sequence's in an order of its own, in splits of 10000 keys:
    several times the page numbers that a workgroup has at hand.  The logits are wide enough that
    keys read in the place of others would be seen."""
    name, batch, news, hq, hkv = form
    cache_dtype, dtype = kind
    _say("windows", name, kind, d)
    n_pages, longest = 1300, 20000
    g = np.random.default_rng(31)
    table = np.stack([g.permutation(n_pages)[:-(-longest // 16)] for _ in range(batch)]).astype(np.int32)
    lengths = [int(x) for x in g.integers(19200, longest + 1, batch)]
    n_new = [news[b % len(news)] for b in range(batch)]
    cache = C.PagedCache(*_pool(cache_dtype, n_pages, hkv, d, gpu, 32), torch.from_numpy(table).to(gpu),
                         torch.tensor(lengths, dtype=torch.int32, device=gpu))
    q = _randn((sum(n_new), hq, d), dtype, gpu, 34)
    scale = 2.5 / np.sqrt(d)
    out = cache.attend(PH.chunk_of(C, n_new, gpu), q, scale=scale)
    only = [0, 1, batch // 2, batch - 1]
    _check(cache, n_new, q, out, scale, only)
    # one 1024 keys read in the place of those before, or of those four before, would be seen
    rows = slice(0, n_new[0])
    want, tol = _reference(cache, cache.page_table[0], lengths[0], q[rows], scale)
    for back in (64, 256):
        stale = cache.page_table[0].clone()
        stale[512:576] = stale[512 - back:576 - back]
        other, _ = _reference(cache, stale, lengths[0], q[rows], scale)
        assert ((other - want).abs() > 2 * tol).any(-1).double().mean() > 0.5


# ------------------------------------------------------------------ pages that are missing
def _gaps(b, segments, g):
    """The missing pages of sequence b: each first page of 8 (where a split of the keys may begin),
    then some of every kind together."""
    firsts = segments // 8
    if b < firsts:
        return [8 * b]
    kinds = [[1], [37], [63], [64], [63, 64, 65], [segments - 6], [segments - 1], [0, 1, 2, 3], [70, 71, 130],
             list(range(40)), list(range(20, 60)), [], list(range(segments))]
    at = b - firsts
    return kinds[at] if at < len(kinds) else sorted(int(x) for x in g.integers(0, segments, 5))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", ["few", "128", "256"])
@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
def test_pages_missing_anywhere(gpu, kind, rows, d):
    """Pages missing in a split's first tile, in the middle of a walk over pages that are all there, at a
    window's border, before the tiles with masks, and in these; in long splits."""
    cache_dtype, dtype = kind
    _say("missing", rows, kind, d)
    m, hq, hkv = {"few": (3, 32, 8), "128": (12, 64, 8), "256": (40, 16, 2)}[rows]
    batch, g = 40, np.random.default_rng(35)
    lengths = [int(x) for x in g.integers(2500, 2561, batch)]
    n_new = [m] * batch
    cache = _cache(cache_dtype, lengths, hkv, d, gpu, 36)
    names = [-1, cache.n_pages, -2 ** 31, 2 ** 31 - 1]
    table = cache.page_table.cpu().numpy().copy()
    for b, n in enumerate(lengths):
        for i in _gaps(b, -(-n // 16), g):
            table[b, i] = names[(b + i) % 4]
    cache.page_table.copy_(torch.from_numpy(table))
    q = _randn((m * batch, hq, d), dtype, gpu, 37)
    scale = 1.0 / np.sqrt(d)
    out = cache.attend(PH.chunk_of(C, n_new, gpu), q)
    _check(cache, n_new, q, out, scale)


# ------------------------------------------------------------------ infinities and NaN in V
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [12, 40], ids=["96rows", "320rows"])
@pytest.mark.parametrize("kind", KINDS, ids=KIND_IDS)
def test_values_that_are_not_finite_in_long_chunks(gpu, kind, m, d):
    """They reach the rows that see them and no other: keys that all rows see, keys among the chunk's own
    (both halves of a tile), keys behind the last one."""
    cache_dtype, dtype = kind
    _say("wild", m, kind, d)
    hq, hkv, n, batch = 16, 2, 2500, 24
    lengths = [n - 7 * b for b in range(batch)]
    cache = _cache(cache_dtype, lengths, hkv, d, gpu, 38)
    table = cache.page_table.cpu().numpy()
    for b, n in enumerate(lengths):
        first = n - m                                         # the chunk's first token
        for j, col, x in ((b * 90 + 5, 3, torch.inf), (b * 90 + 44, 3, -torch.inf if b % 2 else torch.inf),
                          (first + 1, d - 1, torch.inf), (first + m // 2, 33, -torch.inf),
                          (first + m // 2, d - 1, -torch.inf), (first + m - 2, 40, torch.nan)):
            page, slot = int(table[b, j // 16]), j % 16
            if cache_dtype == C.FP8:                          # a NaN code, or a block without values
                if np.isnan(x):
                    cache.v_scale[page, :, slot, col // 32] = 255
                else:
                    cache.v[page, :, slot, col] = 0xFF
            else:
                cache.v[page, :, slot, col] = x
    q = _randn((m * batch, hq, d), dtype, gpu, 39)
    out = cache.attend(PH.chunk_of(C, [m] * batch, gpu), q)
    _check(cache, [m] * batch, q, out, 1.0 / np.sqrt(d))
    assert torch.isfinite(out[0, :, 33:d - 1]).all()          # its row sees none of these


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m", [1, 12, 40], ids=["8rows", "96rows", "320rows"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_infinite_values_of_little_weight(gpu, dtype, m, d):
    """A visible infinity with a weight of 2^-100 of the row's largest, or more, is one in the output,
    wherever its key lies."""
    _say("little weight", dtype, m, d)
    batch, n, hq, hkv = 24, 2500, 16, 2
    lengths = [n - 3 * b for b in range(batch)]
    cache = _cache(dtype, lengths, hkv, d, gpu, 41)
    cache.k[..., 0] = 0.0
    table = cache.page_table.cpu().numpy()
    for b, n in enumerate(lengths):
        j = (3, n // 2, 110 * b, n - m, n - 1)[b % 5]
        page, slot = int(table[b, j // 16]), j % 16
        cache.k[page, :, slot] = 0.0
        cache.k[page, :, slot, 0] = -64.0
        cache.v[page, :, slot, 5] = torch.inf if b % 2 else -torch.inf
    q = _randn((m * batch, hq, d), dtype, gpu, 42) / 32
    q[..., 0] = 1.0
    # the largest other logit is below 69.3 - 64: 5 is 20 deviations of one, at d = 128 14
    out = cache.attend(PH.chunk_of(C, [m] * batch, gpu), q, scale=1.0)
    _check(cache, [m] * batch, q, out, 1.0)
    assert torch.isinf(out.reshape(batch, m, hq, d)[:, -1, :, 5]).all()

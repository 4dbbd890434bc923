"""The bounded cache on the GPU against the oracle: rows in and out (bit for bit),
attention with the slots' weights, eviction (the same slots, rows bit for bit)."""
import sys

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from paper_2606_24467_amd import compresskv as C
from tests import cache_helpers as H

pytestmark = pytest.mark.gpu

BF16, F32, FP4 = torch.bfloat16, torch.float32, C.FP4


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


def _rows(shape, dtype, seed, gpu, wild=False):
    g = np.random.default_rng(seed)
    x = g.standard_normal(shape).astype(np.float32)
    if wild:   # magnitudes over the whole range, zeros, exact ties, blocks of zeros
        x *= np.exp2(g.integers(-140, 127, shape[:-1] + (1,))).astype(np.float32)
        x[..., 0] = 0.0
        x[..., 1::7] = np.round(x[..., 1::7])
        x.reshape(-1, 32)[::5] = 0.0
        x.reshape(-1, 32)[1::11, 3] = -0.0
    return torch.from_numpy(x).to(gpu).to(dtype)


def _encoded(x):
    return CO.fp4_encode(H.values(x))


# --------------------------------------------------------------- load, read
@pytest.mark.parametrize("dtype,rows,d,n", [(FP4, BF16, 128, 77), (FP4, F32, 64, 33),
                                            (FP4, F32, 128, 64), (FP4, BF16, 64, 1),
                                            (BF16, BF16, 128, 50), (F32, F32, 64, 50)])
def test_load_and_read(gpu, dtype, rows, d, n):
    _say("load", dtype, rows, d, n)
    b, h, cap = 3, 2, n + 5
    cache = C.Cache.empty(b, h, cap, d, dtype, gpu)
    for t in (cache.pos, cache.length, cache.seen):
        t.fill_(-9)
    cache.weight.fill_(3.0)
    k, v = (_rows((b, h, n, d), rows, s, gpu, wild=dtype == FP4) for s in (1, 2))
    kept = np.minimum([n, max(1, n // 2), 0], n)
    idx = np.where(np.arange(n)[None, None] < kept[:, None, None],
                   3 * np.arange(n)[None, None] + np.arange(h)[None, :, None], -1).astype(np.int32)
    cu = torch.tensor([0, 400, 900, 907], dtype=torch.int32, device=gpu)
    before = H.state(cache)
    cache.load(k, v, torch.from_numpy(idx).to(gpu), cu)
    after = H.state(cache)
    assert (after["length"] == kept[:, None]).all()
    assert (after["seen"] == np.array([400, 500, 7])[:, None]).all()
    for i in range(b):
        m = kept[i]
        assert (after["pos"][i, :, :m] == idx[i, :, :m]).all() and not after["weight"][i, :, :m].any()
        for name, x in (("k", k), ("v", v)):
            if dtype == FP4:
                codes, scales = _encoded(x)
                assert (after[name][i, :, :m] == codes[i, :, :m]).all()
                assert (after[name + "_scale"][i, :, :m] == scales[i, :, :m]).all()
            else:
                assert (after[name][i, :, :m] == H.bits(x)[i, :, :m]).all()
        for name in after:
            if name not in ("length", "seen"):          # the other slots are left as they were
                assert (after[name][i, :, m:] == before[name][i, :, m:]).all(), name
    for out in ([BF16, F32] if dtype == FP4 else [rows]):
        got = cache.read(out)
        for name, x in zip("kv", got):
            want = H.rows_of(cache, name)
            for i in range(b):
                assert (H.values(x)[i, :, :kept[i]] == want[i, :, :kept[i]]).all()
                assert not H.bits(x)[i, :, kept[i]:].any()


def test_load_blocks_that_are_not_finite(gpu):
    x = _rows((1, 1, 6, 64), F32, 3, gpu)
    x[0, 0, 0, 5], x[0, 0, 1, 40], x[0, 0, 2, 0] = float("inf"), float("nan"), -float("inf")
    cache = C.Cache.empty(1, 1, 32, 64, FP4, gpu)
    idx = torch.arange(6, dtype=torch.int32, device=gpu).reshape(1, 1, 6)
    cache.load(x, x, idx, torch.tensor([0, 6], dtype=torch.int32, device=gpu))
    codes, scales = _encoded(x)
    assert (H.state(cache)["k"][0, 0, :6] == codes).all()
    assert (H.state(cache)["k_scale"][0, 0, :6] == scales).all()
    got = H.values(cache.read(F32)[0])[0, 0, :6]
    want = CO.fp4_decode(codes, scales)[0, 0]
    assert (np.isnan(got) == np.isnan(want)).all() and np.isnan(want).sum() == 3 * 32
    assert (got[~np.isnan(got)] == want[~np.isnan(want)]).all()


def test_load_of_ragged_groups(gpu):
    """Head-level budgets: every group has rows of its own number."""
    b, d, budgets = 2, 128, [5, 40, 17]
    total = sum(budgets)
    k, v = (_rows((b, total, d), BF16, s, gpu) for s in (4, 5))
    idx = np.concatenate([np.arange(n) for n in budgets])[None].repeat(b, 0).astype(np.int32)
    idx[1, 5 + 30:5 + 40] = -1                            # sequence 1, group 1 kept 30 of 40
    cu = torch.tensor([0, 100, 130], dtype=torch.int32, device=gpu)
    cache = C.Cache.empty(b, 3, 64, d, FP4, gpu)
    cache.load(k, v, torch.from_numpy(idx).to(gpu), cu, group_budgets=budgets)
    got = H.state(cache)
    assert got["length"].tolist() == [[5, 40, 17], [5, 30, 17]]
    codes, scales = _encoded(v)
    off = np.cumsum([0] + budgets)
    for i in range(b):
        for g in range(3):
            n = got["length"][i, g]
            assert (got["v"][i, g, :n] == codes[i, off[g]:off[g] + n]).all()
            assert (got["v_scale"][i, g, :n] == scales[i, off[g]:off[g] + n]).all()
            assert (got["pos"][i, g, :n] == np.arange(n)).all()


# ------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype,rows,d,n", [(FP4, BF16, 128, 1), (FP4, F32, 64, 3), (BF16, BF16, 64, 1),
                                            (F32, F32, 128, 2), (FP4, F32, 128, 200),
                                            (BF16, BF16, 128, 300)])
def test_append(gpu, dtype, rows, d, n):
    _say("append", dtype, rows, d, n)
    cap = 256 + 32
    lengths = np.array([[0, 7], [cap - 1, cap], [100, 31]], dtype=np.int32)
    cache = H.make_cache(C, dtype, lengths, cap, d, gpu, 6, past=50)
    kv = _rows((3, n, 2, 2, d), rows, 7, gpu)             # K and V of a token side by side
    k, v = kv[:, :, 0], kv[:, :, 1]
    before = H.state(cache)
    cache.append(k, v)
    after = H.state(cache)
    m = np.minimum(n, cap - lengths)
    assert (after["length"] == lengths + m).all() and (after["seen"] == before["seen"] + n).all()
    for i, g in np.ndindex(3, 2):
        a, e = lengths[i, g], lengths[i, g] + m[i, g]
        assert (after["pos"][i, g, a:e] == before["seen"][i, g] + np.arange(e - a)).all()
        assert not after["weight"][i, g, a:e].any()
        for name, x in (("k", k), ("v", v)):
            x = x[i, :e - a, g]
            if dtype == FP4:
                codes, scales = _encoded(x)
                assert (after[name][i, g, a:e] == codes).all()
                assert (after[name + "_scale"][i, g, a:e] == scales).all()
            else:
                assert (after[name][i, g, a:e] == H.bits(x)).all()
        for name in after:
            if name not in ("length", "seen"):
                assert (after[name][i, g, :a] == before[name][i, g, :a]).all(), name
                assert (after[name][i, g, e:] == before[name][i, g, e:]).all(), name


# ------------------------------------------------------------------ attend
ATTEND = [   # rows, queries, D, Hq, Hkv, n_q, capacity, lengths of (sequence, group)
    (FP4, BF16, 128, 8, 2, 1, 96, [[0, 1], [31, 32], [33, 96]]),
    (FP4, BF16, 128, 28, 4, 1, 1500, [[1500, 700, 999, 1]]),
    (FP4, F32, 128, 8, 2, 1, 300, [[300, 17], [64, 0]]),
    (FP4, F32, 64, 16, 1, 2, 200, [[200], [3], [129]]),
    (FP4, BF16, 64, 8, 8, 1, 130, [[130, 5, 64, 65, 1, 2, 100, 0]]),
    (FP4, BF16, 64, 32, 4, 3, 96, [[96, 2, 1, 33]]),
    (FP4, BF16, 128, 28, 4, 9, 160, [[160, 7, 100, 31]]),       # 63 rows
    (FP4, F32, 128, 32, 2, 4, 100, [[100, 41]]),                # 64 rows, two row blocks
    (BF16, BF16, 128, 8, 2, 1, 101, [[0, 1], [31, 101], [15, 16]]),
    (BF16, BF16, 64, 8, 2, 4, 77, [[77, 3]]),
    (BF16, BF16, 128, 28, 4, 4, 333, [[333, 100, 1, 2]]),
    (BF16, BF16, 128, 64, 1, 1, 50, [[50], [9]]),
    (F32, F32, 64, 8, 2, 1, 65, [[0, 1], [65, 17]]),
    (F32, F32, 128, 8, 2, 5, 203, [[203, 16]]),
    (F32, F32, 128, 32, 1, 2, 40, [[40]]),
    (BF16, BF16, 128, 8, 2, 1, 9000, [[9000, 4097]]),           # split over workgroups
    (FP4, BF16, 128, 4, 1, 2, 20000, [[20000]]),
]


def _check_attend(cache, q, before, out, accumulate, scale=None, bits=16):
    b, n_q, hq, d = q.shape
    hkv = cache.n_kv_heads
    rows = hq // hkv
    k, v, qv, o = H.rows_of(cache, "k"), H.rows_of(cache, "v"), H.values(q), H.values(out)
    c = 1.0 / np.sqrt(d) if scale is None else scale
    weight = cache.weight.cpu().numpy()
    for i, g in np.ndindex(b, hkv):
        n = int(before["length"][i, g])
        qg = qv[i, :, g * rows:(g + 1) * rows]
        kk, vv = k[i, g, :n], v[i, g, :n]
        want, got_w, p, sees = CO.attend(qg, kk, vv, before["pos"][i, g, :n], before["seen"][i, g], c)
        got = o[i, :, g * rows:(g + 1) * rows]
        finite = np.isfinite(want)
        assert (np.isnan(got) == np.isnan(want)).all(), (i, g)
        if n == 0:
            assert not got.any()
        dz = H.logit_error(qg, kk, c)
        if np.isfinite(kk).all() and np.isfinite(vv).all():
            tol = H.attention_tolerance(want, p, sees, dz, vv, q.dtype, H.p_part(q.dtype, bits))
            assert (np.abs(got - want) <= tol).all(), (i, g, np.max(np.abs(got - want) / tol))
        else:   # rows that see a row which is not finite are compared by kind alone
            assert (got[~finite & ~np.isnan(want)] == want[~finite & ~np.isnan(want)]).all()
        old = before["weight"][i, g].view(np.float32)
        if accumulate:
            w0, w1 = old[:n].astype(np.float64), weight[i, g, :n].astype(np.float64)
            err = 2 * np.where(sees, dz, 0).max(-1, initial=0)[..., None] + 2 * n * H.U + 2.0 ** -22
            tol = (p * err).sum((0, 1)) + H.U * (n_q * rows * got_w + np.abs(w0 + got_w))
            ok = np.isfinite(w0 + got_w)
            assert (np.abs(w1 - w0 - got_w) <= tol + 1e-30)[ok].all(), (i, g)
            assert (weight[i, g, n:].view(np.int32) == before["weight"][i, g, n:]).all()
        else:
            assert (weight[i, g].view(np.int32) == before["weight"][i, g]).all()


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[3]}-{c[4]}-{c[5]}-{c[6]}")
@pytest.mark.parametrize("accumulate", [False, True])
def test_attend(gpu, case, accumulate):
    dtype, qt, d, hq, hkv, n_q, cap, lengths = case
    _say("attend", case, accumulate)
    cache = H.make_cache(C, dtype, lengths, cap, d, gpu, 8, past=1000)
    q = _rows((len(lengths), n_q, hq, d), qt, 9, gpu)
    before = H.state(cache)
    out = cache.attend(q, accumulate=accumulate)
    _check_attend(cache, q, before, out, accumulate)
    after = H.state(cache)
    for name in after:
        if name != "weight":
            assert (after[name] == before[name]).all(), name
    again = cache.attend(q)                               # the same bits each time
    assert (H.bits(again) == H.bits(out)).all()


def test_attend_scale_and_large_logits(gpu):
    cache = H.make_cache(C, BF16, [[500, 64]], 500, 64, gpu, 10)
    q = _rows((1, 1, 8, 64), BF16, 11, gpu)
    for scale in (0.02, 1.7):
        before = H.state(cache)
        _check_attend(cache, q, before, cache.attend(q, scale=scale), False, scale)
    q *= 30.0                                             # one key takes nearly everything
    before = H.state(cache)
    _check_attend(cache, q, before, cache.attend(q, accumulate=True), True)


@pytest.mark.parametrize("dtype,qt", [(FP4, BF16), (FP4, F32), (BF16, BF16), (F32, F32)])
def test_attend_tokens_that_see_nothing_or_rubbish(gpu, dtype, qt):
    """Of three query tokens the first sees no slot; slots that only later tokens see hold
    rows that are not finite."""
    cache = H.make_cache(C, dtype, [[40, 40]], 64, 64, gpu, 12, shuffled=False)
    pos = torch.arange(40, dtype=torch.int32, device=gpu) + 100
    cache.pos[:, :, :40] = pos
    cache.seen[0, 0], cache.seen[0, 1] = 102, 141   # tokens at 99, 100, 101; at 138, 139, 140
    for g, slot in ((0, 1), (1, 39)):               # position 101: seen by token 2; 139: by 1 and 2
        if dtype == FP4:
            cache.v_scale[0, g, slot, 1] = 255
        else:
            cache.v[0, g, slot, 5] = float("inf")
            cache.v[0, g, slot, 40] = -float("inf")
            cache.v[0, g, slot, 41] = float("nan")
    q = _rows((1, 3, 4, 64), qt, 13, gpu)
    before = H.state(cache)
    out = cache.attend(q, accumulate=True)
    _check_attend(cache, q, before, out, True)
    got = H.values(out)
    assert not got[0, 0, :2].any() and np.isfinite(got[0, 1, :2]).all()
    assert np.isfinite(got[0, 0, 2:]).all()
    assert not np.isfinite(got[0, 2]).all() and not np.isfinite(got[0, 1, 2:]).all()
    # a key that is not finite: NaN for the tokens that see it, nothing for the others
    if dtype == FP4:
        cache.k_scale[0, 0, 1] = 255
        cache.v_scale[0, 0, 1] = 127
    else:
        cache.k[0, 0, 1] = float("nan")
        cache.v[0, 0, 1] = 0.5
    got = H.values(cache.attend(q))
    assert not got[0, 0, :2].any() and np.isfinite(got[0, 1, :2]).all()
    assert np.isnan(got[0, 2, :2]).all()


def test_attend_lengths_out_of_range(gpu):
    """A length beyond the capacity counts as the capacity, a negative one as none."""
    cache = H.make_cache(C, FP4, [[64, 64]], 64, 128, gpu, 14)
    q = _rows((1, 1, 4, 128), BF16, 15, gpu)
    want = cache.attend(q)
    cache.length[0, 0], cache.length[0, 1] = 1000, -5
    got = cache.attend(q, accumulate=True)
    assert (H.bits(got[:, :, :2]) == H.bits(want[:, :, :2])).all()
    assert not H.bits(got[:, :, 2:]).any()
    cache.append(_rows((1, 1, 2, 128), BF16, 16, gpu), _rows((1, 1, 2, 128), BF16, 17, gpu))
    assert cache.length.tolist() == [[64, 1]]


# ------------------------------------------------------------------- evict
def _evict_oracle(state, budget, sinks, recent):
    want = {n: x.copy() for n, x in state.items()}
    for i, g in np.ndindex(state["length"].shape):
        moves, n = CO.evict(state["weight"][i, g].view(np.float32), state["pos"][i, g],
                            min(max(int(state["length"][i, g]), 0), state["pos"].shape[2]),
                            int(state["seen"][i, g]), budget, sinks, recent)
        want["length"][i, g] = min(state["length"][i, g], n)
        for to, src in moves:
            for name in want:
                if name not in ("length", "seen"):
                    want[name][i, g, to] = state[name][i, g, src]
    return want


EVICT = [   # rows, D, capacity, lengths, budget, sinks, recent
    (FP4, 128, 96, [[0, 1], [64, 65], [66, 96]], 64, 4, 8),
    (BF16, 128, 50, [[50, 49], [10, 11]], 10, 0, 0),
    (F32, 64, 33, [[33, 2]], 1, 0, 1),
    (FP4, 64, 2048, [[2048, 1025, 1024, 2000]], 1000, 4, 64),
    (BF16, 64, 5000, [[5000, 4097]], 4096, 1, 100),
    (F32, 128, 300, [[300, 299]], 299, 4, 298),
    (BF16, 64, 20000, [[20000, 15001]], 2500, 4, 32),
    (FP4, 128, 160, [[160, 150]], 20, 30, 40),        # fewer slots than are held
]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[4]}-{c[5]}-{c[6]}")
@pytest.mark.parametrize("weights", ["random", "ties", "special"])
def test_evict(gpu, case, weights):
    dtype, d, cap, lengths, budget, sinks, recent = case
    _say("evict", case, weights)
    cache = H.make_cache(C, dtype, lengths, cap, d, gpu, 18, past=3)
    g = torch.Generator(device=gpu).manual_seed(19)
    if weights == "ties":
        cache.weight.copy_(torch.randint(0, 3, cache.weight.shape, generator=g, device=gpu) / 2)
    elif weights == "special":
        pick = torch.randint(0, 8, cache.weight.shape, generator=g, device=gpu)
        table = torch.tensor([0.0, -0.0, 1e-40, float("inf"), float("nan"), -1.0, 3e38, 0.5], device=gpu)
        cache.weight.copy_(table[pick])
    before = H.state(cache)
    cache.evict(budget, n_sinks=sinks, n_recent=recent)
    want, got = _evict_oracle(before, budget, sinks, recent), H.state(cache)
    for name in want:
        assert (got[name] == want[name]).all(), name


def test_evict_of_a_budget_of_the_capacity(gpu):
    cache = H.make_cache(C, BF16, [[40]], 40, 64, gpu, 20)
    before = H.state(cache)
    cache.evict(40)
    cache.evict(39)
    cache.evict(40)
    after = H.state(cache)
    assert after["length"].tolist() == [[39]]
    assert _evict_oracle(before, 39, 0, 0)["pos"].tolist() == after["pos"].tolist()

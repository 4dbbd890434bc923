"""Sizes and calls at the edges: offsets past 32 bits, evictions over more slots than are held
in shared memory, windows split over workgroups, calls without queries or keys, inputs
that the caller lets go of while another stream still reads them."""
import sys

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from paper_2606_24467_amd import compresskv as C
from tests import cache_helpers as H
from tests.test_gpu_cache import _check_attend, _evict_oracle, _rows
from tests.test_gpu_window import _check, _inputs

pytestmark = pytest.mark.gpu

BF16, F32, FP4 = torch.bfloat16, torch.float32, C.FP4


def _say(*a):
    print(*a, file=sys.stderr, flush=True)


EVICT = [   # rows, D, capacity, lengths, budget, sinks, recent
    (BF16, 64, 40001, [[40001, 39990]], 39985, 4, 64),          # 16 and 5 slots go
    (BF16, 64, 40001, [[40001, 40000]], 40000, 0, 7),           # one
    (FP4, 64, 40032, [[40032, 2]], 3001, 4, 64),                # most of them
    (BF16, 64, 37003, [[37003, 37000]], 36700, 1, 0),           # more than are ranked
    (F32, 64, 3, [[3, 2]], 2, 0, 0),
    (BF16, 128, 5, [[5, 4], [1, 0]], 1, 0, 0),
    (BF16, 64, 1027, [[1027, 1025]], 1024, 0, 1),
    (BF16, 64, 8193, [[8193]], 8100, 0, 0),
]


@pytest.mark.parametrize("case", EVICT, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}-{c[4]}")
@pytest.mark.parametrize("weights", ["random", "ties", "alike"])
def test_evict(gpu, case, weights):
    dtype, d, cap, lengths, budget, sinks, recent = case
    _say("evict", case, weights)
    cache = H.make_cache(C, dtype, lengths, cap, d, gpu, 50, past=3)
    g = torch.Generator(device=gpu).manual_seed(51)
    if weights == "ties":
        cache.weight.copy_(torch.randint(0, 40, cache.weight.shape, generator=g, device=gpu) / 4)
    elif weights == "alike":
        cache.weight.fill_(0.25)
    before = H.state(cache)
    cache.evict(budget, n_sinks=sinks, n_recent=recent)
    want, got = _evict_oracle(before, budget, sinks, recent), H.state(cache)
    for name in want:
        assert (got[name] == want[name]).all(), name


@pytest.mark.parametrize("dtype,hkv", [(FP4, 5), (F32, 1)], ids=["fp4", "f32"])
def test_cache_of_the_largest_capacity(gpu, dtype, hkv):
    """2^24 slots: rows past 2^32 bytes are appended, attended over, moved."""
    cap, d = 1 << 24, 128
    _say("largest", dtype, hkv)
    cache = C.Cache.empty(1, hkv, cap, d, dtype, gpu)
    cache.length.fill_(cap - 2)
    cache.seen.fill_(cap - 2)
    cache.pos.copy_(torch.arange(cap, dtype=torch.int32, device=gpu))
    cache.weight.copy_(torch.arange(cap, dtype=torch.float32, device=gpu))
    cache.weight[:, :, 5] = -1.0
    rng = np.random.default_rng(52)
    row_t = BF16 if dtype == FP4 else dtype
    # values of the 4-bit format, with a 6 in every block
    values = rng.choice([-6.0, -4, -3, -2, -1.5, -1, -0.5, 0.5, 1, 1.5, 2, 3, 4, 6], (2, hkv, d))
    values[..., ::32] = 6.0
    k_new, v_new = (torch.tensor(x, dtype=row_t, device=gpu)[None, None] for x in values)
    # the logit of the new row is near 60, of all others (rows of zeros) 0: what they add to a
    # sum of 1 is 2^24 e^-55 at most, far below half a step of fp32
    q = k_new.float() * (60.0 / (k_new.float() ** 2).sum(-1, keepdim=True))
    q = q.to(row_t)
    cache.append(k_new, v_new)
    slot = cap - 2
    tol = (H.half_step(row_t) + 2.0 ** -15) * H.values(v_new.abs())

    def attend(accumulate):
        out = cache.attend(q, scale=1.0, accumulate=accumulate)
        assert (np.abs(H.values(out) - H.values(v_new)) <= tol).all()
    attend(True)
    got = cache.weight[0, :, slot].cpu().numpy()
    assert (np.abs(got - 1.0) <= 2.0 ** -15).all()
    assert cache.length.tolist() == [[cap - 1] * hkv]
    cache.weight[:, :, slot] = float(cap)
    moved = [x[0, :, slot].clone() for x in (cache.k, cache.v, cache.pos)]
    cache.evict(cap - 2)
    for x, y in zip((cache.k, cache.v, cache.pos), moved):
        assert torch.equal(x[0, :, 5], y)
    assert cache.length.tolist() == [[cap - 2] * hkv]
    attend(False)


def test_load_and_read_of_the_largest_capacity(gpu):
    cap, d = 1 << 24, 128
    rows = torch.zeros((1, 1, cap, d), device=gpu)
    rng = np.random.default_rng(53)
    last = torch.tensor(rng.standard_normal((300, d)), dtype=F32, device=gpu)
    rows[0, 0, -300:] = last
    idx = torch.arange(cap, dtype=torch.int32, device=gpu)[None, None]
    cache = C.Cache.empty(1, 1, cap, d, FP4, gpu)
    cache.load(rows, rows, idx, torch.tensor([0, cap + 9], dtype=torch.int32, device=gpu))
    codes, scales = CO.fp4_encode(H.values(last))
    assert (cache.k[0, 0, -300:].cpu().numpy() == codes).all()
    assert (cache.v_scale[0, 0, -300:].cpu().numpy() == scales).all()
    assert cache.length.tolist() == [[cap]] and cache.seen.tolist() == [[cap + 9]]
    k, v = cache.read(F32)
    want = CO.fp4_decode(codes, scales)
    for x in (k, v):
        assert (H.values(x[0, 0, -300:]) == want).all()
        assert not x[0, 0, : 1 << 20].any() and not x[0, 0, -(1 << 20):-300].any()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_window_over_keys_past_32_bits(gpu, dtype):
    """The last keys of 2^24 and some: the same bits as over those keys alone."""
    n, near = (1 << 24) + 5000, 6000
    kv = torch.zeros((n, 1, 128), dtype=dtype, device=gpu)
    g = torch.Generator(device=gpu).manual_seed(54)
    kv[-near + 4:] = torch.randn((near - 4, 1, 128), generator=g, device=gpu).to(dtype)
    for lq in (1, 3, 100):
        q = torch.randn((lq, 4, 128), generator=g, device=gpu).to(dtype)
        cu_q = torch.tensor([0, lq], dtype=torch.int32, device=gpu)
        out = []
        for k in (kv, kv[-near:]):
            cu_k = torch.tensor([0, k.shape[0]], dtype=torch.int32, device=gpu)
            p = C.WindowProblem(q, k, k, cu_q, cu_k, window=1000, n_sinks=4)
            out.append(C.window_attention(p, q, k, k))
        assert (H.bits(out[0]) == H.bits(out[1])).all(), lq


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lq,lk,window,sinks", [(70, 5000, 1 << 30, 0), (1, 9000, 8000, 3),
                                                (5, 4000, 3000, 700), (20, 3001, 2900, 4)])
def test_windows_split_over_workgroups(gpu, dtype, lq, lk, window, sinks):
    spans = [(lq, lk), (1, 40)]
    q, k, v, cu_q, cu_k = _inputs(spans, 8, 2, 128, dtype, gpu, 55)
    v[lk - 9, :, 3] = float("inf")                            # the last tokens see it
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=window, n_sinks=sinks)
    _check(q, k, v, spans, window, sinks, C.window_attention(p, q, k, v))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_window_without_queries_or_without_keys(gpu, dtype):
    q, kv = (torch.randn((9, h, 64), device=gpu).to(dtype) for h in (8, 2))
    cu = [torch.tensor(x, dtype=torch.int32, device=gpu) for x in ([0, 0, 0], [0, 4, 9])]
    none = q[:0]
    p = C.WindowProblem(none, kv, kv, cu[0], cu[1], window=4)
    assert C.window_attention(p, none, kv, kv).shape == (0, 8, 64)
    p = C.WindowProblem(q, kv, kv, cu[0], cu[1], window=4)      # rows of none of the sequences
    out = torch.full_like(q, 7.0)
    C.window_attention(p, q, kv, kv, out=out)
    assert (out == 7.0).all()
    p = C.WindowProblem(q, kv[:0], kv[:0], cu[1], cu[0], window=4)
    assert not C.window_attention(p, q, kv[:0], kv[:0]).any()
    many = torch.randn((300, 8, 64), device=gpu).to(dtype)
    cu_m = torch.tensor([0, 1, 300], dtype=torch.int32, device=gpu)
    p = C.WindowProblem(many, kv[:0], kv[:0], cu_m, cu[0], window=4)
    assert not C.window_attention(p, many, kv[:0], kv[:0]).any()


def test_inputs_let_go_while_another_stream_reads_them(gpu):
    """A call on a given stream keeps its inputs' memory until that stream has used it."""
    side = torch.cuda.Stream(gpu)
    q0 = torch.randn((4, 1, 8, 128), device=gpu).to(BF16)
    cache = H.make_cache(C, BF16, [[60, 40]] * 4, 64, 128, gpu, 56)
    new0 = torch.randn((4, 1, 2, 128), device=gpu).to(BF16)
    twin = H.make_cache(C, BF16, [[60, 40]] * 4, 64, 128, gpu, 56)
    twin.append(new0, new0)
    want = twin.attend(q0)
    wq = torch.randn((500, 8, 128), device=gpu).to(BF16)
    kv0 = torch.randn((500, 2, 128), device=gpu).to(BF16)
    cu = torch.tensor([0, 500], dtype=torch.int32, device=gpu)
    p = C.WindowProblem(wq, kv0, kv0, cu, cu, window=100)
    want_w = C.window_attention(p, wq, kv0, kv0)
    big = torch.randn((4096, 4096), device=gpu)
    torch.cuda.synchronize()
    q, new, kv = q0.clone(), new0.clone(), kv0.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = big
        for _ in range(20):
            x = (x @ big) * 1e-2                             # some ms of other work first
    cache.append(new, new, stream=side)
    out = cache.attend(q, stream=side)
    out_w = C.window_attention(p, wq, kv, kv, stream=side)
    shapes = [t.shape for t in (q, new, kv)]
    del q, new, kv
    keep = [torch.full(s, 9.0, dtype=BF16, device=gpu) for s in shapes for _ in range(4)]
    torch.cuda.synchronize()
    assert (H.bits(out) == H.bits(want)).all()
    assert (H.bits(out_w) == H.bits(want_w)).all()
    assert keep[0].shape == shapes[0]


def test_workspaces_elsewhere_are_refused(gpu):
    cache = H.make_cache(C, BF16, [[40]], 64, 128, gpu, 57)
    host = torch.empty(1 << 20, dtype=torch.uint8)
    q = torch.zeros((1, 1, 2, 128), dtype=BF16, device=gpu)
    kv, cu = torch.zeros((9, 2, 128), dtype=BF16, device=gpu), torch.tensor([0, 9], dtype=torch.int32,
                                                                             device=gpu)
    p = C.WindowProblem(kv, kv, kv, cu, cu, window=4)
    for call in (lambda: cache.attend(q, ws=host), lambda: cache.evict(8, ws=host),
                 lambda: C.window_attention(p, kv, kv, kv, ws=host),
                 lambda: cache.attend(q, ws=torch.empty(1 << 20, dtype=torch.uint8, device=gpu)[::2])):
        with pytest.raises(ValueError, match="ws"):
            call()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lq", [1, 2, 5, 16])
@pytest.mark.parametrize("lk,window", [(40, 1 << 30), (700, 500), (4000, 3000)])
def test_every_kernel_of_windows(gpu, dtype, d, lq, lk, window):
    """Each number of row tiles, in one workgroup and split, with the rows of a tile on both
    sides of the window's ends and of the diagonal."""
    spans = [(lq, lk), (1, 33)]
    q, k, v, cu_q, cu_k = _inputs(spans, 8, 2, d, dtype, gpu, 60)
    for sinks in (0, 70):
        p = C.WindowProblem(q, k, v, cu_q, cu_k, window=window, n_sinks=sinks)
        _check(q, k, v, spans, window, sinks, C.window_attention(p, q, k, v))


@pytest.mark.parametrize("dtype,qt", [(FP4, BF16), (FP4, F32), (BF16, BF16), (F32, F32)],
                         ids=["fp4-bf16", "fp4-f32", "bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q", [1, 2, 5, 16])
@pytest.mark.parametrize("cap", [96, 4512])
def test_every_kernel_of_the_cache(gpu, dtype, qt, d, n_q, cap):
    lengths = [[cap, cap - 31], [cap // 2 + 1, 33]]
    cache = H.make_cache(C, dtype, lengths, cap, d, gpu, 61, past=1000)
    q = _rows((2, n_q, 8, d), qt, 62, gpu)
    before = H.state(cache)
    out = cache.attend(q, accumulate=True)
    _check_attend(cache, q, before, out, True)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("cap", [80, 5000])
def test_infinities_that_a_row_sees(gpu, dtype, cap):
    """They reach its output as infinities, or as NaN where both signs meet."""
    cache = H.make_cache(C, dtype, [[cap, cap - 1]], cap, 128, gpu, 63)
    cache.v[0, :, 7, 3] = float("inf")
    cache.v[0, :, 21, 9] = -float("inf")
    cache.v[0, :, 40, 9] = float("inf")
    q = _rows((1, 1, 8, 128), dtype, 64, gpu)
    out = H.values(cache.attend(q))[0, 0]
    assert (out[:, 3] == np.inf).all() and np.isnan(out[:, 9]).all()
    others = np.delete(out, (3, 9), axis=1)
    assert np.isfinite(others).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_windows_over_rows_far_apart(gpu, dtype):
    """More than 2^24 bytes from one key to the next."""
    spans = [(20, 70), (1, 9)]
    q, k, v, cu_q, cu_k = _inputs(spans, 4, 1, 128, dtype, gpu, 70)
    far = torch.zeros((k.shape[0], (1 << 23) + 64), dtype=dtype, device=gpu)
    far[:, 64:192], far[:, -128:] = k[:, 0], v[:, 0]
    kf, vf = far[:, 64:192].unsqueeze(1), far[:, -128:].unsqueeze(1)
    for sinks in (0, 5):
        p = C.WindowProblem(q, kf, vf, cu_q, cu_k, window=30, n_sinks=sinks)
        _check(q, kf, vf, spans, 30, sinks, C.window_attention(p, q, kf, vf))


@pytest.mark.parametrize("budget", [2030, 2098])
def test_evict_of_many_groups(gpu, budget):
    """More groups than CUs, of more slots than few groups have for the small workgroups."""
    lengths = [[2100 - (i % 7)] for i in range(300)]
    cache = H.make_cache(C, BF16, lengths, 2100, 64, gpu, 71)
    before = H.state(cache)
    cache.evict(budget, n_sinks=4, n_recent=32)
    want, got = _evict_oracle(before, budget, 4, 32), H.state(cache)
    for name in want:
        assert (got[name] == want[name]).all(), name


@pytest.mark.parametrize("dtype,qt", [(FP4, BF16), (FP4, F32), (BF16, BF16), (F32, F32)],
                         ids=["fp4-bf16", "fp4-f32", "bf16", "f32"])
@pytest.mark.parametrize("cap", [96, 5024])
def test_a_row_that_is_not_a_number_gives_nothing_to_slots_it_does_not_see(gpu, dtype, qt, cap):
    """Of three query tokens the first holds a NaN: it reaches the weights of the slots that the
    token sees; those of the later tokens get what the later tokens give them."""
    lengths = [[cap, cap - 33]]
    cache = H.make_cache(C, dtype, lengths, cap, 128, gpu, 64, past=1000)
    q = _rows((1, 3, 8, 128), qt, 65, gpu)
    q[0, 0, 1, 5] = float("nan")                              # a head of the first group
    before = H.state(cache)
    out = cache.attend(q, accumulate=True)
    k, v, qv = H.rows_of(cache, "k"), H.rows_of(cache, "v"), H.values(q)
    weight = cache.weight.cpu().numpy().astype(np.float64)
    for g in range(2):
        n, seen = lengths[0][g], before["seen"][0, g]
        pos = before["pos"][0, g, :n]
        qg = qv[0, :, 4 * g:4 * g + 4]
        _, want, p, sees = CO.attend(qg, k[0, g, :n], v[0, g, :n], pos, seen)
        assert np.isnan(want).sum() == (0 if g else n - 2)    # two slots are later tokens'
        assert (np.isnan(weight[0, g, :n]) == np.isnan(want)).all()
        fine = ~np.isnan(want)
        old = before["weight"][0, g].view(np.float32)[:n].astype(np.float64)
        with np.errstate(invalid="ignore"):
            dz = H.logit_error(qg, k[0, g, :n], 128 ** -0.5)
            p, dz = np.where(np.isnan(p), 0.0, p), np.where(np.isnan(dz), 0.0, dz)
        err = 2 * np.where(sees, dz, 0).max(-1, initial=0)[..., None] + 2 * n * H.U + 2.0 ** -22
        tol = (p * err).sum((0, 1)) + H.U * (12 * np.nan_to_num(want) + old + np.nan_to_num(want))
        assert (np.abs(weight[0, g, :n] - old - want) <= tol + 1e-30)[fine].all(), g
    assert np.isnan(H.values(out)[0, 0, 1]).all() and np.isfinite(H.values(out)[0, 1:]).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n_q", [1, 2])
@pytest.mark.parametrize("cap", [80, 5000])
def test_slots_of_logits_of_minus_infinity(gpu, dtype, n_q, cap):
    """They receive nothing; where there are no others, the row gives zeros."""
    cache = H.make_cache(C, dtype, [[cap, cap]], cap, 64, gpu, 66)
    q = _rows((1, n_q, 4, 64), dtype, 67, gpu)
    q[..., 0] = 1.0
    cache.k[0, 0, :, 0] = -float("inf")
    cache.k[0, 1, :cap - 9, 0] = -float("inf")
    before = cache.weight.clone()
    out = H.values(cache.attend(q, accumulate=True))
    assert not out[0, :, :2].any() and (out[0, :, 2:] != 0).all()
    assert (cache.weight[0, 0] == before[0, 0]).all()
    assert (cache.weight[0, 1, :cap - 9] == before[0, 1, :cap - 9]).all()
    received = (cache.weight - before)[0, 1, cap - 9:].double().sum().item()
    assert abs(received - 2 * n_q) <= 2 * n_q * 9 * 2.0 ** -22   # 9 weights below 4, rounded


def test_the_most_groups_that_a_call_takes(gpu):
    """65535 groups: a few of them give what they give in a small cache."""
    n, cap, d = 65535, 32, 64
    g = torch.Generator(device=gpu).manual_seed(68)
    cache = C.Cache.empty(n, 1, cap, d, BF16, gpu)
    cache.length.copy_(torch.randint(0, cap, (n, 1), generator=g, device=gpu))
    cache.seen.copy_(cache.length)
    cache.pos.copy_(torch.arange(cap, dtype=torch.int32, device=gpu).expand(n, 1, cap))
    cache.weight.copy_(torch.rand((n, 1, cap), generator=g, device=gpu))
    for t in (cache.k, cache.v):
        t.copy_(torch.randn(t.shape, generator=g, device=gpu))
    q = torch.randn((n, 1, 4, d), generator=g, device=gpu).to(BF16)
    new = torch.randn((n, 1, 1, d), generator=g, device=gpu).to(BF16)
    some = torch.tensor([0, 1, 255, 256, 32767, 32768, 65533, 65534], device=gpu)
    small = C.Cache.empty(len(some), 1, cap, d, BF16, gpu)
    for a, b in zip(small._tensors(), cache._tensors()):
        if a is not None:
            a.copy_(b[some])

    def steps(cache, q, new):
        cache.append(new, new)
        out = cache.attend(q, accumulate=True)
        cache.evict(20, n_sinks=2, n_recent=4)
        return out, cache.read()[0]
    for got, want in zip(steps(cache, q, new), steps(small, q[some], new[some])):
        assert (H.bits(got[some]) == H.bits(want)).all()
    assert (H.bits(cache.weight[some]) == H.bits(small.weight)).all()
    assert int(cache.length.max()) == 20

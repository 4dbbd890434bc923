"""Windowed attention with sinks on the GPU against the oracle."""
import sys

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from paper_2606_24467_amd import compresskv as C
from tests import cache_helpers as H

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def _inputs(spans, hq, hkv, d, dtype, gpu, seed, layout="kv"):
    """q, k, v of packed sequences with (queries, keys) each; K and V interleaved."""
    g = torch.Generator(device=gpu).manual_seed(seed)
    tq, tk = (sum(s[i] for s in spans) for i in (0, 1))
    q = torch.randn((tq + 3, hq, d), generator=g, device=gpu).to(dtype)   # rows past the end
    kv = torch.randn((tk + 2, 2, hkv, d), generator=g, device=gpu).to(dtype)
    k, v = kv[:, 0], kv[:, 1]
    if layout == "heads":     # [heads, tokens, D] seen as [tokens, heads, D]
        q, k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    k[tk:], v[tk:] = float("nan"), float("nan")
    cu = [torch.tensor(np.cumsum([0] + [s[i] for s in spans]), dtype=torch.int32, device=gpu)
          for i in (0, 1)]
    return q, k, v, cu[0], cu[1]


def _check(q, k, v, spans, window, sinks, out, scale=None, bits=8):
    d, hq, hkv = q.shape[2], q.shape[1], k.shape[1]
    c = 1.0 / np.sqrt(d) if scale is None else scale
    q0 = k0 = 0
    o, qv, kv, vv = (H.values(x) for x in (out, q, k, v))
    for lq, lk in spans:
        t = lk - lq + np.arange(lq)[:, None]
        j = np.arange(lk)[None, :]
        sees = (j <= t) & ((j > t - window) | (j < sinks))
        want = CO.window_attention(qv[q0:q0 + lq], kv[k0:k0 + lk], vv[k0:k0 + lk], window, sinks, c)
        for h in range(hq):
            g = h // (hq // hkv)
            kk, vg = kv[k0:k0 + lk, g], vv[k0:k0 + lk, g]
            got, w = o[q0:q0 + lq, h], want[:, h]
            assert (np.isnan(got) == np.isnan(w)).all()
            with np.errstate(invalid="ignore"):
                p = CO._softmax_rows(c * (qv[q0:q0 + lq, h] @ kk.T), sees)
                dz = H.logit_error(qv[q0:q0 + lq, h], kk, c)
                tol = H.attention_tolerance(w, p, sees, dz, vg, q.dtype, H.p_part(q.dtype, bits))
            fine = np.isfinite(w)
            assert (np.abs(got - w) <= tol)[fine].all(), (lq, lk, h, np.nanmax(np.abs(got - w) / tol))
            assert (got[~fine & ~np.isnan(w)] == w[~fine & ~np.isnan(w)]).all()
        q0, k0 = q0 + lq, k0 + lk


CASES = [   # spans (queries, keys), Hq, Hkv, D, window, sinks
    ([(1, 1), (1, 33), (1, 700)], 8, 2, 128, 64, 4),
    ([(1, 5), (1, 2000)], 28, 4, 128, 1 << 30, 0),
    ([(1, 900)], 16, 1, 64, 100, 130),
    ([(3, 70), (16, 16), (2, 300)], 8, 2, 64, 50, 4),
    ([(130, 130), (65, 200), (0, 40), (1, 1)], 8, 2, 128, 33, 4),
    ([(257, 257)], 28, 4, 128, 1, 0),
    ([(257, 300)], 28, 4, 128, 1, 2),
    ([(128, 128), (64, 64)], 8, 8, 64, 16, 0),
    ([(200, 200)], 16, 1, 128, 77, 100),
    ([(300, 300)], 4, 2, 128, 4096, 0),
    ([(40, 25), (5, 0), (20, 20)], 8, 2, 128, 7, 3),          # more queries than keys
    ([(511, 1030)], 8, 2, 128, 256, 64),
    ([(333, 333)], 6, 2, 64, 128, 16),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0][0]}x{len(c[0])}-{c[1]}-{c[2]}-{c[3]}-{c[4]}-{c[5]}")
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_window_attention(gpu, case, dtype):
    spans, hq, hkv, d, window, sinks = case
    print("window", case, dtype, file=sys.stderr, flush=True)
    q, k, v, cu_q, cu_k = _inputs(spans, hq, hkv, d, dtype, gpu, 1)
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=window, n_sinks=sinks)
    out = torch.full_like(q, 7.0)
    C.window_attention(p, q, k, v, out=out)
    n = sum(s[0] for s in spans)
    _check(q, k, v, spans, window, sinks, out)
    assert (out[n:] == 7.0).all()                             # rows past the last sequence
    again = C.window_attention(p, q, k, v)
    assert (H.bits(again[:n]) == H.bits(out[:n])).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_window_attention_strides_and_scale(gpu, dtype):
    spans = [(150, 150), (20, 90)]
    q, k, v, cu_q, cu_k = _inputs(spans, 8, 2, 64, dtype, gpu, 2, layout="heads")
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=40, n_sinks=4, scale=0.3)
    _check(q, k, v, spans, 40, 4, C.window_attention(p, q, k, v), scale=0.3)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_keys_that_a_query_does_not_see_may_hold_anything(gpu, dtype):
    """Infinities and NaN in K and V reach the queries that see them and no other."""
    spans = [(300, 300), (1, 500)]
    q, k, v, cu_q, cu_k = _inputs(spans, 8, 2, 128, dtype, gpu, 3)
    for j, x in ((5, float("inf")), (100, float("nan")), (177, -float("inf")), (299, float("nan")),
                 (310, float("inf")), (480, float("nan"))):
        v[j, :, 17] = x
    v[178, :, 17] = float("inf")
    k[40] = float("nan")
    k[400] = float("inf")
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=16, n_sinks=4)
    out = C.window_attention(p, q, k, v)
    _check(q, k, v, spans, 16, 4, out)
    assert torch.isfinite(out[300]).all()


def test_a_long_sequence_in_pieces(gpu):
    """Chunks of a prompt and single tokens give what the whole prompt gives."""
    n, window = 1000, 200
    q, k, v, cu, _ = _inputs([(n, n)], 8, 2, 128, BF16, gpu, 4)
    p = C.WindowProblem(q, k, v, cu, cu, window=window, n_sinks=4)
    whole = H.values(C.window_attention(p, q, k, v))
    for a, e in ((0, 130), (130, 999), (999, 1000), (500, 501)):
        qq, kk, vv = q[a:e], k[:e], v[:e]
        cu_q = torch.tensor([0, e - a], dtype=torch.int32, device=gpu)
        cu_k = torch.tensor([0, e], dtype=torch.int32, device=gpu)
        p = C.WindowProblem(qq, kk, vv, cu_q, cu_k, window=window, n_sinks=4)
        got = H.values(C.window_attention(p, qq, kk, vv))
        # both are off by at most half a step of bf16 in the output and in each probability
        size = np.abs(H.values(v[:n])).max()
        assert np.abs(got - whole[a:e]).max() <= 4 * 2.0 ** -8 * size


def test_window_attention_of_many_sequences(gpu):
    """More sequences than a wave looks at together, some of them empty, in the kernel for many rows."""
    rng = np.random.default_rng(11)
    spans = [(int(x), int(x + y)) for x, y in zip(rng.integers(0, 40, 150), rng.integers(0, 30, 150))]
    spans[0] = spans[64] = spans[149] = (0, 7)
    spans[63], spans[128] = (33, 33), (70, 90)
    q, k, v, cu_q, cu_k = _inputs(spans, 4, 1, 64, BF16, gpu, 12)
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=20, n_sinks=2)
    out = torch.full_like(q, 7.0)
    C.window_attention(p, q, k, v, out=out)
    _check(q, k, v, spans, 20, 2, out)
    assert (out[sum(s[0] for s in spans):] == 7.0).all()


def test_window_attention_of_thousands_of_sequences(gpu):
    rng = np.random.default_rng(13)
    spans = [(0, 0)] * 4500
    for s in rng.choice(4500, 120, replace=False):
        spans[s] = (int(rng.integers(1, 40)),) * 2
    spans[4499] = (50, 61)
    q, k, v, cu_q, cu_k = _inputs(spans, 2, 1, 64, BF16, gpu, 14)
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=20, n_sinks=2)
    out = C.window_attention(p, q, k, v)
    keep = [s for s in spans if s[0]]
    _check(q, k, v, keep, 20, 2, out)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
def test_windows_of_mixed_lengths(gpu, dtype, d):
    """Long chunks beside single tokens and sequences without any query, each row block split
    over workgroups: their numbering and their join leave out what is not there."""
    spans = [(0, 9)] * 3 + [(1, 300)] * 5 + [(70, 900)] + [(0, 0)] * 70 + [(3, 40), (0, 5), (33, 700)]
    q, k, v, cu_q, cu_k = _inputs(spans, 8, 2, d, dtype, gpu, 15)
    for window, sinks in ((400, 3), (1 << 20, 0)):
        p = C.WindowProblem(q, k, v, cu_q, cu_k, window=window, n_sinks=sinks)
        assert p._ws_bytes > 256                              # split
        out = torch.full_like(q, 7.0)
        C.window_attention(p, q, k, v, out=out)
        _check(q, k, v, spans, window, sinks, out)
        assert (out[sum(s[0] for s in spans):] == 7.0).all()
        again = torch.full_like(q, 7.0)
        C.window_attention(p, q, k, v, out=again)
        assert (H.bits(again) == H.bits(out)).all()


def test_windows_of_mixed_lengths_over_rows_far_apart(gpu):
    """The same in the kernel for few rows, which bf16 rows far apart take."""
    spans = [(0, 2)] * 70 + [(1, 20)] * 3 + [(20, 300), (0, 0), (5, 9)]
    q, k, v, cu_q, cu_k = _inputs(spans, 4, 1, 128, BF16, gpu, 16)
    far = torch.zeros((k.shape[0], (1 << 23) + 64), dtype=BF16, device=gpu)
    far[:, 64:192], far[:, -128:] = k[:, 0], v[:, 0]
    kf, vf = far[:, 64:192].unsqueeze(1), far[:, -128:].unsqueeze(1)
    p = C.WindowProblem(q, kf, vf, cu_q, cu_k, window=250, n_sinks=5)
    assert p._ws_bytes > 256
    _check(q, kf, vf, spans, 250, 5, C.window_attention(p, q, kf, vf))


@pytest.mark.parametrize("dtype,singles", [(BF16, 300), (F32, 65)], ids=["bf16", "f32"])
def test_a_long_prompt_beside_single_tokens(gpu, dtype, singles):
    """Far more row blocks in one sequence than in the others."""
    n, window, hq, hkv, d = 131072, 19, 32, 8, 64
    spans = [(1, 30)] * singles + [(n, n)]
    print("long prompt", dtype, singles, file=sys.stderr, flush=True)
    q, k, v, cu_q, cu_k = _inputs(spans, hq, hkv, d, dtype, gpu, 17)
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=window)
    out = C.window_attention(p, q, k, v)
    tq, tk = singles + n, 30 * singles + n
    assert torch.isfinite(out[:tq]).all()
    _check(q[:singles], k[:30 * singles], v[:30 * singles], spans[:singles], window, 0, out[:singles])
    for at in (0, 40000, n - 150):                            # pieces of the long one
        back = min(at, window - 1)
        qs, ks = slice(singles + at, singles + at + 150), slice(tk - n + at - back, tk - n + at + 150)
        _check(q[qs], k[ks], v[ks], [(150, 150 + back)], window, 0, out[qs])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("spans,window", [([(1, 300), (1, 40)], 1 << 20), ([(4, 600), (2, 90)], 500),
                                          ([(1, 6000)], 5000), ([(4, 5000), (0, 9), (3, 4000)], 1 << 20)],
                         ids=["tokens", "drafts", "tokens-split", "drafts-split"])
def test_probabilities_of_few_rows_keep_16_bits(gpu, d, spans, window):
    """Up to 16 query rows per group: the output is off by its own rounding and little else."""
    q, k, v, cu_q, cu_k = _inputs(spans, 8, 2, d, BF16, gpu, 18)
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=window, n_sinks=4)
    _check(q, k, v, spans, window, 4, C.window_attention(p, q, k, v), bits=16)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("lq,lk", [(1, 50), (1, 4000), (3, 60), (3, 4000), (150, 150), (150, 4000)])
def test_logits_of_minus_infinity(gpu, dtype, lq, lk):
    """A key whose logit is -infinity receives nothing; a row that sees no other gives zeros."""
    q, k, v, cu_q, cu_k = _inputs([(lq, lk)], 4, 2, 64, dtype, gpu, 19)
    q[:, :, 0] = 1.0                                          # every head: 1 * -infinity
    hidden = lk - lq // 3 - 20                                # keys before it
    k[:hidden, :, 0] = -float("inf")
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=30)
    out = C.window_attention(p, q, k, v)[:lq]
    t = np.arange(lk - lq, lk)
    assert not H.values(out)[t < hidden].any()
    kept = torch.cat((k[hidden:lk], k[lk:])), torch.cat((v[hidden:lk], v[lk:]))
    some = np.nonzero(t >= hidden)[0]
    _check(q[some[0]:lq], *kept, [(len(some), lk - hidden)], 30, 0, out[some[0]:])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_window_attention_of_the_most_sequences(gpu, dtype):
    rng = np.random.default_rng(20)
    spans = [(0, 0)] * 65535
    for s in [0, 63, 64, 1023, 1024, 65472, 65534, *rng.choice(65535, 40, replace=False)]:
        spans[s] = (int(rng.integers(9, 40)),) * 2
    q, k, v, cu_q, cu_k = _inputs(spans, 2, 1, 64, dtype, gpu, 21)
    p = C.WindowProblem(q, k, v, cu_q, cu_k, window=20, n_sinks=2)
    out = C.window_attention(p, q, k, v)
    _check(q, k, v, [s for s in spans if s[0]], 20, 2, out)

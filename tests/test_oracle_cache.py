"""Pins of the oracle of the bounded cache and the windowed attention: worked
examples, exhaustive searches and independent formulations."""
import itertools
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO


def _block(*x):
    return np.array(list(x) + [0.0] * (32 - len(x)))


def test_fp4_worked_block():
    # max 6: e = 0, 2^e = 1.  Ties go to the even code: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1,
    # 1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4
    x = _block(6.0, -6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.3, 0.2, -0.1)
    codes, scales = CO.fp4_encode(x)
    assert scales.tolist() == [127]
    assert codes[:6].tolist() == [0x7 | 0xF << 4, 0x0 | 0x2 << 4, 0x2 | 0x4 << 4, 0x4 | 0x6 << 4,
                                  0x6 | 0x9 << 4, 0x0 | 0x8 << 4]
    assert CO.fp4_decode(codes, scales)[:12].tolist() == [6, -6, 0, 1, 1, 2, 2, 4, 4, -0.5, 0, 0]


@pytest.mark.parametrize("top,e", [(7.0, 0), (np.nextafter(7.0, 8), 1), (3.5, -1),
                                   (np.nextafter(3.5, 4), 0), (4.0, 0), (1.0, -2), (0.0, -100),
                                   (1e-40, -100), (3.3e38, 125), (2.0 ** 127, 125)])
def test_fp4_scale_of_a_block(top, e):
    codes, scales = CO.fp4_encode(_block(0.0, -top))
    assert scales[0] == e + 127
    assert abs(CO.fp4_decode(codes, scales)[1] + top) <= 2.0 ** e + (top > 7 * 2.0 ** 125) * top / 7


def test_fp4_not_finite():
    for bad in (np.inf, -np.inf, np.nan):
        codes, scales = CO.fp4_encode(np.concatenate([_block(1.0, bad), _block(1.0)]))
        assert scales.tolist() == [255, 125] and not codes[:16].any()
        assert np.isnan(CO.fp4_decode(codes, scales)[:32]).all()


def test_fp4_nearest_by_search():
    g = np.random.default_rng(0)
    x = np.concatenate([g.standard_normal((8, 32)), np.round(g.standard_normal((8, 32)) * 8) / 8])
    codes, scales = CO.fp4_encode(x)
    got = CO.fp4_decode(codes, scales)
    for r, c in np.ndindex(x.shape):
        s = Fraction(2) ** (int(scales[r, 0]) - 127)
        far = [abs(abs(Fraction(x[r, c])) - s * Fraction(v)) for v in CO.FP4_STEPS]
        best = [i for i in range(8) if far[i] == min(far)]
        want = best[0] if len(best) == 1 else next(i for i in best if i % 2 == 0)
        assert Fraction(abs(got[r, c])) == s * Fraction(CO.FP4_STEPS[want])
        assert got[r, c] == 0 or np.sign(got[r, c]) == np.sign(x[r, c])


def test_attend_against_torch():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 2, 8), (9, 8), (9, 8)))
    pos = torch.tensor([0, 9, 1, 7, 8, 2, 3, 4, 5])
    out, got, _, _ = CO.attend(q.numpy(), k.numpy(), v.numpy(), pos.numpy(), 10)
    z = (q.reshape(6, 8) @ k.T) / 8 ** 0.5
    t = torch.tensor([7, 7, 8, 8, 9, 9])
    p = torch.softmax(z.masked_fill(pos[None] > t[:, None], -torch.inf), -1)
    np.testing.assert_allclose(out.reshape(6, 8), (p @ v).numpy(), rtol=1e-12)
    np.testing.assert_allclose(got, p.sum(0).numpy(), rtol=1e-12)
    np.testing.assert_allclose(got.sum(), 6.0, rtol=1e-12)


def test_attend_rows_that_see_nothing_and_masked_rubbish():
    q = np.ones((2, 1, 4))
    k, v = np.ones((2, 4)), np.array([[1.0] * 4, [np.nan] * 4])
    out, got, _, _ = CO.attend(q, k, v, np.array([5, 9]), 7)     # tokens at 5 and 6
    assert out[0, 0].tolist() == [1.0] * 4 and out[1, 0].tolist() == [1.0] * 4
    out, got, _, _ = CO.attend(q, k, v, np.array([6, 9]), 7)     # token 5 sees nothing
    assert not out[0].any() and out[1, 0].tolist() == [1.0] * 4 and got.tolist() == [1.0, 0.0]
    out, got, _, _ = CO.attend(q[:1], k[:0], v[:0], np.array([]), 7)
    assert not out.any() and got.shape == (0,)


@pytest.mark.parametrize("lq,lk,window,sinks", [(7, 7, 3, 2), (7, 7, 1, 0), (3, 9, 4, 1),
                                                (1, 9, 5, 0), (5, 3, 2, 1), (6, 6, 99, 3),
                                                (4, 0, 2, 2)])
def test_window_attention_key_by_key(lq, lk, window, sinks):
    g = np.random.default_rng(2)
    q, k, v = (g.standard_normal(s) for s in ((lq, 4, 4), (lk, 2, 4), (lk, 2, 4)))
    got = CO.window_attention(q, k, v, window, sinks, scale=0.7)
    for i, h in itertools.product(range(lq), range(4)):
        t, num, den = lk - lq + i, np.zeros(4), 0.0
        for j in range(lk):
            if j <= t and (t - j < window or j < sinks):
                w = np.exp(0.7 * float(q[i, h] @ k[j, h // 2]))
                num, den = num + w * v[j, h // 2], den + w
        np.testing.assert_allclose(got[i, h], num / den if den else num, rtol=1e-12, atol=1e-15)


def test_window_of_everything_is_causal_attention():
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn((2, 11, 8), generator=g, dtype=torch.float64) for _ in range(3))
    want = torch.softmax((q @ k.mT / 8 ** 0.5).masked_fill(
        torch.ones(11, 11).triu(1).bool(), -torch.inf), -1) @ v
    got = CO.window_attention(*(x.transpose(0, 1).numpy() for x in (q, k, v)), 11, 0)
    np.testing.assert_allclose(got, want.transpose(0, 1).numpy(), rtol=1e-12)


def test_evict_worked():
    #        slot  0    1    2    3    4    5    6    7
    w = np.array([0.9, 0.1, 0.5, 0.1, 0.7, 0.2, 0.0, 0.8])
    pos = np.arange(8)
    # three go: of the two 0.1 both, and 0.2; position 6 is recent, position 1 is not a sink
    assert CO.evict(w, pos, 8, 8, 5, 1, 2) == ([(1, 6), (3, 7)], 5)
    # two go: 0.1 and the higher slot of ... 0.1 (slot 3), then slot 1
    assert CO.evict(w, pos, 8, 8, 7, 0, 2) == ([(3, 7)], 7)
    # slot 1 held as a sink
    assert CO.evict(w, pos, 8, 8, 6, 2, 2) == ([(3, 6), (5, 7)], 6)
    # all held: the highest slots go
    assert CO.evict(w, pos, 8, 8, 6, 8, 0) == ([], 6)
    assert CO.evict(w, pos, 4, 8, 5, 0, 0) == ([], 4)
    w[4] = np.nan
    assert CO.evict(w, pos, 8, 8, 7, 0, 0) == ([(4, 7)], 7)
    w[4] = -np.inf
    w[5] = np.nan
    assert CO.evict(w, pos, 8, 8, 7, 0, 0) == ([(5, 7)], 7)


def test_evict_keeps_the_heaviest():
    g = np.random.default_rng(4)
    for _ in range(50):
        n, budget = g.integers(2, 40), 0
        budget = int(g.integers(1, n))
        w = np.round(g.random(n) * 6) / 6               # many ties
        pos = g.permutation(n)
        moves, new = CO.evict(w, pos, n, n, budget, 0, 0)
        after = list(range(n))
        for to, src in moves:
            after[to] = src
        kept = sorted(after[:new])
        want = sorted(sorted(range(n), key=lambda s: (-w[s], s))[:budget])
        assert kept == want
        assert all(after[s] == s for s in range(budget) if s in want)

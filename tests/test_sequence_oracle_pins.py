"""The fp64 definitions of the sequence operators against what pins them: the explicit sum over earlier tokens, and differences."""
import numpy as np
import pytest

from oracle import sequence_oracle as so


def _random(seed, tokens, hq, hkv, d):
    rng = np.random.default_rng(seed)
    q, k, v = rng.standard_normal((tokens, hq, d)), rng.standard_normal((tokens, hkv, d)), rng.standard_normal((tokens, hkv, d))
    return rng, q, k, v, -rng.random((tokens, hkv))


@pytest.mark.parametrize("rectify", [False, True])
def test_recurrence_is_the_weighted_sum_over_earlier_tokens(rectify):
    rng, q, k, v, g = _random(1, 11, 4, 2, 3)
    spans = [(0, 4), (4, 4), (4, 10)]                   # one empty, the last row in none
    first = rng.standard_normal((3, 2, 3, 3))
    out, last = so.recurrence(q, k, v, g, spans, first, 0.7, rectify)
    rq, rk = (np.maximum(t, 0) if rectify else t for t in (q, k))
    for b, (lo, hi) in enumerate(spans):
        for h in range(4):
            for i in range(lo, hi):
                want = np.exp(g[lo:i + 1, h // 2].sum()) * rq[i, h] @ first[b, h // 2]
                for j in range(lo, i + 1):
                    want = want + np.exp(g[j + 1:i + 1, h // 2].sum()) * (rq[i, h] @ rk[j, h // 2]) * v[j, h // 2]
                np.testing.assert_allclose(out[i, h], 0.7 * want, rtol=1e-12, atol=1e-12)
    assert (out[10] == 0).all()
    np.testing.assert_array_equal(last[1], first[1])


def test_gradient_of_the_recurrence_against_differences():
    rng, q, k, v, g = _random(2, 7, 4, 2, 3)
    spans = [(0, 3), (3, 7)]
    first, do, dl = rng.standard_normal((2, 2, 3, 3)), rng.standard_normal(q.shape), rng.standard_normal((2, 2, 3, 3))

    def value(q, k, v, g, first):
        out, last = so.recurrence(q, k, v, g, spans, first, 0.6, True)
        return (out * do).sum() + (last * dl).sum()

    grads = so.recurrence_backward(q, k, v, g, spans, first, 0.6, do, dl, True)
    args = [q, k, v, g, first]
    for a, (x, got) in enumerate(zip(args, grads)):
        for at in [tuple(rng.integers(0, n) for n in x.shape) for _ in range(12)]:
            moved = []
            for h in (1e-5, -1e-5):
                y = x.copy()
                y[at] += h
                moved.append(value(*args[:a], y, *args[a + 1:]))
            assert abs((moved[0] - moved[1]) / 2e-5 - got[at]) < 1e-7 * max(1.0, abs(got[at]))


def test_norm_and_its_gradient():
    rng = np.random.default_rng(3)
    x, res, w, dy, ds = (rng.standard_normal(s) for s in ((4, 9), (4, 9), (9,), (4, 9), (4, 9)))
    y, r = so.norm(x, res, w, 0.0)
    np.testing.assert_allclose(((y / w) ** 2).mean(-1), 1.0, rtol=1e-12)
    np.testing.assert_array_equal(r, x + res)
    d_r, d_w = so.norm_backward(r, w, dy, ds, 1e-3)
    value = lambda r, w: (so.norm(r, None, w, 1e-3)[0] * dy).sum() + (r * ds).sum()
    for at in [(0, 0), (1, 5), (3, 8)]:
        e = np.zeros_like(r)
        e[at] = 1e-5
        assert abs((value(r + e, w) - value(r - e, w)) / 2e-5 - d_r[at]) < 1e-8
    for c in (0, 4, 8):
        e = np.zeros_like(w)
        e[c] = 1e-5
        assert abs((value(r, w + e) - value(r, w - e)) / 2e-5 - d_w[c]) < 1e-8

"""The fp64 definitions of a selective state space layer's operators against what pins them: explicit sums, closed forms and differences."""
import numpy as np
import pytest

from oracle import layer_oracle as lo


def _scan(seed, tokens=9, channels=4, groups=2, states=3, n=2):
    rng = np.random.default_rng(seed)
    r = rng.standard_normal
    t = dict(x=r((tokens, channels)), delta=r((tokens, channels)), a=-np.abs(r((channels, states))) - 0.1, b=r((tokens, groups, states)),
             c=r((tokens, groups, states)), skip=r(channels), bias=r(channels), gate=r((tokens, channels)), initial=r((n, channels, states)))
    return rng, t


def test_the_scan_is_the_weighted_sum_over_earlier_tokens():
    rng, t = _scan(1, n=3)
    spans = [(0, 4), (4, 4), (4, 8)]                    # one empty, the last row in none
    out, last, _ = lo.scan(t["x"], t["delta"], t["a"], t["b"], t["c"], spans, t["skip"], t["bias"], t["gate"], True, t["initial"])
    step = np.log(1 + np.exp(t["delta"] + t["bias"]))
    for b, (first, end) in enumerate(spans):
        for ch in range(4):
            g = ch // 2
            for i in range(first, end):
                h = np.exp(t["a"][ch] * step[first:i + 1, ch].sum()) * t["initial"][b, ch]
                for j in range(first, i + 1):
                    h = h + np.exp(t["a"][ch] * step[j + 1:i + 1, ch].sum()) * step[j, ch] * t["x"][j, ch] * t["b"][j, g]
                y = h @ t["c"][i, g] + t["skip"][ch] * t["x"][i, ch]
                z = t["gate"][i, ch]
                np.testing.assert_allclose(out[i, ch], y * z / (1 + np.exp(-z)), rtol=1e-12, atol=1e-12)
                if i == end - 1:
                    np.testing.assert_allclose(last[b, ch], h, rtol=1e-12, atol=1e-12)
    assert (out[8] == 0).all()
    np.testing.assert_array_equal(last[1], t["initial"][1])


@pytest.mark.parametrize("softplus", [True, False])
def test_gradient_of_the_scan_against_differences(softplus):
    rng, t = _scan(2)
    if not softplus:
        t["delta"] = np.abs(t["delta"])
    spans = [(0, 5), (5, 9)]
    do, dl = rng.standard_normal((9, 4)), rng.standard_normal((2, 4, 3))

    def value(v):
        out, last, _ = lo.scan(v["x"], v["delta"], v["a"], v["b"], v["c"], spans, v["skip"], v["bias"], v["gate"], softplus, v["initial"])
        return (out * do).sum() + (last * dl).sum()

    g = lo.scan_backward(t["x"], t["delta"], t["a"], t["b"], t["c"], spans, do, t["skip"], t["bias"], t["gate"], softplus, t["initial"], dl)
    for name in t:
        e = rng.standard_normal(t[name].shape)
        h = 1e-6
        got = (value(dict(t, **{name: t[name] + h * e})) - value(dict(t, **{name: t[name] - h * e}))) / (2 * h)
        np.testing.assert_allclose(got, (g[name] * e).sum(), rtol=1e-6, atol=1e-7, err_msg=name)


def test_magnitudes_bound_the_gradient():
    rng, t = _scan(3)
    do = rng.standard_normal((9, 4))
    args = (t["x"], t["delta"], t["a"], t["b"], t["c"], [(0, 9)], do, t["skip"], t["bias"], t["gate"], True, t["initial"][:1])
    g, m = lo.scan_backward(*args), lo.scan_backward(*args, magnitudes=True)
    for name in g:
        assert (np.abs(g[name]) <= m[name] * (1 + 1e-12)).all(), name


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("width", [2, 4])
def test_convolution_and_its_gradient(silu, width):
    rng = np.random.default_rng(4)
    t = dict(x=rng.standard_normal((9, 3)), weight=rng.standard_normal((3, width)), bias=rng.standard_normal(3), initial=rng.standard_normal((3, width - 1, 3)))
    spans = [(0, 1), (1, 1), (1, 9)]
    out, last = lo.conv(t["x"], t["weight"], spans, t["bias"], silu, t["initial"])
    for c in range(3):                                  # numpy's own convolution over the rows of the last sequence
        rows = np.concatenate([t["initial"][2, :, c], t["x"][1:, c]])
        pre = np.convolve(rows, t["weight"][c, ::-1], "valid") + t["bias"][c]
        np.testing.assert_allclose(out[1:, c], pre / (1 + np.exp(-pre)) if silu else pre, rtol=1e-12, atol=1e-12)
    np.testing.assert_array_equal(last[1], t["initial"][1])
    np.testing.assert_array_equal(last[2], t["x"][9 - (width - 1):])
    np.testing.assert_array_equal(last[0], np.concatenate([t["initial"][0], t["x"][:1]])[1:])
    do, dl = rng.standard_normal((9, 3)), rng.standard_normal(t["initial"].shape)

    def value(v):
        out, last = lo.conv(v["x"], v["weight"], spans, v["bias"], silu, v["initial"])
        return (out * do).sum() + (last * dl).sum()

    g = lo.conv(t["x"], t["weight"], spans, t["bias"], silu, t["initial"], do, dl)
    for name, grad in zip(t, g):
        e = rng.standard_normal(t[name].shape)
        got = (value(dict(t, **{name: t[name] + 1e-6 * e})) - value(dict(t, **{name: t[name] - 1e-6 * e}))) / 2e-6
        np.testing.assert_allclose(got, (grad * e).sum(), rtol=1e-6, atol=1e-7, err_msg=name)


def test_layer_norm_and_its_gradient():
    rng = np.random.default_rng(5)
    t = dict(r=rng.standard_normal((4, 7)) + 2, weight=rng.standard_normal(7), bias=rng.standard_normal(7))
    y, _ = lo.layer_norm(t["r"], None, None, None, 0.0)
    np.testing.assert_allclose(y.mean(1), 0, atol=1e-12)
    np.testing.assert_allclose((y * y).mean(1), 1, rtol=1e-12)
    do, ds = rng.standard_normal((4, 7)), rng.standard_normal((4, 7))
    value = lambda v: (lo.layer_norm(v["r"], None, v["weight"], v["bias"], 1e-3)[0] * do).sum() + (v["r"] * ds).sum()
    g = lo.layer_norm_backward(t["r"], t["weight"], do, ds, 1e-3)
    for name, grad in zip(t, g):
        e = rng.standard_normal(t[name].shape)
        got = (value(dict(t, **{name: t[name] + 1e-6 * e})) - value(dict(t, **{name: t[name] - 1e-6 * e}))) / 2e-6
        np.testing.assert_allclose(got, (grad * e).sum(), rtol=1e-6, atol=1e-7, err_msg=name)

"""Layer norm and its gradient, against fp64.

Tolerances: half a step of the result's type, plus fp32 on the way.  A sum over a row is taken in pieces of at most 64 values and a tree above them, 2^-17 of its terms'
magnitudes with all that follows it (the root, the reciprocal, products), as for the root-mean-square norm; the mean's error counts against the deviation, so the
magnitudes hold the mean of |r| over the deviation's root mean square."""
import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from paper_2205_14756_amd import sequence as seq

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
WAY = 2.0 ** -17
EPS = 1e-5


def half_step(dtype):
    return torch.finfo(TDT[dtype]).eps / 2


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def rnd(seed, dtype, *shape, scale=1.0, shift=0.0):
    return (torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)) * scale + shift).to(TDT[dtype]).cuda()


def close(got, want, tol, what):
    got = f64(got)
    assert np.isfinite(got).all(), what
    worst = float(np.max(np.abs(got - want) / tol)) if got.size else 0.0
    print(f"  {what}: {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0, what


def sizes_of(r):
    """(1 / sqrt(var + eps), mean |r|) of every row"""
    d = r - r.mean(-1, keepdims=True)
    return 1 / np.sqrt((d * d).mean(-1, keepdims=True) + EPS), np.abs(r).mean(-1, keepdims=True)


SHAPES = [(1, 1), (5, 7), (3, 16), (130, 33), (64, 64), (9, 128), (257, 520), (2, 2051), (7, 4096), (1025, 4100), (3, 8200), (2, 16385), (1, 32768)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,channels", SHAPES)
@pytest.mark.parametrize("full", [True, False])
def test_layer_norm(dtype, rows, channels, full):
    print(f"layer norm {dtype} {rows} x {channels} {'with' if full else 'without'} residual, weight and bias", flush=True)
    x = rnd(1, dtype, rows, channels, scale=2.0, shift=1.5)
    res, w, b = (rnd(2, dtype, rows, channels), rnd(3, dtype, channels), rnd(4, dtype, channels)) if full else (None, None, None)
    guard = torch.full((rows + 2, channels), 7.0, dtype=TDT[dtype], device="cuda")
    y, r = seq.msla_layer_norm_forward(x, w, b, res, EPS, out=guard[1:-1])
    want, sums = lo.layer_norm(f64(x), f64(res), f64(w), f64(b), EPS)
    rstd, level = sizes_of(sums)
    aw = np.ones(channels) if w is None else np.abs(f64(w))
    # (in a row of one channel the deviation is 0: what is left is the error of the mean over sqrt(eps))
    size = (np.abs(sums) + level) * rstd * aw + (0 if b is None else np.abs(f64(b)))
    close(y, want, half_step(dtype) * np.abs(want) + WAY * size + 2.0 ** -24, "y")
    assert bool((guard[0] == 7.0).all()) and bool((guard[-1] == 7.0).all())
    if full:
        close(r, sums, half_step(dtype) * np.abs(sums) + 1e-7 * (np.abs(f64(x)) + np.abs(f64(res))) + 2.0 ** -25, "sum")
    else:
        assert r is x
    # in place: the sum into the residual, y into x
    x2, res2 = x.clone(), None if res is None else res.clone()
    y2, r2 = seq.msla_layer_norm_forward(x2, w, b, res2, EPS, out=x2, sum_out=res2)
    assert torch.equal(y2, y) and (res is None or torch.equal(res2, r))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,channels", SHAPES + [(0, 64), (3000, 24), (2100, 300)])
@pytest.mark.parametrize("full", [True, False])
def test_layer_norm_backward(dtype, rows, channels, full):
    print(f"layer norm backward {dtype} {rows} x {channels}", flush=True)
    r, dy = rnd(5, dtype, rows, channels, scale=2.0, shift=1.5), rnd(6, dtype, rows, channels)
    w, ds = (rnd(7, dtype, channels), rnd(8, dtype, rows, channels)) if full else (None, None)
    n = seq.msla_layer_norm_backward_workspace_bytes(rows, channels, TDT[dtype])
    ws = torch.full((n + 256,), 0xFF, dtype=torch.uint8, device="cuda")
    d_r, d_w, d_b = seq.msla_layer_norm_backward(r, w, dy, ds, EPS, workspace=ws[:n])
    torch.cuda.synchronize()
    assert bool((ws[n:] == 0xFF).all())
    want_r, want_w, want_b = lo.layer_norm_backward(f64(r), f64(w), f64(dy), f64(ds), EPS)
    rstd, level = sizes_of(f64(r))
    aw = np.ones(channels) if w is None else np.abs(f64(w))
    g, unit = np.abs(f64(dy)) * aw, (np.abs(f64(r)) + level) * rstd
    mag = (g + g.mean(-1, keepdims=True) + unit * (g * unit).mean(-1, keepdims=True)) * rstd + (0 if ds is None else np.abs(f64(ds)))
    close(d_r, want_r, half_step(dtype) * np.abs(want_r) + 4 * WAY * mag + 2.0 ** -24, "d_r")
    close(d_w, want_w, 4 * WAY * (np.abs(f64(dy)) * unit).sum(0) + 1e-30, "d_weight")
    close(d_b, want_b, WAY * np.abs(f64(dy)).sum(0) + 1e-30, "d_bias")
    again = seq.msla_layer_norm_backward(r, w, dy, ds, EPS)
    assert all(torch.equal(p, q) for p, q in zip(again, (d_r, d_w, d_b)))
    if rows:                                # into the gradient that it came from
        dy2 = dy.clone()
        assert torch.equal(seq.msla_layer_norm_backward(r, w, dy2, ds, EPS, d_r=dy2)[0], d_r)


def test_a_mean_that_is_large_beside_the_deviations():
    """rows at 1000 with deviations of 1: the squares less the mean's square would leave 2^-24 * 10^6 of them"""
    x = rnd(9, "f32", 4, 1000, shift=1000.0)
    y, _ = seq.msla_layer_norm_forward(x, eps=EPS)
    want, _ = lo.layer_norm(f64(x), None, None, None, EPS)
    # the mean is off by at most half an ulp of 1000 (2^-15) and its sum's tree (some of those): 2^-12 of a deviation of 1
    assert np.abs(f64(y) - want).max() <= 2.0 ** -12


def test_rows_without_deviations_and_values_that_are_not_finite():
    x = torch.full((4, 96), 3.0, device="cuda")
    b = rnd(10, "f32", 96)
    y, _ = seq.msla_layer_norm_forward(x, None, b, eps=EPS)
    assert torch.equal(y, b.expand(4, 96))
    x = rnd(11, "bf16", 6, 200)
    clean, _ = seq.msla_layer_norm_forward(x)
    x[1, 3], x[4, 199] = float("nan"), float("inf")
    y, _ = seq.msla_layer_norm_forward(x)
    bad = ~torch.isfinite(y)
    assert bool(bad[1].all()) and bool(bad[4].all()) and int(bad.sum()) == 400
    assert torch.equal(y[[0, 2, 3, 5]], clean[[0, 2, 3, 5]])


def test_gradient_against_differences():
    r, w, dy, ds = rnd(12, "f32", 5, 70), rnd(13, "f32", 70), rnd(14, "f32", 5, 70), rnd(15, "f32", 5, 70)
    b = rnd(16, "f32", 70)
    g = seq.msla_layer_norm_backward(r, w, dy, ds, EPS)
    value = lambda r, w, b: float((seq.msla_layer_norm_forward(r, w, b, None, EPS)[0].double() * dy.double()).sum() + (r.double() * ds.double()).sum())
    h, t = 2.0 ** -7, [r, w, b]
    for i, grad in enumerate(g):
        e = rnd(17 + i, "f32", *t[i].shape)
        up, down = ([v + s * h * e if j == i else v for j, v in enumerate(t)] for s in (1, -1))
        got, want = (value(*up) - value(*down)) / (2 * h), float((grad.double() * e.double()).sum())
        # h^2 / 6 of the third derivative, which is of the size of the value's own terms
        assert abs(got - want) <= h * h * float((grad.double().abs() * e.double().abs()).sum()) + 2e-3, (got, want)


@pytest.mark.parametrize("offset", [1, 3])
def test_rows_that_start_anywhere(offset):
    flat = rnd(20, "bf16", offset + 6 * 130)
    x = flat[offset:].view(6, 130)
    assert torch.equal(seq.msla_layer_norm_forward(x)[0], seq.msla_layer_norm_forward(x.clone())[0])
    g = rnd(21, "bf16", offset + 6 * 130)[offset:].view(6, 130)
    assert all(torch.equal(p, q) for p, q in zip(seq.msla_layer_norm_backward(x, None, g), seq.msla_layer_norm_backward(x.clone(), None, g.clone())))

"""The short causal convolution through the C ABI against oracle/layer_oracle.py (fp64, tap by tap).

Tolerances, element by element: half a step of the type that a result is rounded to once, plus fp32 on the way in units of 2^-24 of the terms' magnitudes:
at most five multiply-adds in a row and some ulps of the sigmoid (and its derivative) with an argument of up to 16: 64 of them; sums over tokens add one a
token of a run of 64, and of at most 32 runs in a row, and 32 more: 160."""
import functools

import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from paper_2205_14756_amd import sequence as seq

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
WAY, SUM = 64 * 2.0 ** -24, 224 * 2.0 ** -24


def half_step(dtype):
    return torch.finfo(TDT[dtype]).eps / 2


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


@functools.lru_cache(maxsize=None)
def _numbers(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape))


def num(seed, dtype, *shape):
    return _numbers(seed, *shape).to(TDT[dtype]).cuda()


def close(got, want, tol, what):
    got = f64(got)
    assert np.isfinite(got).all(), what
    worst = float(np.max(np.abs(got - want) / tol)) if got.size else 0.0
    print(f"  {what}: {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0, what


def check(dtype, lens, channels, width, silu=True, full=True, initial=True, start=0, tail=0, packed=True, seed=1):
    tokens = start + sum(lens) + tail
    print(f"conv {dtype} lens={lens if len(lens) < 12 else len(lens)} channels={channels} width={width} silu={silu} full={full} initial={initial}", flush=True)
    x, d_out = num(seed, dtype, tokens, channels), num(seed + 100, dtype, tokens, channels)
    w, bias = num(seed + 200, dtype, channels, width), num(seed + 300, dtype, channels) if full else None
    first = num(seed + 400, dtype, len(lens), width - 1, channels) if initial else None
    d_last = num(seed + 500, dtype, len(lens), width - 1, channels) if initial else None
    offs = [start + sum(lens[:i]) for i in range(len(lens) + 1)]
    spans = list(zip(offs[:-1], offs[1:]))
    kw = dict(silu=silu, sequences=len(lens), offsets=torch.tensor(offs, dtype=torch.int32, device="cuda") if packed else None, initial_state=first)
    live = np.zeros(tokens, bool)
    live[offs[0]:offs[-1]] = True
    rows = torch.from_numpy(live).cuda()
    half = half_step(dtype)
    tiny = 2.0 ** -24 if dtype == "f16" else 1e-30
    mag = lambda v: None if v is None else np.abs(f64(v))
    want, last = lo.conv(f64(x), f64(w), spans, f64(bias), silu, f64(first))
    size, _ = lo.conv(mag(x), mag(w), spans, mag(bias), False, mag(first))
    to = torch.full((tokens, channels), 7.0, dtype=TDT[dtype], device="cuda")
    got, state = seq.msla_causal_conv_forward(x, w, bias, out=to, **kw)
    assert bool((got[~rows] == 7.0).all()), "rows of no sequence were written"
    close(got[rows], want[live], half * np.abs(want[live]) + WAY * size[live] + tiny, "out")
    assert np.array_equal(f64(state), last), "the state is not the last rows"
    want = lo.conv(f64(x), f64(w), spans, f64(bias), silu, f64(first), f64(d_out), f64(d_last))
    # silu's derivative is at most 1.1, and moves by at most half of what its argument does
    slack = 1.1 + 0.5 * size.max(initial=0)
    sizes = [slack * v for v in lo.conv(mag(x), mag(w), spans, mag(bias), False, mag(first), mag(d_out), mag(d_last))]
    n_ws = seq.msla_causal_conv_backward_workspace_bytes(len(lens), tokens, channels, width, TDT[dtype], packed=packed)
    ws = torch.full((n_ws + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    run = lambda ws: seq.msla_causal_conv_backward(x, w, d_out, bias, d_final_state=d_last, d_x=torch.full_like(x, 7.0), workspace=ws, **kw)
    dx, dw, db, ds = run(ws[:n_ws])
    assert bool((ws[n_ws:] == 0xFF).all()), "bytes past the workspace were written"
    assert bool((dx[~rows] == 7.0).all()), "rows of no sequence were written"
    close(dx[rows], want[0][live], half * np.abs(want[0][live]) + WAY * sizes[0][live] + tiny, "d_x")
    close(dw, want[1], SUM * sizes[1] + 1e-30, "d_weight")
    if full:
        close(db, want[2], SUM * sizes[2] + 1e-30, "d_bias")
    if initial:
        close(ds, want[3], half * np.abs(want[3]) + WAY * sizes[3] + tiny, "d_initial")
    for p, q in zip((dx, dw, db, ds), run(None)):       # the same bits again
        assert p is None and q is None or torch.equal(p, q)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("lens", [[1], [2], [3], [5], [16], [17, 0, 1, 2, 3, 64, 65], [200]])
def test_sizes(dtype, width, lens):
    check(dtype, lens, 40, width)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("channels", [1, 3, 7, 8, 9, 15, 64, 513, 2047, 2050, 4104])
def test_channels(dtype, channels):
    check(dtype, [21, 2, 40], channels, 4, seed=2)


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("full,initial", [(True, False), (False, True), (False, False)])
def test_optional_operands(silu, full, initial):
    check("bf16", [33, 70], 24, 4, silu, full, initial, seed=3)
    check("f32", [50, 50], 24, 3, silu, full, initial, seed=4, packed=False)


def test_rows_of_no_sequence_are_left_alone():
    check("f32", [10, 0, 97], 20, 4, start=5, tail=9, seed=5)
    check("bf16", [0, 0, 0], 20, 4, start=5, tail=9, seed=5)
    check("bf16", [0], 20, 2, start=0, tail=0, seed=5, packed=False)


def test_long_runs_of_many_tokens():
    check("bf16", [5000, 3001], 512, 4, seed=6)
    check("f32", [1] * 300, 100, 4, seed=7, packed=False)


def test_parts_of_wider_rows():
    x, w, bias, d = num(8, "bf16", 60, 50), num(9, "bf16", 50, 4), num(10, "bf16", 50), num(11, "bf16", 60, 50)
    want, state = seq.msla_causal_conv_forward(x, w, bias, silu=True)
    wide = torch.full((60, 111), 3.0, dtype=torch.bfloat16, device="cuda")
    room = torch.full((60, 61), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 1:51], wide[:, 61:111] = x, d
    got, state2 = seq.msla_causal_conv_forward(wide[:, 1:51], w, bias, silu=True, out=room[:, 3:53])
    assert torch.equal(got, want) and torch.equal(state, state2) and bool((room[:, :3] == 7).all()) and bool((room[:, 53:] == 7).all())
    p = seq.msla_causal_conv_backward(x, w, d, bias, silu=True)
    q = seq.msla_causal_conv_backward(wide[:, 1:51], w, wide[:, 61:111], bias, silu=True, d_x=room[:, 5:55])
    assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(p, q))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("width", [2, 3, 4])
@pytest.mark.parametrize("sequences,channels", [(1, 1), (3, 9), (5, 515), (130, 64), (1, 4096)])
def test_step(dtype, width, sequences, channels):
    x, w, bias = num(12, dtype, sequences, channels), num(13, dtype, channels, width), num(14, dtype, channels)
    state = num(15, dtype, sequences, width - 1, channels)
    spans = [(i, i + 1) for i in range(sequences)]
    want, last = lo.conv(f64(x), f64(w), spans, f64(bias), True, f64(state))
    size, _ = lo.conv(np.abs(f64(x)), np.abs(f64(w)), spans, np.abs(f64(bias)), False, np.abs(f64(state)))
    got, new = seq.msla_causal_conv_step(x, w, state, bias, silu=True, new_state=torch.full_like(state, 7.0))
    close(got, want, half_step(dtype) * np.abs(want) + WAY * size + (2.0 ** -24 if dtype == "f16" else 1e-30), "out")
    assert np.array_equal(f64(new), last)
    there = state.clone()
    again, s = seq.msla_causal_conv_step(x, w, there, bias, silu=True)
    assert s is there and torch.equal(there, new) and torch.equal(again, got)
    whole, ends = seq.msla_causal_conv_forward(x, w, bias, silu=True, sequences=sequences, initial_state=state)
    assert torch.equal(whole, got) and torch.equal(ends, new)


def test_values_that_are_not_finite_reach_their_own_window_alone():
    x, w = num(16, "f32", 40, 8), num(17, "f32", 8, 4)
    clean, _ = seq.msla_causal_conv_forward(x, w, sequences=2)
    x[18, 3] = float("nan")
    got, _ = seq.msla_causal_conv_forward(x, w, sequences=2)
    bad = torch.isnan(got)
    assert bool(bad[18:20, 3].all()) and int(bad.sum()) == 2        # (the next sequence starts at 20)
    assert torch.equal(got[~bad], clean[~bad])


def test_gradient_against_differences():
    x, w, bias, d = num(18, "f32", 50, 12), num(19, "f32", 12, 4), num(20, "f32", 12), num(21, "f32", 50, 12)
    first, d_last = num(22, "f32", 2, 3, 12), num(23, "f32", 2, 3, 12)
    offs = torch.tensor([0, 2, 50], dtype=torch.int32, device="cuda")
    t = dict(x=x, weight=w, bias=bias, initial_state=first)

    def value(**v):
        out, last = seq.msla_causal_conv_forward(silu=True, offsets=offs, **v)
        return float((out.double() * d.double()).sum() + (last.double() * d_last.double()).sum())

    g = seq.msla_causal_conv_backward(x, w, d, bias, silu=True, offsets=offs, initial_state=first, d_final_state=d_last)
    h = 2.0 ** -8
    for i, (name, grad) in enumerate(zip(t, g)):
        e = num(30 + i, "f32", *t[name].shape)
        got = (value(**dict(t, **{name: t[name] + h * e})) - value(**dict(t, **{name: t[name] - h * e}))) / (2 * h)
        want = float((grad.double() * e.double()).sum())
        # h^2 / 6 of the third derivative, of the size of the terms, and fp32's rounding over h
        assert abs(got - want) <= 4 * h * h * float((grad.double().abs() * e.double().abs()).sum()) + 2e-2, (name, got, want)

"""Rows in 8-bit integers and their projection: integers and sums are exact, so the oracle is integer arithmetic.

Tolerances of the projection: the integer's conversion to fp32 and two products, 3 * 2^-24 relative, and half a step of the output's type."""
import numpy as np
import pytest
import torch

from paper_2205_14756_amd import sequence as seq

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def f64(t):
    return t.detach().double().cpu().numpy()


def rnd(seed, dtype, *shape, scale=1.0):
    return (torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)) * scale).to(TDT[dtype]).cuda()


def ints(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).integers(-128, 128, shape).astype(np.int8)).cuda()


def rows_oracle(x):
    """the definition in fp32 as IEEE rounds it (numpy multiplies and divides that way)"""
    x = x.detach().float().cpu().numpy()
    scale = (np.abs(x).max(-1) * (np.float32(1) / np.float32(127))).astype(np.float32)
    q = np.rint(x / np.where(scale > 0, scale, np.float32(1))[..., None])
    return q.astype(np.int8), scale


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,channels", [(1, 1), (5, 7), (3, 16), (130, 33), (64, 64), (257, 520), (2, 2051), (7, 4096), (3, 8200), (2, 16385), (1, 32768)])
def test_rows_into_integers(dtype, rows, channels):
    x = rnd(1, dtype, rows, channels, scale=3.0)
    guard = torch.full((rows + 2, channels), 7, dtype=torch.int8, device="cuda")
    x8, scale = seq.msla_quantize_rows_integer(x, out8=guard[1:-1])
    q, s = rows_oracle(x)
    assert np.array_equal(x8.cpu().numpy(), q) and np.array_equal(scale.cpu().numpy(), s)
    assert bool((guard[0] == 7).all()) and bool((guard[-1] == 7).all())


def test_rows_of_any_values():
    x = rnd(2, "f32", 9, 200)
    x[0] = 0
    x[1] *= 1e-38                            # a scale below fp32's normal range
    x[2] *= 1e36
    x[3, 5] = float("nan")
    x[4, 6] = float("inf")
    x[5] = torch.arange(200, device="cuda") - 100.5       # halves, to even: 127 / 100.5 of them are not
    x[6] = (torch.arange(200, device="cuda") % 255 - 127).float() / 2
    x[6, 0], x[6, 1] = 63.5, -63.5                          # a scale of some 1/2: whole numbers
    x[7] = torch.where(torch.arange(200, device="cuda") % 2 == 0, 0.5, 1.5)
    x[7, 0] = 127.0                                        # a scale of 1 to within its last place: halves go to one side, or tie to even
    x8, scale = seq.msla_quantize_rows_integer(x)
    fine = [0, 1, 2, 5, 6, 7, 8]
    q, s = rows_oracle(x[fine])
    assert np.array_equal(x8[fine].cpu().numpy(), q) and np.array_equal(scale[fine].cpu().numpy(), s)
    assert bool((x8[0] == 0).all()) and float(scale[0]) == 0.0
    assert bool(torch.isnan(scale[3])) and bool(torch.isinf(scale[4])) and bool((x8[3:5] == 0).all())
    assert set(x8[7, 1:].tolist()) <= {0, 1, 2}
    one = float(np.float32(127) * (np.float32(1) / np.float32(127)))
    assert float(scale[7]) == one and (one != 1.0 or set(x8[7, 1:].tolist()) == {0, 2})


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,c_in,c_out", [(1, 16, 16), (1, 64, 48), (3, 80, 16), (16, 4096, 64), (17, 144, 32), (33, 1040, 80), (48, 4096, 256), (64, 112, 512),
                                             (65, 128, 128), (129, 272, 144), (200, 16, 1040), (300, 4112, 272), (513, 512, 784), (1100, 1024, 1296)])
def test_projection(dtype, rows, c_in, c_out):
    print(f"projection of integers {dtype} {rows} x {c_in} -> {c_out}", flush=True)
    x8, w8 = ints(3, rows, c_in), ints(4, c_out, c_in)
    xs, ws = rnd(5, "f32", rows).abs() * 1e-3, rnd(6, "f32", c_out).abs() * 1e-2
    guard = torch.full((rows + 2, c_out), 7.0, dtype=TDT[dtype], device="cuda")
    y = seq.msla_linear_integer(x8, xs, w8, ws, out=guard[1:-1])
    want = (f64(x8) @ f64(w8).T) * f64(xs)[:, None] * f64(ws)
    tol = (torch.finfo(TDT[dtype]).eps / 2 + 3 * 2.0 ** -24) * np.abs(want) + (2.0 ** -24 if dtype == "f16" else 1e-30)
    got = f64(y)
    worst = np.max(np.abs(got - want) / tol)
    print(f"  y: {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0
    assert bool((guard[0] == 7.0).all()) and bool((guard[-1] == 7.0).all())


def test_sums_of_the_largest_products_are_exact():
    c_in = 131056
    for rows in (2, 70):
        x8 = torch.full((rows, c_in), -128, dtype=torch.int8, device="cuda")
        w8 = torch.full((16, c_in), -128, dtype=torch.int8, device="cuda")
        w8[1] = 127
        w8[2, ::2] = 127
        one = torch.ones(rows, device="cuda")
        y = seq.msla_linear_integer(x8, one, w8, torch.ones(16, device="cuda"), torch.float32)
        want = np.float32((f64(x8[:1]) @ f64(w8).T))
        assert np.array_equal(y.cpu().numpy(), np.repeat(want, rows, 0))


def test_rows_and_their_projection_together():
    x, w = rnd(7, "bf16", 90, 640), rnd(8, "f32", 304, 640, scale=640 ** -0.5)
    w8, ws = seq.msla_quantize_rows_integer(w)
    x8, xs = seq.msla_quantize_rows_integer(x)
    y = seq.msla_linear_integer(x8, xs, w8, ws)
    # both sides are rounded to half a step of max / 127: errors of a row of 640 products, in the mean square
    want = f64(x) @ f64(w).T
    xe, we = f64(xs)[:, None] / np.sqrt(12), f64(ws) / np.sqrt(12)
    spread = np.sqrt(640 * (xe * np.sqrt((f64(w) ** 2).mean(-1))) ** 2 + 640 * (we * np.sqrt((f64(x) ** 2).mean(-1, keepdims=True))) ** 2)
    assert (np.abs(f64(y) - want) <= 6 * spread + 2.0 ** -8 * np.abs(want)).all()

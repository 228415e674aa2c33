"""The projection of 8-bit rows into many outputs (a vocabulary), on both sides of the border between its two kernels."""
import numpy as np
import pytest
import torch

import test_gpu_norm as base
from paper_2205_14756_amd import sequence as seq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 16, 17, 33, 48, 49])
@pytest.mark.parametrize("c_in,c_out", [(272, 16000), (144, 32000), (64, 128000)])
def test_many_outputs(dtype, rows, c_in, c_out):
    """Within test_gpu_norm.test_linear_quantized's tolerance: half a step, and fp32 sums of c_in exact products, in steps of 32, and three factors."""
    x8, sx = seq.msla_quantize_rows(base.rnd(rows, "f32", rows, c_in))
    w8, sw = seq.msla_quantize_rows(base.rnd(30, "f32", c_out, c_in))
    guard = torch.full((rows + 2, c_out), 7.0, dtype=base.TDT[dtype], device="cuda")
    y = seq.msla_linear_quantized(x8, sx, w8, sw, out=guard[1:-1])
    torch.cuda.synchronize()
    assert bool((guard[0] == 7.0).all()) and bool((guard[-1] == 7.0).all())
    a, b = x8.double(), w8.double()
    scales = sx.double()[:, None] * sw.double()
    want, size = base.f64((a @ b.t()) * scales), base.f64((a.abs() @ b.abs().t()) * scales)
    base.close(y, want, (base.half_step(dtype) + 2.0 ** -22) * np.abs(want) + (c_in / 32 + 8) * 2.0 ** -24 * size + 2.0 ** -24, "y")

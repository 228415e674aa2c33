"""The gradient of the scan with a decay for each state where its kernel goes by in other ways than for a few tokens of one sequence, against
oracle/layer_oracle.py.  Inputs, tolerances and checks are those of test_gpu_selective_scan.py."""
import numpy as np
import pytest

from test_gpu_selective_scan import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("states", [8, 16, 32, 64])
def test_sequences_shorter_than_a_tile(dtype, states):
    """Many workgroups of one tile with few tokens: a wave that has none goes ahead to the sums of d_skip and d_delta_bias while another still reads the last
    tile's sums over states, which d_x, d_delta and d_gate come from."""
    lens = [int(v) for v in np.random.default_rng(20 + states).integers(5, 17, 400)]
    check(dtype, lens, 64, 1, states, seed=15)
    check(dtype, [12] * 400, 64, 1, states, seed=16, packed=False)

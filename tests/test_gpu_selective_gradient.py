"""The gradient of the scan with a decay for each state where its kernel goes by in other ways than for a few tokens of one sequence, against
oracle/layer_oracle.py.  Inputs, tolerances and checks are those of test_gpu_selective_scan.py."""
import numpy as np
import pytest

from paper_2205_14756_amd import sequence as seq
from test_gpu_selective_scan import TDT, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("states", [8, 16, 32, 64])
def test_sequences_shorter_than_a_tile(dtype, states):
    """Many workgroups of one tile with few tokens: a wave that has none goes ahead to the sums of d_skip and d_delta_bias while another still reads the last
    tile's sums over states, which d_x, d_delta and d_gate come from."""
    lens = [int(v) for v in np.random.default_rng(20 + states).integers(5, 17, 400)]
    check(dtype, lens, 64, 1, states, seed=15)
    check(dtype, [12] * 400, 64, 1, states, seed=16, packed=False)


def slots_of(dtype, lens, channels, groups, states, packed):
    """(runs of tokens that sequences are cut into, whether any may be), from the bytes that a call's workspace takes: marks at every 16 tokens (8 of 8 states), sums
    over tokens of each run, sums over channels of each 32 of a group, and what only sequences that are cut have."""
    n, tokens, mark = len(lens), sum(lens), 8 if states == 8 else 16
    up = lambda floats: (4 * floats + 255) // 256 * 256
    marks = tokens // mark + n if packed else n * max(1, -(-(tokens // n) // mark))
    tiles, per = groups * -(-(channels // groups) // 32), channels * states
    got = seq.msla_selective_scan_workspace_bytes(n, tokens, channels, groups, states, TDT[dtype], packed=packed, backward=True)
    for slots in range(1, tokens + n + 1):
        whole = up(marks * per) + up(slots * (per + 2 * channels)) + up(tiles * tokens * 2 * states)
        if whole == got:
            return slots, False
        if whole + 2 * up(slots * per) + up(slots * channels) + up(marks * channels) == got:
            return slots, True
    raise AssertionError("the workspace has other parts than these")


KINDS = [("f32", 8), ("f32", 16), ("f32", 32), ("f32", 64), ("f16", 16), ("f16", 64), ("bf16", 8), ("bf16", 16), ("bf16", 32), ("bf16", 64)]


# A tile has 64 tokens (32 of 8 states).
@pytest.mark.parametrize("dtype,states", KINDS)
@pytest.mark.parametrize("length", [192, 203])
def test_whole_sequences_of_several_tiles(dtype, states, length):
    """groups of 36 channels: 32 and 4"""
    lens, channels, groups = [length] * 13, 360, 10
    assert slots_of(dtype, lens, channels, groups, states, False) == (13, False)
    check(dtype, lens, channels, groups, states, seed=17, packed=False)


@pytest.mark.parametrize("dtype,states", KINDS)
def test_equal_sequences_that_are_cut_into_slots_of_several_tiles(dtype, states):
    lens, channels, groups = [1003, 1003], 192, 48
    slots, cut = slots_of(dtype, lens, channels, groups, states, False)
    assert cut and 4 <= slots and sum(lens) / slots > 3 * 64
    check(dtype, lens, channels, groups, states, seed=18, packed=False)


@pytest.mark.parametrize("dtype,states", KINDS)
def test_packed_sequences_that_are_cut_into_slots_of_several_tiles(dtype, states):
    """sequences of several slots, of one that is full, of one and a token, of a part of one, and of nothing"""
    lens, channels, groups = [700, 0, 256, 257, 1000, 1, 192, 193, 100, 903], 240, 60
    slots, cut = slots_of(dtype, lens, channels, groups, states, True)
    run = sum(lens) // (slots - len(lens))      # (slots are tokens / run and one a sequence)
    assert cut and 3 * 64 <= run < 500
    check(dtype, lens, channels, groups, states, seed=19)


def test_packed_sequences_of_wide_groups():
    """every wave of a tile has channels"""
    lens, channels, groups = [500, 77, 0, 1001], 2048, 32
    slots, cut = slots_of("bf16", lens, channels, groups, 16, True)
    assert cut and 100 <= sum(lens) // (slots - len(lens)) < 500
    check("bf16", lens, channels, groups, 16, seed=20)

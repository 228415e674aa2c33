"""CPU-only: what include/msla_sequence.h says of the most that the scan and the convolution of a selective state space layer take.  Workspace sizes are asked for, and
single tokens are called with a state that is not there where they fit (which is refused behind the shape), so nothing touches a GPU."""
import ctypes
import os
import random

import pytest

from paper_2205_14756_amd import build as msla_build
from paper_2205_14756_amd import sequence as seq

OK, UNSUPPORTED = 0, -2
F32, BF16 = 0, 2
MOST = 1 << 23


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(msla_build.LIB):
        msla_build.build(True)
    return seq._lib()


def scan(lib, sequences, tokens, channels, groups, states, packed, backward, dt=BF16):
    n = ctypes.c_size_t(0)
    s = seq._Scan(sequences, tokens, 4 if packed else None, channels, groups, states, 1)
    return lib.msla_selective_scan_workspace_bytes(ctypes.byref(s), backward, dt, ctypes.byref(n))


def conv(lib, sequences, tokens, channels, width, packed, dt):
    n = ctypes.c_size_t(0)
    s = seq._Conv(sequences, tokens, 4 if packed else None, channels, width, 1)
    return lib.msla_causal_conv_backward_workspace_bytes(ctypes.byref(s), dt, ctypes.byref(n))


def scan_fits(sequences, tokens, channels, groups, states, backward):
    tile = 32 if states == 8 else 64
    return ((sequences + tokens / tile) * groups * -(-(channels // groups) // 32) < MOST and sequences * -(-channels * states // 256) < MOST and
            (not backward or tokens * groups * states < 1 << 30) and tokens < (1 << 31) - 4096)


def log(rng, low, high):
    return min(high, int(low * (high / low) ** rng.random()))


def test_scans_of_the_stated_sizes_are_taken(lib):
    rng, taken, refused = random.Random(1), 0, 0
    for _ in range(20000):
        groups, states = 1 << rng.randrange(10), rng.choice([8, 16, 32, 64])
        sequences, channels = log(rng, 1, 1 << 22), groups * log(rng, 1, (1 << 20) // groups)
        packed, backward = rng.random() < 0.5, rng.random() < 0.5
        tokens = log(rng, 1, (1 << 31) - 4097)
        if not packed:
            tokens = sequences * (tokens // sequences)
        got = scan(lib, sequences, tokens, channels, groups, states, packed, backward)
        if scan_fits(sequences, tokens, channels, groups, states, backward):
            assert got == OK, (sequences, tokens, channels, groups, states, packed, backward)
            taken += 1
        else:
            assert got in (OK, UNSUPPORTED)
            refused += got == UNSUPPORTED
    assert taken > 2000 and refused > 2000, (taken, refused)


@pytest.mark.parametrize("packed", [True, False])
def test_scans_beyond_them(lib, packed):
    assert scan(lib, 1, (1 << 24) - 64, 32, 1, 64, packed, 1) == OK
    assert scan(lib, 1, 1 << 24, 32, 1, 64, packed, 1) == UNSUPPORTED           # 2^30 states of d_b
    assert scan(lib, 1, 1 << 24, 32, 1, 64, packed, 0) == OK
    assert scan(lib, 1 << 18, 1 << 18, 1024, 1, 8, packed, 0) == UNSUPPORTED     # 2^18 sequences of 32 workgroups
    assert scan(lib, 1 << 17, 1 << 17, 1024, 1, 8, packed, 0) == OK


def test_single_tokens_beyond_them(lib):
    def step(sequences, channels):
        r = seq._Rows(1 << 20, channels)
        s = seq._Scan(sequences, sequences, None, channels, 1, 8, 1)
        return lib.msla_selective_scan_step(ctypes.byref(s), r, r, 1 << 20, r, r, None, None, seq._Rows(None, 0), 1 << 21, seq._Rows(1 << 22, channels), 1 << 21, BF16, None)
    # (what fits would run)
    assert step(1 << 22, 128) == step((1 << 17) + 1, 4096) == UNSUPPORTED


def test_convolutions_of_the_stated_sizes_are_taken(lib):
    rng, taken, refused = random.Random(2), 0, 0
    for _ in range(20000):
        sequences, channels, dt, packed = log(rng, 1, 1 << 23), log(rng, 1, 1 << 20), rng.choice([F32, BF16]), rng.random() < 0.5
        tokens = log(rng, 1, (1 << 31) - 4097)
        if not packed:
            tokens = sequences * (tokens // sequences)
        got = conv(lib, sequences, tokens, channels, rng.choice([2, 3, 4]), packed, dt)
        if (sequences + tokens / 32) * (channels * (4 if dt == F32 else 2) / 1024 + 2) < MOST:
            assert got == OK, (sequences, tokens, channels, dt, packed)
            taken += 1
        else:
            assert got in (OK, UNSUPPORTED)
            refused += got == UNSUPPORTED
    assert taken > 2000 and refused > 2000, (taken, refused)

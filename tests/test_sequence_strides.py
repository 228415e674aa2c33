"""CPU-only: how far apart the heads of a tile may lie.  A workgroup of the scan has 64 / head_dim state heads, and the 32-bit offset of a
lane reaches from the first row of the first one's operand to the last row of the last one's: with rows of ts bytes, heads of hs and
`group` query heads a state that is 63 ts + (64 / head_dim - 1) group hs + a head's row, which has to end before 2^32 - 16.

No call here gets as far as a launch: the workspace is a byte, so a call whose strides are in order is refused for that."""
import ctypes
import os

import pytest

from paper_2205_14756_amd import build as msla_build
from paper_2205_14756_amd import sequence

UNSUPPORTED, WORKSPACE = -2, -3
F32, F16, BF16 = 0, 1, 2
P = 1 << 20                     # stands for a buffer: no call here reads it

REACH = 2 ** 32 - 16
SIZE = {F32: 4, F16: 2, BF16: 2}


def widest(d, group, dt, ts, kv=4, rows=63):
    """the largest head stride (elements) that a lane's offset reaches, and the one above it"""
    e, others = SIZE[dt], min(64 // d, kv) - 1
    unit = 16 // e
    hs = (REACH - d * e - rows * ts * e) // (others * group * e) // unit * unit
    return min(hs, 2 ** 29 // e), hs + unit


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(msla_build.LIB):
        msla_build.build(True)
    return sequence._lib()


def call(lib, s, which, hs, ts, dt):
    """forward and backward with head stride hs at operand `which`: 0 q, 1 d_out, 2 k, 3 v.  (A forward of few tokens needs no workspace, and
    would be launched: not called.)"""
    at = lambda n, wide: sequence._Heads(n * P, ts, hs if wide else s.head_dim)
    q, d_out, k, v = (at(i + 1, which == i) for i in range(4))
    fresh = lambda n, heads: sequence._Heads(n * P, heads * s.head_dim, s.head_dim)
    back = lib.msla_recurrence_backward(ctypes.byref(s), q, k, v, None, 0, None, d_out, None, fresh(5, s.heads_q), fresh(6, s.heads_kv),
                                        fresh(7, s.heads_kv), None, 0, None, P, 1, dt, None)
    forth = lib.msla_recurrence_forward(ctypes.byref(s), q, k, v, None, 0, None, fresh(8, s.heads_q), None, P, 1, dt, None) if which != 1 and s.tokens > 64 else back
    return forth, back


def shape(d, group, kv=4, tokens=1 << 16):
    return sequence._Shape(1, tokens, None, kv * group, kv, d, 1.0, 0)


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("d,group", [(16, 3), (16, 4), (16, 16), (16, 512), (32, 9), (32, 16), (32, 256)])
@pytest.mark.parametrize("which", [0, 1])
def test_grouped_heads(lib, dt, d, group, which):
    for ts in (64, (2 ** 24 - 16) // SIZE[dt]):
        fits, beyond = widest(d, group, dt, ts)
        s = shape(d, group)
        assert call(lib, s, which, fits, ts, dt) == (WORKSPACE, WORKSPACE)
        assert call(lib, s, which, beyond, ts, dt) == (UNSUPPORTED, UNSUPPORTED)


def test_two_calls_that_read_other_rows(lib):
    """head-major maps of 12.5 million tokens, 16 heads over 4 states of 16; and of 3 million, 64 over 4"""
    assert call(lib, shape(16, 4), 0, 12_500_000 * 16, 16, BF16) == (UNSUPPORTED, UNSUPPORTED)
    assert call(lib, shape(16, 16), 1, 3_000_000 * 16, 16, BF16) == (UNSUPPORTED, UNSUPPORTED)


@pytest.mark.parametrize("dt", [F32, BF16])
def test_what_one_offset_reaches_is_taken(lib, dt):
    """a state head's own operands, ungrouped heads, heads of 64 and 128 (one to a workgroup) and a single state head"""
    e = SIZE[dt]
    top, ts = 2 ** 29 // e, (2 ** 24 - 16) // e
    for s, which in ((shape(16, 16), 2), (shape(32, 16), 3), (shape(16, 1), 0), (shape(32, 4), 0), (shape(64, 16), 0), (shape(128, 16), 1),
                     (shape(16, 16, kv=1), 0)):
        assert call(lib, s, which, top, ts, dt) == (WORKSPACE, WORKSPACE)
        assert call(lib, s, which, top + 16 // e, ts, dt) == (UNSUPPORTED, UNSUPPORTED)


def test_few_states_and_few_rows(lib):
    """two states of 16 have one between them, and eight tokens seven"""
    e, ts = 2, (2 ** 24 - 16) // 2
    fits, beyond = widest(16, 16, BF16, ts, kv=2)
    assert call(lib, shape(16, 16, kv=2), 0, fits, ts, BF16) == (WORKSPACE, WORKSPACE)
    assert call(lib, shape(16, 16, kv=2), 0, beyond, ts, BF16) == (UNSUPPORTED, UNSUPPORTED)
    fits, beyond = widest(16, 16, BF16, ts, rows=7)
    assert call(lib, shape(16, 16, tokens=8), 0, fits, ts, BF16) == (WORKSPACE, WORKSPACE)
    assert call(lib, shape(16, 16, tokens=8), 0, beyond, ts, BF16) == (UNSUPPORTED, UNSUPPORTED)

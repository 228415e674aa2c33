"""CPU-only checks of include/msla_sequence.h: every declared function is exported and bound, and bad arguments are refused on the
host before any launch (so none of these calls touches a GPU)."""
import ctypes
import os
import re

import pytest

from paper_2205_14756_amd import build as msla_build
from paper_2205_14756_amd import sequence

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
F32, F16, BF16 = 0, 1, 2
P = 1 << 20                     # stands for a buffer: no call here reads it


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(msla_build.LIB):
        msla_build.build(True)
    return sequence._lib()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "msla_sequence.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(msla_[a-z_]+)\s*\(", text))
    assert names == set(sequence.EXPORTS)
    for n in names:
        assert getattr(lib, n) is not None and callable(getattr(sequence, n))


def shape(**kw):
    s = dict(sequences=2, tokens=128, offsets=None, heads_q=4, heads_kv=2, head_dim=64, scale=0.125, rectify=0)
    s.update(kw)
    return sequence._Shape(*s.values())


def heads(p=P, ts=256, hs=64):
    return sequence._Heads(p, ts, hs)


def size_of(lib, s, backward=0, dt=F16):
    n = ctypes.c_size_t(77)
    st = lib.msla_recurrence_workspace_bytes(ctypes.byref(s), backward, dt, ctypes.byref(n))
    return st, n.value


BAD_SHAPES = [(dict(sequences=0), INVALID), (dict(sequences=-1), INVALID), (dict(tokens=-1), INVALID), (dict(tokens=127), INVALID),
              (dict(heads_q=0), INVALID), (dict(heads_kv=0), INVALID), (dict(heads_q=3), INVALID), (dict(head_dim=0), INVALID),
              (dict(head_dim=48), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED), (dict(scale=float("inf")), INVALID),
              (dict(scale=float("nan")), INVALID), (dict(rectify=2), INVALID), (dict(offsets=P + 2), INVALID),
              (dict(heads_q=1 << 16, heads_kv=1), UNSUPPORTED), (dict(tokens=1 << 32), UNSUPPORTED),
              (dict(sequences=1 << 21, tokens=1 << 21), UNSUPPORTED)]


@pytest.mark.parametrize("change,want", BAD_SHAPES)
def test_shapes_are_refused(lib, change, want):
    s = shape(**change)
    assert size_of(lib, s) == (want, 77)
    assert lib.msla_recurrence_forward(ctypes.byref(s), heads(), heads(), heads(), None, 0, None, heads(2 * P), None, P, 1 << 40, F16, None) == want
    assert lib.msla_recurrence_backward(ctypes.byref(s), heads(), heads(), heads(), None, 0, None, heads(), None, heads(2 * P), heads(3 * P),
                                        heads(4 * P), None, 0, None, P, 1 << 40, F16, None) == want
    if "offsets" not in change and "tokens" not in change and "sequences" not in change:
        s.sequences, s.tokens = 128, 128
        assert lib.msla_recurrence_step(ctypes.byref(s), heads(), heads(), heads(), None, 0, P, heads(2 * P), 3 * P, F16, None) == want


def test_workspace_sizes(lib):
    assert size_of(lib, shape()) == (OK, 0)                                     # two short sequences: nothing is cut
    st, n = size_of(lib, shape(sequences=1, tokens=65536, heads_q=2, heads_kv=2, head_dim=128))
    assert st == OK and n >= 65536 // 1024 * 2 * 128 * 128 * 4
    st, more = size_of(lib, shape(sequences=1, tokens=65536, heads_q=2, heads_kv=2, head_dim=128), backward=1)
    assert st == OK and more > 2 * n
    assert size_of(lib, shape(), dt=3) == (INVALID, 77)
    assert lib.msla_recurrence_workspace_bytes(ctypes.byref(shape()), 0, F16, None) == INVALID
    assert lib.msla_recurrence_workspace_bytes(None, 0, F16, ctypes.byref(ctypes.c_size_t())) == INVALID
    big = shape(sequences=1, tokens=65536, heads_q=2, heads_kv=2, head_dim=128)
    h = heads(ts=256, hs=128)
    assert lib.msla_recurrence_forward(ctypes.byref(big), h, h, h, None, 0, None, heads(2 * P, 256, 128), None, P, n - 1, F16, None) == WORKSPACE
    assert lib.msla_recurrence_forward(ctypes.byref(big), h, h, h, None, 0, None, heads(2 * P, 256, 128), None, None, n, F16, None) == INVALID
    assert lib.msla_recurrence_forward(ctypes.byref(big), h, h, h, None, 0, None, heads(2 * P, 256, 128), None, P + 8, n, F16, None) == INVALID


BAD_HEADS = [heads(None), heads(P + 8), heads(ts=-256), heads(hs=-64), heads(ts=252), heads(hs=68), heads(ts=1 << 60)]


@pytest.mark.parametrize("bad", range(len(BAD_HEADS)))
@pytest.mark.parametrize("place", range(4))
def test_operands_are_refused(lib, bad, place):
    s = shape()
    args = [heads(), heads(2 * P), heads(3 * P), heads(4 * P)]
    args[place] = BAD_HEADS[bad]
    q, k, v, o = args
    assert lib.msla_recurrence_forward(ctypes.byref(s), q, k, v, None, 0, None, o, None, None, 0, F16, None) == INVALID
    for t in range(3):
        outs = [heads(5 * P), heads(6 * P), heads(7 * P)]
        outs[t] = BAD_HEADS[bad]
        assert lib.msla_recurrence_backward(ctypes.byref(s), heads(), heads(2 * P), heads(3 * P), None, 0, None, heads(4 * P), None, *outs, None, 0,
                                            None, P, 1 << 40, F16, None) == INVALID


def test_outputs_that_overlap_are_refused(lib):
    s = shape()
    f = lambda o, **kw: lib.msla_recurrence_forward(ctypes.byref(s), heads(), heads(2 * P), heads(3 * P), None, 0, None, o, None, None, 0, F16, None)
    assert f(heads()) == f(heads(2 * P)) == f(heads(3 * P)) == INVALID                  # an input itself
    assert f(heads(4 * P, ts=0)) == f(heads(4 * P, hs=0)) == f(heads(4 * P, ts=128)) == INVALID
    assert f(heads(4 * P, ts=64, hs=64 * 127)) == INVALID                               # head-major, one row short
    b = lambda *outs, **kw: lib.msla_recurrence_backward(ctypes.byref(s), heads(), heads(2 * P), heads(3 * P), kw.get("g"), 2, None, heads(4 * P), None,
                                                         *outs, kw.get("dg"), kw.get("dgs", 2), kw.get("di"), P, kw.get("n", 1 << 40), F16, None)
    x, y, z = heads(5 * P), heads(6 * P), heads(7 * P)
    assert b(x, x, z) == b(x, y, x) == b(x, y, y) == b(heads(4 * P), y, z) == INVALID
    assert b(x, y, z, dg=P) == INVALID                                                  # no gate, yet its gradient
    assert b(x, y, z, g=P, dg=2 * P, dgs=1) == b(x, y, z, g=P + 1) == INVALID
    assert b(x, y, z, di=P + 4) == INVALID
    assert b(x, y, z, n=64) == WORKSPACE


def test_the_state_s_gradient_has_a_place_of_its_own(lib):
    s = shape()
    for first, d_last in ((8 * P, None), (None, 8 * P), (8 * P, 8 * P)):
        st = lib.msla_recurrence_backward(ctypes.byref(s), heads(), heads(2 * P), heads(3 * P), None, 0, first, heads(4 * P), d_last, heads(5 * P),
                                          heads(6 * P), heads(7 * P), None, 0, 8 * P, P, 1 << 40, F16, None)
        assert st == INVALID


def test_step_is_refused(lib):
    f = lambda s, state=P, new=2 * P, dt=F16: lib.msla_recurrence_step(ctypes.byref(s), heads(), heads(2 * P), heads(3 * P), None, 0, state,
                                                                       heads(4 * P), new, dt, None)
    one = dict(sequences=128)
    assert f(shape()) == INVALID                                                        # two tokens to a sequence
    assert f(shape(**one), new=None) == f(shape(**one), new=P + 4) == f(shape(**one), state=P + 4) == f(shape(**one), dt=7) == INVALID
    assert f(shape(offsets=P, **one)) == INVALID


def test_norm_is_refused(lib):
    n = lambda x=P, res=None, w=None, y=2 * P, s=None, rows=4, ch=64, eps=1e-6, dt=F16: lib.msla_norm_forward(x, res, w, y, s, rows, ch, eps, dt, None)
    for kw in (dict(x=None), dict(y=None), dict(rows=-1), dict(ch=0), dict(ch=-4), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(dt=3), dict(x=P + 1), dict(res=P + 1), dict(w=P + 1), dict(y=P + 1), dict(s=P + 1), dict(s=2 * P), dict(res=2 * P)):
        assert n(**kw) == INVALID, kw
    assert n(ch=32769) == n(rows=1 << 31) == UNSUPPORTED
    assert n(rows=0) == OK
    q = lambda x=P, y=2 * P, sc=3 * P, **kw: lib.msla_norm_quantized(x, None, None, y, sc, None, kw.get("rows", 4), 64, 1e-6, F16, None)
    assert q(sc=None) == q(sc=P + 2) == q(y=P) == q(y=None) == q(x=None) == INVALID
    r = lambda x=P, y=2 * P, sc=3 * P, dt=F16: lib.msla_quantize_rows(x, y, sc, 4, 64, dt, None)
    assert r(sc=None) == r(y=P) == r(x=None) == r(dt=9) == INVALID
    b = lambda s=P, dy=2 * P, dr=3 * P, dw=4 * P, ws=5 * P, nb=1 << 30, rows=4, ch=64, eps=0.0, dt=F16: lib.msla_norm_backward(
        s, None, dy, None, dr, dw, ws, nb, rows, ch, eps, dt, None)
    assert b(s=None) == b(dy=None) == b(dr=None) == b(dr=P) == b(ws=None) == b(ws=P + 8) == b(dw=P + 2) == b(rows=-1) == b(eps=-1.0) == INVALID
    assert b(nb=64) == WORKSPACE
    size = ctypes.c_size_t(5)
    assert lib.msla_norm_backward_workspace_bytes(4, 0, F16, ctypes.byref(size)) == INVALID and size.value == 5
    assert lib.msla_norm_backward_workspace_bytes(4, 64, F16, None) == INVALID
    assert lib.msla_norm_backward_workspace_bytes(4, 64, F16, ctypes.byref(size)) == OK and size.value >= 256


def test_linear_quantized_is_refused(lib):
    f = lambda x=P, sx=2 * P, w=3 * P, sw=4 * P, y=5 * P, rows=4, i=64, o=32, dt=F16: lib.msla_linear_quantized(x, sx, w, sw, y, rows, i, o, dt, None)
    for kw in (dict(x=None), dict(sx=None), dict(w=None), dict(sw=None), dict(y=None), dict(rows=-1), dict(i=0), dict(o=0), dict(dt=3), dict(x=P + 8),
               dict(w=P + 8), dict(y=P + 8), dict(sx=P + 2), dict(sw=P + 2), dict(y=P), dict(y=3 * P)):
        assert f(**kw) == INVALID, kw
    assert f(i=40) == f(o=40) == f(rows=1 << 31) == UNSUPPORTED
    assert f(rows=0) == OK


def test_the_binding_refuses_what_is_not_on_the_gpu():
    import torch
    x = torch.zeros(4, 2, 16, dtype=torch.float16)
    with pytest.raises(ValueError):
        sequence.msla_recurrence_forward(x, x, x)
    with pytest.raises(ValueError):
        sequence.msla_norm_forward(x)
    with pytest.raises(ValueError):
        sequence.msla_quantize_rows(x)


def test_rows_of_strided_heads():
    import torch
    m = torch.zeros(2, 5, 3, 3, 16)
    h, n = sequence._rows(m[:, :, :, 1], "q")
    assert n == 10 and (h.token_stride, h.head_stride) == (144, 48) and h.data == m.data_ptr() + 64
    h, n = sequence._rows(torch.zeros(3, 10, 16).transpose(0, 1), "q")                  # head-major
    assert n == 10 and (h.token_stride, h.head_stride) == (16, 160)
    h, n = sequence._rows(torch.zeros(10, 1, 16).expand(10, 4, 16), "k")                # one head for four
    assert n == 10 and (h.token_stride, h.head_stride) == (16, 0)
    with pytest.raises(ValueError):
        sequence._rows(torch.zeros(2, 6, 3, 16)[:, :5], "q")                            # a gap between the sequences
    with pytest.raises(ValueError):
        sequence._rows(torch.zeros(4, 3, 32)[..., ::2], "q")

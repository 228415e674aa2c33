"""Thin ctypes binding of the sequence operators of libmsla.so (the C ABI of include/msla_sequence.h).

The linear attention of Eq. (3) as a running state over a sequence, the root-mean-square norm with the residual's addition, and
the projection of rows in 8 bits.  Like ``msla``: argument marshalling only, no CPU fallback, tensors on the current GPU, work on
its current stream unless one is given.  Buffers that are not passed in are allocated here with torch, for the stream that they are
used on.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import msla as _msla
from .msla import MSLA_OK, MslaError, _DTYPES, _ptr, _stream

EXPORTS = ("msla_recurrence_workspace_bytes", "msla_recurrence_forward", "msla_recurrence_backward", "msla_recurrence_step",
           "msla_norm_forward", "msla_norm_quantized", "msla_norm_backward_workspace_bytes", "msla_norm_backward", "msla_quantize_rows",
           "msla_linear_quantized")

HEAD_DIMS = (16, 32, 64, 128)


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _Shape(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int), ("tokens", ctypes.c_int64), ("offsets", ctypes.c_void_p), ("heads_q", ctypes.c_int),
                ("heads_kv", ctypes.c_int), ("head_dim", ctypes.c_int), ("scale", ctypes.c_float), ("rectify", ctypes.c_int)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = _msla.load_library()
        vp, i, i64, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        shape, size = ctypes.POINTER(_Shape), ctypes.POINTER(sz)
        lib.msla_recurrence_workspace_bytes.argtypes = [shape, i, i, size]
        lib.msla_recurrence_forward.argtypes = [shape, _Heads, _Heads, _Heads, vp, i64, vp, _Heads, vp, vp, sz, i, vp]
        lib.msla_recurrence_backward.argtypes = [shape, _Heads, _Heads, _Heads, vp, i64, vp, _Heads, vp, _Heads, _Heads, _Heads, vp, i64, vp,
                                                 vp, sz, i, vp]
        lib.msla_recurrence_step.argtypes = [shape, _Heads, _Heads, _Heads, vp, i64, vp, _Heads, vp, i, vp]
        lib.msla_norm_forward.argtypes = [vp, vp, vp, vp, vp, i64, i, f, i, vp]
        lib.msla_norm_quantized.argtypes = [vp, vp, vp, vp, vp, vp, i64, i, f, i, vp]
        lib.msla_norm_backward_workspace_bytes.argtypes = [i64, i, i, size]
        lib.msla_norm_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, sz, i64, i, f, i, vp]
        lib.msla_quantize_rows.argtypes = [vp, vp, vp, i64, i, i, vp]
        lib.msla_linear_quantized.argtypes = [vp, vp, vp, vp, vp, i64, i, i, i, vp]
        for name in EXPORTS:
            getattr(lib, name).restype = i
        _ready = lib
    return _ready


def _check(status, where):
    if status != MSLA_OK:
        raise MslaError(status, where)


def _refuse(what):
    raise ValueError("msla: " + what)


# Small calls wait for the host (a call on one token is some us on the GPU), so the checks below are made of few attribute reads: contiguous
# operands, which most are, are recognised by one, and shapes are compared as they come.
_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on_gpu(*tensors):
    """All on the current device (whose stream the work goes to)."""
    here = -1
    for t in tensors:
        if t is not None:
            at = t.get_device()
            if at != here or at < 0:
                if not (at >= 0 and t.is_cuda):
                    _refuse("tensors must live in GPU memory")
                if at != _device():
                    _refuse("tensors must live on the current device")
                here = at


def _new(like, stream, shape=None, dtype=None):
    """Memory for a call on ``stream``: of that stream, so that it is not handed on before the call's work is done."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return _new(like, None, shape, dtype)
    if shape is None:
        return torch.empty_like(like) if dtype is None else torch.empty_like(like, dtype=dtype)
    return like.new_empty(shape, dtype=dtype)


def _plain(t, name, shape, dtype):
    if t is not None and not (t.shape == shape and t.dtype == dtype and t.is_contiguous()):
        if not t.is_contiguous():
            _refuse(f"{name} must be contiguous")
        if not (tuple(t.shape) == tuple(shape)):
            _refuse(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
        if not (t.dtype == dtype):
            _refuse(f"{name} must be {dtype}, not {t.dtype}")


def _rows(t, name, like=None):
    """A [..., heads, head_dim] tensor as rows of tokens: (data, token stride, head stride), tokens in order."""
    shape = t.shape
    if like is not None and shape != like:
        _refuse(f"{name} must have the shape {tuple(like)}, not {tuple(shape)}")
    if not (len(shape) >= 3):
        _refuse(f"{name} must be [..., heads, head_dim]")
    heads, dim = shape[-2:]
    if t.is_contiguous():
        row = heads * dim
        return _Heads(t.data_ptr(), row, dim), t.numel() // row if row else 0
    strides = t.stride()
    if not (strides[-1] == 1 or dim == 1):
        _refuse(f"{name}'s channels must lie next to each other")
    tokens, step = 1, strides[-3]
    for size, stride in zip(shape[-3::-1], strides[-3::-1]):
        if not (size == 1 or tokens == 1 or stride == step * tokens):
            _refuse(f"{name}'s tokens must lie at equal distances")
        if tokens == 1 and size != 1:
            step = stride
        tokens *= size
    # (the stride of an axis of length one says nothing, and torch leaves anything there)
    return _Heads(t.data_ptr(), step if tokens > 1 else 0, strides[-2] if heads > 1 else 0), tokens


def _gate(t, tokens, heads, dtype, name):
    if t is None:
        return None, 0
    if not (t.dtype == dtype):
        _refuse(f"{name} must be {dtype}, not {t.dtype}")
    if not (t.shape[-1] == heads and t.numel() == tokens * heads):
        _refuse(f"{name} must be [..., heads_kv]")
    if t.is_contiguous():
        return t.data_ptr(), heads
    try:
        flat = t if t.dim() == 2 else t.view(-1, heads)
    except RuntimeError:
        _refuse(f"{name}'s tokens must lie at equal distances")
    if not (heads == 1 or flat.stride(1) == 1):
        _refuse(f"{name}'s heads must lie next to each other")
    return flat.data_ptr(), flat.stride(0) if tokens > 1 else heads


class _Call:
    """The arguments that forward, backward and step share, checked."""
    __slots__ = ("q", "k", "v", "gate", "gate_stride", "tokens", "heads_kv", "shape", "dt", "state_shape")

    def __init__(self, q, k, v, log_gate, sequences, offsets, scale, rectify):
        dtype = q.dtype
        self.dt = dt = _DTYPES.get(dtype)
        if dt is None:
            _refuse(f"{dtype} is not a storage type")
        if not (dtype == k.dtype and dtype == v.dtype):
            _refuse("q, k and v must have one type")
        kv = k.shape
        self.q, tokens = _rows(q, "q")
        self.k, tokens_k = _rows(k, "k")
        if not (tokens_k == tokens):
            _refuse("q and k must have the same tokens")
        self.v, _ = _rows(v, "v", kv)
        heads_q, head_dim = q.shape[-2:]
        heads_kv = kv[-2]
        if not (kv[-1] == head_dim):
            _refuse("q and k must have the same head_dim")
        if offsets is not None:
            if not (offsets.dtype == torch.int32 and offsets.dim() == 1 and offsets.is_contiguous() and offsets.numel() >= 2):
                _refuse("offsets must be int32 [sequences + 1]")
            if not (sequences is None or sequences == offsets.numel() - 1):
                _refuse("offsets must be int32 [sequences + 1]")
            sequences = offsets.numel() - 1
            offsets = offsets.data_ptr()
        elif sequences is None:
            sequences = q.shape[0] if q.dim() == 4 else 1
        self.gate, self.gate_stride = _gate(log_gate, tokens, heads_kv, dtype, "log_gate")
        self.tokens, self.heads_kv = tokens, heads_kv
        self.shape = _Shape(int(sequences), tokens, offsets, heads_q, heads_kv, head_dim, head_dim ** -0.5 if scale is None else scale,
                            1 if rectify else 0)
        self.state_shape = (sequences, heads_kv, head_dim, head_dim)

    def workspace(self, given, backward, like, stream):
        if given is not None:
            if not (given.is_contiguous() and given.dtype == torch.uint8):
                _refuse("the workspace must be contiguous bytes")
            return given
        size = ctypes.c_size_t(0)
        _check(_lib().msla_recurrence_workspace_bytes(self.shape, backward, self.dt, size), "msla_recurrence_workspace_bytes")
        return _new(like, stream, size.value, torch.uint8) if size.value else None


def msla_recurrence_workspace_bytes(sequences, tokens, heads_q, heads_kv, head_dim, dtype, packed=False, backward=False) -> int:
    """Bytes that msla_recurrence_forward (or _backward) needs; packed: with offsets."""
    shape = _Shape(sequences, tokens, 4 if packed else None, heads_q, heads_kv, head_dim, 1.0, 0)
    size = ctypes.c_size_t(0)
    _check(_lib().msla_recurrence_workspace_bytes(shape, int(backward), _DTYPES[dtype], size),
           "msla_recurrence_workspace_bytes")
    return int(size.value)


def msla_recurrence_forward(q, k, v, log_gate=None, sequences: Optional[int] = None, offsets=None, initial_state=None, scale=None,
                            rectify=False, out=None, final_state=None, workspace=None, stream=None):
    """S_i = exp(log_gate_i) S_{i-1} + k_i v_i^T, out_i = scale q_i^T S_i over every sequence and head.

    q [..., heads_q, d], k and v [..., heads_kv, d], any strides over tokens and heads (so parts of a projected map will do); log_gate
    [..., heads_kv] in the same type.  The tokens are those of ``sequences`` equally long sequences (by default q.shape[0] of a
    four-dimensional q, else one), or of sequences packed behind each other that start at ``offsets`` (int32, on the GPU, one more than
    sequences).  scale: d ** -0.5 by default; rectify: max(., 0) of q and k.  Returns (out, final_state [sequences, heads_kv, d, d] fp32);
    rows that belong to no sequence are left as they are in a given ``out``."""
    _on_gpu(q, k, v, log_gate, offsets, initial_state, out, final_state, workspace)
    c = _Call(q, k, v, log_gate, sequences, offsets, scale, rectify)
    _plain(initial_state, "initial_state", c.state_shape, torch.float32)
    _plain(final_state, "final_state", c.state_shape, torch.float32)
    if out is None:
        out = _new(q, stream)
    elif not (out.dtype == q.dtype):
        _refuse("out must have q's type")
    o, _ = _rows(out, "out", q.shape)
    if final_state is None:
        final_state = _new(q, stream, c.state_shape, torch.float32)
    ws = c.workspace(workspace, 0, q, stream)
    _check(_lib().msla_recurrence_forward(c.shape, c.q, c.k, c.v, c.gate, c.gate_stride, _ptr(initial_state), o,
                                          _ptr(final_state), _ptr(ws), 0 if ws is None else ws.numel(), c.dt, _stream(stream)),
           "msla_recurrence_forward")
    return out, final_state


def msla_recurrence_backward(q, k, v, d_out, log_gate=None, sequences: Optional[int] = None, offsets=None, initial_state=None,
                             d_final_state=None, scale=None, rectify=False, d_q=None, d_k=None, d_v=None, d_log_gate=None,
                             d_initial_state=None, workspace=None, stream=None):
    """The gradient of msla_recurrence_forward: (d_q, d_k, d_v, d_log_gate, d_initial_state), the last two None where log_gate or
    initial_state is."""
    _on_gpu(q, k, v, d_out, log_gate, offsets, initial_state, d_final_state, d_q, d_k, d_v, d_log_gate, d_initial_state, workspace)
    c = _Call(q, k, v, log_gate, sequences, offsets, scale, rectify)
    _plain(initial_state, "initial_state", c.state_shape, torch.float32)
    _plain(d_final_state, "d_final_state", c.state_shape, torch.float32)
    _plain(d_initial_state, "d_initial_state", c.state_shape, torch.float32)
    if not (d_out.dtype == q.dtype):
        _refuse("d_out must have q's type")
    do, _ = _rows(d_out, "d_out", q.shape)
    grads = []
    for t, like, name in ((d_q, q, "d_q"), (d_k, k, "d_k"), (d_v, v, "d_v")):
        if t is None:
            t = _new(like, stream)
        if not (t.dtype == q.dtype):
            _refuse(f"{name} must have q's type")
        grads.append((t, _rows(t, name, like.shape)[0]))
    if not (log_gate is not None or d_log_gate is None):
        _refuse("d_log_gate needs a log_gate")
    if d_log_gate is None and log_gate is not None:
        d_log_gate = _new(log_gate, stream, log_gate.shape)
    dg, dg_stride = _gate(d_log_gate, c.tokens, c.heads_kv, q.dtype, "d_log_gate")
    if d_initial_state is None and initial_state is not None:
        d_initial_state = _new(q, stream, c.state_shape, torch.float32)
    ws = c.workspace(workspace, 1, q, stream)
    _check(_lib().msla_recurrence_backward(c.shape, c.q, c.k, c.v, c.gate, c.gate_stride, _ptr(initial_state), do,
                                           _ptr(d_final_state), grads[0][1], grads[1][1], grads[2][1], dg, dg_stride,
                                           _ptr(d_initial_state), _ptr(ws), 0 if ws is None else ws.numel(), c.dt, _stream(stream)),
           "msla_recurrence_backward")
    return grads[0][0], grads[1][0], grads[2][0], d_log_gate, d_initial_state


def msla_recurrence_step(q, k, v, state, log_gate=None, scale=None, rectify=False, out=None, new_state=None, stream=None):
    """One token for each of q.shape[0] sequences: q [sequences, heads_q, d], k and v [sequences, heads_kv, d], state [sequences,
    heads_kv, d, d] fp32.  The state is updated in place unless new_state is given.  Returns (out, new_state)."""
    if new_state is None:
        new_state = state
    _on_gpu(q, k, v, state, log_gate, out, new_state)
    if not (q.dim() == 3):
        _refuse("q must be [sequences, heads_q, head_dim]")
    c = _Call(q, k, v, log_gate, q.shape[0], None, scale, rectify)
    _plain(state, "state", c.state_shape, torch.float32)
    if new_state is not state:
        _plain(new_state, "new_state", c.state_shape, torch.float32)
    if out is None:
        out = _new(q, stream)
    elif not (out.dtype == q.dtype):
        _refuse("out must have q's type")
    o, _ = _rows(out, "out", q.shape)
    _check(_lib().msla_recurrence_step(c.shape, c.q, c.k, c.v, c.gate, c.gate_stride, _ptr(state), o, _ptr(new_state), c.dt,
                                       _stream(stream)), "msla_recurrence_step")
    return out, new_state


def _norm_arguments(x, weight, residual, total, names=("x", "residual", "sum_out")):
    _on_gpu(x, weight, residual, total)
    if not (x.dtype in _DTYPES):
        _refuse(f"{x.dtype} is not a storage type")
    if not (x.dim() >= 1 and x.is_contiguous()):
        _refuse(f"{names[0]} must be contiguous rows")
    shape = x.shape
    channels = shape[-1]
    if weight is not None:
        _plain(weight, "weight", (channels,), x.dtype)
    if residual is not None:
        _plain(residual, names[1], shape, x.dtype)
    if total is not None:
        _plain(total, names[2], shape, x.dtype)
    return x.numel() // channels if channels else 0, channels


def msla_norm_forward(x, weight=None, residual=None, eps=1e-6, out=None, sum_out=None, stream=None):
    """(y, r): r = x + residual, y = r / sqrt(mean(r^2) + eps) * weight over the last axis.  Without a residual r is x itself and is not
    written, unless sum_out is given."""
    rows, channels = _norm_arguments(x, weight, residual, sum_out)
    if out is None:
        out = _new(x, stream)
    else:
        _on_gpu(out)
        _plain(out, "out", x.shape, x.dtype)
    if sum_out is None and residual is not None:
        sum_out = _new(x, stream)
    _check(_lib().msla_norm_forward(_ptr(x), _ptr(residual), _ptr(weight), _ptr(out), _ptr(sum_out), rows, channels, float(eps),
                                    _DTYPES[x.dtype], _stream(stream)), "msla_norm_forward")
    return out, x if sum_out is None else sum_out


def _rows8(x, out8, scale, stream):
    if out8 is None:
        out8 = _new(x, stream, None, torch.float8_e4m3fn)
    else:
        _on_gpu(out8)
        _plain(out8, "out8", x.shape, torch.float8_e4m3fn)
    if scale is None:
        scale = _new(x, stream, x.shape[:-1], torch.float32)
    else:
        _on_gpu(scale)
        _plain(scale, "scale", x.shape[:-1], torch.float32)
    return out8, scale


def msla_norm_quantized(x, weight=None, residual=None, eps=1e-6, out8=None, scale=None, sum_out=None, stream=None):
    """(y8, scale, r): msla_norm_forward with y as e4m3 rows, y ~ y8 * scale[..., None]."""
    rows, channels = _norm_arguments(x, weight, residual, sum_out)
    out8, scale = _rows8(x, out8, scale, stream)
    if sum_out is None and residual is not None:
        sum_out = _new(x, stream)
    _check(_lib().msla_norm_quantized(_ptr(x), _ptr(residual), _ptr(weight), _ptr(out8), _ptr(scale), _ptr(sum_out), rows, channels,
                                      float(eps), _DTYPES[x.dtype], _stream(stream)), "msla_norm_quantized")
    return out8, scale, x if sum_out is None else sum_out


def msla_quantize_rows(x, out8=None, scale=None, stream=None):
    """(x8, scale): rows of x as e4m3, x ~ x8 * scale[..., None]."""
    rows, channels = _norm_arguments(x, None, None, None)
    out8, scale = _rows8(x, out8, scale, stream)
    _check(_lib().msla_quantize_rows(_ptr(x), _ptr(out8), _ptr(scale), rows, channels, _DTYPES[x.dtype], _stream(stream)),
           "msla_quantize_rows")
    return out8, scale


def msla_norm_backward_workspace_bytes(rows, channels, dtype) -> int:
    size = ctypes.c_size_t(0)
    _check(_lib().msla_norm_backward_workspace_bytes(rows, channels, _DTYPES[dtype], size),
           "msla_norm_backward_workspace_bytes")
    return int(size.value)


def msla_norm_backward(r, weight, d_y, d_sum=None, eps=1e-6, d_r=None, d_weight=None, workspace=None, stream=None):
    """(d_r, d_weight): the gradient of msla_norm_forward at r (what it returned); d_sum: the gradient that reaches r past the norm.
    d_r is that of x and of residual alike; d_weight is fp32."""
    rows, channels = _norm_arguments(r, weight, d_y, d_sum, ("r", "d_y", "d_sum"))
    _on_gpu(d_r, d_weight, workspace)
    _plain(d_r, "d_r", r.shape, r.dtype)
    _plain(d_weight, "d_weight", (channels,), torch.float32)
    if d_r is None:
        d_r = _new(r, stream)
    if d_weight is None:
        d_weight = _new(r, stream, channels, torch.float32)
    if workspace is None:
        workspace = _new(r, stream, msla_norm_backward_workspace_bytes(rows, channels, r.dtype), torch.uint8)
    else:
        if not (workspace.is_contiguous() and workspace.dtype == torch.uint8):
            _refuse("the workspace must be contiguous bytes")
    _check(_lib().msla_norm_backward(_ptr(r), _ptr(weight), _ptr(d_y), _ptr(d_sum), _ptr(d_r), _ptr(d_weight), _ptr(workspace),
                                     workspace.numel(), rows, channels, float(eps), _DTYPES[r.dtype], _stream(stream)),
           "msla_norm_backward")
    return d_r, d_weight


def msla_linear_quantized(x8, x_scale, w8, w_scale, dtype=torch.bfloat16, out=None, stream=None):
    """y[..., o] = x_scale[...] * w_scale[o] * sum_c x8[..., c] * w8[o, c]: x8, w8 e4m3, scales fp32, y in ``dtype`` (out's, if given)."""
    _on_gpu(x8, x_scale, w8, w_scale, out)
    shape = x8.shape
    if not (w8.dim() == 2 and len(shape) >= 1 and shape[-1] == w8.shape[1]):
        _refuse("x8 must be [..., c_in] and w8 [c_out, c_in]")
    c_out, c_in = w8.shape
    _plain(x8, "x8", shape, torch.float8_e4m3fn)
    _plain(w8, "w8", (c_out, c_in), torch.float8_e4m3fn)
    _plain(x_scale, "x_scale", shape[:-1], torch.float32)
    _plain(w_scale, "w_scale", (c_out,), torch.float32)
    if out is not None:
        dtype = out.dtype
    dt = _DTYPES.get(dtype)
    if dt is None:
        _refuse(f"{dtype} is not a storage type")
    to = shape[:-1] + (c_out,)
    if out is None:
        out = _new(x8, stream, to, dtype)
    else:
        _plain(out, "out", to, dtype)
    rows = x8.numel() // c_in if c_in else 0
    _check(_lib().msla_linear_quantized(x8.data_ptr(), x_scale.data_ptr(), w8.data_ptr(), w_scale.data_ptr(), out.data_ptr(), rows, c_in, c_out, dt,
                                        _stream(stream)), "msla_linear_quantized")
    return out

"""Thin ctypes binding of the sequence operators of libmsla.so (the C ABI of include/msla_sequence.h).

The linear attention of Eq. (3) as a running state over a sequence, the root-mean-square norm with the residual's addition, and
the projection of rows in 8 bits; the scan with a decay for each state, the short causal convolution in front of it, layer norm, and the
projection in 8-bit integers.  Like ``msla``: argument marshalling only, no CPU fallback, tensors on the current GPU, work on
its current stream unless one is given.  Buffers that are not passed in are allocated here with torch, for the stream that they are
used on.
"""
from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

import torch

from . import msla as _msla
from .msla import MSLA_OK, MslaError, _DTYPES, _ptr, _stream

EXPORTS = ("msla_recurrence_workspace_bytes", "msla_recurrence_forward", "msla_recurrence_backward", "msla_recurrence_step",
           "msla_norm_forward", "msla_norm_quantized", "msla_norm_backward_workspace_bytes", "msla_norm_backward", "msla_quantize_rows",
           "msla_linear_quantized",
           "msla_selective_scan_workspace_bytes", "msla_selective_scan_forward", "msla_selective_scan_backward", "msla_selective_scan_step",
           "msla_causal_conv_forward", "msla_causal_conv_backward_workspace_bytes", "msla_causal_conv_backward", "msla_causal_conv_step",
           "msla_layer_norm_forward", "msla_layer_norm_backward_workspace_bytes", "msla_layer_norm_backward", "msla_quantize_rows_integer",
           "msla_linear_integer")

HEAD_DIMS = (16, 32, 64, 128)


class _Heads(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class _Shape(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int), ("tokens", ctypes.c_int64), ("offsets", ctypes.c_void_p), ("heads_q", ctypes.c_int),
                ("heads_kv", ctypes.c_int), ("head_dim", ctypes.c_int), ("scale", ctypes.c_float), ("rectify", ctypes.c_int)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64)]


class _Scan(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int), ("tokens", ctypes.c_int64), ("offsets", ctypes.c_void_p), ("channels", ctypes.c_int),
                ("groups", ctypes.c_int), ("states", ctypes.c_int), ("softplus", ctypes.c_int)]


class _Conv(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int), ("tokens", ctypes.c_int64), ("offsets", ctypes.c_void_p), ("channels", ctypes.c_int),
                ("width", ctypes.c_int), ("silu", ctypes.c_int)]


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
        scan, conv, rows = ctypes.POINTER(_Scan), ctypes.POINTER(_Conv), _Rows
        lib.msla_selective_scan_workspace_bytes.argtypes = [scan, i, i, size]
        lib.msla_selective_scan_forward.argtypes = [scan, rows, rows, vp, rows, rows, vp, vp, rows, vp, rows, vp, vp, sz, i, vp]
        lib.msla_selective_scan_backward.argtypes = [scan, rows, rows, vp, rows, rows, vp, vp, rows, vp, rows, vp, rows, rows, vp, rows, rows, vp,
                                                     vp, rows, vp, vp, sz, i, vp]
        lib.msla_selective_scan_step.argtypes = [scan, rows, rows, vp, rows, rows, vp, vp, rows, vp, rows, vp, i, vp]
        lib.msla_causal_conv_forward.argtypes = [conv, rows, vp, vp, vp, rows, vp, i, vp]
        lib.msla_causal_conv_backward_workspace_bytes.argtypes = [conv, i, size]
        lib.msla_causal_conv_backward.argtypes = [conv, rows, vp, vp, vp, rows, vp, rows, vp, vp, vp, vp, sz, i, vp]
        lib.msla_causal_conv_step.argtypes = [conv, rows, vp, vp, vp, rows, vp, i, vp]
        lib.msla_layer_norm_forward.argtypes = [vp, vp, vp, vp, vp, vp, i64, i, f, i, vp]
        lib.msla_layer_norm_backward_workspace_bytes.argtypes = [i64, i, i, size]
        lib.msla_layer_norm_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, sz, i64, i, f, i, vp]
        lib.msla_quantize_rows_integer.argtypes = [vp, vp, vp, i64, i, i, vp]
        lib.msla_linear_integer.argtypes = [vp, vp, vp, vp, vp, i64, i, i, i, vp]
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


# ------------------------------------------------------------------------------------------------ a selective state space layer
def _tokens(t, name, dtype, like=None):
    """A [..., channels] tensor as rows of tokens: (data and token stride, tokens in order)."""
    shape = t.shape
    if t.dtype != dtype:
        _refuse(f"{name} must be {dtype}, not {t.dtype}")
    if like is not None and shape != like:
        _refuse(f"{name} must have the shape {tuple(like)}, not {tuple(shape)}")
    if not (len(shape) >= 2):
        _refuse(f"{name} must be [..., channels]")
    channels = shape[-1]
    if t.is_contiguous():
        return _Rows(t.data_ptr(), channels), t.numel() // channels if channels else 0
    strides = t.stride()
    if not (strides[-1] == 1 or channels == 1):
        _refuse(f"{name}'s channels must lie next to each other")
    tokens, step = 1, strides[-2]
    for size, stride in zip(shape[-2::-1], strides[-2::-1]):
        if not (size == 1 or tokens == 1 or stride == step * tokens):
            _refuse(f"{name}'s tokens must lie at equal distances")
        if tokens == 1 and size != 1:
            step = stride
        tokens *= size
    # (the stride of an axis of length one says nothing, and torch leaves anything there)
    return _Rows(t.data_ptr(), step if tokens > 1 else channels), tokens


def _alike(t, name, dtype, shape):
    """... of a known shape: most are contiguous, and are recognised by few reads."""
    if t.is_contiguous() and t.dtype == dtype and t.shape == shape and len(shape) >= 2:
        return _Rows(t.data_ptr(), shape[-1])
    return _tokens(t, name, dtype, shape)[0]


_NONE = _Rows(None, 0)


def _sequences(x, sequences, offsets):
    """(sequences, offsets' address): those of ``offsets``, the given number, or x.shape[0] of a three-dimensional x, else one."""
    if offsets is None:
        return (x.shape[0] if x.dim() == 3 else 1) if sequences is None else int(sequences), None
    if not (offsets.dtype == torch.int32 and offsets.dim() == 1 and offsets.is_contiguous() and offsets.numel() >= 2):
        _refuse("offsets must be int32 [sequences + 1]")
    if not (sequences is None or sequences == offsets.numel() - 1):
        _refuse("offsets must be int32 [sequences + 1]")
    return offsets.numel() - 1, offsets.data_ptr()


def _bytes(workspace):
    if not (workspace.is_contiguous() and workspace.dtype == torch.uint8):
        _refuse("the workspace must be contiguous bytes")
    return workspace


def _storage(dtype):
    dt = _DTYPES.get(dtype)
    if dt is None:
        _refuse(f"{dtype} is not a storage type")
    return dt


class _ScanCall:
    """The arguments that the scan's forward, backward and step share, checked."""
    __slots__ = ("x", "delta", "b", "c", "gate", "shape", "dt", "state_shape", "rows")

    def __init__(self, x, delta, a, b, c, skip, delta_bias, gate, softplus, sequences, offsets):
        dtype, self.rows = x.dtype, x.shape
        self.dt = _storage(dtype)
        self.x, tokens = _tokens(x, "x", dtype)
        channels = self.rows[-1]
        self.delta = _alike(delta, "delta", dtype, self.rows)
        self.gate = _NONE if gate is None else _alike(gate, "gate", dtype, self.rows)
        of_a = a.shape
        if not (len(of_a) == 2 and of_a[0] == channels):
            _refuse("a must be [channels, states]")
        states = of_a[1]
        _plain(a, "a", of_a, torch.float32)
        if skip is not None:
            _plain(skip, "skip", (channels,), torch.float32)
        if delta_bias is not None:
            _plain(delta_bias, "delta_bias", (channels,), torch.float32)
        of_b = b.shape
        if len(of_b) < 2 or of_b[-1] != states or (of_b[:-1] != self.rows[:-1] and of_b[:-2] != self.rows[:-1]):
            _refuse("b must be [..., states] or [..., groups, states]")
        groups = 1 if len(of_b) == len(self.rows) else of_b[-2]
        self.b = self.shared(b, "b", dtype, of_b, groups * states)
        self.c = self.shared(c, "c", dtype, of_b, groups * states)
        sequences, at = _sequences(x, sequences, offsets)
        self.shape = _Scan(sequences, tokens, at, channels, groups, states, 1 if softplus else 0)
        self.state_shape = (sequences, channels, states)

    def shared(self, t, name, dtype, shape, width):
        """b, c or their gradients, of a known shape ([..., states] or [..., groups, states]), as rows of ``width``."""
        if t.is_contiguous() and t.dtype == dtype and t.shape == shape:
            return _Rows(t.data_ptr(), width)
        if t.dtype != dtype:
            _refuse(f"{name} must be {dtype}, not {t.dtype}")
        if t.shape != shape:
            _refuse(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
        if len(shape) == len(self.rows):
            return _tokens(t, name, dtype)[0]
        if t.is_contiguous():
            return _Rows(t.data_ptr(), width)
        strides = t.stride()
        if not (shape[-2] == 1 or (strides[-2] == shape[-1] and (strides[-1] == 1 or shape[-1] == 1))):
            _refuse(f"{name}'s groups must lie next to each other")
        return _tokens(t.as_strided(shape[:-2] + (width,), strides[:-2] + strides[-1:]), name, dtype)[0]

    def workspace(self, given, backward, like, stream):
        if given is not None:
            return _bytes(given)
        s = self.shape
        size = _scan_bytes(s.sequences, s.tokens, s.offsets is not None, s.channels, s.groups, s.states, backward, self.dt)
        return _new(like, stream, size, torch.uint8) if size or backward else None


@functools.lru_cache(maxsize=256)
def _scan_bytes(sequences, tokens, packed, channels, groups, states, backward, dt):
    """(a function of numbers alone, so what it says of the last shapes is kept)"""
    shape = _Scan(sequences, tokens, 4 if packed else None, channels, groups, states, 0)
    size = ctypes.c_size_t(0)
    _check(_lib().msla_selective_scan_workspace_bytes(shape, backward, dt, size), "msla_selective_scan_workspace_bytes")
    return size.value


def msla_selective_scan_workspace_bytes(sequences, tokens, channels, groups, states, dtype, packed=False, backward=False) -> int:
    """Bytes that msla_selective_scan_forward (or _backward) needs; packed: with offsets."""
    return _scan_bytes(sequences, tokens, bool(packed), channels, groups, states, int(backward), _DTYPES[dtype])


def msla_selective_scan_forward(x, delta, a, b, c, skip=None, delta_bias=None, gate=None, softplus=False, sequences: Optional[int] = None,
                                offsets=None, initial_state=None, out=None, final_state=None, workspace=None, stream=None):
    """h_i = exp(t_i a) h_{i-1} + t_i x_i b_i, y_i = sum(c_i h_i) + skip x_i, out = y silu(gate), over every sequence and channel.

    x, delta, gate [..., channels]: a token's step t is delta + delta_bias, or softplus of that; b, c [..., states], or [..., groups, states] where groups of
    channels have their own; any strides over tokens (so parts of a projected map will do).  a [channels, states], skip and delta_bias [channels] fp32.
    The tokens are those of ``sequences`` equally long sequences (by default x.shape[0] of a three-dimensional x, else one), or of sequences
    packed behind each other that start at ``offsets`` (int32, on the GPU, one more than sequences).  Returns (out, final_state [sequences, channels,
    states] fp32); rows that belong to no sequence are left as they are in a given ``out``."""
    _on_gpu(x, delta, a, b, c, skip, delta_bias, gate, offsets, initial_state, out, final_state, workspace)
    k = _ScanCall(x, delta, a, b, c, skip, delta_bias, gate, softplus, sequences, offsets)
    _plain(initial_state, "initial_state", k.state_shape, torch.float32)
    _plain(final_state, "final_state", k.state_shape, torch.float32)
    if out is None:
        out = _new(x, stream, x.shape)
    o = _alike(out, "out", x.dtype, x.shape)
    if final_state is None:
        final_state = _new(x, stream, k.state_shape, torch.float32)
    ws = k.workspace(workspace, 0, x, stream)
    _check(_lib().msla_selective_scan_forward(k.shape, k.x, k.delta, a.data_ptr(), k.b, k.c, _ptr(skip), _ptr(delta_bias), k.gate, _ptr(initial_state), o,
                                              _ptr(final_state), _ptr(ws), 0 if ws is None else ws.numel(), k.dt, _stream(stream)),
           "msla_selective_scan_forward")
    return out, final_state


class SelectiveScanGradients(NamedTuple):
    """What msla_selective_scan_backward returns; None where the input is."""
    d_x: torch.Tensor
    d_delta: torch.Tensor
    d_a: torch.Tensor
    d_b: torch.Tensor
    d_c: torch.Tensor
    d_skip: Optional[torch.Tensor]
    d_delta_bias: Optional[torch.Tensor]
    d_gate: Optional[torch.Tensor]
    d_initial_state: Optional[torch.Tensor]


def msla_selective_scan_backward(x, delta, a, b, c, d_out, skip=None, delta_bias=None, gate=None, softplus=False,
                                 sequences: Optional[int] = None, offsets=None, initial_state=None, d_final_state=None, d_x=None, d_delta=None,
                                 d_a=None, d_b=None, d_c=None, d_skip=None, d_delta_bias=None, d_gate=None, d_initial_state=None, workspace=None,
                                 stream=None) -> SelectiveScanGradients:
    """The gradient of msla_selective_scan_forward; those of a, skip, delta_bias and the initial state are fp32."""
    _on_gpu(x, delta, a, b, c, d_out, skip, delta_bias, gate, offsets, initial_state, d_final_state, d_x, d_delta, d_a, d_b, d_c, d_skip, d_delta_bias,
            d_gate, d_initial_state, workspace)
    k = _ScanCall(x, delta, a, b, c, skip, delta_bias, gate, softplus, sequences, offsets)
    f32, channels = torch.float32, x.shape[-1]
    _plain(initial_state, "initial_state", k.state_shape, f32)
    _plain(d_final_state, "d_final_state", k.state_shape, f32)
    do = _alike(d_out, "d_out", x.dtype, x.shape)
    for t, of, name in ((d_skip, skip, "skip"), (d_delta_bias, delta_bias, "delta_bias"), (d_gate, gate, "gate"),
                        (d_initial_state, initial_state, "initial_state")):
        if t is not None and of is None:
            _refuse(f"d_{name} needs a {name}")

    def rows(t, of, name):
        if of is None:
            return None, _NONE
        if t is None:
            t = _new(of, stream, k.rows)
        return t, _alike(t, name, x.dtype, k.rows)

    def shared(t, of, name):
        if t is None:
            t = _new(of, stream, of.shape)
        return t, k.shared(t, name, x.dtype, of.shape, k.shape.groups * k.shape.states)

    def single(t, of, name, shape):
        if of is None:
            return None
        if t is None:
            return _new(x, stream, shape, f32)
        _plain(t, name, shape, f32)
        return t

    d_x, rx = rows(d_x, x, "d_x")
    d_delta, rd = rows(d_delta, delta, "d_delta")
    d_gate, rg = rows(d_gate, gate, "d_gate")
    d_b, rb = shared(d_b, b, "d_b")
    d_c, rc = shared(d_c, c, "d_c")
    d_a = single(d_a, a, "d_a", tuple(a.shape))
    d_skip = single(d_skip, skip, "d_skip", (channels,))
    d_delta_bias = single(d_delta_bias, delta_bias, "d_delta_bias", (channels,))
    d_initial_state = single(d_initial_state, initial_state, "d_initial_state", k.state_shape)
    ws = k.workspace(workspace, 1, x, stream)
    _check(_lib().msla_selective_scan_backward(k.shape, k.x, k.delta, a.data_ptr(), k.b, k.c, _ptr(skip), _ptr(delta_bias), k.gate, _ptr(initial_state),
                                               do, _ptr(d_final_state), rx, rd, _ptr(d_a), rb, rc, _ptr(d_skip), _ptr(d_delta_bias), rg,
                                               _ptr(d_initial_state), _ptr(ws), ws.numel(), k.dt, _stream(stream)), "msla_selective_scan_backward")
    return SelectiveScanGradients(d_x, d_delta, d_a, d_b, d_c, d_skip, d_delta_bias, d_gate, d_initial_state)


def msla_selective_scan_step(x, delta, a, b, c, state, skip=None, delta_bias=None, gate=None, softplus=False, out=None, new_state=None, stream=None):
    """One token for each of x.shape[0] sequences: x, delta, gate [sequences, channels], b, c [sequences, states] or [sequences, groups, states], state
    [sequences, channels, states] fp32.  The state is updated in place unless new_state is given.  Returns (out, new_state)."""
    if new_state is None:
        new_state = state
    _on_gpu(x, delta, a, b, c, state, skip, delta_bias, gate, out, new_state)
    if not (x.dim() == 2):
        _refuse("x must be [sequences, channels]")
    k = _ScanCall(x, delta, a, b, c, skip, delta_bias, gate, softplus, x.shape[0], None)
    _plain(state, "state", k.state_shape, torch.float32)
    if new_state is not state:
        _plain(new_state, "new_state", k.state_shape, torch.float32)
    if out is None:
        out = _new(x, stream, x.shape)
    o = _alike(out, "out", x.dtype, x.shape)
    _check(_lib().msla_selective_scan_step(k.shape, k.x, k.delta, a.data_ptr(), k.b, k.c, _ptr(skip), _ptr(delta_bias), k.gate, state.data_ptr(), o,
                                           new_state.data_ptr(), k.dt, _stream(stream)), "msla_selective_scan_step")
    return out, new_state


def _conv_arguments(x, weight, bias, silu, sequences, offsets):
    """(shape, x's rows, storage type, state's shape)"""
    dtype = x.dtype
    dt = _storage(dtype)
    rows, tokens = _tokens(x, "x", dtype)
    channels = x.shape[-1]
    if not (weight.dim() == 2 and weight.shape[0] == channels):
        _refuse("weight must be [channels, width]")
    width = weight.shape[1]
    _plain(weight, "weight", weight.shape, dtype)
    if bias is not None:
        _plain(bias, "bias", (channels,), dtype)
    sequences, at = _sequences(x, sequences, offsets)
    return _Conv(sequences, tokens, at, channels, width, 1 if silu else 0), rows, dt, (sequences, max(width - 1, 0), channels)


def msla_causal_conv_forward(x, weight, bias=None, silu=False, sequences: Optional[int] = None, offsets=None, initial_state=None, out=None,
                             final_state=None, stream=None):
    """pre_i = bias + sum_k weight[:, k] x_{i - width + 1 + k}, out = pre, or pre sigmoid(pre) with ``silu``, over every sequence.

    x [..., channels], any strides over tokens; weight [channels, width], bias [channels] in x's type; sequences and offsets as in
    msla_selective_scan_forward.  initial_state [sequences, width - 1, channels] in x's type: the rows in front of each sequence, oldest first.
    Returns (out, final_state), the same rows behind each sequence."""
    _on_gpu(x, weight, bias, offsets, initial_state, out, final_state)
    shape, rows, dt, state_shape = _conv_arguments(x, weight, bias, silu, sequences, offsets)
    _plain(initial_state, "initial_state", state_shape, x.dtype)
    _plain(final_state, "final_state", state_shape, x.dtype)
    if out is None:
        out = _new(x, stream, x.shape)
    o = _alike(out, "out", x.dtype, x.shape)
    if final_state is None:
        final_state = _new(x, stream, state_shape)
    _check(_lib().msla_causal_conv_forward(shape, rows, weight.data_ptr(), _ptr(bias), _ptr(initial_state), o, _ptr(final_state), dt, _stream(stream)),
           "msla_causal_conv_forward")
    return out, final_state


@functools.lru_cache(maxsize=256)
def _conv_bytes(sequences, tokens, packed, channels, width, dt):
    shape = _Conv(sequences, tokens, 4 if packed else None, channels, width, 0)
    size = ctypes.c_size_t(0)
    _check(_lib().msla_causal_conv_backward_workspace_bytes(shape, dt, size), "msla_causal_conv_backward_workspace_bytes")
    return size.value


def msla_causal_conv_backward_workspace_bytes(sequences, tokens, channels, width, dtype, packed=False) -> int:
    return _conv_bytes(sequences, tokens, bool(packed), channels, width, _DTYPES[dtype])


def msla_causal_conv_backward(x, weight, d_out, bias=None, silu=False, sequences: Optional[int] = None, offsets=None, initial_state=None,
                              d_final_state=None, d_x=None, d_weight=None, d_bias=None, d_initial_state=None, workspace=None, stream=None):
    """(d_x, d_weight, d_bias, d_initial_state): the gradient of msla_causal_conv_forward, d_weight and d_bias fp32, the last two None where bias or
    initial_state is."""
    _on_gpu(x, weight, d_out, bias, offsets, initial_state, d_final_state, d_x, d_weight, d_bias, d_initial_state, workspace)
    shape, rows, dt, state_shape = _conv_arguments(x, weight, bias, silu, sequences, offsets)
    do = _alike(d_out, "d_out", x.dtype, x.shape)
    _plain(initial_state, "initial_state", state_shape, x.dtype)
    _plain(d_final_state, "d_final_state", state_shape, x.dtype)
    _plain(d_initial_state, "d_initial_state", state_shape, x.dtype)
    _plain(d_weight, "d_weight", tuple(weight.shape), torch.float32)
    _plain(d_bias, "d_bias", (weight.shape[0],), torch.float32)
    for t, of, name in ((d_bias, bias, "bias"), (d_initial_state, initial_state, "initial_state")):
        if t is not None and of is None:
            _refuse(f"d_{name} needs a {name}")
    if d_x is None:
        d_x = _new(x, stream, x.shape)
    dx = _alike(d_x, "d_x", x.dtype, x.shape)
    if d_weight is None:
        d_weight = _new(x, stream, tuple(weight.shape), torch.float32)
    if d_bias is None and bias is not None:
        d_bias = _new(x, stream, tuple(bias.shape), torch.float32)
    if d_initial_state is None and initial_state is not None:
        d_initial_state = _new(x, stream, state_shape)
    if workspace is None:
        workspace = _new(x, stream, _conv_bytes(shape.sequences, shape.tokens, offsets is not None, shape.channels, shape.width, dt), torch.uint8)
    _check(_lib().msla_causal_conv_backward(shape, rows, weight.data_ptr(), _ptr(bias), _ptr(initial_state), do, _ptr(d_final_state), dx, _ptr(d_weight),
                                            _ptr(d_bias), _ptr(d_initial_state), _ptr(_bytes(workspace)), workspace.numel(), dt, _stream(stream)),
           "msla_causal_conv_backward")
    return d_x, d_weight, d_bias, d_initial_state


def msla_causal_conv_step(x, weight, state, bias=None, silu=False, out=None, new_state=None, stream=None):
    """One token for each of x.shape[0] sequences: x [sequences, channels], state [sequences, width - 1, channels].  The state is updated in place unless
    new_state is given.  Returns (out, new_state)."""
    if new_state is None:
        new_state = state
    _on_gpu(x, weight, state, bias, out, new_state)
    if not (x.dim() == 2):
        _refuse("x must be [sequences, channels]")
    shape, rows, dt, state_shape = _conv_arguments(x, weight, bias, silu, x.shape[0], None)
    _plain(state, "state", state_shape, x.dtype)
    if new_state is not state:
        _plain(new_state, "new_state", state_shape, x.dtype)
    if out is None:
        out = _new(x, stream, x.shape)
    o = _alike(out, "out", x.dtype, x.shape)
    _check(_lib().msla_causal_conv_step(shape, rows, weight.data_ptr(), _ptr(bias), state.data_ptr(), o, new_state.data_ptr(), dt, _stream(stream)),
           "msla_causal_conv_step")
    return out, new_state


def msla_layer_norm_forward(x, weight=None, bias=None, residual=None, eps=1e-5, out=None, sum_out=None, stream=None):
    """(y, r): r = x + residual, y = (r - mean(r)) / sqrt(var(r) + eps) * weight + bias over the last axis.  Without a residual r is x itself and is not
    written, unless sum_out is given."""
    rows, channels = _norm_arguments(x, weight, residual, sum_out)
    _on_gpu(bias)
    _plain(bias, "bias", (channels,), x.dtype)
    if out is None:
        out = _new(x, stream)
    else:
        _on_gpu(out)
        _plain(out, "out", x.shape, x.dtype)
    if sum_out is None and residual is not None:
        sum_out = _new(x, stream)
    _check(_lib().msla_layer_norm_forward(_ptr(x), _ptr(residual), _ptr(weight), _ptr(bias), _ptr(out), _ptr(sum_out), rows, channels, float(eps),
                                          _DTYPES[x.dtype], _stream(stream)), "msla_layer_norm_forward")
    return out, x if sum_out is None else sum_out


@functools.lru_cache(maxsize=256)
def _layer_norm_bytes(rows, channels, dt):
    size = ctypes.c_size_t(0)
    _check(_lib().msla_layer_norm_backward_workspace_bytes(rows, channels, dt, size), "msla_layer_norm_backward_workspace_bytes")
    return size.value


def msla_layer_norm_backward_workspace_bytes(rows, channels, dtype) -> int:
    return _layer_norm_bytes(rows, channels, _DTYPES[dtype])


def msla_layer_norm_backward(r, weight, d_y, d_sum=None, eps=1e-5, d_r=None, d_weight=None, d_bias=None, workspace=None, stream=None):
    """(d_r, d_weight, d_bias): the gradient of msla_layer_norm_forward at r (what it returned); d_sum: the gradient that reaches r past the norm.
    d_r is that of x and of residual alike; d_weight and d_bias are fp32."""
    rows, channels = _norm_arguments(r, weight, d_y, d_sum, ("r", "d_y", "d_sum"))
    _on_gpu(d_r, d_weight, d_bias, workspace)
    if d_r is None:
        d_r = _new(r, stream)
    else:
        _plain(d_r, "d_r", r.shape, r.dtype)
    if d_weight is None:
        d_weight = _new(r, stream, channels, torch.float32)
    else:
        _plain(d_weight, "d_weight", (channels,), torch.float32)
    if d_bias is None:
        d_bias = _new(r, stream, channels, torch.float32)
    else:
        _plain(d_bias, "d_bias", (channels,), torch.float32)
    if workspace is None:
        workspace = _new(r, stream, _layer_norm_bytes(rows, channels, _DTYPES[r.dtype]), torch.uint8)
    _check(_lib().msla_layer_norm_backward(_ptr(r), _ptr(weight), _ptr(d_y), _ptr(d_sum), _ptr(d_r), _ptr(d_weight), _ptr(d_bias),
                                           _ptr(_bytes(workspace)), workspace.numel(), rows, channels, float(eps), _DTYPES[r.dtype], _stream(stream)),
           "msla_layer_norm_backward")
    return d_r, d_weight, d_bias


def msla_quantize_rows_integer(x, out8=None, scale=None, stream=None):
    """(x8, scale): rows of x in 8-bit integers, x ~ x8 * scale[..., None].  scale is the fp32 product of max |x| and fp32's 1 / 127 (which is not always the
    quotient's rounding), x8 is x / scale to the nearest whole number, ties to even; a row whose scale is 0 or not finite has zeros."""
    rows, channels = _norm_arguments(x, None, None, None)
    if out8 is None:
        out8 = _new(x, stream, None, torch.int8)
    else:
        _on_gpu(out8)
        _plain(out8, "out8", x.shape, torch.int8)
    if scale is None:
        scale = _new(x, stream, x.shape[:-1], torch.float32)
    else:
        _on_gpu(scale)
        _plain(scale, "scale", x.shape[:-1], torch.float32)
    _check(_lib().msla_quantize_rows_integer(_ptr(x), _ptr(out8), _ptr(scale), rows, channels, _DTYPES[x.dtype], _stream(stream)),
           "msla_quantize_rows_integer")
    return out8, scale


def msla_linear_integer(x8, x_scale, w8, w_scale, dtype=torch.bfloat16, out=None, stream=None):
    """y[..., o] = x_scale[...] * w_scale[o] * sum_c x8[..., c] * w8[o, c]: x8, w8 int8, scales fp32, y in ``dtype`` (out's, if given)."""
    _on_gpu(x8, x_scale, w8, w_scale, out)
    shape = x8.shape
    if not (w8.dim() == 2 and len(shape) >= 1 and shape[-1] == w8.shape[1]):
        _refuse("x8 must be [..., c_in] and w8 [c_out, c_in]")
    c_out, c_in = w8.shape
    _plain(x8, "x8", shape, torch.int8)
    _plain(w8, "w8", (c_out, c_in), torch.int8)
    _plain(x_scale, "x_scale", shape[:-1], torch.float32)
    _plain(w_scale, "w_scale", (c_out,), torch.float32)
    if out is not None:
        dtype = out.dtype
    dt = _storage(dtype)
    to = shape[:-1] + (c_out,)
    if out is None:
        out = _new(x8, stream, to, dtype)
    else:
        _plain(out, "out", to, dtype)
    rows = x8.numel() // c_in if c_in else 0
    _check(_lib().msla_linear_integer(x8.data_ptr(), x_scale.data_ptr(), w8.data_ptr(), w_scale.data_ptr(), out.data_ptr(), rows, c_in, c_out, dt,
                                      _stream(stream)), "msla_linear_integer")
    return out

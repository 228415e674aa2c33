"""Plain fp64 definitions of the sequence operators (include/msla_sequence.h), token by token, in numpy.

Test infrastructure only: written from the recurrences themselves, nothing of the chunked forms that the kernels use."""
import numpy as np


def sequences_of(tokens, sequences=1, offsets=None):
    """[(first row, last row + 1)] of every sequence."""
    if offsets is not None:
        return list(zip(offsets[:-1], offsets[1:]))
    n = tokens // sequences
    return [(b * n, (b + 1) * n) for b in range(sequences)]


def _inputs(q, k, v, gate, rectify):
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    if rectify:
        q, k = np.maximum(q, 0), np.maximum(k, 0)
    keep = np.ones(k.shape[:2]) if gate is None else np.exp(np.asarray(gate, np.float64))
    return q, k, v, keep


def recurrence(q, k, v, gate, spans, initial, scale, rectify=False):
    """out [T, Hq, d] (zero in rows of no sequence) and the last states [n, Hkv, d, d]."""
    q, k, v, keep = _inputs(q, k, v, gate, rectify)
    hkv, d = k.shape[1:]
    group = q.shape[1] // hkv
    out = np.zeros_like(q)
    last = np.zeros((len(spans), hkv, d, d)) if initial is None else np.array(initial, np.float64)
    for b, (lo, hi) in enumerate(spans):
        s = last[b]
        for t in range(lo, hi):
            s = keep[t][:, None, None] * s + k[t][:, :, None] * v[t][:, None, :]
            out[t] = scale * (q[t].reshape(hkv, group, d) @ s).reshape(-1, d)
        last[b] = s
    return out, last


def recurrence_backward(q, k, v, gate, spans, initial, scale, d_out, d_last=None, rectify=False, magnitudes=False):
    """(d_q, d_k, d_v, d_gate, d_initial), from the recurrence of the state's own gradient.  magnitudes: for inputs that are magnitudes, what
    every gradient's terms add up to without their signs (no rectifier's mask then)."""
    q, k, v, keep = _inputs(q, k, v, gate, rectify)
    d_out = np.asarray(d_out, np.float64)
    hkv, d = k.shape[1:]
    group = q.shape[1] // hkv
    dq, dk, dv, dg = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros_like(keep)
    di = np.zeros((len(spans), hkv, d, d)) if d_last is None else np.array(d_last, np.float64)
    for b, (lo, hi) in enumerate(spans):
        s = np.zeros((hkv, d, d)) if initial is None else np.array(initial[b], np.float64)
        states = [s]
        for t in range(lo, hi):
            s = keep[t][:, None, None] * s + k[t][:, :, None] * v[t][:, None, :]
            states.append(s)
        ds = di[b]
        for t in range(hi - 1, lo - 1, -1):
            qt, dot = q[t].reshape(hkv, group, d), d_out[t].reshape(hkv, group, d)
            ds = ds + scale * np.swapaxes(qt, 1, 2) @ dot
            dq[t] = scale * (dot @ np.swapaxes(states[t - lo + 1], 1, 2)).reshape(-1, d)
            dk[t] = (ds @ v[t][:, :, None])[:, :, 0]
            dv[t] = (k[t][:, None, :] @ ds)[:, 0]
            dg[t] = keep[t] * (ds * states[t - lo]).sum((1, 2))
            ds = keep[t][:, None, None] * ds
        di[b] = ds
    if rectify and not magnitudes:
        dq, dk = dq * (q > 0), dk * (k > 0)
    return dq, dk, dv, dg, di


def norm(x, residual, weight, eps):
    """(y, r)"""
    r = np.asarray(x, np.float64) + (0 if residual is None else np.asarray(residual, np.float64))
    y = r / np.sqrt((r * r).mean(-1, keepdims=True) + eps)
    return y * (1 if weight is None else np.asarray(weight, np.float64)), r


def norm_backward(r, weight, d_y, d_sum, eps):
    """(d_r, d_weight): d_r through r and through the mean of its squares."""
    r, d_y = np.asarray(r, np.float64), np.asarray(d_y, np.float64)
    w = np.ones(r.shape[-1]) if weight is None else np.asarray(weight, np.float64)
    size = np.sqrt((r * r).mean(-1, keepdims=True) + eps)
    d_size = -(d_y * w * r / size ** 2).sum(-1, keepdims=True)
    d_r = d_y * w / size + d_size * r / (r.shape[-1] * size)
    if d_sum is not None:
        d_r = d_r + np.asarray(d_sum, np.float64)
    return d_r, (d_y * r / size).sum(tuple(range(r.ndim - 1)))

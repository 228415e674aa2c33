"""Plain fp64 definitions of a selective state space layer's operators (include/msla_sequence.h), token by token, in numpy.

Test infrastructure only: written from the recurrences themselves.  ``magnitudes`` wherever it stands: for inputs that are magnitudes, what the terms of
every result add up to without their signs (what errors of rounding are measured by)."""
import numpy as np


def f64(t):
    return None if t is None else np.asarray(t, np.float64)


def sigmoid(v):
    e = np.exp(-np.abs(v))
    return np.where(v >= 0, 1 / (1 + e), e / (1 + e))


def steps_of(delta, bias, softplus):
    pre = f64(delta) + (0 if bias is None else f64(bias))
    return pre, (np.maximum(pre, 0) + np.log1p(np.exp(-np.abs(pre))) if softplus else pre)


def scan(x, delta, a, b, c, spans, skip=None, bias=None, gate=None, softplus=False, initial=None):
    """out [T, C] (zero in rows of no sequence), last states [n, C, N], and y before the gate."""
    x, a, b, c, gate = map(f64, (x, a, b, c, gate))
    per = x.shape[1] // b.shape[1]
    _, dt = steps_of(delta, bias, softplus)
    skip = np.zeros(x.shape[1]) if skip is None else f64(skip)
    y = np.zeros_like(x)
    last = np.zeros((len(spans),) + a.shape) if initial is None else np.array(initial, np.float64)
    for i, (lo, hi) in enumerate(spans):
        h = last[i]
        for t in range(lo, hi):
            h = np.exp(dt[t][:, None] * a) * h + (dt[t] * x[t])[:, None] * np.repeat(b[t], per, 0)
            y[t] = (h * np.repeat(c[t], per, 0)).sum(1) + skip * x[t]
        last[i] = h
    return (y if gate is None else y * gate * sigmoid(gate)), last, y


def scan_backward(x, delta, a, b, c, spans, d_out, skip=None, bias=None, gate=None, softplus=False, initial=None, d_last=None, magnitudes=False):
    """dict of gradients by their arguments' names.  magnitudes: of |x|, |b|, ... with the true steps, decays and gates."""
    absolute = np.abs if magnitudes else (lambda v: v)
    pre, dt = steps_of(delta, bias, softplus)
    decays = f64(a)
    x, a, b, c, d_out = (absolute(f64(v)) for v in (x, a, b, c, d_out))
    gate = f64(gate)
    skip = np.zeros(x.shape[1]) if skip is None else absolute(f64(skip))
    groups = b.shape[1]
    per = x.shape[1] // groups
    dy, g = d_out, {}
    if gate is not None:
        s = sigmoid(gate)
        dy = d_out * absolute(gate * s)
    out = {k: np.zeros_like(v) for k, v in (("x", x), ("delta", x), ("a", a), ("b", b), ("c", c))}
    out["initial"] = np.zeros((len(spans),) + a.shape) if d_last is None else absolute(np.array(d_last, np.float64))
    y = np.zeros_like(x)
    for i, (lo, hi) in enumerate(spans):
        h = np.zeros_like(a) if initial is None else absolute(np.array(initial[i], np.float64))
        states = [h]
        for t in range(lo, hi):
            h = np.exp(dt[t][:, None] * decays) * h + (dt[t] * x[t])[:, None] * np.repeat(b[t], per, 0)
            states.append(h)
            y[t] = (h * np.repeat(c[t], per, 0)).sum(1) + skip * x[t]
        dh = out["initial"][i]
        for t in range(hi - 1, lo - 1, -1):
            dh = dh + dy[t][:, None] * np.repeat(c[t], per, 0)
            keep = np.exp(dt[t][:, None] * decays)
            out["c"][t] = (dy[t][:, None] * states[t - lo + 1]).reshape(groups, per, -1).sum(1)
            out["b"][t] = (dh * (dt[t] * x[t])[:, None]).reshape(groups, per, -1).sum(1)
            inflow = (dh * np.repeat(b[t], per, 0)).sum(1)
            through = dh * keep * states[t - lo]
            out["x"][t] = dt[t] * inflow + skip * dy[t]
            out["delta"][t] = x[t] * inflow + (through * a).sum(1)
            out["a"] += through * dt[t][:, None]
            dh = keep * dh
        out["initial"][i] = dh
    if softplus:
        out["delta"] = out["delta"] * sigmoid(pre)
    rows = np.zeros(len(x), bool)
    for lo, hi in spans:
        rows[lo:hi] = True
    out["skip"] = (dy * x)[rows].sum(0)
    out["bias"] = out["delta"].sum(0)
    if gate is not None:
        # (two terms of the derivative, 1 and gate (1 - s), cancel near a gate of -1.28: magnitudes add them up)
        out["gate"] = d_out * y * s * (1 + absolute(gate) * (1 - s)) * rows[:, None]
    return out


def conv(x, weight, spans, bias=None, silu=False, initial=None, d_out=None, d_last=None):
    """(out, last) or, with d_out, (d_x, d_weight, d_bias, d_initial), tap by tap."""
    x, weight = f64(x), f64(weight)
    channels, w = weight.shape
    bias = np.zeros(channels) if bias is None else f64(bias)
    out, dx = np.zeros_like(x), np.zeros_like(x)
    last, d_initial = np.zeros((len(spans), w - 1, channels)), np.zeros((len(spans), w - 1, channels))
    dw, db = np.zeros_like(weight), np.zeros(channels)
    for i, (lo, hi) in enumerate(spans):
        rows = np.concatenate([np.zeros((w - 1, channels)) if initial is None else f64(initial[i]), x[lo:hi]])
        n = hi - lo
        pre = bias + sum(weight[:, k] * rows[k:k + n] for k in range(w))
        s = sigmoid(pre)
        out[lo:hi] = pre * s if silu else pre
        last[i] = rows[n:]
        if d_out is None:
            continue
        d = f64(d_out)[lo:hi] * ((s * (1 + pre * (1 - s))) if silu else 1)
        back = np.zeros_like(rows)
        if d_last is not None:
            back[n:] += f64(d_last[i])
        for k in range(w):
            back[k:k + n] += weight[:, k] * d
            dw[:, k] += (d * rows[k:k + n]).sum(0)
        db += d.sum(0)
        dx[lo:hi], d_initial[i] = back[w - 1:], back[:w - 1]
    return (out, last) if d_out is None else (dx, dw, db, d_initial)


def layer_norm(x, residual, weight, bias, eps):
    """(y, r)"""
    r = f64(x) + (0 if residual is None else f64(residual))
    d = r - r.mean(-1, keepdims=True)
    y = d / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return y * (1 if weight is None else f64(weight)) + (0 if bias is None else f64(bias)), r


def layer_norm_backward(r, weight, d_y, d_sum, eps):
    """(d_r, d_weight, d_bias): d_r through r, through the mean, and through the mean of the squares."""
    r, d_y = f64(r), f64(d_y)
    n = r.shape[-1]
    g = d_y * (1 if weight is None else f64(weight))
    d = r - r.mean(-1, keepdims=True)
    size = np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    d_size = -(g * d / size ** 2).sum(-1, keepdims=True)
    d_d = g / size + d_size * d / (n * size)
    d_r = d_d - d_d.mean(-1, keepdims=True)
    if d_sum is not None:
        d_r = d_r + f64(d_sum)
    return d_r, (d_y * d / size).reshape(-1, n).sum(0), d_y.reshape(-1, n).sum(0)

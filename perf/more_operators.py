"""The operators of a selective state space layer as timed cases: the scan (over sequences, its gradient, one token a sequence), the
short causal convolution before it (the same three), layer norm and its gradient, and the projection in 8-bit integers.

A case is a dict; ``op`` says which entry point of ``paper_2205_14756_amd.sequence`` it is about:

* ``scan`` / ``scan_backward``: ``dtype``, ``seqs`` sequences of ``tokens`` rows in all, equally long or cut at random places
  (``packed``; some may be empty), ``channels``, in ``groups`` that share B and C, ``states`` a channel, ``gated`` (out * silu(z)),
  ``softplus`` (steps are softplus(delta + bias), else delta), ``initial`` (the sequences go on from a state).
* ``scan_step``: the same with one token for each of ``seqs`` sequences.
* ``conv`` / ``conv_backward`` / ``conv_step``: ``seqs``, ``tokens``, ``packed``, ``channels``, ``width``, ``silu``, ``initial``.
* ``layer_norm`` / ``layer_norm_backward``: ``rows``, ``channels``, ``residual`` (backward: a gradient that arrives through the sum).
* ``integer``: ``rows``, ``c_in``, ``c_out``; ``dtype`` is that of the rows and of the output; ``quantize``: the rows arrive in ``dtype`` and are
  brought into 8 bits first.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------ the cases
def _scan(name, op, dtype, seqs, tokens, channels, groups, states, packed=False, gated=True, softplus=True, initial=False):
    return {"name": name, "op": op, "dtype": dtype, "seqs": seqs, "tokens": tokens, "channels": channels, "groups": groups,
            "states": states, "packed": packed, "gated": gated, "softplus": softplus, "initial": initial}


def _conv(name, op, dtype, seqs, tokens, channels, width, packed=False, silu=True, initial=False):
    return {"name": name, "op": op, "dtype": dtype, "seqs": seqs, "tokens": tokens, "channels": channels, "width": width,
            "packed": packed, "silu": silu, "initial": initial}


def _norm(name, op, dtype, rows, channels, residual=True):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "channels": channels, "residual": residual}


def _integer(name, dtype, rows, c_in, c_out, quantize):
    return {"name": name, "op": "integer", "dtype": dtype, "rows": rows, "c_in": c_in, "c_out": c_out, "quantize": quantize}


def listed():
    return [
        # one short prompt of a small model that goes on from a state: latency
        _scan("scan_prompt", "scan", "bf16", 1, 203, 1024, 1, 16, initial=True),
        # a training batch
        _scan("scan_training", "scan", "bf16", 4, 8192, 4096, 1, 16),
        # prompts of many lengths packed behind each other, groups of channels with a B and C of their own, large states
        _scan("scan_packed", "scan", "f16", 24, 5003, 2048, 4, 64, packed=True, initial=True),
        # the gradient of a training batch
        _scan("scan_gradient", "scan_backward", "bf16", 4, 8192, 4096, 1, 16),
        # one token for each of many conversations
        _scan("scan_step_many", "scan_step", "bf16", 192, 192, 4096, 1, 16),
        # the convolution of a training batch
        _conv("conv_training", "conv", "bf16", 4, 16384, 4096, 4),
        # its gradient over packed sequences
        _conv("conv_gradient", "conv_backward", "bf16", 16, 16384, 4096, 4, packed=True),
        # one token of one conversation
        _conv("conv_step_one", "conv_step", "bf16", 1, 1, 4096, 4),
        # between the halves of a block, training
        _norm("layer_norm_training", "layer_norm", "bf16", 16384, 4096),
        # the gradient, an odd width
        _norm("layer_norm_gradient", "layer_norm_backward", "f16", 8192, 2051),
        # a batch of single tokens, whose rows arrive in the storage type: the weights outweigh everything
        _integer("integer_decode", "bf16", 48, 4096, 4096, True),
        # a batch of prompts
        _integer("integer_prompt", "bf16", 4096, 4096, 8192, False),
    ]


def _log(rng, low, high):
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    op = rng.choice(["scan", "scan", "scan_backward", "scan_backward", "scan_step", "conv", "conv_backward", "conv_step",
                     "layer_norm", "layer_norm_backward", "integer", "integer"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if op.startswith("scan") or op.startswith("conv"):
        step = op.endswith("step")
        channels = _log(rng, 16, 4096)
        if rng.random() < 0.7:
            channels = channels // 16 * 16
        seqs = _log(rng, 1, 192 if step else 16)
        length = 1 if step else _log(rng, 1, 8192)
        c = {"op": op, "dtype": dtype, "seqs": seqs, "tokens": 0, "channels": channels, "packed": not step and rng.random() < 0.5,
             "initial": step or rng.random() < 0.5}
        if op.startswith("scan"):
            states = rng.choice([8, 16, 16, 32, 64])
            groups = rng.choice([1, 1, 2, 4])
            c.update(groups=groups if channels % groups == 0 else 1, states=states, gated=rng.random() < 0.7, softplus=rng.random() < 0.7)
            most = 8192 * 4096 * 16 // (channels * states)
        else:
            c.update(width=rng.choice([2, 3, 4, 4]), silu=rng.random() < 0.7)
            most = 16384 * 4096 // channels
        while seqs * length > most:
            length = (length + 1) // 2
        c["tokens"] = seqs * length
        return c
    if op.startswith("layer_norm"):
        channels = _log(rng, 16, 8192)
        if rng.random() < 0.7:
            channels = channels // 16 * 16
        rows = _log(rng, 1, 16384)
        while rows * channels > 8192 * 4096:
            rows = (rows + 1) // 2
        return {"op": op, "dtype": dtype, "rows": rows, "channels": channels, "residual": rng.random() < 0.7}
    rows, c_in, c_out = _log(rng, 1, 4096), 16 * _log(rng, 4, 512), 16 * _log(rng, 4, 512)
    while rows * c_in * c_out > 4096 * 4096 * 8192:
        rows = (rows + 1) // 2
    return {"op": op, "dtype": dtype, "rows": rows, "c_in": c_in, "c_out": c_out, "quantize": rng.random() < 0.5}


# ------------------------------------------------------------------------------------------------ inputs
def _starts(case, seed):
    """Where the sequences start, and the end of the last one."""
    seqs, tokens = case["seqs"], case["tokens"]
    if not case["packed"]:
        return [i * (tokens // seqs) for i in range(seqs + 1)]
    cuts = np.sort(np.random.RandomState(seed % (1 << 31)).randint(0, tokens + 1, seqs - 1))
    return [0] + [int(c) for c in cuts] + [tokens]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, op = DTYPES[case["dtype"]], case["op"]

    def normal(*shape, dtype=None, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype or dt)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    s = {"case": case}
    if op.startswith("scan") or op.startswith("conv"):
        tokens, channels, seqs = case["tokens"], case["channels"], case["seqs"]
        if not op.endswith("step"):
            s["starts"] = _starts(case, seed)
            s["offsets"] = torch.tensor(s["starts"], dtype=torch.int32, device="cuda") if case["packed"] else None
        s["x"] = normal(tokens, channels)
        if op.endswith("backward"):
            s["d_out"] = normal(tokens, channels)
    if op.startswith("scan"):
        n, groups = case["states"], case["groups"]
        # steps from 0.001 to 0.1, decays from those of a state that remembers hundreds of tokens to those of one that forgets in a few
        steps = torch.exp(uniform(channels) * math.log(100.0) + math.log(1e-3))
        if case["softplus"]:
            s["bias"], s["delta"] = torch.log(torch.expm1(steps)), normal(tokens, channels, std=0.5)
        else:
            s["bias"], s["delta"] = None, (steps * torch.exp(normal(tokens, channels, dtype=torch.float32, std=0.3))).to(dt)
        s["a"] = -(torch.arange(1, n + 1, device="cuda") * (0.75 + 0.5 * uniform(channels, n)))
        s["b"], s["c"] = normal(tokens, groups, n), normal(tokens, groups, n)
        s["skip"] = 1.0 + normal(channels, dtype=torch.float32, std=0.1)
        s["z"] = normal(tokens, channels) if case["gated"] else None
        s["state"] = normal(seqs, channels, n, dtype=torch.float32, std=0.3) if case["initial"] or op == "scan_step" else None
        if op == "scan_step":
            s["new_state"] = torch.empty_like(s["state"])
    elif op.startswith("conv"):
        w = case["width"]
        s["weight"], s["bias"] = normal(channels, w, std=w ** -0.5), normal(channels, std=0.1)
        s["state"] = normal(seqs, w - 1, channels) if case["initial"] or op == "conv_step" else None
        if op == "conv_step":
            s["new_state"] = torch.empty_like(s["state"])
    elif op.startswith("layer_norm"):
        rows, channels = case["rows"], case["channels"]
        s["x"] = (normal(rows, channels, dtype=torch.float32) + 0.5).to(dt)
        s["weight"], s["bias"] = (1.0 + normal(channels, dtype=torch.float32, std=0.1)).to(dt), normal(channels, std=0.1)
        s["residual"] = normal(rows, channels) if case["residual"] else None
        if op == "layer_norm_backward":
            s["d_out"] = normal(rows, channels)
    else:
        # activations: some channels much larger than the others
        x = normal(case["rows"], case["c_in"], dtype=torch.float32) * torch.where(uniform(case["c_in"]) < 0.01, 8.0, 1.0)
        s["x"] = x.to(dt)
        w8, scale = _integer_rows(normal(case["c_out"], case["c_in"], dtype=torch.float32, std=case["c_in"] ** -0.5))
        s["w8"], s["w_scale"] = w8, scale
        if not case["quantize"]:
            s["x8"], s["x_scale"] = _integer_rows(s.pop("x"))
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _integer_rows(x):
    x = x.float()
    scale = x.abs().amax(1) / 127.0
    return torch.round(x / torch.where(scale > 0, scale, 1.0)[:, None]).to(torch.int8), scale


def _silu(z):
    return z * torch.sigmoid(z)


def _spans(s):
    """First and last rows of the sequences that have any, their numbers, and the longest one's length."""
    starts = np.array(s["starts"])
    full = np.nonzero(starts[1:] > starts[:-1])[0]
    at = lambda v: torch.tensor(v, device="cuda", dtype=torch.long)
    return at(starts[full]), at(starts[full + 1] - 1), at(full), int((starts[1:] - starts[:-1]).max())


def _recur(keep, add, longest):
    """h_i = keep_i h_{i-1} + add_i along the first axis (keep is 0 where a sequence starts), by pairs, fours, eights ..."""
    step = 1
    while step < longest:
        add = torch.cat([add[:step], torch.addcmul(add[step:], keep[step:], add[:-step])])
        keep = torch.cat([keep[:step], keep[step:] * keep[:-step]])
        step *= 2
    return add


def _scan_terms(s):
    case = s["case"]
    per = case["channels"] // case["groups"]
    pre = s["delta"].float() if s["bias"] is None else s["delta"].float() + s["bias"]
    dt = torch.nn.functional.softplus(pre) if case["softplus"] else pre
    x = s["x"].float()
    b, c = (s[k].float().repeat_interleave(per, 1) for k in "bc")                       # [tokens, channels, states]
    return pre, dt, x, b, c, torch.exp(dt[..., None] * s["a"])


def _scan_plain(s, backward):
    case = s["case"]
    dtype, groups = s["x"].dtype, case["groups"]
    first, last, full, longest = _spans(s)
    pre, dt, x, b, c, decay = _scan_terms(s)
    state = s["state"] if s["state"] is not None else torch.zeros(case["seqs"], case["channels"], case["states"], device="cuda")
    add = (dt * x)[..., None] * b
    add[first] += decay[first] * state[full]
    keep = decay.clone()
    keep[first] = 0
    h = _recur(keep, add, longest)
    y = (h * c).sum(-1) + s["skip"] * x
    z = None if s["z"] is None else s["z"].float()
    if not backward:
        end = state.clone()
        end[full] = h[last]
        return (y if z is None else y * _silu(z)).to(dtype), end
    do = s["d_out"].float()
    outs = {}
    dy = do
    if z is not None:
        gate = torch.sigmoid(z)
        dy = do * z * gate
        outs["d_gate"] = (do * y * gate * (1 + z * (1 - gate))).to(dtype)
    behind = torch.cat([decay[1:], decay[:1]])
    behind[last] = 0
    dh = _recur(behind.flip(0), (dy[..., None] * c).flip(0), longest).flip(0)
    shared = lambda t: t.unflatten(1, (groups, -1)).sum(2).to(dtype)
    outs["d_c"] = shared(dy[..., None] * h)
    outs["d_b"] = shared(dh * (dt * x)[..., None])
    before = torch.cat([h[:1], h[:-1]])
    before[first] = state[full]
    through = dh * decay * before
    along = (dh * b).sum(-1)
    d_dt = x * along + (through * s["a"]).sum(-1)
    if case["softplus"]:
        d_dt = d_dt * torch.sigmoid(pre)
    outs["d_a"] = (through * dt[..., None]).sum(0)
    outs["d_skip"] = (dy * x).sum(0)
    outs["d_x"] = (dt * along + s["skip"] * dy).to(dtype)
    outs["d_delta"] = d_dt.to(dtype)
    if s["bias"] is not None:
        outs["d_bias"] = d_dt.sum(0)
    if s["state"] is not None:
        outs["d_state"] = torch.zeros_like(state)
        outs["d_state"][full] = decay[first] * dh[first]
    return outs


def _scan_step_plain(s):
    pre, dt, x, b, c, decay = _scan_terms(s)
    h = decay * s["state"] + (dt * x)[..., None] * b
    y = (h * c).sum(-1) + s["skip"] * x
    return (y if s["z"] is None else y * _silu(s["z"].float())).to(s["x"].dtype), h


def _conv_windows(s):
    """Rows of the padded [seqs, width - 1 + longest, channels] sequences, their windows, and which tokens are rows."""
    case = s["case"]
    w, starts = case["width"], torch.tensor(s["starts"], device="cuda")
    lengths = starts[1:] - starts[:-1]
    longest = max(1, max(b - a for a, b in zip(s["starts"], s["starts"][1:])))
    at = torch.arange(longest, device="cuda")
    live = at[None, :] < lengths[:, None]
    rows = torch.where(live, starts[:-1, None] + at[None, :], 0)
    x = torch.where(live[..., None], s["x"].float()[rows], 0.0)
    head = torch.zeros(case["seqs"], w - 1, case["channels"], device="cuda") if s["state"] is None else s["state"].float()
    x = torch.cat([head, x], 1)
    return x, x.unfold(1, w, 1), live, rows, lengths


def _conv_plain(s, backward):
    case = s["case"]
    w, dtype = case["width"], s["x"].dtype
    x, windows, live, rows, lengths = _conv_windows(s)
    weight = s["weight"].float()
    pre = (windows * weight).sum(-1) + s["bias"].float()
    ends = lengths[:, None] + torch.arange(w - 1, device="cuda")
    which = torch.arange(case["seqs"], device="cuda")[:, None]
    if not backward:
        out = _silu(pre) if case["silu"] else pre
        return out[live].to(dtype), x[which, ends].to(dtype)
    d = torch.where(live[..., None], s["d_out"].float()[rows], 0.0)
    if case["silu"]:
        gate = torch.sigmoid(pre)
        d = d * gate * (1 + pre * (1 - gate))
    dx = (torch.nn.functional.pad(d, (0, 0, w - 1, w - 1)).unfold(1, w, 1) * weight.flip(1)).sum(-1)
    outs = {"d_x": dx[:, w - 1:][live].to(dtype), "d_weight": (d[..., None] * windows).sum((0, 1)), "d_bias": d.sum((0, 1))}
    if s["state"] is not None:
        outs["d_state"] = dx[:, :w - 1].to(dtype)
    return outs


def _conv_step_plain(s):
    rows = torch.cat([s["state"], s["x"][:, None]], 1)
    pre = (rows.float() * s["weight"].float().t()).sum(1) + s["bias"].float()
    return (_silu(pre) if s["case"]["silu"] else pre).to(s["x"].dtype), rows[:, 1:].contiguous()


def _layer_norm_plain(s):
    r = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
    d = r - r.mean(1, keepdim=True)
    y = d * torch.rsqrt(d.square().mean(1, keepdim=True) + EPS) * s["weight"].float() + s["bias"].float()
    return y.to(s["x"].dtype), r.to(s["x"].dtype)


def _layer_norm_backward_plain(s):
    r, dy, w = s["x"].float(), s["d_out"].float(), s["weight"].float()
    d = r - r.mean(1, keepdim=True)
    rstd = torch.rsqrt(d.square().mean(1, keepdim=True) + EPS)
    unit = d * rstd
    g = w * dy
    dx = rstd * (g - g.mean(1, keepdim=True) - unit * (g * unit).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return dx.to(s["x"].dtype), (dy * unit).sum(0), dy.sum(0)


def _integer_plain(s):
    x8, x_scale = _integer_rows(s["x"]) if s["case"]["quantize"] else (s["x8"], s["x_scale"])
    y = ((x8.float() @ s["w8"].float().t()) * x_scale[:, None] * s["w_scale"]).to(DTYPES[s["case"]["dtype"]])
    return (x8, x_scale, y) if s["case"]["quantize"] else y


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "scan_step":
            return _scan_step_plain(s)
        if op.startswith("scan"):
            return _scan_plain(s, op.endswith("backward"))
        if op == "conv_step":
            return _conv_step_plain(s)
        if op.startswith("conv"):
            return _conv_plain(s, op.endswith("backward"))
        if op == "layer_norm":
            return _layer_norm_plain(s)
        return _layer_norm_backward_plain(s) if op == "layer_norm_backward" else _integer_plain(s)
    from paper_2205_14756_amd import sequence
    if op.startswith("scan"):
        rest = {"skip": s["skip"], "delta_bias": s["bias"], "gate": s["z"], "softplus": case["softplus"]}
        args = (s["x"], s["delta"], s["a"], s["b"], s["c"])
        if op == "scan_step":
            return sequence.msla_selective_scan_step(*args, s["state"], new_state=s["new_state"], **rest)
        rest.update(sequences=case["seqs"], offsets=s["offsets"], initial_state=s["state"])
        if op == "scan":
            return sequence.msla_selective_scan_forward(*args, **rest)
        g = sequence.msla_selective_scan_backward(*args, s["d_out"], **rest)
        outs = {"d_x": g.d_x, "d_delta": g.d_delta, "d_a": g.d_a, "d_b": g.d_b, "d_c": g.d_c, "d_skip": g.d_skip}
        outs.update({k: v for k, v in (("d_bias", g.d_delta_bias), ("d_gate", g.d_gate), ("d_state", g.d_initial_state)) if v is not None})
        return outs
    if op == "conv_step":
        return sequence.msla_causal_conv_step(s["x"], s["weight"], s["state"], s["bias"], silu=case["silu"], new_state=s["new_state"])
    if op == "conv":
        return sequence.msla_causal_conv_forward(s["x"], s["weight"], s["bias"], silu=case["silu"], sequences=case["seqs"],
                                                 offsets=s["offsets"], initial_state=s["state"])
    if op == "conv_backward":
        dx, dw, db, ds = sequence.msla_causal_conv_backward(s["x"], s["weight"], s["d_out"], s["bias"], silu=case["silu"],
                                                            sequences=case["seqs"], offsets=s["offsets"], initial_state=s["state"])
        outs = {"d_x": dx, "d_weight": dw, "d_bias": db}
        if ds is not None:
            outs["d_state"] = ds
        return outs
    if op == "layer_norm":
        return sequence.msla_layer_norm_forward(s["x"], s["weight"], s["bias"], residual=s["residual"], eps=EPS)
    if op == "layer_norm_backward":
        return sequence.msla_layer_norm_backward(s["x"], s["weight"], s["d_out"], d_sum=s["residual"], eps=EPS)
    if not case["quantize"]:
        return sequence.msla_linear_integer(s["x8"], s["x_scale"], s["w8"], s["w_scale"], DTYPES[case["dtype"]])
    x8, x_scale = sequence.msla_quantize_rows_integer(s["x"])
    return x8, x_scale, sequence.msla_linear_integer(x8, x_scale, s["w8"], s["w_scale"], s["x"].dtype)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_steps(s):
    pre = s["delta"].double()
    if s["bias"] is not None:
        pre = pre + s["bias"].double()
    return pre, torch.logaddexp(pre, torch.zeros_like(pre)) if s["case"]["softplus"] else pre


def _exact_scan(s, backward):
    """Token by token, all sequences at once (a sequence that has ended hands its state on)."""
    case = s["case"]
    per, seqs, channels, n = case["channels"] // case["groups"], case["seqs"], case["channels"], case["states"]
    starts = torch.tensor(s["starts"], device="cuda")
    lengths, longest = starts[1:] - starts[:-1], max(b - a for a, b in zip(s["starts"], s["starts"][1:]))
    pre, dt = _exact_steps(s)
    x, a, skip = s["x"].double(), s["a"].double(), s["skip"].double()
    b, c = s["b"].double(), s["c"].double()
    wide = lambda t: t.repeat_interleave(per, 1)
    state = torch.zeros(seqs, channels, n, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()
    first, h, y, kept = state, state, torch.zeros_like(x), []
    z = None if s["z"] is None else s["z"].double()
    for t in range(longest):
        on = (t < lengths).nonzero()[:, 0] if case["packed"] else torch.arange(seqs, device="cuda")
        i = starts[on] + t
        if backward:
            kept.append(h)
        now = torch.exp(dt[i][..., None] * a) * h[on] + (dt[i] * x[i])[..., None] * wide(b[i])
        h = h.clone()
        h[on] = now
        y[i] = (now * wide(c[i])).sum(-1) + skip * x[i]
    if not backward:
        return (y if z is None else y * z / (1 + torch.exp(-z))), h
    do, dy, outs = s["d_out"].double(), s["d_out"].double(), {}
    if z is not None:
        e = torch.exp(-z)
        dy = do * z / (1 + e)
        outs["d_gate"] = do * y * ((1 + e) + z * e) / (1 + e) ** 2
    dx, dd, db, dc = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(b), torch.zeros_like(c)
    da, carry = torch.zeros_like(a), torch.zeros_like(state)
    for t in reversed(range(longest)):
        on = (t < lengths).nonzero()[:, 0] if case["packed"] else torch.arange(seqs, device="cuda")
        i = starts[on] + t
        decay = torch.exp(dt[i][..., None] * a)
        here = decay * kept[t][on] + (dt[i] * x[i])[..., None] * wide(b[i])
        dh = carry[on] + dy[i][..., None] * wide(c[i])
        db[i] = (dh * (dt[i] * x[i])[..., None]).unflatten(1, (case["groups"], per)).sum(2)
        dc[i] = (here * dy[i][..., None]).unflatten(1, (case["groups"], per)).sum(2)
        inflow = (dh * wide(b[i])).sum(2)
        log = dh * decay * kept[t][on]
        dx[i] = dt[i] * inflow + skip * dy[i]
        dd[i] = x[i] * inflow + (log * a).sum(2)
        da += (log * dt[i][..., None]).sum(0)
        carry[on] = decay * dh
    if case["softplus"]:
        dd = dd / (1 + torch.exp(-pre))
    outs.update(d_c=dc, d_b=db, d_a=da, d_skip=(dy * x).sum(0), d_x=dx, d_delta=dd)
    if s["bias"] is not None:
        outs["d_bias"] = dd.sum(0)
    if s["state"] is not None:
        outs["d_state"] = torch.where((lengths > 0)[:, None, None], carry, torch.zeros_like(first))
    return outs


def _exact_conv(s, backward):
    """Tap by tap over each sequence."""
    case = s["case"]
    w, weight, bias = case["width"], s["weight"].double(), s["bias"].double()
    x = s["x"].double()
    out, ends, dx, dstate = torch.zeros_like(x), [], torch.zeros_like(x), []
    dw, db = torch.zeros_like(weight), torch.zeros_like(bias)
    for i, (lo, hi) in enumerate(zip(s["starts"], s["starts"][1:])):
        head = torch.zeros(w - 1, case["channels"], dtype=torch.float64, device="cuda") if s["state"] is None else s["state"][i].double()
        rows, n = torch.cat([head, x[lo:hi]]), hi - lo
        pre = bias.expand(n, -1).clone()
        for k in range(w):
            pre += weight[:, k] * rows[k:k + n]
        sig = 1 / (1 + torch.exp(-pre))
        if not backward:
            out[lo:hi] = pre * sig if case["silu"] else pre
            ends.append(rows[n:])
            continue
        d = s["d_out"][lo:hi].double()
        if case["silu"]:
            d = d * (sig + pre * sig * (1 - sig))
        back = torch.zeros_like(rows)
        for k in range(w):
            back[k:k + n] += weight[:, k] * d
            dw[:, k] += (d * rows[k:k + n]).sum(0)
        db += d.sum(0)
        dx[lo:hi] = back[w - 1:]
        dstate.append(back[:w - 1])
    if not backward:
        return out, torch.stack(ends)
    outs = {"d_x": dx, "d_weight": dw, "d_bias": db}
    if s["state"] is not None:
        outs["d_state"] = torch.stack(dstate)
    return outs


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "scan_step":
        per = case["channels"] // case["groups"]
        _, dt = _exact_steps(s)
        x = s["x"].double()
        h = torch.exp(dt[:, :, None] * s["a"].double()) * s["state"].double()
        h = h + (dt * x)[:, :, None] * s["b"].double().repeat_interleave(per, 1)
        y = (h * s["c"].double().repeat_interleave(per, 1)).sum(-1) + s["skip"].double() * x
        return (y if s["z"] is None else y * s["z"].double() / (1 + torch.exp(-s["z"].double()))), h
    if op.startswith("scan"):
        return _exact_scan(s, op.endswith("backward"))
    if op == "conv_step":
        pre = s["bias"].double() + s["weight"][:, -1].double() * s["x"].double()
        for k in range(case["width"] - 1):
            pre = pre + s["weight"][:, k].double() * s["state"][:, k].double()
        state = torch.cat([s["state"][:, 1:], s["x"][:, None]], 1)
        return (pre / (1 + torch.exp(-pre)) if case["silu"] else pre), state.double()
    if op.startswith("conv"):
        return _exact_conv(s, op.endswith("backward"))
    if op.startswith("layer_norm"):
        r = s["x"].double()
        if op == "layer_norm" and s["residual"] is not None:
            r = r + s["residual"].double()
        n, w = case["channels"], s["weight"].double()
        centre = torch.sum(r, 1, keepdim=True) / n
        size = torch.sqrt(torch.sum((r - centre) ** 2, 1, keepdim=True) / n + EPS)
        if op == "layer_norm":
            return (r - centre) / size * w + s["bias"].double(), r
        # of sum(dy w (r - centre) / size): by r itself, by size (whose gradient is (r - centre) / (n size)), and by the centre
        dy = s["d_out"].double()
        by_size = -torch.sum(dy * w * (r - centre), 1, keepdim=True) / size ** 2
        dx = dy * w / size + by_size * (r - centre) / (n * size)
        dx = dx - torch.sum(dy * w, 1, keepdim=True) / (n * size)
        if s["residual"] is not None:
            dx = dx + s["residual"].double()
        return dx, torch.sum(dy * (r - centre) / size, 0), torch.sum(dy, 0)
    x8, x_scale = _integer_rows(s["x"]) if case["quantize"] else (s["x8"], s["x_scale"])
    y = (x8.double() @ s["w8"].double().t()) * x_scale.double()[:, None] * s["w_scale"].double()
    return (None, s["x"].double().abs().amax(1) / 127, y) if case["quantize"] else y


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    e = 4 if case["dtype"] == "f32" else 2
    if op.startswith("scan"):
        size, n, seqs = case["tokens"] * case["channels"], case["states"], case["seqs"]
        shared = e * case["tokens"] * case["groups"] * n * 2
        state = 4 * seqs * case["channels"] * n
        weights = 4 * case["channels"] * (n + 1 + case["softplus"])
        if op == "scan_step":
            return {"bytes": e * size * (3 + case["gated"]) + shared + weights + 2 * state, "flops": 7 * size * n}
        if op == "scan":
            return {"bytes": e * size * (3 + case["gated"]) + shared + weights + state * (1 + case["initial"]), "flops": 7 * size * n}
        # the decays and states again, the state's gradient, and five sums of its products
        return {"bytes": e * size * (5 + 2 * case["gated"]) + 2 * shared + 2 * weights + 2 * state * case["initial"], "flops": 22 * size * n}
    if op.startswith("conv"):
        size, w = case["tokens"] * case["channels"], case["width"]
        state, weights = e * case["seqs"] * (w - 1) * case["channels"], case["channels"] * (w + 1)
        if op == "conv_backward":
            return {"bytes": e * size * 3 + (e + 4) * weights + 2 * state * case["initial"], "flops": size * (6 * w + 10 * case["silu"])}
        return {"bytes": e * size * 2 + e * weights + state * (1 + case["initial"]), "flops": size * (2 * w + 5 * case["silu"])}
    if op.startswith("layer_norm"):
        size, channels = case["rows"] * case["channels"], case["channels"]
        if op == "layer_norm_backward":
            return {"bytes": e * size * (3 + case["residual"]) + channels * (e + 8), "flops": 14 * size}
        return {"bytes": e * size * (2 + 2 * case["residual"]) + 2 * e * channels, "flops": 8 * size}
    rows, c_in, c_out = case["rows"], case["c_in"], case["c_out"]
    rest = (e + 1) * rows * c_in if case["quantize"] else rows * c_in
    return {"bytes": rest + c_in * c_out + 4 * (rows + c_out) + e * rows * c_out, "flops": 2 * rows * c_in * c_out}

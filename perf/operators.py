"""Sequence operators as timed cases: the gated linear recurrence (over a sequence, its gradient, one token a
sequence), the root-mean-square norm with the residual's addition (plain, with an 8-bit output, its gradient) and the
projection of 8-bit rows.

A case is a dict; ``op`` says which entry point of ``paper_2205_14756_amd.sequence`` it is about:

* ``recurrence`` / ``recurrence_backward``: ``dtype``, ``seqs`` sequences of ``tokens`` rows in all, equally long or cut
  at random places (``packed``; some may be empty), ``heads_q`` query heads that share ``heads_kv`` states, ``head_dim``,
  ``gated``, ``rectify`` (ReLU on q and k), ``initial`` (the sequences go on from a state).
* ``recurrence_step``: the same with one token for each of ``seqs`` sequences.
* ``norm`` / ``norm_quantized`` / ``norm_backward``: ``rows``, ``channels``, ``residual`` (backward: a gradient that arrives
  through the sum).
* ``linear_quantized``: ``rows``, ``c_in``, ``c_out``; ``dtype`` is the output's.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
CHUNK = 64
E4M3_MAX = 448.0


# ------------------------------------------------------------------------------------------------ the cases
def _scan(name, op, dtype, seqs, tokens, heads_q, heads_kv, head_dim, packed=False, gated=True, rectify=False, initial=False):
    return {"name": name, "op": op, "dtype": dtype, "seqs": seqs, "tokens": tokens, "heads_q": heads_q, "heads_kv": heads_kv,
            "head_dim": head_dim, "packed": packed, "gated": gated, "rectify": rectify, "initial": initial}


def _norm(name, op, dtype, rows, channels, residual=True):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "channels": channels, "residual": residual}


def _linear(name, dtype, rows, c_in, c_out):
    return {"name": name, "op": "linear_quantized", "dtype": dtype, "rows": rows, "c_in": c_in, "c_out": c_out}


def listed():
    return [
        # one short prompt of a small model: latency
        _scan("scan_prompt", "recurrence", "bf16", 1, 203, 8, 8, 64, initial=True),
        # a training batch of long sequences
        _scan("scan_training", "recurrence", "bf16", 4, 16384, 16, 16, 128),
        # prompts of many lengths packed behind each other, four query heads to a state
        _scan("scan_packed", "recurrence", "f16", 24, 20011, 16, 4, 64, packed=True, initial=True),
        # the gradient of a training batch
        _scan("scan_gradient", "recurrence_backward", "bf16", 4, 16384, 16, 16, 128),
        # the gradient with this library's heads of 16, rectified, in single precision
        _scan("scan_gradient_d16", "recurrence_backward", "f32", 2, 4 * 1021, 16, 16, 16, rectify=True),
        # one token of one conversation
        _scan("step_one", "recurrence_step", "bf16", 1, 1, 16, 16, 128),
        # one token for each of many conversations
        _scan("step_many", "recurrence_step", "bf16", 192, 192, 32, 16, 128),
        # between the halves of a block, training
        _norm("norm_training", "norm", "bf16", 16384, 4096),
        # before an 8-bit projection, a batch of single tokens
        _norm("norm_decode_e4m3", "norm_quantized", "f16", 48, 4096),
        # the gradient, an odd width
        _norm("norm_gradient", "norm_backward", "bf16", 8192, 2051),
        # a batch of single tokens: the weights outweigh everything
        _linear("linear_decode_e4m3", "bf16", 48, 4096, 4096),
        # a batch of prompts
        _linear("linear_prompt_e4m3", "bf16", 4096, 4096, 8192),
    ]


def _log(rng, low, high):
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    op = rng.choice(["recurrence", "recurrence", "recurrence_backward", "recurrence_backward", "recurrence_step",
                     "norm", "norm_quantized", "norm_backward", "linear_quantized"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if op.startswith("recurrence"):
        heads_kv = rng.choice([1, 2, 3, 4, 8, 16])
        heads_q = heads_kv * rng.choice([1, 1, 2, 4])
        head_dim = rng.choice([16, 32, 64, 128])
        seqs = _log(rng, 1, 160 if op.endswith("step") else 16)
        length = 1 if op.endswith("step") else _log(rng, 1, 8192)
        # no more than the largest listed case
        while seqs * length * heads_q * head_dim > 4 * 4096 * 16 * 128:
            length = (length + 1) // 2
        packed = not op.endswith("step") and rng.random() < 0.5
        return {"op": op, "dtype": dtype, "seqs": seqs, "tokens": seqs * length, "heads_q": heads_q, "heads_kv": heads_kv,
                "head_dim": head_dim, "packed": packed, "gated": rng.random() < 0.8, "rectify": rng.random() < 0.3,
                "initial": rng.random() < 0.5}
    if op.startswith("norm"):
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
    return {"op": op, "dtype": rng.choice(["bf16", "f16"]), "rows": rows, "c_in": c_in, "c_out": c_out}


# ------------------------------------------------------------------------------------------------ inputs
def _offsets(case, seed):
    """Where the sequences start, and the end of the last one."""
    seqs, tokens = case["seqs"], case["tokens"]
    if not case["packed"]:
        return [i * (tokens // seqs) for i in range(seqs + 1)]
    cuts = np.sort(np.random.RandomState(seed % (1 << 31)).randint(0, tokens + 1, seqs - 1))
    return [0] + [int(c) for c in cuts] + [tokens]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape, dtype=None, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype or dt)

    dt, op = DTYPES[case["dtype"]], case["op"]
    s = {"case": case}
    if op.startswith("recurrence"):
        hq, hkv, d, seqs = case["heads_q"], case["heads_kv"], case["head_dim"], case["seqs"]
        tokens = case["tokens"]
        s["q"], s["k"], s["v"] = normal(tokens, hq, d), normal(tokens, hkv, d), normal(tokens, hkv, d)
        s["gate"] = None
        if case["gated"]:   # heads that forget within some tokens, others that remember some hundreds
            bias = torch.linspace(1.0, 6.0, hkv, device="cuda")
            s["gate"] = torch.nn.functional.logsigmoid(normal(tokens, hkv, dtype=torch.float32) + bias).to(dt)
        if op == "recurrence_step":
            s["state"] = normal(seqs, hkv, d, d, dtype=torch.float32, std=4.0)
            s["new_state"] = torch.empty_like(s["state"])
            return s
        s["state"] = normal(seqs, hkv, d, d, dtype=torch.float32) if case["initial"] else None
        s["starts"] = _offsets(case, seed)
        s["offsets"] = torch.tensor(s["starts"], dtype=torch.int32, device="cuda") if case["packed"] else None
        if op == "recurrence_backward":
            s["d_out"] = normal(tokens, hq, d)
        return s
    if op.startswith("norm"):
        rows, channels = case["rows"], case["channels"]
        s["x"] = normal(rows, channels)
        s["weight"] = (1.0 + normal(channels, dtype=torch.float32, std=0.1)).to(dt)
        s["residual"] = normal(rows, channels) if case["residual"] else None
        if op == "norm_backward":
            s["d_out"] = normal(rows, channels)
        return s

    def rows8(rows, channels):
        values = normal(rows, channels, dtype=torch.float32)
        scale = values.abs().amax(1) / E4M3_MAX
        return (values / scale[:, None]).to(torch.float8_e4m3fn), scale

    s["x8"], s["x_scale"] = rows8(case["rows"], case["c_in"])
    s["w8"], s["w_scale"] = rows8(case["c_out"], case["c_in"])
    s["w_scale"] = s["w_scale"] / math.sqrt(case["c_in"])
    return s


# ------------------------------------------------------------------------------------------------ the plain forms
def _cumulative(x, dim):
    return torch.cumsum(x.double(), dim)


def _scan_plain(q, k, v, g, state):
    """out_i = q_i^T S_i with S_i = exp(g_i) S_{i-1} + k_i v_i^T, S_{-1} = state: chunks of 64 tokens, the chunks' states joined
    by one product with the matrix of decays between them.  q, k, v [seqs, heads, group, N, d], g [seqs, heads, 1, N],
    state [seqs, heads, group, d, d].  Returns out and the last state."""
    n, d = q.shape[-2], q.shape[-1]
    pad = -n % CHUNK
    q, k, v = (torch.nn.functional.pad(t, (0, 0, 0, pad)) for t in (q, k, v))
    g = torch.nn.functional.pad(g, (0, pad))
    nc = (n + pad) // CHUNK
    q, k, v = (t.unflatten(-2, (nc, CHUNK)) for t in (q, k, v))
    within = _cumulative(g.unflatten(-1, (nc, CHUNK)), -1)
    total = within[..., -1]
    ends = _cumulative(total, -1)
    # decay from token j to token i of a chunk, and from the end of chunk c' to the start of chunk c
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=q.device).tril()
    decay = torch.where(low, within[..., :, None] - within[..., None, :], -math.inf).exp().float()
    before = torch.cat([torch.zeros_like(ends[..., :1]), ends], -1)                     # nc + 1 chunk borders
    earlier = torch.ones(nc + 1, nc, dtype=torch.bool, device=q.device).tril(-1)
    between = torch.where(earlier, before[..., :, None] - ends[..., None, :], -math.inf).exp().float()
    own_state = (k * (total[..., None] - within).exp().float()[..., None]).transpose(-1, -2) @ v
    states = (between @ own_state.flatten(-2)).unflatten(-1, (d, d)) + before.exp().float()[..., None, None] * state[..., None, :, :]
    out = ((q @ k.transpose(-1, -2)) * decay) @ v + (q * within.exp().float()[..., None]) @ states[..., :-1, :, :]
    return out.flatten(-3, -2)[..., :n, :], states[..., -1, :, :]


def _padded(s):
    """Indices [seqs, longest] of the rows of each sequence, and which of them are rows."""
    starts = torch.tensor(s["starts"], device="cuda")
    lengths = starts[1:] - starts[:-1]
    at = torch.arange(max(1, int(max(b - a for a, b in zip(s["starts"], s["starts"][1:])))), device="cuda")
    live = at[None, :] < lengths[:, None]
    return torch.where(live, starts[:-1, None] + at[None, :], 0), live


def _recurrence_plain(s, backward):
    case = s["case"]
    hkv, group, d = case["heads_kv"], case["heads_q"] // case["heads_kv"], case["head_dim"]
    scale = 1.0 / math.sqrt(d)
    rows, live = _padded(s)

    def heads(x):      # [tokens, heads, d] -> [seqs, heads_kv, group, N, d], zeros behind each sequence
        x = torch.where(live[..., None, None], x.float()[rows], 0.0)
        return x.unflatten(2, (hkv, -1)).permute(0, 2, 3, 1, 4)

    def flat(x):       # ... and back
        return x.permute(0, 3, 1, 2, 4).flatten(2, 3)[live]

    q, k, v = heads(s["q"]), heads(s["k"]), heads(s["v"])
    if case["rectify"]:
        q, k = q.clamp(min=0), k.clamp(min=0)
    g = torch.zeros(live.shape[0], hkv, 1, live.shape[1], device="cuda")
    if s["gate"] is not None:
        g = torch.where(live[..., None], s["gate"].float()[rows], 0.0).permute(0, 2, 1)[:, :, None, :]
    state = torch.zeros(live.shape[0], hkv, 1, d, d, device="cuda") if s["state"] is None else s["state"][:, :, None]
    if not backward:
        out, last = _scan_plain(q * scale, k, v, g, state)
        return flat(out).to(s["q"].dtype), last[:, :, 0]
    # the gradient: of q by the same scan with the places of k and v exchanged, of k and v by scans from the end
    do = heads(s["d_out"])
    back = torch.cat([torch.zeros_like(g[..., :1]), g.flip(-1)[..., :-1]], -1)
    none = torch.zeros(live.shape[0], hkv, group, d, d, device="cuda")
    dq, _ = _scan_plain(do * scale, v, k, g, state.transpose(-1, -2))
    q_, k_, v_, do_ = ((t * w).flip(-2) for t, w in ((q, scale), (k, 1.0), (v, 1.0), (do, 1.0)))
    dk, _ = _scan_plain(v_, do_, q_, back, none)
    dv, dstate = _scan_plain(k_, q_, do_, back, none)
    dk, dv = dk.flip(-2).sum(2, keepdim=True), dv.flip(-2).sum(2, keepdim=True)
    outs = {}
    if s["gate"] is not None:
        through = ((q * dq).sum(-1).double().sum(2) - (k * dk).sum(-1).double().sum(2)).flip(-1)
        outs["d_gate"] = _cumulative(through, -1).flip(-1).permute(0, 2, 1)[live].to(s["q"].dtype)
    if s["state"] is not None:
        outs["d_state"] = dstate.sum(2) * g[..., 0, :1, None].exp()
    if case["rectify"]:
        dq, dk = torch.where(q > 0, dq, 0.0), torch.where(k > 0, dk, 0.0)
    return {"dq": flat(dq).to(s["q"].dtype), "dk": flat(dk).to(s["q"].dtype), "dv": flat(dv).to(s["q"].dtype), **outs}


def _step_plain(s):
    case = s["case"]
    hkv, d = case["heads_kv"], case["head_dim"]
    q, k, v = s["q"].float().unflatten(1, (hkv, -1)), s["k"].float(), s["v"].float()
    if case["rectify"]:
        q, k = q.clamp(min=0), k.clamp(min=0)
    state = s["state"] if s["gate"] is None else s["state"] * s["gate"].float().exp()[..., None, None]
    state = state + k[..., :, None] * v[..., None, :]
    return ((q / math.sqrt(d)) @ state).flatten(1, 2).to(s["q"].dtype), state


def _norm_plain(s):
    r = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
    y = r * torch.rsqrt(r.square().mean(1, keepdim=True) + EPS) * s["weight"].float()
    total = r.to(s["x"].dtype)
    if s["case"]["op"] == "norm":
        return y.to(s["x"].dtype), total
    scale = y.abs().amax(1) / E4M3_MAX
    return (y / torch.where(scale > 0, scale, 1.0)[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale, total


def _norm_backward_plain(s):
    r, dy, w = s["x"].float(), s["d_out"].float(), s["weight"].float()
    rstd = torch.rsqrt(r.square().mean(1, keepdim=True) + EPS)
    unit = r * rstd
    dx = rstd * (w * dy - unit * (w * dy * unit).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return dx.to(s["x"].dtype), (dy * unit).sum(0)


def _linear_plain(s):
    y = s["x8"].float() @ s["w8"].float().t()
    return (y * s["x_scale"][:, None] * s["w_scale"]).to(DTYPES[s["case"]["dtype"]])


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        if op == "recurrence_step":
            return _step_plain(s)
        if op.startswith("recurrence"):
            return _recurrence_plain(s, op.endswith("backward"))
        if op == "norm_backward":
            return _norm_backward_plain(s)
        return _norm_plain(s) if op.startswith("norm") else _linear_plain(s)
    from paper_2205_14756_amd import sequence
    if op == "recurrence_step":
        return sequence.msla_recurrence_step(s["q"], s["k"], s["v"], s["state"], s["gate"], rectify=case["rectify"],
                                             new_state=s["new_state"])
    if op == "recurrence":
        return sequence.msla_recurrence_forward(s["q"], s["k"], s["v"], s["gate"], sequences=case["seqs"], offsets=s["offsets"],
                                                initial_state=s["state"], rectify=case["rectify"])
    if op == "recurrence_backward":
        dq, dk, dv, dg, ds = sequence.msla_recurrence_backward(
            s["q"], s["k"], s["v"], s["d_out"], s["gate"], sequences=case["seqs"], offsets=s["offsets"], initial_state=s["state"],
            rectify=case["rectify"])
        outs = {"dq": dq, "dk": dk, "dv": dv}
        if dg is not None:
            outs["d_gate"] = dg
        if ds is not None:
            outs["d_state"] = ds
        return outs
    if op == "norm":
        return sequence.msla_norm_forward(s["x"], s["weight"], residual=s["residual"], eps=EPS)
    if op == "norm_quantized":
        return sequence.msla_norm_quantized(s["x"], s["weight"], residual=s["residual"], eps=EPS)
    if op == "norm_backward":
        return sequence.msla_norm_backward(s["x"], s["weight"], s["d_out"], d_sum=s["residual"], eps=EPS)
    return sequence.msla_linear_quantized(s["x8"], s["x_scale"], s["w8"], s["w_scale"], DTYPES[case["dtype"]])


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_sequence(q, k, v, g, state, do):
    """One sequence of one state with its query heads, by the whole N x N matrix of decays.  q, do [N, group, d], k, v [N, d], g [N],
    state [d, d]."""
    n, d = k.shape
    scale = d ** -0.5
    upto = torch.cumsum(g, 0)
    decay = torch.exp(torch.where(torch.ones(n, n, dtype=torch.bool, device=g.device).tril(), upto[:, None] - upto[None, :], -math.inf))
    outs, grads = [], None
    end = torch.exp(upto[-1]) * state + (k * torch.exp(upto[-1] - upto)[:, None]).t() @ v
    if do is None:
        for h in range(q.shape[1]):
            outs.append(scale * ((decay * (q[:, h] @ k.t())) @ v + torch.exp(upto)[:, None] * (q[:, h] @ state)))
        return torch.stack(outs, 1), end
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dstate, crossing = torch.zeros_like(state), torch.zeros_like(g)
    for h in range(q.shape[1]):
        scores, dots = decay * (q[:, h] @ k.t()) * scale, do[:, h] @ v.t()
        dscores = decay * dots * scale
        carried = torch.exp(upto)[:, None] * scale
        dq[:, h] = dscores @ k + carried * (do[:, h] @ state.t())
        dk += dscores.t() @ q[:, h]
        dv += scores.t() @ do[:, h]
        dstate += (carried * q[:, h]).t() @ do[:, h]
        # what crosses the border before token t: pairs (i >= t > j), and the state's part of every i >= t
        pairs = scores * dots
        from_state = (carried * (q[:, h] @ state) * do[:, h]).sum(1)
        inflow = torch.flip(torch.cumsum(torch.flip(pairs.sum(1) + from_state, [0]), 0), [0])
        crossing += inflow - torch.flip(torch.cumsum(torch.flip(pairs.sum(0), [0]), 0), [0])
    return dq, dk, dv, crossing, dstate


def _exact_recurrence(s, backward):
    case = s["case"]
    hkv, group = case["heads_kv"], case["heads_q"] // case["heads_kv"]
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    if case["rectify"]:
        q, k = torch.relu(q), torch.relu(k)
    g = torch.zeros(case["tokens"], hkv, dtype=torch.float64, device="cuda") if s["gate"] is None else s["gate"].double()
    first = torch.zeros(case["seqs"], hkv, case["head_dim"], case["head_dim"], dtype=torch.float64, device="cuda")
    if s["state"] is not None:
        first = s["state"].double()
    out, last = torch.zeros_like(q), first.clone()
    dq, dk, dv, dg, ds = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(g), torch.zeros_like(first)
    for b, (lo, hi) in enumerate(zip(s["starts"], s["starts"][1:])):
        for h in range(hkv) if hi > lo else ():
            mine = slice(h * group, (h + 1) * group)
            do = s["d_out"][lo:hi, mine].double() if backward else None
            got = _exact_sequence(q[lo:hi, mine], k[lo:hi, h], v[lo:hi, h], g[lo:hi, h], first[b, h], do)
            if backward:
                dq[lo:hi, mine], dk[lo:hi, h], dv[lo:hi, h], dg[lo:hi, h], ds[b, h] = got
            else:
                out[lo:hi, mine], last[b, h] = got
    if not backward:
        return out, last
    if case["rectify"]:
        dq, dk = dq * (q > 0), dk * (k > 0)
    outs = {"dq": dq, "dk": dk, "dv": dv}
    if s["gate"] is not None:
        outs["d_gate"] = dg
    if s["state"] is not None:
        outs["d_state"] = ds
    return outs


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("recurrence", "recurrence_backward"):
        return _exact_recurrence(s, op.endswith("backward"))
    if op == "recurrence_step":
        group = case["heads_q"] // case["heads_kv"]
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        if case["rectify"]:
            q, k = torch.relu(q), torch.relu(k)
        keep = 1.0 if s["gate"] is None else torch.exp(s["gate"].double())[:, :, None, None]
        state = keep * s["state"].double() + k[:, :, :, None] * v[:, :, None, :]
        out = (q[:, :, :, None] * state.repeat_interleave(group, 1)).sum(2) * case["head_dim"] ** -0.5
        return out, state
    if op.startswith("norm"):
        r = s["x"].double()
        if op != "norm_backward" and s["residual"] is not None:
            r = r + s["residual"].double()
        size = torch.sqrt(torch.sum(r * r, 1) / case["channels"] + EPS)[:, None]
        w = s["weight"].double()
        if op == "norm_backward":
            # of sum(dy r w / size): by r itself, and by size, whose own gradient is r / (channels size)
            dy = s["d_out"].double()
            by_size = -torch.sum(dy * w * r, 1, keepdim=True) / size ** 2
            dx = dy * w / size + by_size * r / (case["channels"] * size)
            if s["residual"] is not None:
                dx = dx + s["residual"].double()
            return dx, torch.sum(dy * r / size, 0)
        y = r / size * w
        if op == "norm":
            return y, r
        top = y.abs().max(1).values / E4M3_MAX
        return y / torch.where(top > 0, top, torch.ones_like(top))[:, None], top, r
    y = s["x8"].double() @ s["w8"].double().t()
    return y * s["x_scale"].double()[:, None] * s["w_scale"].double()[None, :]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    e = 4 if case["dtype"] == "f32" else 2
    if op.startswith("recurrence"):
        n, hq, hkv, d, seqs = case["tokens"], case["heads_q"], case["heads_kv"], case["head_dim"], case["seqs"]
        state = 4 * seqs * hkv * d * d
        gate = e * n * hkv if case["gated"] else 0
        if op == "recurrence_step":
            return {"bytes": 2 * state + e * n * d * (2 * hq + 2 * hkv) + gate, "flops": n * d * d * (3 * hkv + 2 * hq)}
        # chunks of 64 tokens: half of two 64-wide products, one with the state a query head, one into the state a state
        pair = 2 * d * CHUNK
        if op == "recurrence":
            return {"bytes": e * n * d * (2 * hq + 2 * hkv) + gate + state * (1 + case["initial"]),
                    "flops": n * (hq * (pair + 2 * d * d) + hkv * 2 * d * d)}
        return {"bytes": e * n * d * (3 * hq + 4 * hkv) + 2 * gate + state * 2 * case["initial"],
                "flops": n * hq * (2.5 * pair + 4 * 2 * d * d) + n * hkv * 2 * d * d}
    if op.startswith("norm"):
        rows, channels = case["rows"], case["channels"]
        size = rows * channels
        if op == "norm_backward":
            return {"bytes": e * size * (3 + case["residual"]) + channels * (e + 4), "flops": 10 * size}
        out = size + 4 * rows if op == "norm_quantized" else e * size
        return {"bytes": e * size * (2 + case["residual"]) + out + e * channels, "flops": 6 * size}
    rows, c_in, c_out = case["rows"], case["c_in"], case["c_out"]
    return {"bytes": c_in * (rows + c_out) + 4 * (rows + c_out) + e * rows * c_out, "flops": 2 * rows * c_in * c_out}

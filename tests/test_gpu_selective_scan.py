"""The scan with a decay for each state through the C ABI against oracle/layer_oracle.py (fp64, token by token).

Tolerances, element by element: half a step of the type that a result is rounded to once, plus WAY times the sum of the magnitudes of the result's
terms (the same recurrence on magnitudes).  WAY covers fp32 on the way, in units of 2^-24: a token that a state passes costs it the rounding of its decay's
exponent, the exponential (2) and the multiply-add (1); the step and the gate (softplus, sigmoid: some ulps each), the exponent's own relative error
times an exponent of up to 16, and sums over states, channels (tree) and tokens the rest: (256 + 4 tokens) 2^-24."""
import functools

import numpy as np
import pytest
import torch

from oracle import layer_oracle as lo
from paper_2205_14756_amd import sequence as seq

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def half_step(dtype):
    return torch.finfo(TDT[dtype]).eps / 2


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


@functools.lru_cache(maxsize=None)
def _numbers(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape))


def offsets_of(lens, start=0):
    return [start + sum(lens[:i]) for i in range(len(lens) + 1)]


def make(seed, dtype, tokens, channels, groups, states, n, softplus=True, gated=True, full=True, initial=True):
    num = lambda i, *s: _numbers(seed * 16 + i, *s)
    store = lambda v: v.to(TDT[dtype]).cuda()
    t = dict(x=store(num(0, tokens, channels)), b=store(num(1, tokens, groups, states)), c=store(num(2, tokens, groups, states)),
             d_out=store(num(3, tokens, channels)))
    steps = torch.exp(num(4, channels) - 3.5).clamp(1e-3, 0.4)
    t["bias"] = torch.log(torch.expm1(steps)).float().cuda() if softplus and full else None
    t["delta"] = store(num(5, tokens, channels) * 0.5 - (0 if full else 3)) if softplus else store(steps * torch.exp(0.3 * num(5, tokens, channels)))
    t["a"] = -(torch.arange(1, states + 1) * torch.exp(0.2 * num(6, channels, states))).float().cuda()
    t["skip"] = num(7, channels).float().cuda() if full else None
    t["gate"] = store(num(8, tokens, channels)) if gated else None
    t["first"] = num(9, n, channels, states).float().cuda() if initial else None
    t["d_last"] = num(10, n, channels, states).float().cuda() if initial else None
    return t


def close(got, want, size, dtype, what, way, half=True):
    got = f64(got)
    assert np.isfinite(got).all(), what
    tol = (half_step(dtype) * np.abs(want) if half else 0) + way * size + (2.0 ** -24 if dtype == "f16" and half else 1e-30)
    worst = np.max(np.abs(got - want) / tol) if got.size else 0.0
    print(f"  {what}: {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1.0, what


def args_of(t):
    return t["x"], t["delta"], t["a"], t["b"], t["c"]


def rest_of(t, softplus):
    return dict(skip=t["skip"], delta_bias=t["bias"], gate=t["gate"], softplus=softplus)


def check(dtype, lens, channels, groups, states, softplus=True, gated=True, full=True, initial=True, start=0, tail=0, packed=True, seed=1, backward=True):
    tokens = start + sum(lens) + tail
    print(f"scan {dtype} lens={lens if len(lens) < 12 else len(lens)} channels={channels}/{groups} states={states} softplus={softplus} gated={gated} "
          f"full={full} initial={initial}", flush=True)
    t = make(seed, dtype, tokens, channels, groups, states, len(lens), softplus, gated, full, initial)
    offs = offsets_of(lens, start)
    spans = list(zip(offs[:-1], offs[1:]))
    dev_offs = torch.tensor(offs, dtype=torch.int32, device="cuda") if packed else None
    way = (256 + 4 * max(lens)) * 2.0 ** -24
    live = np.zeros(tokens, bool)
    for lo_, hi in spans:
        live[lo_:hi] = True
    rows = torch.from_numpy(live).cuda()
    args = [f64(v) for v in args_of(t)]
    rest = {k: f64(t[v]) for k, v in (("skip", "skip"), ("bias", "bias"), ("gate", "gate"))}
    rest["softplus"] = softplus
    first, d_last = f64(t["first"]), f64(t["d_last"])
    mag = lambda v: None if v is None else np.abs(v)
    out, last, _ = lo.scan(*args, spans, initial=first, **rest)
    # magnitudes: |x|, |b|, |c|, |skip|, |first| with the true steps and decays, and |silu|
    _, steps = lo.steps_of(args[1], rest["bias"], softplus)
    _, size_last, size = lo.scan(mag(args[0]), steps, args[2], mag(args[3]), mag(args[4]), spans, skip=mag(rest["skip"]), initial=mag(first))
    if gated:
        size = size * np.abs(rest["gate"] * lo.sigmoid(rest["gate"]))
    kw = dict(sequences=len(lens), offsets=dev_offs, initial_state=t["first"], **rest_of(t, softplus))
    n_ws = seq.msla_selective_scan_workspace_bytes(len(lens), tokens, channels, groups, states, TDT[dtype], packed=packed)
    ws = torch.full((n_ws + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    to = torch.full((tokens, channels), 7.0, dtype=TDT[dtype], device="cuda")
    got, state = seq.msla_selective_scan_forward(*args_of(t), out=to, workspace=ws[:n_ws], **kw)
    torch.cuda.synchronize()
    assert bool((ws[n_ws:] == 0xFF).all()), "bytes past the workspace were written"
    assert bool((got[~rows] == 7.0).all()), "rows of no sequence were written"
    close(got[rows], out[live], size[live], dtype, "out", way)
    close(state, last, size_last, dtype, "state", way, half=False)
    if not backward:
        return
    want = lo.scan_backward(*args, spans, f64(t["d_out"]), initial=first, d_last=d_last, **rest)
    sizes = lo.scan_backward(*args, spans, f64(t["d_out"]), initial=first, d_last=d_last, magnitudes=True, **rest)
    n_ws = seq.msla_selective_scan_workspace_bytes(len(lens), tokens, channels, groups, states, TDT[dtype], packed=packed, backward=True)
    ws = torch.full((n_ws + 512,), 0xFF, dtype=torch.uint8, device="cuda")
    seven = lambda v: None if v is None else torch.full_like(v, 7.0)
    run = lambda ws: seq.msla_selective_scan_backward(*args_of(t), t["d_out"], d_final_state=t["d_last"], d_x=seven(t["x"]), d_delta=seven(t["x"]),
                                                      d_b=seven(t["b"]), d_c=seven(t["c"]), d_gate=seven(t["gate"]), workspace=ws, **kw)
    g = run(ws[:n_ws])
    torch.cuda.synchronize()
    assert bool((ws[n_ws:] == 0xFF).all()), "bytes past the workspace were written"
    for name, v in (("x", g.d_x), ("delta", g.d_delta), ("b", g.d_b), ("c", g.d_c), ("gate", g.d_gate)):
        if v is not None:
            assert bool((v[~rows] == 7.0).all()), "rows of no sequence were written: " + name
            close(v[rows], want[name][live], sizes[name][live], dtype, "d_" + name, way)
    for name, v in (("a", g.d_a), ("skip", g.d_skip), ("bias", g.d_delta_bias), ("initial", g.d_initial_state)):
        if v is not None:
            size = sizes[name] if name != "bias" else sizes["delta"].sum(0)
            close(v, want[name], size, dtype, "d_" + name, (256 + 4 * sum(lens)) * 2.0 ** -24, half=False)
    for p, q in zip(g, run(None)):                  # the same bits again
        assert p is None and q is None or torch.equal(p, q)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("states", [8, 16, 32, 64])
@pytest.mark.parametrize("lens", [[1], [2], [5], [33], [64], [65, 1, 0, 130]])
def test_sizes(dtype, states, lens):
    check(dtype, lens, 80, 2, states)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("channels,groups", [(1, 1), (3, 1), (63, 1), (64, 1), (65, 1), (195, 3), (24, 24), (2048, 1)])
def test_channels(dtype, channels, groups):
    check(dtype, [37, 20], channels, groups, 16)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("states", [8, 16, 64])
def test_long(dtype, states):
    check(dtype, [600], 48, 1, states, seed=2)
    check(dtype, [300, 300], 48, 1, states, seed=3, packed=False)


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("full,initial", [(True, True), (False, True), (True, False), (False, False)])
def test_optional_operands(softplus, gated, full, initial):
    check("bf16", [70, 131], 33, 1, 16, softplus, gated, full, initial, seed=4)


def test_rows_of_no_sequence_are_left_alone():
    check("f32", [10, 0, 97], 20, 2, 16, start=5, tail=9, seed=5)
    check("bf16", [0, 0, 0], 20, 2, 16, start=5, tail=9, seed=5)


def test_many_sequences():
    lens = [int(v) for v in np.random.default_rng(6).integers(0, 9, 300)]
    check("f16", lens, 70, 1, 16, seed=6)
    check("f32", [3] * 200, 70, 1, 32, seed=7, packed=False)


def test_parts_of_wider_rows_in_any_place():
    """x, gate, delta, b and c as parts of rows that start at odd elements, outputs as well; one row for all tokens"""
    t = make(8, "bf16", 90, 50, 1, 16, 2)
    kw = dict(sequences=2, initial_state=t["first"], **rest_of(t, True))
    want, state = seq.msla_selective_scan_forward(*args_of(t), **kw)
    grads = seq.msla_selective_scan_backward(*args_of(t), t["d_out"], d_final_state=t["d_last"], **kw)
    wide = torch.full((90, 2 * 50 + 3 + 32 + 50), 3.0, dtype=torch.bfloat16, device="cuda")
    place = lambda at, v: wide[:, at:at + v.shape[-1]].copy_(v.flatten(1))
    x, gate, delta = place(1, t["x"]), place(51, t["gate"]), place(101 + 34, t["delta"])
    b, c = place(102, t["b"]).unflatten(1, (1, 16)), place(118, t["c"])
    room = torch.full((90, 53), 7.0, dtype=torch.bfloat16, device="cuda")
    kw["gate"] = gate
    got, state2 = seq.msla_selective_scan_forward(x, delta, t["a"], b, c.unflatten(1, (1, 16)), out=room[:, 2:52], **kw)
    assert torch.equal(got, want) and torch.equal(state, state2)
    assert bool((room[:, :2] == 7.0).all()) and bool((room[:, 52:] == 7.0).all())
    dwide = torch.full_like(wide, 7.0)
    g = seq.msla_selective_scan_backward(x, delta, t["a"], b, c.unflatten(1, (1, 16)), t["d_out"], d_final_state=t["d_last"], d_x=dwide[:, 1:51],
                                         d_gate=dwide[:, 51:101], d_b=dwide[:, 102:118].unflatten(1, (1, 16)),
                                         d_c=dwide[:, 118:134].unflatten(1, (1, 16)), d_delta=dwide[:, 135:185], **kw)
    for p, q in zip(g, grads):
        assert torch.equal(p, q)
    assert bool((dwide[:, 101] == 7.0).all()) and bool((dwide[:, 134] == 7.0).all()) and bool((dwide[:, 0] == 7.0).all())
    # one row of b and of the steps for all tokens
    one = t["b"][:1].expand(90, 1, 16), t["delta"][:1].expand(90, 50)
    p = seq.msla_selective_scan_forward(t["x"], one[1], t["a"], one[0], t["c"], **rest_of(t, True))
    q = seq.msla_selective_scan_forward(t["x"], one[1].contiguous(), t["a"], one[0].contiguous(), t["c"], **rest_of(t, True))
    assert torch.equal(p[0], q[0]) and torch.equal(p[1], q[1])


def test_the_state_in_place_and_a_sequence_in_pieces():
    t = make(9, "bf16", 300, 96, 1, 16, 1)
    rest = rest_of(t, True)
    whole, state = seq.msla_selective_scan_forward(*args_of(t), initial_state=t["first"], **rest)
    s = t["first"].clone()
    outs = []
    for lo_, hi in ((0, 1), (1, 130), (130, 300)):
        part = {k: (v[lo_:hi] if k in ("x", "delta", "b", "c", "gate", "d_out") and v is not None else v) for k, v in t.items()}
        outs.append(seq.msla_selective_scan_forward(*args_of(part), initial_state=s, final_state=s, **rest_of(part, True))[0])
    way = (256 + 4 * 300) * 2.0 ** -24
    torch.testing.assert_close(s, state, rtol=way, atol=way * float(state.abs().max()))
    torch.testing.assert_close(torch.cat(outs).float(), whole.float(), rtol=2.0 ** -7, atol=way * float(whole.abs().max()))


@pytest.mark.parametrize("lens", [[2000], [900, 0, 3, 700]])
def test_the_state_in_place_where_sequences_are_cut(lens):
    """many slots to a sequence, more workgroups than run at once: the last may end before the first begins"""
    t = make(14, "bf16", sum(lens), 2048, 1, 16, len(lens))
    offs = torch.tensor(offsets_of(lens), dtype=torch.int32, device="cuda")
    assert seq.msla_selective_scan_workspace_bytes(len(lens), sum(lens), 2048, 1, 16, torch.bfloat16, packed=True) > 0
    want, state = seq.msla_selective_scan_forward(*args_of(t), offsets=offs, initial_state=t["first"], **rest_of(t, True))
    for _ in range(3):
        s = t["first"].clone()
        got, _ = seq.msla_selective_scan_forward(*args_of(t), offsets=offs, initial_state=s, final_state=s, **rest_of(t, True))
        assert torch.equal(got, want) and torch.equal(s, state)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("states", [8, 16, 32, 64])
@pytest.mark.parametrize("sequences,channels,groups", [(1, 1, 1), (3, 100, 2), (150, 64, 1)])
def test_step(dtype, states, sequences, channels, groups):
    print(f"scan step {dtype} {sequences} x {channels}/{groups} states {states}", flush=True)
    t = make(10, dtype, sequences, channels, groups, states, sequences)
    spans = [(i, i + 1) for i in range(sequences)]
    rest = {k: f64(t[v]) for k, v in (("skip", "skip"), ("bias", "bias"), ("gate", "gate"))}
    args = [f64(v) for v in args_of(t)]
    out, last, _ = lo.scan(*args, spans, initial=f64(t["first"]), softplus=True, **rest)
    _, steps = lo.steps_of(args[1], rest["bias"], True)
    _, size_last, size = lo.scan(np.abs(args[0]), steps, args[2], np.abs(args[3]), np.abs(args[4]), spans, skip=np.abs(rest["skip"]),
                                 initial=np.abs(f64(t["first"])))
    size = size * np.abs(rest["gate"] * lo.sigmoid(rest["gate"]))
    new = torch.full_like(t["first"], 7.0)
    got, new = seq.msla_selective_scan_step(*args_of(t), t["first"], new_state=new, **rest_of(t, True))
    way = 260 * 2.0 ** -24
    close(got, out, size, dtype, "out", way)
    close(new, last, size_last, dtype, "state", way, half=False)
    s = t["first"].clone()
    again, s2 = seq.msla_selective_scan_step(*args_of(t), s, **rest_of(t, True))
    assert s2 is s and torch.equal(s, new) and torch.equal(again, got)
    full, state = seq.msla_selective_scan_forward(*args_of(t), sequences=sequences, initial_state=t["first"], **rest_of(t, True))
    close(full, out, size, dtype, "the same as sequences of one token", way)
    close(state, last, size_last, dtype, "their states", way, half=False)


def test_steps_of_every_size():
    """softplus over its whole range, relative to its own size: the state behind one token of x = b = 1 is the step"""
    v = torch.cat([torch.linspace(-80, 80, 1601), torch.tensor([-87.0, -1e-3, 0.0, 1e-3, 16.6, 88.0, 1e4])])
    n = len(v)
    one = lambda *s: torch.ones(*s, device="cuda")
    _, h = seq.msla_selective_scan_forward(one(1, n), v.float()[None].cuda(), -one(n, 8), one(1, 8), one(1, 8), softplus=True)
    _, want = lo.steps_of(v.float().numpy(), None, True)
    got = f64(h[0, :, 0])
    rel = np.abs(got - want) / want
    # exp's argument is off by half an ulp of itself (|v| 2^-24 of the result), and some ulps
    assert (rel <= (16 + 2 * np.abs(v.numpy())) * 2.0 ** -24).all(), (v[int(rel.argmax())], rel.max())


def test_values_that_are_not_finite_stay_in_their_channel_and_behind_their_token():
    t = make(11, "f32", 200, 40, 2, 16, 2)
    kw = dict(sequences=2, **rest_of(t, True))
    clean, _ = seq.msla_selective_scan_forward(*args_of(t), **kw)
    x = t["x"].clone()
    x[50, 7], x[160, 9] = float("nan"), float("inf")
    got, state = seq.msla_selective_scan_forward(x, *args_of(t)[1:], **kw)
    bad = ~torch.isfinite(got)
    assert bool(bad[50:100, 7].all()) and bool(bad[160:, 9].all())
    bad[50:100, 7] = False
    bad[160:, 9] = False
    assert not bool(bad.any())
    keep = torch.isfinite(got)
    assert torch.equal(got[keep], clean[keep])
    b = t["b"].clone()
    b[120, 1] = float("inf")
    got, _ = seq.msla_selective_scan_forward(t["x"], t["delta"], t["a"], b, t["c"], **kw)
    bad = ~torch.isfinite(got)
    assert not bool(bad[:120].any()) and not bool(bad[:, :20].any()) and bool(bad[120:, 20:].all())
    # the last token of a run of two: nothing that is not finite comes from behind it
    b = t["b"][:2].clone()
    b[1] = float("inf")
    _, state = seq.msla_selective_scan_forward(t["x"][:2].abs(), t["delta"][:2], t["a"], b, t["c"][:2], softplus=True)
    assert bool(torch.isinf(state).all())


def test_decays_of_any_size():
    """everything forgotten, nothing forgotten, and decays below fp32's range"""
    t = make(12, "f32", 70, 32, 1, 16, 1, softplus=False)
    for size in (0.0, -1e-8, -1e4, -1e30, -float("inf")):
        a = torch.full_like(t["a"], size)
        t["delta"] = t["delta"].abs()
        out, state = seq.msla_selective_scan_forward(t["x"], t["delta"], a, t["b"], t["c"], initial_state=t["first"])
        want, last, _ = lo.scan(*(f64(v) for v in (t["x"], t["delta"], a, t["b"], t["c"])), [(0, 70)], initial=f64(t["first"]))
        np.testing.assert_allclose(f64(out), want, rtol=1e-4, atol=1e-4 * np.abs(want).max())
        np.testing.assert_allclose(f64(state), last, rtol=1e-4, atol=1e-4 * np.abs(last).max())
        g = seq.msla_selective_scan_backward(t["x"], t["delta"], a, t["b"], t["c"], t["d_out"], initial_state=t["first"])
        if np.isfinite(size):
            assert all(bool(torch.isfinite(v).all()) for v in g if v is not None)


def test_gradient_against_differences():
    t = make(13, "f32", 75, 20, 1, 16, 2)
    offs = torch.tensor([0, 31, 75], dtype=torch.int32, device="cuda")
    names = ("x", "delta", "a", "b", "c", "skip", "bias", "gate", "first")
    w = _numbers(999, 2, 20, 16).cuda()

    def value(v):
        out, state = seq.msla_selective_scan_forward(*args_of(v), offsets=offs, initial_state=v["first"], **rest_of(v, True))
        return float((out.double() * t["d_out"].double()).sum() + (state.double() * w).sum())

    g = seq.msla_selective_scan_backward(*args_of(t), t["d_out"], offsets=offs, initial_state=t["first"], d_final_state=w.float(), **rest_of(t, True))
    grads = dict(zip(("x", "delta", "a", "b", "c", "skip", "bias", "gate", "first"), g))
    h = 2.0 ** -8
    for i, name in enumerate(names):
        e = _numbers(1000 + i, *t[name].shape).float().cuda()
        e = e * t[name].abs() if name == "a" else e
        up, down = (dict(t, **{name: t[name] + s * h * e}) for s in (1, -1))
        got = (value(up) - value(down)) / (2 * h)
        want = float((grads[name].double() * e.double()).sum())
        # h^2 / 6 of the third derivative, of the size of the terms, and fp32's rounding over h
        bound = 4 * h * h * float((grads[name].double().abs() * e.double().abs()).sum()) + 2e-2
        print(f"  {name}: {got:.4f} {want:.4f} (within {bound:.4f})", flush=True)
        assert abs(got - want) <= bound, name

"""The recurrence where its numbers are hard: sums that are exact in fp32, whatever its operands are split into on the way."""
import numpy as np
import pytest
import torch

import test_gpu_recurrence as base
from oracle import sequence_oracle as so
from paper_2205_14756_amd import sequence as seq

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
DTYPES = ["f32", "f16", "bf16"]


def whole(seed, top, *shape):
    return torch.from_numpy(np.random.default_rng(seed).integers(-top, top + 1, shape)).double()


def single(seed, tokens, heads, d):
    """one channel of every row is 1 or -1, token t's is t mod d: a column sums tokens / d rows"""
    x = torch.zeros(tokens, heads, d, dtype=torch.float64)
    t = torch.arange(tokens)
    x[t, :, t % d] = whole(seed, 1, tokens, heads).mul(2).add(1).sign()
    return x


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_whole_numbers_are_exact(dtype, d):
    """Whole numbers up to 255 (8 bits: every type has them), two chunks of 64 tokens, a scale of 2^-9 and no gates: scores stay below
    128 * 255^2 < 2^23, and so do all sums of them, so fp32 holds every one of them exactly and an output is the exact sum, rounded once."""
    tokens, heads = 128, 4
    a, b, one = whole(1, 255, tokens, heads, d), whole(2, 255, tokens, heads, d), single(3, tokens, heads, d)
    scale = 2.0 ** -9
    to = lambda x: x.to(TDT[dtype]).cuda()
    low = torch.ones(tokens, tokens, dtype=torch.float64).tril()
    scores = torch.einsum("ihc,jhc->hij", a, b) * scale

    def same(got, want, what):
        want = want.to(TDT[dtype])
        assert bool(torch.isfinite(want.float()).all())
        wrong = int((got.cpu() != want).sum())
        print(f"  {what}: {wrong} of {want.numel()} differ", flush=True)
        assert wrong == 0, what

    print(f"whole numbers {dtype} d={d}", flush=True)
    out, state = seq.msla_recurrence_forward(to(a), to(b), to(one), scale=scale)
    same(out, torch.einsum("hij,jhe->ihe", scores * low, one), "out")
    assert torch.equal(state[0].cpu().double(), torch.einsum("jhc,jhe->hce", b, one))
    # scores of d_out and v: of d_q (a: d_out, b: v) over the keys, of d_k (a: v, b: d_out) over the queries
    back = torch.einsum("ihc,jhc->hij", a, b) * scale
    d_q, d_k, d_v, *_ = seq.msla_recurrence_backward(to(one), to(one), to(b), to(a), scale=scale)
    same(d_q, torch.einsum("hij,jhe->ihe", back * low, one), "d_q")
    same(d_k, torch.einsum("hij,ihe->jhe", back * low, one), "d_k")
    same(d_v, torch.einsum("hij,ihe->jhe", torch.einsum("ihc,jhc->hij", one, one) * low * scale, a), "d_v")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d", [16, 32, 64, 128])
def test_a_state_of_whole_numbers_is_read_exactly(dtype, d):
    """A state of numbers up to 2^20 and queries of one 1 and one -1: differences below 2^21, exact in fp32, rounded once.  The rows behind
    the state's own tokens are zero, so every token reads the same state."""
    tokens, heads = 70, 4
    first = whole(4, 2 ** 20, 1, heads, d, d)
    q = torch.zeros(tokens, heads, d, dtype=torch.float64)
    t = torch.arange(tokens)
    q[t, :, t % d], q[t, :, (t + 1 + t // d) % d] = 1.0, -1.0
    none = torch.zeros(tokens, heads, d, dtype=TDT[dtype], device="cuda")
    scale = 2.0 ** -8
    want = (torch.einsum("ihc,hce->ihe", q, first[0]) * scale).to(TDT[dtype])
    print(f"state {dtype} d={d}", flush=True)
    out, state = seq.msla_recurrence_forward(q.to(TDT[dtype]).cuda(), none, none, initial_state=first.float().cuda(), scale=scale)
    wrong = int((out.cpu() != want).sum())
    print(f"  out: {wrong} of {want.numel()} differ", flush=True)
    assert wrong == 0
    assert torch.equal(state.cpu().double(), first)


@pytest.mark.parametrize("d", [16, 32])
def test_grouped_heads_as_far_apart_as_they_may_be(d):
    """Head-major queries and gradients whose last row of a workgroup's last state head ends right below 2^32 - 16 bytes behind the first."""
    tokens, hkv, group = 150, 64 // d, 4 if d == 16 else 9
    hq = hkv * group
    stride = (2 ** 32 - 16 - 2 * d - 63 * 2 * d) // ((64 // d - 1) * group * 2) // 8 * 8
    n = lambda seed, *s: torch.from_numpy(np.random.default_rng(seed).standard_normal(s)).bfloat16().cuda()
    q, k, v, d_out = n(1, tokens, hq, d), n(2, tokens, hkv, d), n(3, tokens, hkv, d), n(4, tokens, hq, d)

    def apart(x):
        room = torch.empty((hq - 1) * stride + tokens * d, dtype=x.dtype, device="cuda")
        y = room.as_strided(x.shape, (d, stride, 1))
        y.copy_(x)
        return y

    fq, fd = apart(q), apart(d_out)
    for a, b in zip(seq.msla_recurrence_forward(q, k, v), seq.msla_recurrence_forward(fq, k, v, out=torch.empty_like(q))):
        assert torch.equal(a, b)
    for a, b in zip(seq.msla_recurrence_backward(q, k, v, d_out)[:3], seq.msla_recurrence_backward(fq, k, v, fd, d_q=torch.empty_like(q))[:3]):
        assert torch.equal(a, b)


NANS = {"f32": (torch.int32, (0x7FC00000, 0xFFC00000, 0xFF800001)), "f16": (torch.int16, (0x7E00, 0xFE00, 0xFC01)),
        "bf16": (torch.int16, (0x7FC0, 0xFFC0, 0xFF81))}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("which", range(3))
@pytest.mark.parametrize("operand", ["q", "k"])
def test_a_rectified_nan_stays_one(dtype, which, operand):
    """NaNs of both signs, in the scan and in the step: what reads one is a NaN, and nothing else is touched."""
    ints, codes = NANS[dtype]
    code = codes[which] - (1 << (8 * ints.itemsize)) if codes[which] >> (8 * ints.itemsize - 1) else codes[which]
    n, h, d, at, head = 150, 3, 64, 100, 1
    x = {m: torch.from_numpy(np.random.default_rng(i).standard_normal((n, h, d))).to(TDT[dtype]).cuda() for i, m in enumerate("qkv")}
    x["q"][3, 0, :2], x["k"][3, 0, :2] = float("-inf"), float("-inf")                     # (rectified: 0)
    first = torch.from_numpy(np.random.default_rng(5).standard_normal((n, h, d, d))).float().cuda()
    clean, last = seq.msla_recurrence_forward(x["q"], x["k"], x["v"], initial_state=first[:1], rectify=True)
    one, states = seq.msla_recurrence_step(x["q"], x["k"], x["v"], first, rectify=True, new_state=torch.empty_like(first))
    assert all(bool(torch.isfinite(t.float()).all()) for t in (clean, last, one, states))
    x[operand].view(ints)[at, head, 5] = code
    assert bool(torch.isnan(x[operand][at, head, 5]))
    got, end = seq.msla_recurrence_forward(x["q"], x["k"], x["v"], initial_state=first[:1], rectify=True)
    hit = torch.zeros(n, h, dtype=torch.bool, device="cuda")
    hit[slice(at, at + 1 if operand == "q" else None), head] = True
    assert bool(torch.isnan(got[hit].float()).all())
    if dtype != "f16":          # (fp16: a chunk's normaliser hangs on its largest value, which may be another one now)
        assert torch.equal(got[~hit], clean[~hit])
    assert bool(torch.isfinite(got[~hit].float()).all())
    assert bool(torch.isnan(end[0, head, 5]).all()) if operand == "k" else bool(torch.isfinite(end).all())
    got, after = seq.msla_recurrence_step(x["q"], x["k"], x["v"], first, rectify=True, new_state=torch.empty_like(first))
    hit = torch.zeros(n, h, dtype=torch.bool, device="cuda")
    hit[at, head] = True
    assert bool(torch.isnan(got[hit].float()).all()) and torch.equal(got[~hit], one[~hit])
    assert bool(torch.isnan(after[at, head, 5]).all()) if operand == "k" else torch.equal(after, states)


# sizes of q, k, v, d_out of every other head and of the heads between: results are not lost in fp16's smallest steps
HEAD_SIZES = [((100.0, 100.0, 1e-3, 1.0), (1e-2, 1e-2, 300.0, 50.0)), ((1e-2, 1.0, 1e4, 1e-2), (30.0, 30.0, 1e-4, 1.0))]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [16, 32, 64])
@pytest.mark.parametrize("group", [1, 2])
@pytest.mark.parametrize("sizes", HEAD_SIZES)
@pytest.mark.parametrize("tokens", [150, 700])
def test_heads_of_different_size_side_by_side(dtype, d, group, sizes, tokens):
    """A head's precision is its own: each within the tolerance of its own terms (base.close), whatever its neighbours' sizes."""
    hkv, scale = 5, 0.02
    t = base.make(31, dtype, tokens, hkv * group, hkv, d, [tokens], initial=False)
    for i, n in enumerate(("q", "k", "v", "d_out")):
        heads = t[n].shape[1] // hkv
        size = torch.tensor([sizes[h % 2][i] for h in range(hkv) for _ in range(heads if n in ("q", "d_out") else 1)], device="cuda")
        t[n] = (t[n].float() * size[:, None]).to(TDT[dtype])
    args = [base.f64(t[n]) for n in ("q", "k", "v", "gate")] + [[(0, tokens)]]
    mag = [np.abs(a) for a in args[:3]] + args[3:]
    print(f"heads of different size {dtype} d={d} group={group} tokens={tokens}", flush=True)
    out, state = seq.msla_recurrence_forward(t["q"], t["k"], t["v"], t["gate"], scale=scale)
    want, last = so.recurrence(*args, None, scale)
    size, size_last = so.recurrence(*mag, None, scale)
    base.close(out, want, size, dtype, "out")
    base.close(state, last, size_last, dtype, "state", base.STATE, half=False)
    got = seq.msla_recurrence_backward(t["q"], t["k"], t["v"], t["d_out"], t["gate"], scale=scale)
    ref = so.recurrence_backward(*args, None, scale, base.f64(t["d_out"]))
    m, _ = base.gate_magnitudes(t, [(0, tokens)], scale, False)
    for i, name in enumerate(("d_q", "d_k", "d_v")):
        # (some of the large head's d_v, sums of 10^4 * sqrt(d) * scale over the tokens, are above fp16's 65504; a result is an infinity from 65520 on)
        fits = np.abs(ref[i]) < 65504 * (1 - 2.0 ** -10) if dtype == "f16" else np.ones(ref[i].shape, bool)
        beyond = np.abs(ref[i]) > 65520 * (1 + 2.0 ** -10) if dtype == "f16" else ~fits
        assert np.isinf(base.f64(got[i])[beyond]).all()
        base.close(got[i][torch.from_numpy(fits).cuda()], ref[i][fits], m[i][fits], dtype, name)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens,group", [(150, 1), (700, 2)])
@pytest.mark.parametrize("large", [1e30, 1e32])
def test_small_values_behind_a_large_state(dtype, tokens, group, large):
    """A state of 1e30 or 1e32 (fp32 has it), values of 1e-4, and a gate that forgets the state at token 100: rows before it see the state times some
    ten (fp16: an infinity), rows behind it what the values make, and so does the last state.  The gradient likewise from a d_final_state of that size:
    tokens before 100 know nothing of it.  The short ones run whole, through three chunks, the long ones in segments of one."""
    hkv, d, reset = 2, 64, 100
    t = base.make(33, dtype, tokens, hkv * group, hkv, d, [tokens])
    t["v"] = (t["v"].float() * 1e-4).to(TDT[dtype])
    t["d_out"] = (t["d_out"].float() * 1e-4).to(TDT[dtype])
    t["gate"][reset] = -200.0
    t["first"] *= large
    t["d_last"] *= large
    assert (seq.msla_recurrence_workspace_bytes(1, tokens, hkv * group, hkv, d, TDT[dtype]) == 0) == (tokens == 150)
    spans = [(0, tokens)]
    args = [base.f64(t[n]) for n in ("q", "k", "v", "gate")] + [spans]
    mag = [np.abs(a) for a in args[:3]] + args[3:]
    first, d_last = base.f64(t["first"]), base.f64(t["d_last"])
    print(f"state of {large} {dtype} tokens={tokens}", flush=True)
    out, state = seq.msla_recurrence_forward(t["q"], t["k"], t["v"], t["gate"], initial_state=t["first"], scale=1.0)
    want, last = so.recurrence(*args, first, 1.0)
    size, size_last = so.recurrence(*mag, np.abs(first), 1.0)
    base.close(out[reset:], want[reset:], size[reset:], dtype, "out")
    base.close(state, last, size_last, dtype, "state", base.STATE, half=False)
    before = base.f64(out[:reset])
    if dtype == "f16":
        far = np.abs(want[:reset]) > 2.0 ** 20
        assert np.isinf(before[far]).all() and not np.isnan(before).any()
    else:
        base.close(out[:reset], want[:reset], size[:reset], dtype, "out before")
    got = seq.msla_recurrence_backward(t["q"], t["k"], t["v"], t["d_out"], t["gate"], d_final_state=t["d_last"], scale=1.0)
    ref = so.recurrence_backward(*args, None, 1.0, base.f64(t["d_out"]), d_last)
    m = so.recurrence_backward(*mag, None, 1.0, np.abs(base.f64(t["d_out"])), np.abs(d_last), magnitudes=True)
    base.close(got[0], ref[0], m[0], dtype, "d_q")
    for i, name in ((1, "d_k"), (2, "d_v")):
        base.close(got[i][:reset], ref[i][:reset], m[i][:reset], dtype, name)
        if dtype != "f16":
            base.close(got[i][reset:], ref[i][reset:], m[i][reset:], dtype, name + " behind")

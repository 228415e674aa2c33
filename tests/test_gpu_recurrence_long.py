"""Segments of many chunks: the loops over chunks of the scan, of its gradient and of the segments' sums, against the fp64 oracle on a sample of
sequences and heads.  How many chunks a segment has is asserted, from the workspace that the call asks for.

Tolerances: those of test_gpu_recurrence, whose sums are over a chunk.  A state adds to that, for every chunk that it goes through, its products (at
most 16 instructions, each rounding once) and a decay: 17 * 2^-24 a chunk, 2^-16.4 of the terms' magnitudes for ten chunks; segments are joined by one
more product and sum each, 2^-20 for eight.  Both stay below the 2^-16 (PART in fp32, and STATE) of that file."""
import math

import numpy as np
import pytest
import torch

import test_gpu_recurrence as base
from oracle import sequence_oracle as so
from paper_2205_14756_amd import sequence as seq

pytestmark = pytest.mark.gpu

DTYPES = ["f32", "f16", "bf16"]
# a head's gate a token, on average: mild ones, whose sum passes 16 powers of two several times in ten chunks or does not at all, a hard one, and
# one above 0
RATES = [-0.06, -0.004, 0.02, -0.15, -2.0]


def numbers(seed, dtype, seqs, length, hkv, group, d, spread=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, hq = seqs * length, hkv * group
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")
    to = lambda x: x.to(base.TDT[dtype])
    t = dict(q=to(normal(n, hq, d)), k=to(normal(n, hkv, d)), d_out=to(normal(n, hq, d)))
    v = normal(n, hkv, d)
    if spread:                  # chunks of different size
        v *= 10.0 ** torch.randint(-2, 2, (n // 64 + 1,), generator=g, device="cuda").repeat_interleave(64)[:n, None, None]
    t["v"] = to(v)
    rate = torch.tensor([RATES[h % len(RATES)] for h in range(hkv)], device="cuda")
    t["gate"] = to(rate * (0.5 + torch.rand(n, hkv, generator=g, device="cuda")))
    t["first"], t["d_last"] = normal(seqs, hkv, d, d), normal(seqs, hkv, d, d)
    return t


def close(got, want, size, dtype, what):
    """base.close; in fp16 the head whose gate is above 0 grows by e^0.02 a token, e^12 and more in all, out of fp16's range: what is above 65504 there
    has to be an infinity (from 65520 on)."""
    if dtype != "f16":
        return base.close(got, want, size, dtype, what)
    fits, beyond = np.abs(want) < 65504 * (1 - 2.0 ** -10), np.abs(want) > 65520 * (1 + 2.0 ** -10)
    assert (base.f64(got)[beyond] == np.sign(want[beyond]) * np.inf).all(), what
    base.close(got[torch.from_numpy(fits).cuda()], want[fits], size[fits], dtype, what)


def compare(dtype, t, seqs, length, group, scale, sample, heads, backward=True):
    """The calls on everything, the oracle on the sequences `sample` and the state heads `heads`."""
    hkv = t["k"].shape[1]
    kw = dict(sequences=seqs, initial_state=t["first"], scale=scale)
    rows = torch.cat([torch.arange(b * length, (b + 1) * length) for b in sample]).cuda()
    hs = torch.tensor(heads, device="cuda")
    hqs = (hs[:, None] * group + torch.arange(group, device="cuda")).flatten()
    part = lambda x, which: x[rows][:, which]
    s = dict(q=part(t["q"], hqs), k=part(t["k"], hs), v=part(t["v"], hs), d_out=part(t["d_out"], hqs), gate=part(t["gate"], hs),
             first=t["first"][sample][:, hs], d_last=t["d_last"][sample][:, hs])
    spans = [(i * length, (i + 1) * length) for i in range(len(sample))]
    args = [base.f64(s[n]) for n in ("q", "k", "v", "gate")] + [spans]
    mag = [np.abs(a) for a in args[:3]] + args[3:]
    first = base.f64(s["first"])
    out, state = seq.msla_recurrence_forward(t["q"], t["k"], t["v"], t["gate"], **kw)
    want, last = so.recurrence(*args, first, scale)
    size, size_last = so.recurrence(*mag, np.abs(first), scale)
    close(part(out, hqs), want, size, dtype, "out")
    base.close(state[sample][:, hs], last, size_last, dtype, "state", base.STATE, half=False)
    if not backward:
        return
    got = seq.msla_recurrence_backward(t["q"], t["k"], t["v"], t["d_out"], t["gate"], d_final_state=t["d_last"], **kw)
    ref = so.recurrence_backward(*args, first, scale, base.f64(s["d_out"]), base.f64(s["d_last"]))
    m, size_g = base.gate_magnitudes(s, spans, scale, False)
    for i, (name, which) in enumerate((("d_q", hqs), ("d_k", hs), ("d_v", hs))):
        close(part(got[i], which), ref[i], m[i], dtype, name)
    close(part(got[3], hs), ref[3], size_g, dtype, "d_gate")
    base.close(got[4][sample][:, hs], ref[4], m[4], dtype, "d_state", base.STATE, half=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,hkv,group", [(16, 4, 1), (16, 3, 2), (32, 2, 1), (32, 2, 3), (64, 1, 1), (64, 1, 2), (128, 1, 1), (128, 1, 2)])
def test_whole_sequences_of_many_chunks(dtype, d, hkv, group):
    """256 equal sequences fill the GPU, so each runs whole: ten chunks (six with several query heads), the last one ragged."""
    seqs, length = 256, 600 if group == 1 else 333
    assert seq.msla_recurrence_workspace_bytes(seqs, seqs * length, hkv * group, hkv, d, base.TDT[dtype]) == 0
    print(f"whole sequences {dtype} d={d} heads={hkv * group}/{hkv}", flush=True)
    t = numbers(40 + d + group, dtype, seqs, length, hkv, group, d)
    if hkv == 1:                # (heads of 64 and 128: a sequence each for the rates)
        t["gate"] = (t["gate"].float() * (torch.arange(seqs, device="cuda") % 4 + 0.25).repeat_interleave(length)[:, None]).to(t["gate"].dtype)
    compare(dtype, t, seqs, length, group, 0.3, [0, 101, 255], list(range(hkv)))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("d,group", [(16, 1), (16, 2), (32, 1), (32, 3), (64, 1), (64, 2), (128, 1), (128, 2)])
def test_segments_of_many_chunks(dtype, d, group):
    """So many heads that a sequence is cut into eight segments alone: four or five chunks each."""
    hkv, length = 64 * max(1, 64 // d) - (1 if d < 64 else 0), 1613
    slots = seq.msla_recurrence_workspace_bytes(1, length, hkv * group, hkv, d, base.TDT[dtype]) / (hkv * (d * d + 1) * 4)
    assert 5 <= slots <= length / 256 + 1.1, slots           # segments of 256 tokens and more
    print(f"segments {dtype} d={d} heads={hkv * group}/{hkv}", flush=True)
    compare(dtype, numbers(60 + d + group, dtype, 1, length, hkv, group, d), 1, length, group, 0.3, [0], [0, 2, hkv - 1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("exponent", [100, -60])
@pytest.mark.parametrize("d", [16, 64, 128])
def test_values_far_from_one_over_many_chunks(dtype, exponent, d):
    """A state on the way stands for up to 2^16 times its value, or as much less, over chunk after chunk; its values stay in fp32's range."""
    seqs, length, hkv = 256, 640, max(1, 64 // d)
    assert seq.msla_recurrence_workspace_bytes(seqs, seqs * length, hkv, hkv, d, base.TDT[dtype]) == 0
    t = numbers(80 + d, dtype, seqs, length, hkv, 1, d, spread=False)
    t["v"] = (t["v"].float() * 2.0 ** exponent).to(base.TDT[dtype])
    t["first"] *= 2.0 ** exponent
    if hkv == 1:
        t["gate"][::2] *= -0.25         # (some above 0)
    compare(dtype, t, seqs, length, 1, 0.01, [3, 200], list(range(hkv)), backward=False)


def test_a_state_that_is_forgotten_slowly():
    """2^24 tokens that add nothing, and a gate that leaves e^-8.8 of the state in all: 128 segments of 2048 chunks.  A segment's decay is the
    exponential of its gates' sum (one step of fp32, 2^-23, and half a step of its argument, below 0.1), and the join multiplies (half a step):
    2^-22 a segment at most, 2^-15 in all."""
    tokens, h, d = 2 ** 24, 16, 16
    rate = -141 / 128 * 2.0 ** -21              # (bf16 has it)
    slots = seq.msla_recurrence_workspace_bytes(1, tokens, h, h, d, torch.bfloat16) / (h * (d * d + 1) * 4)
    assert slots <= tokens / (64 * 1024) + 2, slots
    none = torch.zeros(1, 1, d, dtype=torch.bfloat16, device="cuda").expand(tokens, h, d)
    gate = torch.full((1, h), rate, dtype=torch.bfloat16, device="cuda").expand(tokens, h)
    assert float(gate[0, 0]) == rate
    first = torch.randn(1, h, d, d, device="cuda")
    out = torch.empty(tokens, h, d, dtype=torch.bfloat16, device="cuda")
    _, last = seq.msla_recurrence_forward(none, none, none, gate, initial_state=first, out=out)
    want = first.double() * math.exp(tokens * rate)
    worst = float(((last.double() - want) / want).abs().max())
    print(f"  {worst:.3g}", flush=True)
    assert worst <= 2.0 ** -15
    assert bool((out[::4096] == 0).all())

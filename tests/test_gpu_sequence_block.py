"""The sequence operators together, as a language model's layer uses them: norm into 8 bits -> 8-bit projection to q, k, v and the gate ->
recurrence -> norm of every head -> 8-bit projection back -> norm with the residual; a packed batch of prompts, then single tokens,
eager and from a captured graph; and a training step of the same layer in the storage type."""
import numpy as np
import pytest
import torch

from oracle import sequence_oracle as so
from paper_2205_14756_amd import msla
from paper_2205_14756_amd import sequence as seq

pytestmark = pytest.mark.gpu

HEADS, D, C = 4, 32, 128


def rnd(seed, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)) * scale).to(dtype).cuda()


class Layer:
    def __init__(self):
        self.norm_in, self.norm_head, self.norm_out = (1 + rnd(i, n, scale=0.1) for i, n in ((1, C), (2, D), (3, C)))
        # rows in msla_linear's order of heads, and 16 more for the gates (a multiple of 16)
        self.w_in = seq.msla_quantize_rows(rnd(4, 3 * C + 16, C, scale=C ** -0.5))
        self.w_back = seq.msla_quantize_rows(rnd(5, C, C, scale=C ** -0.5))

    def project(self, x, residual):
        y8, scale, r = seq.msla_norm_quantized(x, self.norm_in, residual)
        m = seq.msla_linear_quantized(y8, scale, *self.w_in, dtype=x.dtype)
        qkv = m[:, :3 * C].unflatten(1, (HEADS, 3, D))
        gate = torch.nn.functional.logsigmoid(m[:, 3 * C:3 * C + HEADS].float() + 2).to(x.dtype)
        return qkv[:, :, 0], qkv[:, :, 1], qkv[:, :, 2], gate, r

    def finish(self, o, r):
        h, _ = seq.msla_norm_forward(o, self.norm_head)
        h8, scale = seq.msla_quantize_rows(h.flatten(1))
        return seq.msla_norm_forward(seq.msla_linear_quantized(h8, scale, *self.w_back, dtype=r.dtype), self.norm_out, r)

    def prompts(self, x, residual, offsets):
        q, k, v, gate, r = self.project(x, residual)
        o, state = seq.msla_recurrence_forward(q, k, v, gate, offsets=offsets, rectify=True)
        return self.finish(o, r) + (state,)

    def step(self, x, residual, state):
        q, k, v, gate, r = self.project(x, residual)
        o, state = seq.msla_recurrence_step(q, k, v, state, gate, rectify=True)
        return self.finish(o, r)


def test_a_layer_serves_prompts_and_tokens():
    layer = Layer()
    lens, n_new = [70, 1, 300], 5
    whole = [l + n_new for l in lens]
    offs = lambda ls: torch.tensor([sum(ls[:i]) for i in range(len(ls) + 1)], dtype=torch.int32, device="cuda")
    x, res = rnd(6, sum(whole), C), rnd(7, sum(whole), C)
    y, r, state = layer.prompts(x, res, offs(whole))
    assert bool(torch.isfinite(y.float()).all())
    starts = [sum(whole[:i]) for i in range(len(whole))]
    rows = torch.cat([torch.arange(s, s + l) for s, l in zip(starts, lens)]).cuda()
    y0, r0, state0 = layer.prompts(x[rows], res[rows], offs(lens))
    assert torch.equal(y0, y[rows]) and torch.equal(r0, r[rows])        # (tokens see what is before them alone)
    # single tokens: eager, and the captured step on the same inputs, replayed with eager work between the replays
    eager, fixed = state0.clone(), state0.clone()
    xin, rin = torch.empty(3, C, dtype=x.dtype, device="cuda"), torch.empty(3, C, dtype=x.dtype, device="cuda")
    at = lambda i: torch.tensor([s + l + i for s, l in zip(starts, lens)], device="cuda")
    xin.copy_(x[at(0)])
    rin.copy_(res[at(0)])
    warm = fixed.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(xin, rin, warm)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        yg, rg = layer.step(xin, rin, fixed)
    for i in range(n_new):
        ye, re = layer.step(x[at(i)], res[at(i)], eager)
        xin.copy_(x[at(i)])
        rin.copy_(res[at(i)])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ye, yg) and torch.equal(re, rg) and torch.equal(eager, fixed)
        # against the whole sequence in one call: the recurrence's rounding can move a value over a border of the 8-bit rows behind it, a
        # step of 2^-3 of one of C values, each of which weighs C^-0.5 in a row of size 1, and the norm keeps rows at size 1
        err = (ye.float() - y[at(i)].float()).norm(dim=1) / y[at(i)].float().norm(dim=1)
        assert float(err.max()) < 2 ** -3 * C ** -0.5 * 4, err
    torch.testing.assert_close(eager, state, rtol=2 ** -14, atol=2 ** -14 * float(state.abs().max()))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_layer_trains(dtype):
    """norm -> msla_linear -> recurrence -> head norm -> msla_linear -> residual, forward and backward, against the fp64 oracle's chain.
    Every stage rounds once to the storage type, forwards and backwards (about eight roundings of half a step in a row, each
    carried on with a factor of order one): 8 * eps / 2 of the gradient's norm, three times that as a bound."""
    tokens, lens = 260, [100, 160]
    offs = torch.tensor([0, 100, 260], dtype=torch.int32, device="cuda")
    x, dz = rnd(8, tokens, C, dtype=dtype), rnd(9, tokens, C, dtype=dtype)
    n1, n2 = 1 + rnd(10, C, dtype=dtype, scale=0.1), 1 + rnd(11, D, dtype=dtype, scale=0.1)
    w_qkv, w_o = rnd(12, 3 * C, C, dtype=dtype, scale=C ** -0.5), rnd(13, C, C, dtype=dtype, scale=C ** -0.5)
    gate = torch.nn.functional.logsigmoid(rnd(14, tokens, HEADS, dtype=torch.float32) + 2).to(dtype)
    # forward and backward on the GPU
    y, _ = seq.msla_norm_forward(x, n1)
    qkv = msla.msla_linear(y, w_qkv).unflatten(1, (HEADS, 3, D))
    q, k, v = (qkv[:, :, i] for i in range(3))
    o, _ = seq.msla_recurrence_forward(q, k, v, gate, offsets=offs)
    h, _ = seq.msla_norm_forward(o, n2)
    z = msla.msla_linear(h.flatten(1), w_o) + x
    dh = msla.msla_linear(dz, w_o.t().contiguous())
    do, dn2 = seq.msla_norm_backward(o, n2, dh.view(tokens, HEADS, D))
    dqkv = torch.empty_like(qkv)
    _, _, _, dg, _ = seq.msla_recurrence_backward(q, k, v, do, gate, offsets=offs, d_q=dqkv[:, :, 0], d_k=dqkv[:, :, 1], d_v=dqkv[:, :, 2])
    dy = msla.msla_linear(dqkv.flatten(1), w_qkv.t().contiguous())
    dx, dn1 = seq.msla_norm_backward(x, n1, dy, d_sum=dz)
    # the same in fp64
    f = lambda t: t.double().cpu().numpy()
    Y, _ = so.norm(f(x), None, f(n1), 1e-6)
    QKV = (Y @ f(w_qkv).T).reshape(tokens, HEADS, 3, D)
    spans = [(0, 100), (100, 260)]
    args = (QKV[:, :, 0], QKV[:, :, 1], QKV[:, :, 2], f(gate), spans)
    O, _ = so.recurrence(*args, None, D ** -0.5)
    H, _ = so.norm(O, None, f(n2), 1e-6)
    Z = H.reshape(tokens, C) @ f(w_o).T + f(x)
    dH = (f(dz) @ f(w_o)).reshape(tokens, HEADS, D)
    dO, dN2 = so.norm_backward(O, f(n2), dH, None, 1e-6)
    dQ, dK, dV, dG, _ = so.recurrence_backward(*args, None, D ** -0.5, dO)
    dQKV = np.stack([dQ, dK, dV], 2).reshape(tokens, 3 * C)
    dX, dN1 = so.norm_backward(f(x), f(n1), dQKV @ f(w_qkv), f(dz), 1e-6)
    bound = 3 * 8 * torch.finfo(dtype).eps / 2
    for name, got, want in (("z", z, Z), ("dx", dx, dX), ("dqkv", dqkv.flatten(1), dQKV), ("dgate", dg, dG), ("dn1", dn1, dN1), ("dn2", dn2, dN2)):
        err = np.linalg.norm(f(got) - want) / np.linalg.norm(want)
        print(f"  {name}: {err:.2e} of {bound:.2e}", flush=True)
        assert err <= bound, name

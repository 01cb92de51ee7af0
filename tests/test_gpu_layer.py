"""The delta rule, the head-wise norm and gate, and the norms around blocks as a layer uses them together, against the same
layer in 64 bits; and what single calls have to keep: streams, neighbours in memory, offsets past 32 bits, NaN.

Bounds of the layer, as relative 2-norms: each step's own bound (delta rule 1e-2 in bf16 and 2e-5 in fp32; any other step
one rounding, 2^-8 = 3.9e-3, or 2e-6), and no step of this layer enlarges a relative error on its way.  Forward: the delta
rule and six others, 1e-2 + 6 x 3.9e-3 = 3.4e-2, in fp32 2e-5 + 6 x 2e-6 = 3.2e-5.  A gradient takes those and as many again
on the way back: 6.8e-2 and 6.4e-5.
"""
import math

import pytest
import torch

import paper_2307_14995_amd as ltn
from _delta_ref import block_norm, gradients, make, recurrence, rel
from _helpers import dev

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-5
FWD = {BF: 3.4e-2, F32: 3.2e-5}
NAMES = ("dq", "dk", "dv", "dg", "dbeta")


class Delta(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g, beta, cu, scale):
        ctx.save_for_backward(q, k, v, g, beta)
        ctx.cu, ctx.scale = cu, scale
        return ltn.ltn_delta_fwd(q, k, v, g, beta, cu=cu, scale=scale)

    @staticmethod
    def backward(ctx, d_o):
        dq, dk, dv, dg, dbeta = ltn.ltn_delta_bwd(*ctx.saved_tensors, d_o.contiguous(), cu=ctx.cu, scale=ctx.scale)
        return dq, dk, dv, dg.float(), dbeta.float(), None, None


class Gate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, u):
        ctx.save_for_backward(x, u)
        return ltn.ltn_gate_fwd(x, u, EPS)

    @staticmethod
    def backward(ctx, d_y):
        return ltn.ltn_gate_bwd(*ctx.saved_tensors, d_y.contiguous(), EPS)


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, w_after, w_before):
        ctx.save_for_backward(x, y, w_after, w_before)
        return ltn.ltn_block_norm_fwd(x, y, w_after=w_after, w_before=w_before, scale=0.5, eps=EPS)

    @staticmethod
    def backward(ctx, d_x, d_h):
        x, y, wa, wb = ctx.saved_tensors
        dx, dy, _, dwa, dwb = ltn.ltn_block_norm_bwd(x, y, d_x.contiguous(), d_h.contiguous(), w_after=wa, w_before=wb, scale=0.5, eps=EPS)
        return dx, dy, dwa, dwb


def unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def heads(x, Bt, H):
    return x.view(Bt, x.shape[0] // Bt, H, -1).transpose(1, 2).contiguous()


def rows(x):
    return x.transpose(1, 2).reshape(x.shape[0] * x.shape[2], -1)


def inputs_of(p, h, Bt, Hk, H):
    """q, k, v, u, g, beta of a mixer whose input is h [tokens, C]."""
    q, k = (unit(heads(h @ p[n], Bt, Hk)) for n in ("wq", "wk"))
    v, u = (heads(h @ p[n], Bt, H) for n in ("wv", "wu"))
    gates = heads(h.to(p["wg"].dtype) @ p["wg"], Bt, H)
    return q, k, v, u, -torch.nn.functional.softplus(gates[..., 0]).contiguous(), torch.sigmoid(gates[..., 1]).contiguous()


def layer(p, x, h, Bt, Hk, H, delta, gate, norm):
    q, k, v, u, g, beta = inputs_of(p, h, Bt, Hk, H)
    y = rows(gate(delta(q, k, v, g, beta), u)) @ p["wo"]
    return norm(x, y, p["wa"], p["wb"])


def parameters(C, Hk, H, Dk, Dv, dtype, seed):
    r = torch.Generator().manual_seed(seed)
    shapes = dict(wq=(C, Hk * Dk), wk=(C, Hk * Dk), wv=(C, H * Dv), wu=(C, H * Dv), wo=(H * Dv, C))
    p = {n: (torch.randn(*s, generator=r) / s[0] ** 0.5).to(dtype) for n, s in shapes.items()}
    p["wg"] = torch.randn(C, 2 * H, generator=r) / C**0.5
    p["wa"], p["wb"] = (1 + 0.2 * torch.randn(C, generator=r) for _ in range(2))
    return {n: t.to(dev()) for n, t in p.items()}


def exact_gate(o, u):
    return o / (o.square().mean(-1, keepdim=True) + EPS).sqrt() * u


def exact_norm(x, y, wa, wb):
    return block_norm(x, y, None, wa, wb, 0.5, EPS, True)


def grads(outs, leaves, by):
    return torch.autograd.grad(outs, leaves, by)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cuts", [None, [0, 37, 38, 150]])
def test_a_layer_and_its_gradients(dtype, cuts):
    Bt, N, C, Hk, H, D = (2, 100, 256, 2, 4, 64) if cuts is None else (1, 150, 256, 2, 4, 64)
    p = parameters(C, Hk, H, D, D, dtype, 3)
    r = torch.Generator().manual_seed(4)
    x, h, dx, dh = (torch.randn(Bt * N, C, generator=r).to(dtype).to(dev()) for _ in range(4))
    cu = None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device=dev())

    leaves = {n: t.clone().requires_grad_() for n, t in {**p, "x": x, "h": h}.items()}
    outs = layer(leaves, leaves["x"], leaves["h"], Bt, Hk, H, lambda *t: Delta.apply(*t, cu, D**-0.5), Gate.apply, Norm.apply)
    got = grads(outs, list(leaves.values()), (dx, dh))

    def exact_delta(*t):
        if cuts is None:
            return recurrence(*t, D**-0.5)[0]
        return torch.cat([recurrence(*(y[:, :, a:b] for y in t), D**-0.5)[0] for a, b in zip(cuts[:-1], cuts[1:])], 2)

    exact = {n: t.detach().double().requires_grad_() for n, t in leaves.items()}
    want_outs = layer(exact, exact["x"], exact["h"], Bt, Hk, H, exact_delta, exact_gate, exact_norm)
    want = grads(want_outs, list(exact.values()), (dx.double(), dh.double()))
    for a, b in zip(outs, want_outs):
        assert rel(a.detach(), b.detach()) <= FWD[dtype]
    for n, a, b in zip(leaves, got, want):
        assert rel(a, b) <= 2 * FWD[dtype], n


@pytest.mark.parametrize("dtype", [F32, BF])
def test_a_prompt_and_then_tokens_through_two_layers(dtype):
    Bt, N, steps, C, Hk, H, D = 3, 70, 4, 128, 1, 2, 128
    ps = [parameters(C, Hk, H, D, D, dtype, s) for s in (5, 6)]
    r = torch.Generator().manual_seed(7)
    x, h = (torch.randn(Bt, N + steps, C, generator=r).to(dtype).to(dev()) for _ in range(2))

    def run(a, b, mixers):
        xs, hs = (t[:, a:b].reshape(-1, C).contiguous() for t in (x, h))
        for p, delta in zip(ps, mixers):
            xs, hs = layer(p, xs, hs, Bt, Hk, H, delta, lambda o, u: ltn.ltn_gate_fwd(o, u, EPS),
                           lambda x, y, wa, wb: ltn.ltn_block_norm_fwd(x, y, w_after=wa, w_before=wb, scale=0.5, eps=EPS))
        return xs.view(Bt, b - a, C), hs.view(Bt, b - a, C)

    states = [torch.zeros(Bt, H, D, D, device=dev()) for _ in ps]
    parts = [run(0, N, [lambda *t, s=s: ltn.ltn_delta_fwd(*t, kv_in=s, kv_out=s, scale=D**-0.5)[0] for s in states])]
    for i in range(N, N + steps):
        parts.append(run(i, i + 1, [lambda q, k, v, g, b, s=s: ltn.ltn_delta_decode_steps(q, k, v, s, g, b, scale=D**-0.5) for s in states]))

    xs, hs = x.double().view(-1, C), h.double().view(-1, C)
    for p in ps:
        xs, hs = layer({n: t.double() for n, t in p.items()}, xs, hs, Bt, Hk, H, lambda *t: recurrence(*t, D**-0.5)[0], exact_gate, exact_norm)
    for got, want in zip(zip(*parts), (xs, hs)):
        assert rel(torch.cat(got, 1).reshape(-1, C), want) <= 2 * FWD[dtype]     # (two layers)


@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128)])
def test_fp32_calls_that_fill_the_device(Dk, Dv):
    """More workgroups than half of the compute units: a wave has all features of its columns."""
    Bt, H, N = (5, 32, 70) if Dv == 64 else (5, 16, 70)
    *x, d_o = (t.to(dev()) for t in make(Bt, H // 2, H, N, Dk, Dv, F32, 8))
    kv0 = 0.3 * torch.randn(Bt, H, Dk, Dv, generator=torch.Generator().manual_seed(9)).to(dev())
    o, kv = ltn.ltn_delta_fwd(*x, kv_in=kv0, return_state=True)
    o_ref, kv_ref = recurrence(*x, 1.0, kv0)
    assert rel(o, o_ref) <= 2e-5 and rel(kv, kv_ref) <= 2e-5
    for n, a, b in zip(NAMES, ltn.ltn_delta_bwd(*x, d_o), gradients(*x, d_o, 1.0)[1:]):
        assert rel(a, b) <= 2e-5, n


def calls(seed):
    """Every call on inputs of its own: a function that makes them, and returns what they wrote."""
    *x, d_o = (t.to(dev()) for t in make(2, 2, 4, 150, 128, 128, BF, seed))
    kv0 = torch.ones(2, 4, 128, 128, device=dev())
    a, b, c = (t.flatten(0, 2) for t in (x[2], d_o, x[2].flip(0).contiguous()))
    w = torch.full((128,), 1.5, device=dev())

    def run():
        kv = kv0.clone()
        one = [t[:, :, :1].contiguous() for t in x]
        return (*ltn.ltn_delta_fwd(*x, return_state=True), *ltn.ltn_delta_bwd(*x, d_o),
                ltn.ltn_delta_decode_steps(*one[:3], kv, *one[3:]), kv,
                *ltn.ltn_block_norm_fwd(a, b, w_after=w, eps=EPS), *(t for t in ltn.ltn_block_norm_bwd(a, b, c, c, w_after=w, eps=EPS) if t is not None))

    return run


def test_two_streams_at_once():
    runs = [calls(s) for s in (11, 12)]
    want = [f() for f in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        got = []
        for f, s in zip(runs, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(f())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))


def test_two_graphs_and_eager_calls_in_turn():
    runs = [calls(s) for s in (13, 14)]
    want = [f() for f in runs]
    side = torch.cuda.Stream()
    graphs, outs = [], []
    for f in runs:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            f()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(f())
        graphs.append(graph)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
        eager = runs[0]()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip((*outs, eager), (*want, want[0])) for a, b in zip(g, w))
        for g in outs:
            for t in g:
                t.zero_()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("N", [1, 63, 130])
def test_neighbours_of_the_outputs_stay(dtype, N):
    Hk, H, Dk, Dv, mark = 1, 3, 64, 128, 77.0
    *x, d_o = (t.to(dev()) for t in make(1, Hk, H, N, Dk, Dv, dtype, 15))

    def padded(like, t):
        n = math.prod(like)
        pad = torch.full((n + 1024,), mark, dtype=t, device=dev())
        return pad, pad[512 : 512 + n].view(like)

    pads, outs = zip(*(padded(s, dtype) for s in ((1, Hk, N, Dk), (1, Hk, N, Dk), (1, H, N, Dv), (1, H, N), (1, H, N))))
    o_pad, o = padded((1, H, N, Dv), dtype)
    kv_pad, kv = padded((1, H, Dk, Dv), F32)
    ltn.ltn_delta_fwd(*x, kv_out=kv, out=o)
    ltn.ltn_delta_bwd(*x, d_o, out=outs)
    step_pad, step = padded((1, H, N, Dv), dtype)
    ltn.ltn_delta_decode_steps(*x[:3], kv, *x[3:], out=step)
    for pad in (*pads, o_pad, kv_pad, step_pad):
        assert (pad[:512] == mark).all() and (pad[-512:] == mark).all() and (pad[512:-512] != mark).all() and torch.isfinite(pad.float()).all()


def test_not_a_number_stays_in_its_sequence_and_behind_its_chunk():
    cuts = [0, 200, 330]
    *x, d_o = (t.to(dev()) for t in make(1, 2, 2, 330, 64, 64, BF, 16))
    cu = torch.tensor(cuts, dtype=torch.int32, device=dev())
    o, kv = ltn.ltn_delta_fwd(*x, cu=cu, return_state=True)
    grad = ltn.ltn_delta_bwd(*x, d_o, cu=cu)
    for at, value in ((2, float("nan")), (1, float("inf"))):
        y = list(x)
        y[at] = x[at].clone()
        y[at][0, 0, 140] = value           # the first sequence's third chunk: 128 .. 191
        o2, kv2 = ltn.ltn_delta_fwd(*y, cu=cu, return_state=True)
        assert torch.equal(o2[:, :, :128], o[:, :, :128]) and torch.equal(o2[:, :, 200:], o[:, :, 200:]) and torch.equal(kv2[1], kv[1])
        assert torch.equal(o2[:, 1], o[:, 1]) and not torch.isfinite(o2[:, 0, 140].float()).all()
        for a, b in zip(ltn.ltn_delta_bwd(*y, d_o, cu=cu), grad):
            assert torch.equal(a[:, :, 200:], b[:, :, 200:]) and torch.equal(a[:, 1], b[:, 1])


def test_offsets_past_32_bits():
    H, N, D = 40, 430_000, 128                         # 2.2e9 elements
    r = torch.Generator(dev()).manual_seed(17)

    def randn():
        return torch.randn(1, H, N, D, dtype=BF, device=dev(), generator=r)

    q, k = randn(), randn()
    for t in (q, k):
        for h in range(H):
            t[:, h] /= t[:, h].float().norm(dim=-1, keepdim=True).to(BF)
    v, d_o = randn(), randn()
    g = -torch.rand(1, H, N, device=dev(), generator=r)
    beta = torch.rand(1, H, N, device=dev(), generator=r)
    last = [t[:, -1:].contiguous() for t in (q, k, v, g, beta, d_o)]
    want = (*ltn.ltn_delta_fwd(*last[:5], return_state=True), *ltn.ltn_delta_bwd(*last))
    o, kv = ltn.ltn_delta_fwd(q, k, v, g, beta, return_state=True)
    assert torch.equal(o[:, -1:], want[0]) and torch.equal(kv[:, -1:], want[1])
    del o
    for n, a, b in zip(NAMES, ltn.ltn_delta_bwd(q, k, v, g, beta, d_o), want[2:]):
        assert torch.equal(a[:, -1:], b), n


def test_states_past_32_bits():
    Bt, H, D = 1100, 128, 128                          # 2.3e9 elements of states
    x = make(1, H, H, 1, D, D, BF, 18)[:5]
    q, k, v, g, beta = (t.expand(Bt, *t.shape[1:]).contiguous().to(dev()) for t in x)
    kv = torch.zeros(Bt, H, D, D, device=dev())
    kv[-1] = 0.5
    one = kv[-1:].clone()
    o = ltn.ltn_delta_decode_steps(q, k, v, kv, g, beta)
    o1 = ltn.ltn_delta_decode_steps(q[-1:], k[-1:], v[-1:], one, g[-1:], beta[-1:])
    assert torch.equal(o[-1:], o1) and torch.equal(kv[-1:], one) and torch.equal(kv[0], kv[Bt - 2])


def test_norm_rows_past_32_bits():
    n, C = 270_000, 8192                               # 2.2e9 elements
    r = torch.Generator(dev()).manual_seed(19)
    x, y, d = (torch.randn(n, C, dtype=BF, device=dev(), generator=r) for _ in range(3))
    tail = [t[-500:].contiguous() for t in (x, y, d)]
    got = ltn.ltn_block_norm_fwd(x, y, scale=0.5, eps=EPS)
    want = ltn.ltn_block_norm_fwd(*tail[:2], scale=0.5, eps=EPS)
    assert all(torch.equal(a[-500:], b) for a, b in zip(got, want))
    del got
    got = ltn.ltn_block_norm_bwd(x, y, d, d, scale=0.5, eps=EPS)[:2]
    want = ltn.ltn_block_norm_bwd(*tail, tail[2], scale=0.5, eps=EPS)[:2]
    assert all(torch.equal(a[-500:], b) for a, b in zip(got, want))

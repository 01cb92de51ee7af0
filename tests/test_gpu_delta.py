"""GPU parity of the gated delta rule against its recurrence in 64 bits (tests/_delta_ref.py).

Bounds, as relative 2-norms, derived from the roundings: a rounding to bf16 is off by at most 2^-8 of the value, by
2^-8 / sqrt(6) in the mean over a binade.  o: P, U, S and o itself, four roundings that add up independently, at most
4 x 2^-8 = 1.6e-2, expected 2 x 1.6e-3.  Gradients: up to nine (Z, dY, S0, dS, P, T, dU, dP or E, the gradient), expected
3 x 1.6e-3 = 4.8e-3; 1e-2 is the bound that the other bf16 gradients of this suite are held to.  fp32 states of bf16 tensors:
parts of 16 bits, 2^-16 per rounding, four of them: 6e-5 at most, expected 4e-6 .. 6e-6; bound 2e-5.  fp32: 2^-24 times the
square root of some thousand terms, 4e-6; bound 2e-5.
"""
import pytest
import torch

import paper_2307_14995_amd as ltn
from _delta_ref import gradients, make, packed, recurrence, rel
from _helpers import dev

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
TOL = {BF: 1e-2, F32: 2e-5}
TOL_STATE = 2e-5
NAMES = ("dq", "dk", "dv", "dg", "dbeta")
WIDTHS = [(64, 64), (64, 128), (128, 64), (128, 128)]


def gpu(*ts):
    return tuple(None if t is None else t.to(dev()) for t in ts)


def states(rows, H, Dk, Dv, seed):
    return 0.3 * torch.randn(rows, H, Dk, Dv, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("Dk,Dv", WIDTHS)
@pytest.mark.parametrize("N", [1, 5, 64, 65, 200])
def test_forward(dtype, Dk, Dv, N):
    x = make(2, 2, 4, N, Dk, Dv, dtype, 11 * N + Dk)[:5]
    kv0 = states(2, 4, Dk, Dv, N)
    for S in (None, kv0):
        o, kv = ltn.ltn_delta_fwd(*gpu(*x), kv_in=None if S is None else S.to(dev()), scale=0.125, return_state=True)
        o_ref, kv_ref = recurrence(*gpu(*x), 0.125, None if S is None else S.to(dev()))
        assert rel(o, o_ref) <= TOL[dtype] and rel(kv, kv_ref) <= TOL_STATE


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("Dk,Dv", WIDTHS)
@pytest.mark.parametrize("N", [1, 7, 64, 129, 200])
def test_backward(dtype, Dk, Dv, N):
    *x, d_o = gpu(*make(2, 2, 4, N, Dk, Dv, dtype, 7 * N + Dv))
    got = ltn.ltn_delta_bwd(*x, d_o, scale=0.125)
    _, *want = gradients(*x, d_o, 0.125)
    for n, a, b in zip(NAMES, got, want):
        assert a.dtype == dtype and a.shape == b.shape
        if N == 1 and n == "dg":           # the state before the first token is zero: so is its decay's gradient
            assert (a == 0).all()
            continue
        assert rel(a, b) <= TOL[dtype], n


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("Hk,H", [(1, 1), (1, 3), (3, 3), (4, 8)])
def test_shared_key_heads(dtype, Hk, H):
    *x, d_o = gpu(*make(3, Hk, H, 100, 128, 128, dtype, 31 + H))
    got = (ltn.ltn_delta_fwd(*x), *ltn.ltn_delta_bwd(*x, d_o))
    want = gradients(*x, d_o, 1.0)
    for n, a, b in zip(("o", *NAMES), got, want):
        assert rel(a, b) <= TOL[dtype], n


CUTS = [[0, 130], [0, 0, 1, 1, 65, 130, 130], [3, 67, 68, 120], [0, 64, 128], [5, 5, 5, 9], [0, 63, 126, 130]]


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("cuts", CUTS)
def test_packed_sequences(dtype, cuts):
    N, H, D = 130, 2, 64
    *x, d_o = gpu(*make(1, 1, H, N, D, D, dtype, sum(cuts)))
    cu = torch.tensor(cuts, dtype=torch.int32, device=dev())
    seqs = len(cuts) - 1
    kv0 = states(seqs, H, D, D, 5).to(dev())
    mark = 77.0
    o = torch.full_like(x[2], mark)
    _, kv = ltn.ltn_delta_fwd(*x, kv_in=kv0, cu=cu, return_state=True, out=o)
    outside = torch.ones(N, dtype=torch.bool, device=dev())
    outside[cuts[0] : cuts[-1]] = False
    assert (o[:, :, outside] == mark).all()
    for i, (a, b) in enumerate(zip(cuts[:-1], cuts[1:])):
        if a == b:
            assert torch.equal(kv[i], kv0[i])
            continue
        o_ref, kv_ref = recurrence(*(t[:, :, a:b] for t in x), 1.0, kv0[i : i + 1])
        assert rel(o[:, :, a:b], o_ref) <= TOL[dtype] and rel(kv[i : i + 1], kv_ref) <= TOL_STATE
    out = [torch.full_like(t, mark) for t in (x[0], x[1], x[2])] + [torch.full((1, H, N), mark, dtype=dtype, device=dev()) for _ in range(2)]
    ltn.ltn_delta_bwd(*x, d_o, cu=cu, out=out)
    want = packed(cuts, lambda *t: gradients(*t, 1.0)[1:], (*x, d_o))
    for n, a, b in zip(NAMES, out, want):
        assert (a[:, :, outside] == mark).all(), n
        assert rel(a[:, :, ~outside], b[:, :, ~outside]) <= TOL[dtype], n


def test_packed_ends_out_of_order_stay_within_the_tensors():
    """Not a supported call: what is checked is that rows outside [0, N) and other tensors stay untouched."""
    N, H, D = 130, 2, 64
    *x, d_o = gpu(*make(1, 2, H, N, D, D, BF, 3))
    for cuts in ([-5, 400, 20], [100, 20, 130], [2**31 - 1, 0, -(2**31)]):
        cu = torch.tensor(cuts, dtype=torch.int32, device=dev())
        pad = torch.full((3, *x[2].shape), 77.0, dtype=BF, device=dev())
        ltn.ltn_delta_fwd(*x, cu=cu, out=pad[1])
        assert (pad[0] == 77).all() and (pad[2] == 77).all()
        ltn.ltn_delta_bwd(*x, d_o, cu=cu)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("case", ["no_decay", "strong", "dropped", "beta_zero", "beta_one", "same_keys"])
def test_gates_at_their_ends(dtype, case):
    N = 150
    q, k, v, g, beta, d_o = make(1, 2, 2, N, 64, 64, dtype, 17)
    if case == "no_decay":
        g = torch.zeros_like(g)
    if case == "strong":                   # sums of log decays far below what exp can hold
        g = g * 60
    if case == "dropped":                  # the state is dropped at some tokens
        g[:, :, ::13] = float("-inf")
    if case == "beta_zero":
        beta[:, :, ::3] = 0.0
    if case == "beta_one":
        beta = torch.ones_like(beta)
    if case == "same_keys":                # every key nearly the same: the chunk's triangle is full
        k = (k[:, :, :1].float() + 0.05 * k.float()).to(dtype)
        k = (k.float() / k.float().norm(dim=-1, keepdim=True)).to(dtype)
    q, k, v, g, beta, d_o = gpu(q, k, v, g, beta, d_o)
    o, kv = ltn.ltn_delta_fwd(q, k, v, g, beta, return_state=True)
    _, kv_ref = recurrence(q, k, v, g, beta, 1.0)
    want = gradients(q, k, v, g.clamp(min=-1e30), beta, d_o, 1.0)
    assert rel(kv, kv_ref) <= TOL_STATE
    for n, a, b in zip(("o", *NAMES), (o, *ltn.ltn_delta_bwd(q, k, v, g, beta, d_o)), want):
        assert torch.isfinite(a.float()).all(), n
        assert rel(a, b) <= TOL[dtype], n


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("Dk,Dv", WIDTHS)
def test_decode_steps(dtype, Dk, Dv):
    Bt, Hk, H, S = 3, 2, 4, 5
    x = gpu(*make(Bt, Hk, H, S, Dk, Dv, dtype, 5)[:5])
    kv0 = states(Bt, H, Dk, Dv, 9).to(dev())
    o_ref, kv_ref = recurrence(*x, 0.5, kv0)
    kv = kv0.clone()
    o = ltn.ltn_delta_decode_steps(*x[:3], kv, *x[3:], scale=0.5)
    assert rel(o, o_ref) <= (2.0**-8 if dtype == BF else 2e-6) and rel(kv, kv_ref) <= 2e-6
    one = kv0.clone()
    for t in range(S):
        part = ltn.ltn_delta_decode_steps(*(y[:, :, t : t + 1].contiguous() for y in x[:3]), one,
                                          *(y[:, :, t : t + 1].contiguous() for y in x[3:]), scale=0.5)
        assert torch.equal(part, o[:, :, t : t + 1])
    assert torch.equal(one, kv)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_a_prompt_in_pieces_and_then_tokens(dtype):
    """Forward, forward from its state (in place), then decode: one sequence."""
    Bt, H, D, N = 2, 2, 128, 150
    x = gpu(*make(Bt, H, H, N, D, D, dtype, 23)[:5])
    o_ref, kv_ref = recurrence(*x, 1.0)

    def cut(a, b):
        return [t[:, :, a:b].contiguous() for t in x]

    o1, kv = ltn.ltn_delta_fwd(*cut(0, 70), return_state=True)
    o2, kv = ltn.ltn_delta_fwd(*cut(70, 147), kv_in=kv, kv_out=kv)
    p = cut(147, 150)
    o3 = ltn.ltn_delta_decode_steps(*p[:3], kv, *p[3:])
    assert rel(torch.cat((o1, o2, o3), 2), o_ref) <= TOL[dtype] and rel(kv, kv_ref) <= TOL_STATE


def test_empty_calls():
    x = gpu(*make(2, 2, 2, 0, 64, 64, BF, 1))
    kv0 = states(2, 2, 64, 64, 1).to(dev())
    o, kv = ltn.ltn_delta_fwd(*x[:5], kv_in=kv0, return_state=True)
    assert o.numel() == 0 and torch.equal(kv, kv0)
    _, kv = ltn.ltn_delta_fwd(*x[:5], return_state=True)
    assert (kv == 0).all()
    assert all(t.numel() == 0 for t in ltn.ltn_delta_bwd(*x))
    assert ltn.ltn_delta_decode_steps(*x[:3], kv0, *x[3:5]).numel() == 0
    x = gpu(*make(1, 2, 2, 8, 64, 64, BF, 1))
    cu = torch.zeros(3, dtype=torch.int32, device=dev())
    _, kv = ltn.ltn_delta_fwd(*x[:5], kv_in=kv0, cu=cu, return_state=True)
    assert torch.equal(kv, kv0)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_same_bits_every_run_and_in_a_batch(dtype):
    *x, d_o = gpu(*make(3, 2, 4, 200, 128, 64, dtype, 41))
    first = (*ltn.ltn_delta_fwd(*x, return_state=True), *ltn.ltn_delta_bwd(*x, d_o))
    again = (*ltn.ltn_delta_fwd(*x, return_state=True), *ltn.ltn_delta_bwd(*x, d_o))
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    alone = [t[1:2].contiguous() for t in (*x, d_o)]
    one = (*ltn.ltn_delta_fwd(*alone[:5], return_state=True), *ltn.ltn_delta_bwd(*alone))
    assert all(torch.equal(a[1:2], b) for a, b in zip(first, one))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_captured_calls_replay(dtype):
    *x, d_o = gpu(*make(1, 2, 2, 100, 64, 64, dtype, 43))
    cu = torch.tensor([0, 30, 100], dtype=torch.int32, device=dev())
    kv0 = states(1, 2, 64, 64, 3).to(dev())
    kv = kv0.clone()

    def step():
        o = ltn.ltn_delta_fwd(*x, cu=cu)
        p = [t[:, :, :2].contiguous() for t in x]
        return (o, *ltn.ltn_delta_bwd(*x, d_o, cu=cu), ltn.ltn_delta_decode_steps(*p[:3], kv, *p[3:]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(3):
        x[2].copy_(torch.randn_like(x[2]))
        kv.copy_(kv0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        kv.copy_(kv0)
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i

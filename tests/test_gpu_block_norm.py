"""GPU parity of the norms around a block against their definition in 64 bits (autograd).

Bounds as relative 2-norms: everything is computed in fp32 and rounded once: bf16 outputs 2^-8 at most (half a step); fp32
outputs and the weights' gradients some roundings of 2^-24 and means over up to 8192 terms, 2e-6.
"""
import pytest
import torch

import paper_2307_14995_amd as ltn
from _delta_ref import block_norm, rel
from _helpers import dev

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
TOL = {BF: 2.0**-8, F32: 2e-6}


def make(rows, C, gates, wa, wb, dtype, seed):
    r = torch.Generator().manual_seed(seed)

    def randn(*shape):
        return torch.randn(*shape, generator=r)

    x, y, dx, dh = (randn(rows, C).to(dtype).to(dev()) for _ in range(4))
    gate = randn(gates, C).to(dtype).to(dev()) if gates else None
    return x, y, dx, dh, gate, (1 + 0.3 * randn(C)).to(dev()) if wa else None, (1 + 0.3 * randn(C)).to(dev()) if wb else None


def check(rows, C, gates, wa, wb, dtype, after=True, scale=0.7, eps=1e-5, seed=0, with_dx=True):
    x, y, dx, dh, gate, w_after, w_before = make(rows, C, gates, wa, wb, dtype, seed + rows + C)
    kw = dict(gate=gate, w_after=w_after, w_before=w_before, scale=scale, eps=eps, after=after)
    xo, h = ltn.ltn_block_norm_fwd(x, y, **kw)
    got = ltn.ltn_block_norm_bwd(x, y, dx if with_dx else None, dh, **kw)
    leaves = [None if t is None else t.double().requires_grad_() for t in (x, y, gate, w_after, w_before)]
    xo_ref, h_ref = block_norm(*leaves, scale, eps, after)
    there = [t for t in leaves if t is not None]
    grads = iter(torch.autograd.grad((xo_ref, h_ref), there, (dx.double() if with_dx else torch.zeros_like(xo_ref), dh.double())))
    want = [None if t is None else next(grads) for t in leaves]
    assert rel(xo, xo_ref.detach()) <= TOL[dtype] and rel(h, h_ref.detach()) <= TOL[dtype]
    for n, a, b in zip(("dx", "dy", "dgate", "dw_after", "dw_before"), got, want):
        assert (a is None) == (b is None), n
        if a is not None:
            assert a.shape == b.shape and a.dtype == (F32 if n[1] == "w" else dtype), n
            assert rel(a, b) <= TOL[a.dtype], n


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("C", [8, 72, 512, 520, 1024, 1032, 2048, 2056, 4096, 4104, 8192])
def test_widths(dtype, C):
    check(5, C, 0, True, True, dtype)
    check(3, C, 3, False, True, dtype)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 63, 1025, 8200])
def test_rows(dtype, rows):
    check(rows, 96, 0, True, True, dtype)
    check(rows, 96, 1, True, False, dtype)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("rows,gates", [(12, 12), (12, 6), (12, 4), (12, 1), (300, 100), (300, 3), (9000, 9), (9000, 4500), (4099, 4099), (4099, 1), (12288, 2)])
@pytest.mark.parametrize("C", [64, 1536, 4096])
def test_gates(dtype, rows, gates, C):
    """Gates that lie within a team's rows, cross them, or hold many teams'."""
    check(rows, C, gates, True, True, dtype)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_without_the_norm_behind_or_weights(dtype):
    check(33, 1152, 0, False, False, dtype)
    check(33, 1152, 11, False, True, dtype, after=False)
    check(33, 1152, 33, False, False, dtype, after=False, scale=1.0)
    check(33, 1152, 0, True, True, dtype, with_dx=False)


@pytest.mark.parametrize("dtype", [F32, BF])
def test_rows_of_zeros(dtype):
    x, y, dx, dh, *_ = make(6, 256, 0, False, False, dtype, 1)
    x[2], y[2], y[4] = 0, 0, 0
    xo, h = ltn.ltn_block_norm_fwd(x, y, eps=1e-6)
    assert (xo[2] == 0).all() and (h[2] == 0).all() and torch.equal(xo[4], x[4]) and torch.isfinite(h.float()).all()
    g = ltn.ltn_block_norm_bwd(x, y, dx, dh, eps=1e-6)
    assert all(torch.isfinite(t.float()).all() for t in g[:2])
    h = ltn.ltn_block_norm_fwd(x, y, after=False)[1]       # eps = 0: the formula's NaN, in that row alone
    assert h[2].isnan().all() and torch.isfinite(h[[0, 1, 3, 4, 5]].float()).all()


def test_no_rows():
    x = torch.empty(0, 64, dtype=BF, device=dev())
    w = torch.ones(64, device=dev())
    xo, h = ltn.ltn_block_norm_fwd(x, x.clone(), w_before=w)
    assert xo.shape == h.shape == (0, 64)
    gate = torch.ones(3, 64, dtype=BF, device=dev())
    _, _, dgate, dwa, dwb = ltn.ltn_block_norm_bwd(x, x.clone(), None, x.clone(), gate=gate, w_after=w, w_before=w.clone())
    assert (dgate == 0).all() and (dwa == 0).all() and (dwb == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF])
def test_in_place_and_same_bits(dtype):
    x, y, dx, dh, gate, wa, wb = make(1000, 1000, 10, True, True, dtype, 2)
    kw = dict(gate=gate, w_after=wa, w_before=wb, scale=0.5, eps=1e-6)
    xo, h = ltn.ltn_block_norm_fwd(x, y, **kw)
    first, again = (ltn.ltn_block_norm_bwd(x, y, dx, dh, **kw) for _ in range(2))
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    x2, h2 = x.clone(), torch.empty_like(x)
    ltn.ltn_block_norm_fwd(x2, y, **kw, out=(x2, h2))
    assert torch.equal(x2, xo) and torch.equal(h2, h)


def test_nothing_outside_the_outputs_is_written():
    rows, C = 37, 1032
    for dtype in (BF, F32):
        x, y, dx, dh, gate, wa, wb = make(rows, C, 37, True, True, dtype, 4)
        pads = [torch.full((rows + 2, C), 5.0, dtype=dtype, device=dev()) for _ in range(2)]
        ltn.ltn_block_norm_fwd(x, y, gate=gate, w_after=wa, w_before=wb, eps=1e-6, out=[p[1:-1] for p in pads])
        assert all((p[[0, -1]] == 5).all() for p in pads)


def test_captured_calls_replay():
    x, y, dx, dh, gate, wa, wb = make(200, 256, 4, True, True, BF, 5)

    def step():
        kw = dict(gate=gate, w_after=wa, w_before=wb, eps=1e-6)
        return (*ltn.ltn_block_norm_fwd(x, y, **kw), *ltn.ltn_block_norm_bwd(x, y, dx, dh, **kw))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        y.copy_(torch.randn_like(y))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
        torch.cuda.synchronize()

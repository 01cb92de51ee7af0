"""Host-side checks (no GPU) of the gated delta rule's and the block norm's entry points: refusals before any launch,
workspace sizes, the binding's argument errors; and the tests' own reference against difference quotients."""
import pytest
import torch

import paper_2307_14995_amd as ltn
from _delta_ref import block_norm, gradients, make, recurrence

OK, E_NULL, E_SHAPE, E_UNSUP, E_ALIGN = range(5)
G = 1 << 36              # fake, aligned, never dereferenced; tensors sit 64 GiB apart
F32, BF = 0, 1


@pytest.fixture(scope="module")
def lib():
    return ltn.load_library()


def fwd(lib, q=G, k=2 * G, v=3 * G, o=4 * G, g=5 * G, beta=6 * G, cu=None, kv_in=None, kv_out=None, Bt=1, Hk=2, H=2, N=100, Dk=64,
        Dv=64, seqs=0, dtype=BF, ws=9 * G, ws_bytes=1 << 30):
    return lib.ltn_delta_fwd(q, k, v, o, g, beta, cu, kv_in, kv_out, 1.0, Bt, Hk, H, N, Dk, Dv, seqs, dtype, ws, ws_bytes, None)


def bwd(lib, q=G, k=2 * G, v=3 * G, d_o=4 * G, dq=10 * G, dk=11 * G, dv=12 * G, dg=13 * G, db=14 * G, g=5 * G, beta=6 * G, cu=None,
        Bt=1, Hk=2, H=2, N=100, Dk=64, Dv=64, seqs=0, dtype=BF, ws=9 * G, ws_bytes=1 << 30):
    return lib.ltn_delta_bwd(q, k, v, d_o, dq, dk, dv, dg, db, g, beta, cu, 1.0, Bt, Hk, H, N, Dk, Dv, seqs, dtype, ws, ws_bytes, None)


def decode(lib, q=G, k=2 * G, v=3 * G, o=4 * G, kv=7 * G, g=5 * G, beta=6 * G, Bt=1, Hk=2, H=2, S=1, Dk=64, Dv=64, dtype=BF):
    return lib.ltn_delta_decode_steps(q, k, v, o, kv, g, beta, 1.0, Bt, Hk, H, S, Dk, Dv, dtype, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_delta_refusals(lib, call):
    for name in ("q", "k", "v", "g", "beta", "ws", *(("o",) if call is fwd else ("d_o", "dq", "dk", "dv", "dg", "db"))):
        assert call(lib, **{name: None}) == E_NULL, name
    for bad in (dict(Bt=-1), dict(H=-2), dict(N=-1), dict(Dk=0), dict(Hk=0), dict(Hk=2, H=3), dict(N=2**31), dict(ws_bytes=100),
                dict(Bt=1 << 20, H=1 << 12, Hk=1 << 12), dict(cu=15 * G, Bt=2, seqs=3), dict(cu=15 * G, seqs=-1)):
        assert call(lib, **bad) == E_SHAPE, bad
    for bad in (dict(Dk=96), dict(Dv=256), dict(Dk=128, Dv=96), dict(dtype=2), dict(dtype=-7)):
        assert call(lib, **bad) == E_UNSUP, bad
    for name in ("q", "k", "v", "ws", *(("o", "kv_in", "kv_out") if call is fwd else ("d_o", "dq", "dk", "dv"))):
        assert call(lib, **{name: 16 * G + 8}) == E_ALIGN, name
    for name in ("g", "beta", "cu", *(() if call is fwd else ("dg", "db"))):
        assert call(lib, **{name: 16 * G + 2}) == E_ALIGN, name
    assert call(lib, Bt=0) == OK and call(lib, H=0, Hk=0) == OK and call(lib, N=0) == OK


def test_delta_overlaps(lib):
    tb = 2 * 100 * 64 * 2
    for out in (G, 2 * G + tb - 16, 3 * G, 5 * G, 6 * G + 16, 9 * G):
        assert fwd(lib, o=out) == E_UNSUP, out
    assert fwd(lib, kv_out=3 * G) == E_UNSUP and fwd(lib, kv_out=4 * G) == E_UNSUP
    assert fwd(lib, kv_in=7 * G, kv_out=7 * G + 16) == E_UNSUP
    assert fwd(lib, cu=15 * G, seqs=3, o=15 * G) == E_UNSUP
    for name in ("dq", "dk", "dv", "dg", "db"):
        for out in (G, 4 * G, 5 * G, 9 * G):
            assert bwd(lib, **{name: out}) == E_UNSUP, (name, out)
    assert bwd(lib, dq=11 * G) == E_UNSUP and bwd(lib, dg=14 * G) == E_UNSUP


def test_decode_refusals(lib):
    for name in ("q", "k", "v", "o", "kv", "g", "beta"):
        assert decode(lib, **{name: None}) == E_NULL, name
    for bad in (dict(Bt=-1), dict(S=-1), dict(Hk=2, H=5), dict(Dk=-64)):
        assert decode(lib, **bad) == E_SHAPE, bad
    for bad in (dict(Dk=96), dict(Dv=32), dict(dtype=3), dict(o=G), dict(kv=3 * G), dict(kv=4 * G)):
        assert decode(lib, **bad) == E_UNSUP, bad
    assert decode(lib, kv=7 * G + 4) == E_ALIGN and decode(lib, g=5 * G + 1) == E_ALIGN
    assert decode(lib, Bt=0) == OK and decode(lib, S=0) == OK


def test_delta_workspace(lib):
    ws = ltn.ltn_delta_workspace_bytes
    for dtype in (torch.bfloat16, torch.float32):
        one = ws(1, 1, 64, 128, 128, 0, dtype, 0)
        assert one > 0 and ws(2, 3, 640, 128, 128, 0, dtype, 0) == 60 * one
        assert ws(1, 1, 65, 128, 128, 0, dtype, 0) == 2 * one
        assert ws(1, 1, 640, 128, 128, 7, dtype, 0) == 17 * one        # a chunk more for each sequence at most
        assert ws(1, 1, 64, 128, 128, 0, dtype, 1) > one
        assert ws(0, 1, 64, 128, 128, 0, dtype, 0) == ws(1, 1, 0, 128, 128, 0, dtype, 0) == ws(1, 1, 64, 96, 128, 0, dtype, 0) == 0
        assert ws(2, 1, 64, 128, 128, 3, dtype, 0) == 0                # packed: one row
        assert ws(1, 1, 64, 128, 128, 0, dtype, 2) == 0
        need = ws(1, 2, 100, 64, 64, 0, dtype, 0)
        code = BF if dtype == torch.bfloat16 else F32
        assert fwd(lib, ws_bytes=need - 1, dtype=code) == E_SHAPE


def norm_fwd(lib, x=G, y=2 * G, gate=None, wa=None, wb=None, xo=3 * G, h=4 * G, eps=0.0, after=1, rows=10, gates=0, C=64, dtype=BF):
    return lib.ltn_block_norm_fwd(x, y, gate, wa, wb, xo, h, 1.0, eps, after, rows, gates, C, dtype, None)


def norm_bwd(lib, x=G, y=2 * G, gate=None, wa=None, wb=None, dxo=5 * G, dh=6 * G, dx=3 * G, dy=4 * G, dgate=None, dwa=None, dwb=None,
             eps=0.0, after=1, rows=10, gates=0, C=64, dtype=BF, ws=9 * G, ws_bytes=1 << 30):
    return lib.ltn_block_norm_bwd(x, y, gate, wa, wb, dxo, dh, dx, dy, dgate, dwa, dwb, 1.0, eps, after, rows, gates, C, dtype, ws, ws_bytes, None)


def test_block_norm_refusals(lib):
    for call in (norm_fwd, norm_bwd):
        for bad in (dict(rows=-1), dict(C=0), dict(eps=-1e-6), dict(eps=float("nan")), dict(gate=7 * G, gates=0), dict(gate=7 * G, gates=3),
                    dict(rows=1 << 31)):
            assert call(lib, **bad) == E_SHAPE, bad
        for bad in (dict(C=60), dict(C=8200), dict(dtype=2), dict(after=0, wa=8 * G)):
            assert call(lib, **bad) == E_UNSUP, bad
        for name in ("x", "y", "wb"):
            assert call(lib, **{name: 16 * G + 4}, **({"dwb": 11 * G} if name == "wb" and call is norm_bwd else {})) == E_ALIGN, name
    for name in ("x", "y", "xo", "h"):
        assert norm_fwd(lib, **{name: None}) == E_NULL
    for name in ("x", "y", "dh", "dx", "dy", "ws"):
        assert norm_bwd(lib, **{name: None}) == E_NULL
    # a gradient for everything that has one, and for nothing else
    assert norm_bwd(lib, gate=7 * G, gates=5) == E_NULL and norm_bwd(lib, dgate=7 * G) == E_NULL
    assert norm_bwd(lib, wa=7 * G) == E_NULL and norm_bwd(lib, dwb=7 * G) == E_NULL
    assert norm_bwd(lib, ws_bytes=16) == E_SHAPE
    assert norm_fwd(lib, h=G) == E_UNSUP and norm_fwd(lib, xo=2 * G) == E_UNSUP and norm_fwd(lib, xo=G + 64) == E_UNSUP
    assert norm_fwd(lib, xo=4 * G) == E_UNSUP
    for out in ("dx", "dy"):
        for at in (G, 2 * G, 5 * G, 6 * G, 9 * G):
            assert norm_bwd(lib, **{out: at}) == E_UNSUP
    assert ltn.ltn_block_norm_workspace_bytes(0, 64) == ltn.ltn_block_norm_workspace_bytes(5, 60) == 0
    assert norm_fwd(lib, rows=0) == OK


def test_the_binding_refuses():
    *x, d_o = make(1, 2, 4, 8, 64, 64, torch.bfloat16, 1)
    for fn in (lambda: ltn.ltn_delta_fwd(*x), lambda: ltn.ltn_delta_bwd(*x, d_o),
               lambda: ltn.ltn_delta_decode_steps(*x[:3], torch.zeros(1, 4, 64, 64), *x[3:]),
               lambda: ltn.ltn_block_norm_fwd(d_o, d_o), lambda: ltn.ltn_block_norm_bwd(d_o, d_o, None, d_o)):
        with pytest.raises(ValueError, match="GPU"):
            fn()


def test_the_reference_against_differences():
    torch.manual_seed(0)
    x = [t.double() for t in make(1, 1, 2, 5, 4, 3, torch.float64, 3)]
    *leaves, d_o = x
    _, *grads = gradients(*leaves, d_o, 0.5)
    for i, t in enumerate(leaves):
        step = torch.randn_like(t) * 1e-6
        up, down = ([a + s * step if j == i else a for j, a in enumerate(leaves)] for s in (1, -1))
        slope = ((recurrence(*up, 0.5)[0] - recurrence(*down, 0.5)[0]) * d_o).sum() / 2
        assert torch.isclose(slope, (grads[i] * step).sum(), rtol=1e-6, atol=1e-14)
    x, y, gate, w = (torch.randn(s, dtype=torch.float64, requires_grad=True) for s in ((4, 6), (4, 6), (2, 6), (6,)))
    assert torch.autograd.gradcheck(lambda x, y, g, w: block_norm(x, y, g, w, w * 2, 0.7, 1e-5, True), (x, y, gate, w))


@pytest.mark.parametrize("call", [fwd, bwd])
def test_more_than_a_launch_holds_is_refused(lib, call):
    big = dict(ws_bytes=1 << 60, q=1 << 50, ws=1 << 60)
    assert call(lib, Bt=1 << 21, N=1, **big) == E_SHAPE                             # 2^22 chains
    assert call(lib, N=1 << 28, **big) == E_SHAPE                                   # 2^23 chunks and heads
    assert call(lib, cu=15 * G, seqs=1 << 21, N=1, **big) == E_SHAPE
    assert ltn.ltn_delta_workspace_bytes(1 << 21, 2, 1, 64, 64, 0, torch.bfloat16, 0) == 0
    assert ltn.ltn_delta_workspace_bytes(1, 2, 1 << 28, 64, 64, 0, torch.bfloat16, 0) == 0
    assert ltn.ltn_delta_workspace_bytes(1, 2, (1 << 28) - 64, 64, 64, 0, torch.bfloat16, 0) > 0


class Stub:
    """A tensor as the binding's checks see one, on a GPU that need not exist."""

    def __init__(self, index, dtype, *shape):
        self.device, self.dtype, self.shape, self.is_cuda = torch.device("cuda", index), dtype, torch.Size(shape), True

    dim = lambda self: len(self.shape)
    numel = lambda self: self.shape.numel()
    is_contiguous = lambda self: True


def test_an_output_on_another_gpu_is_refused(monkeypatch):
    from paper_2307_14995_amd import binding

    class NoFast:                          # (its marshalling passes on what it does not take)
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(binding, "_fast", NoFast)
    bf, f32 = torch.bfloat16, torch.float32
    q, v, g, s, x = Stub(0, bf, 1, 2, 8, 64), Stub(0, bf, 1, 2, 8, 64), Stub(0, f32, 1, 2, 8), Stub(0, f32, 1, 2, 64, 64), Stub(0, bf, 8, 64)
    v1, g1, s1, x1 = (Stub(1, t.dtype, *t.shape) for t in (v, g, s, x))
    dg = Stub(0, bf, 1, 2, 8)
    for fn in (lambda: ltn.ltn_delta_fwd(q, q, v, g, g, out=v1), lambda: ltn.ltn_delta_fwd(q, q, v, g, g, kv_in=s1, out=v),
               lambda: ltn.ltn_delta_fwd(q, q, v, g, g, kv_out=s1, out=v), lambda: ltn.ltn_delta_fwd(q, q, v1, g, g, out=v),
               lambda: ltn.ltn_delta_bwd(q, q, v, g, g, v, out=(q, q, v, dg, Stub(1, bf, 1, 2, 8))),
               lambda: ltn.ltn_delta_decode_steps(q, q, v, s, g, g, out=v1), lambda: ltn.ltn_delta_decode_steps(q, q, v, s, g1, g, out=v),
               lambda: ltn.ltn_block_norm_fwd(x, x, out=(x, x1))):
        with pytest.raises(ValueError, match="one GPU"):
            fn()

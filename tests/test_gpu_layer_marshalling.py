"""The native marshalling of the gated delta rule's and the block norm's entry points against the Python path behind it."""
import pytest
import torch

import paper_2307_14995_amd as ltn
from paper_2307_14995_amd import binding
from _delta_ref import make
from _helpers import dev
from test_gpu_marshalling import Recorder, Refuses, flat

pytestmark = pytest.mark.gpu

Bt, Hk, H, N, D = 1, 2, 4, 70, 64
ENTRIES = ("delta_fwd", "delta_bwd", "delta_decode_steps", "block_norm_fwd", "block_norm_bwd")


def inputs(dtype):
    x = [t.to(dev()) for t in make(Bt, Hk, H, N, D, D, dtype, 3)]
    r = torch.Generator().manual_seed(4)
    kv = torch.randn(Bt, H, D, D, generator=r).to(dev())
    cu = torch.tensor([0, 70], dtype=torch.int32, device=dev())
    w = torch.rand(D, generator=r).to(dev())
    gate = torch.randn(H, D, generator=r).to(dtype).to(dev())
    return x, kv, cu, w, gate


def calls(dtype):
    (q, k, v, g, beta, d_o), kv, cu, w, gate = inputs(dtype)
    s = kv.clone()
    norm = dict(gate=gate, w_after=w, w_before=w, scale=0.5, eps=1e-6)
    return {
        "delta_fwd": [lambda: ltn.ltn_delta_fwd(q, k, v, g, beta), lambda: ltn.ltn_delta_fwd(q, k, v, g, beta, kv_in=kv, cu=cu, scale=0.5, return_state=True)],
        "delta_bwd": [lambda: ltn.ltn_delta_bwd(q, k, v, g, beta, d_o), lambda: ltn.ltn_delta_bwd(q, k, v, g, beta, d_o, cu=cu, scale=2)],
        "delta_decode_steps": [lambda: (ltn.ltn_delta_decode_steps(q, k, v, s.copy_(kv), g, beta, scale=0.5), s.clone())],
        "block_norm_fwd": [lambda: ltn.ltn_block_norm_fwd(v, d_o, eps=1e-6), lambda: ltn.ltn_block_norm_fwd(v, d_o, **norm),
                           lambda: ltn.ltn_block_norm_fwd(v, d_o, eps=1e-6, after=False)],
        "block_norm_bwd": [lambda: tuple(t for t in ltn.ltn_block_norm_bwd(v, d_o, None, v, eps=1e-6) if t is not None),
                           lambda: ltn.ltn_block_norm_bwd(v, d_o, v, d_o, **norm)],
    }


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_same_bits_as_the_python_path(dtype, monkeypatch):
    recorder = Recorder(binding._fast())
    monkeypatch.setattr(binding, "_native", recorder)
    native = {n: [flat(f()) for f in fs] for n, fs in calls(dtype).items()}
    assert {n: all(d) for n, d in recorder.did.items()} == {n: True for n in ENTRIES}
    monkeypatch.setattr(binding, "_native", Refuses())
    for n, fs in calls(dtype).items():
        for f, want in zip(fs, native[n]):
            got = flat(f())
            assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want)), n


def native_arguments(dtype):
    (q, k, v, g, beta, d_o), kv, cu, w, gate = inputs(dtype)
    return {
        "delta_fwd": [q, k, v, g, beta, kv, cu, 0.5, True, None, None],
        "delta_bwd": [q, k, v, g, beta, d_o, cu, 0.5],
        "delta_decode_steps": [q, k, v, kv, g, beta, 0.5, None],
        "block_norm_fwd": [v, d_o, gate, w, w, 0.5, 1e-6, True],
        "block_norm_bwd": [v, d_o, v, d_o, gate, w, w, 0.5, 1e-6, True],
    }


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_entry_refuses_each_wrong_argument(entry, dtype):
    native, args = getattr(binding._fast(), entry), native_arguments(dtype)[entry]
    assert native(*args) is not None
    for i, a in enumerate(args):
        if isinstance(a, torch.Tensor):
            wrong = [a.cpu(), a.half(), a[..., :-1], a[..., :-1].contiguous()[..., :0], torch.cat((a, a), -1)[..., ::2], 1, "x"]
            if i == 6 and entry != "block_norm_bwd":
                wrong[3] = a[:1].contiguous()                            # (one end is no sequence)
        elif a is None:
            wrong = [1, "x", torch.empty(1, device="cuda"), torch.empty(Bt, H, N, 2 * D, dtype=torch.half, device="cuda")]
        elif isinstance(a, bool):
            wrong = [1, None, "x"]
        else:
            wrong = [None, "x", torch.zeros(1)]
        for w in wrong:
            if a is w or (isinstance(a, torch.Tensor) and isinstance(w, torch.Tensor) and a.dtype == w.dtype and a.shape == w.shape and w.is_contiguous() and w.is_cuda):
                continue
            assert native(*args[:i], w, *args[i + 1 :]) is None, (i, w)
    assert native(*args[:-1]) is None and native(*args, None) is None


def test_the_binding_refuses():
    (q, k, v, g, beta, d_o), kv, cu, w, gate = inputs(torch.bfloat16)
    bad = [
        lambda: ltn.ltn_delta_fwd(q, k, v[:, :3].contiguous(), g[:, :3].contiguous(), beta[:, :3].contiguous()),     # 3 value heads, 2 key heads
        lambda: ltn.ltn_delta_fwd(q, k[..., :32].contiguous(), v, g, beta),
        lambda: ltn.ltn_delta_fwd(q, k, v, g.bfloat16(), beta),
        lambda: ltn.ltn_delta_fwd(q, k, v, g, beta[..., :-1].contiguous()),
        lambda: ltn.ltn_delta_fwd(q, k, v, g, beta, cu=cu.long()),
        lambda: ltn.ltn_delta_fwd(q, k, v, g, beta, cu=cu.cpu()),
        lambda: ltn.ltn_delta_fwd(q.repeat(2, 1, 1, 1), k.repeat(2, 1, 1, 1), v.repeat(2, 1, 1, 1), g.repeat(2, 1, 1), beta.repeat(2, 1, 1), cu=cu),
        lambda: ltn.ltn_delta_fwd(q, k, v, g, beta, kv_in=kv[:, :2].contiguous()),
        lambda: ltn.ltn_delta_fwd(q, k, v.transpose(1, 2), g, beta),
        lambda: ltn.ltn_delta_bwd(q, k, v, g, beta, d_o.float()),
        lambda: ltn.ltn_delta_decode_steps(q, k, v, kv.double(), g, beta),
        lambda: ltn.ltn_block_norm_fwd(v, d_o.float()),
        lambda: ltn.ltn_block_norm_fwd(v, d_o, gate=gate.float()),
        lambda: ltn.ltn_block_norm_fwd(v, d_o, gate=gate[:3]),           # 3 gates for 280 rows
        lambda: ltn.ltn_block_norm_fwd(v, d_o, w_after=w.bfloat16()),
        lambda: ltn.ltn_block_norm_fwd(v, d_o, w_after=w, after=False),
        lambda: ltn.ltn_block_norm_bwd(v, d_o, None, d_o[..., :32].contiguous()),
    ]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ltn.ltn_delta_fwd(*(t[..., :48].contiguous() for t in (q, k, v)), g, beta),
              lambda: ltn.ltn_block_norm_fwd(v[..., :4].contiguous(), d_o[..., :4].contiguous()),
              lambda: ltn.ltn_block_norm_fwd(v, d_o, eps=-1.0),
              lambda: ltn.ltn_block_norm_fwd(v, d_o, out=(d_o, torch.empty_like(v)))):
        with pytest.raises(ltn.LtnError):
            f()
    with pytest.raises(TypeError):
        ltn.ltn_delta_fwd(q.half(), k.half(), v.half(), g, beta)

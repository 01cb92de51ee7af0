"""The gated delta rule and the norms around a block in 64 bits, from their definitions (test infrastructure).

Token by token, by torch's autograd: S_t = A_t + k_t u_t^T with A_t = exp(g_t) S_{t-1}, u_t = beta_t (v_t - A_t^T k_t),
o_t = scale S_t^T q_t.  Nothing here is shared with the library or with its chunked form.
"""
import torch


def unit(x):
    return x / x.norm(dim=-1, keepdim=True)


def make(Bt, Hk, H, N, Dk, Dv, dtype, seed, device="cpu"):
    """(q, k, v, g, beta, d_o): unit queries and keys, log decays of -0.001 .. -2 a token."""
    r = torch.Generator().manual_seed(seed)
    q, k = (unit(torch.randn(Bt, Hk, N, Dk, generator=r)).to(dtype) for _ in range(2))
    v, d_o = (torch.randn(Bt, H, N, Dv, generator=r).to(dtype) for _ in range(2))
    g = -torch.exp(torch.empty(Bt, H, N).uniform_(-7.0, 0.7, generator=r))
    beta = torch.sigmoid(torch.randn(Bt, H, N, generator=r))
    return tuple(t.to(device) for t in (q, k, v, g, beta, d_o))


def recurrence(q, k, v, g, beta, scale, S=None):
    """(o, last state) in 64 bits; differentiable."""
    H = v.shape[1]
    q, k = (t.double().repeat_interleave(H // t.shape[1], dim=1) for t in (q, k))
    v, g, beta = v.double(), g.double(), beta.double()
    S = v.new_zeros((*v.shape[:2], q.shape[-1], v.shape[-1])) if S is None else S.double()
    o = []
    for t in range(v.shape[2]):
        A = torch.exp(g[:, :, t])[..., None, None] * S
        u = beta[:, :, t, None] * (v[:, :, t] - (k[:, :, t, :, None] * A).sum(-2))
        S = A + k[:, :, t, :, None] * u[..., None, :]
        o.append(scale * (q[:, :, t, :, None] * S).sum(-2))
    return (torch.stack(o, 2) if o else torch.zeros_like(v)), S


def gradients(q, k, v, g, beta, d_o, scale):
    """(o, dq, dk, dv, dg, dbeta) in 64 bits."""
    with torch.enable_grad():
        leaves = [t.detach().double().requires_grad_() for t in (q, k, v, g, beta)]
        o, _ = recurrence(*leaves, scale)
        grads = torch.autograd.grad(o, leaves, d_o.double())
    return (o.detach(), *grads)


def packed(cu, fn, tensors, fill=0.0):
    """fn over each sequence of one packed row, its results put together along the token axis (`fill` outside of them)."""
    N, out = tensors[0].shape[2], None
    for a, b in zip(cu[:-1], cu[1:]):
        if a == b:
            continue
        part = fn(*(t[:, :, a:b] for t in tensors))
        if out is None:
            out = [torch.full((*p.shape[:2], N, *p.shape[3:]), fill, dtype=p.dtype, device=p.device) for p in part]
        for t, p in zip(out, part):
            t[:, :, a:b] = p
    return out


def rel(got, want):
    """2-norm of the difference over that of `want` (which is not zero)."""
    want = want.double()
    return ((got.double().to(want.device) - want).norm() / want.norm()).item()


def block_norm(x, y, gate, w_after, w_before, scale, eps, after):
    """(x_out, h) in the inputs' precision; differentiable.  gate: [gates, C]."""
    def norm(t, w):
        t = t / (t.square().mean(-1, keepdim=True) + eps).sqrt()
        return t if w is None else t * w

    z = norm(y, w_after) if after else y
    if gate is not None:
        z = z * gate.repeat_interleave(x.shape[0] // gate.shape[0], dim=0)
    x = x + scale * z
    return x, norm(x, w_before)

"""The gated delta rule and the norms around a block, as timed cases.

Five kinds of pass, each through the public entry points of the Python binding:

  delta_train    one layer's training step: forward, then the gradients of q, k, v and of both gates
  delta_prefill  a prompt, or the next chunk of one: forward with the state handed on
  delta_decode   one decode call: `N` tokens per sequence against the running states
  norm_train     what stands between two blocks in training: the norm behind a block, its gate, the residual
                 scale and sum, the norm before the next block, and the gradients of all of them
  norm_infer     the same in inference

Shapes are [Bt, H, N, D]; `Hk` heads of queries and keys serve `H` heads of values.  With `seqs` the one row of N
tokens is packed: that many sequences of different lengths.  Sizes: the paper's models (8 / 16 / 32 heads of 128
features; widths of 1024, 2048, 4096), the training lengths, decode batch and chunk lengths that perf/cases.py has, and
the odd lengths, widths and small batches that training and serving meet.
"""
import math

import torch

own = False

EPS = 1e-6                       # under the root of a norm
CHUNK = 64                       # tokens of a chunk of the plain form
#: work of the largest listed case, in token-heads x Dk x Dv (bf16); fp32 products run at a sixteenth of the rate
BUDGET = 4 * 32 * 8192 * 128 ** 2
FP32_SHARE = 16
NORM_BUDGET = 4 * 8192 * 4096    # elements of the largest listed norm


def _delta(name, kind, Bt, Hk, H, N, Dk, Dv, dtype="bf16", seqs=0, state_in=False):
    return {"name": name, "kind": kind, "Bt": Bt, "Hk": Hk, "H": H, "N": N, "Dk": Dk, "Dv": Dv, "dtype": dtype,
            "seqs": seqs, "state_in": state_in}


def _norm(name, kind, Bt, N, C, dtype="bf16", gate="none", after=True, weights=True):
    return {"name": name, "kind": kind, "Bt": Bt, "N": N, "C": C, "dtype": dtype, "gate": gate, "after": after,
            "weights": weights}


def listed():
    return [
        # pre-training: a 7B-shaped layer at the paper's training length
        _delta("delta_train_7b", "delta_train", 4, 32, 32, 8192, 128, 128),
        # pre-training: a 385M-shaped layer, two heads of values to one of keys
        _delta("delta_train_385m", "delta_train", 8, 4, 8, 2048, 128, 128),
        # packed documents of different lengths, a total that is no multiple of anything, narrow keys
        _delta("delta_train_packed", "delta_train", 1, 16, 16, 15999, 64, 128, seqs=11),
        # numerics checks and small-model training
        _delta("delta_train_fp32", "delta_train", 2, 4, 8, 700, 64, 64, dtype="fp32"),
        # serving: one user's prompt
        _delta("delta_prefill_prompt", "delta_prefill", 1, 16, 32, 3001, 128, 128),
        # serving: the next chunk of a few prompts
        _delta("delta_prefill_chunk", "delta_prefill", 4, 8, 8, 200, 128, 128, state_in=True),
        # serving: one token for a full batch
        _delta("delta_decode_batch", "delta_decode", 64, 16, 32, 1, 128, 128),
        # serving: one token for one user
        _delta("delta_decode_one", "delta_decode", 1, 32, 32, 1, 128, 128),
        # pre-training: between two blocks of the 7B shape
        _norm("norm_train_7b", "norm_train", 4, 8192, 4096),
        # heads of 96 features: an odd width and length, a gate for each sequence
        _norm("norm_train_gated", "norm_train", 8, 1999, 1152, gate="sequence"),
        # a whole batch of prompts, gated element by element, the paper's norm without weights, fp32
        _norm("norm_infer_fp32", "norm_infer", 8, 1000, 2048, dtype="fp32", gate="element", weights=False),
        # serving: one token for a full batch
        _norm("norm_infer_step", "norm_infer", 64, 1, 4096),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(("delta_train", "delta_prefill", "delta_decode", "norm_train", "norm_infer"), (30, 22, 18, 18, 12))[0]
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    if kind.startswith("norm"):
        C = 8 * _log_int(rng, 8, 1024)
        N = _log_int(rng, 1, max(1, min(8192, NORM_BUDGET // (2 if dtype == "fp32" else 1) // C)))
        Bt = _log_int(rng, 1, max(1, min(64, NORM_BUDGET // (2 if dtype == "fp32" else 1) // (C * N))))
        return {"kind": kind, "Bt": Bt, "N": N, "C": C, "dtype": dtype, "gate": rng.choice(("none", "vector", "sequence", "element")),
                "after": rng.random() < 0.75, "weights": rng.random() < 0.7}
    Dk, Dv = rng.choice(((64, 64), (64, 128), (128, 64), (128, 128), (128, 128), (128, 128)))
    budget = BUDGET // (FP32_SHARE if dtype == "fp32" else 1) // (Dk * Dv)
    H = rng.choice((4, 6, 8, 12, 16, 20, 24, 32, 40))
    Hk = H // rng.choice((1, 1, 2))
    seqs = 0
    if kind == "delta_decode":
        N = rng.choice((1, 1, 1, 2, 3, 5, 8))
        Bt = _log_int(rng, 1, 96)
    else:
        N = _log_int(rng, 16, min(2048 if dtype == "fp32" else 16384, budget // H))
        Bt = _log_int(rng, 1, max(1, min(32, budget // (H * N))))
        if rng.random() < 0.3:
            N, Bt = min(N * Bt, 32768), 1
            seqs = _log_int(rng, 2, max(2, min(64, N // 8)))
    return {"kind": kind, "Bt": Bt, "Hk": Hk, "H": H, "N": N, "Dk": Dk, "Dv": Dv, "dtype": dtype, "seqs": seqs,
            "state_in": kind == "delta_prefill" and rng.random() < 0.5}


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def prepare(case, seed):
    dt, dev = _dtype(case), torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    def uniform(lo, hi, *shape):
        return torch.rand(shape, generator=g, device=dev).mul_(hi - lo).add_(lo)

    st = {"case": case}
    if case["kind"].startswith("norm"):
        Bt, N, C = case["Bt"], case["N"], case["C"]
        st.update(x=randn(Bt, N, C, dtype=dt), y=randn(Bt, N, C, dtype=dt).mul_(0.5), scale=0.7,
                  w_before=1 + 0.1 * randn(C) if case["weights"] else None,
                  w_after=1 + 0.1 * randn(C) if case["weights"] and case["after"] else None)
        shape = {"none": None, "vector": (1, C), "sequence": (Bt, C), "element": (Bt, N, C)}[case["gate"]]
        st["gate"] = None if shape is None else randn(*shape, dtype=dt)
        if case["kind"] == "norm_train":
            st.update(d_x=randn(Bt, N, C, dtype=dt), d_h=randn(Bt, N, C, dtype=dt))
        return st
    Bt, Hk, H, N, Dk, Dv = (case[n] for n in ("Bt", "Hk", "H", "N", "Dk", "Dv"))

    def activated(heads, D):     # what a convolution and its activation leave
        return torch.nn.functional.silu(randn(Bt, heads, N, D))

    def unit(x):
        return x.div_(x.square().sum(-1, keepdim=True).add_(EPS).sqrt_())

    st.update(q=unit(activated(Hk, Dk)).to(dt), k=unit(activated(Hk, Dk)).to(dt), v=activated(H, Dv).to(dt),
              beta=torch.sigmoid(randn(Bt, H, N)), scale=Dk ** -0.5)
    # log decays -a softplus(x + b): rates a of 1 .. 16, steps of 1e-3 .. 0.1 at x = 0
    b = torch.log(torch.expm1(torch.exp(uniform(math.log(1e-3), math.log(0.1), 1, H, 1))))
    st["g"] = -uniform(1.0, 16.0, 1, H, 1) * torch.nn.functional.softplus(0.5 * randn(Bt, H, N) + b)
    if case["kind"] == "delta_train":
        st["d_o"] = randn(Bt, H, N, Dv, dtype=dt)
    if case["kind"] == "delta_decode" or case["state_in"]:
        st["kv"] = 0.2 * randn(case["seqs"] or Bt, H, Dk, Dv)
    st["cu"] = None
    if case["seqs"]:             # cuts at random places: lengths from one token (now and then none) to most of the row
        cuts = torch.randint(0, N + 1, (case["seqs"] - 1,), generator=g, device=dev).sort().values
        ends = torch.tensor([0, N], device=dev)
        st["cu"] = torch.cat((ends[:1], cuts, ends[1:])).to(torch.int32)
        st["longest"] = int((st["cu"][1:] - st["cu"][:-1]).max())
    return st


# ---- the plain forms -------------------------------------------------------------------------------------------


def _heads(x, H):
    return x.float().repeat_interleave(H // x.shape[1], dim=1)


def _unpack(st, x):
    """[1, H, N, ...] -> [seqs, H, longest, ...] with zeros behind each sequence."""
    at = st["cu"][:-1, None].long() + torch.arange(st["longest"], device=x.device)
    inside = at < st["cu"][1:, None]
    return (x[0][:, at.clamp(max=x.shape[2] - 1)] * inside.view(1, *inside.shape, *(1,) * (x.dim() - 3))).transpose(0, 1)


def _pack(st, x):
    """The reverse of _unpack: token n sits in the sequence that ends behind it."""
    n = torch.arange(st["q"].shape[2], device=x.device)
    seq = torch.searchsorted(st["cu"][1:].long(), n, right=True)
    return x.transpose(0, 1)[:, seq, n - st["cu"].long()[seq]][None]


def _chunks(x, n):
    """[B, H, N, ...] -> [B H, n, CHUNK, ...], zeros behind the last token."""
    x = x.reshape(-1, *x.shape[2:])
    out = x.new_zeros((x.shape[0], n * CHUNK, *x.shape[2:]))
    out[:, : x.shape[1]] = x
    return out.view(x.shape[0], n, CHUNK, *x.shape[2:])


def _inverse(A):
    """(I + A)^-1 of strictly lower triangles, blocks of 1, 2, 4 ... merged in pairs."""
    i = torch.arange(CHUNK, device=A.device)
    T = torch.eye(CHUNK, device=A.device, dtype=A.dtype).expand_as(A)
    s = 1
    while s < CHUNK:
        pair = (i[:, None] // (2 * s) == i // (2 * s)) & (i[:, None] // s != i // s)
        T = T - T @ (A * pair) @ T
        s *= 2
    return T


def _plain_delta(st, gradients):
    """The chunked form in 32 bits; cumulated log decays in 64."""
    H, scale, cu = st["v"].shape[1], st["scale"], st["cu"]
    x = {n: _heads(st[n], H) for n in ("q", "k")}
    x.update({n: st[n].float() for n in ("v", "g", "beta", "d_o") if n in st})
    if cu is not None:
        x = {n: _unpack(st, t) for n, t in x.items()}
    B, _, N = x["g"].shape
    n = -(-N // CHUNK)
    q, k, v, beta = (_chunks(x[name], n) for name in ("q", "k", "v", "beta"))
    G = _chunks(x["g"].double(), n).cumsum(2)
    gam, to_end, whole = torch.exp(G).float()[..., None], torch.exp(G[:, :, -1:] - G).float()[..., None], torch.exp(G[:, :, -1]).float()
    ratio = torch.exp((G[..., :, None] - G[..., None, :]).clamp_(max=0)).float().tril()
    L = (ratio * (k @ k.transpose(-1, -2))).tril(-1)
    T = _inverse(beta[..., None] * L)
    P = ratio * (q @ k.transpose(-1, -2)) * scale
    kT = k.transpose(-1, -2)
    S = st["kv"].reshape(-1, *st["kv"].shape[2:]) if "kv" in st else q.new_zeros((B * H, q.shape[-1], v.shape[-1]))
    U, S0 = torch.empty_like(v), q.new_empty((B * H, n, *S.shape[1:]))
    # (the recurrence over chunks: each needs the state that the one before it leaves)
    for i in range(n):
        S0[:, i] = S
        U[:, i] = T[:, i] @ (beta[:, i, :, None] * (v[:, i] - gam[:, i] * (k[:, i] @ S)))
        S = whole[:, i, None, None] * S + kT[:, i] @ (to_end[:, i] * U[:, i])
    o = gam * (q @ S0) * scale + P @ U

    def back(t, name):           # chunks -> the layout and type of an input
        t = t.reshape(B, H, n * CHUNK, *t.shape[3:])[:, :, :N]
        t = _pack(st, t) if cu is not None else t
        like = st[name]
        if like.shape[1] != H:
            t = t.unflatten(1, (like.shape[1], -1)).sum(2)
        return t.to(st["q"].dtype)

    out = {"o": back(o, "v")}
    if not gradients:
        out["kv"] = S.view(B, H, *S.shape[1:])
        return out
    do = _chunks(x["d_o"], n)
    dS, dS1, dY = torch.zeros_like(S), torch.empty_like(S0), torch.empty_like(v)
    qT, PT, TT = (q * gam * scale).transpose(-1, -2), P.transpose(-1, -2), T.transpose(-1, -2)
    for i in reversed(range(n)):
        dS1[:, i] = dS
        dY[:, i] = TT[:, i] @ (PT[:, i] @ do[:, i] + to_end[:, i] * (k[:, i] @ dS))
        dS = whole[:, i, None, None] * dS + qT[:, i] @ do[:, i] - kT[:, i] @ ((gam * beta[..., None])[:, i] * dY[:, i])
    dv = beta[..., None] * dY
    dP = (do @ U.transpose(-1, -2)).tril() * scale * ratio
    dL = -(dY @ U.transpose(-1, -2)).tril(-1)
    E = dL * beta[..., None] * ratio
    q_state = gam * scale * (do @ S0.transpose(-1, -2))
    k_state = -gam * (dv @ S0.transpose(-1, -2))
    k_end = to_end * (U @ dS1.transpose(-1, -2))
    z = v - gam * (k @ S0) - L @ U
    MP, MA = dP * (q @ k.transpose(-1, -2)), dL * beta[..., None] * L
    end = (k * k_end).sum(-1)
    dG = (q * q_state).sum(-1) + (k * k_state).sum(-1) - end + (MP + MA).sum(-1) - (MP + MA).sum(-2)
    dG[:, :, -1] += end.sum(-1) + whole * (S0 * dS1).sum((-1, -2))
    out.update(dq=back(q_state + dP @ k, "q"), dk=back(k_state + k_end + dP.transpose(-1, -2) @ q + E @ k + E.transpose(-1, -2) @ k, "k"),
               dv=back(dv, "v"), dg=back(dG.flip(-1).cumsum(-1).flip(-1), "g"), dbeta=back((dY * z).sum(-1), "beta"))
    return out


def _plain_decode(st):
    q, k, v = _heads(st["q"], st["v"].shape[1]), _heads(st["k"], st["v"].shape[1]), st["v"].float()
    S, o = st["kv"], torch.empty_like(v)
    for t in range(v.shape[2]):
        S = S * torch.exp(st["g"][:, :, t, None, None])
        u = st["beta"][:, :, t, None] * (v[:, :, t] - (k[:, :, t, :, None] * S).sum(-2))
        S = S + k[:, :, t, :, None] * u[..., None, :]
        o[:, :, t] = st["scale"] * (q[:, :, t, :, None] * S).sum(-2)
    st["kv"].copy_(S)
    return {"o": o.to(st["v"].dtype), "kv": st["kv"]}


def _plain_norm(st):
    x, y, dt = st["x"].float(), st["y"].float(), st["x"].dtype
    wa, wb = (1.0 if st[n] is None else st[n] for n in ("w_after", "w_before"))
    gate = 1.0 if st["gate"] is None else st["gate"].float()
    gate = gate[:, None] if st["gate"] is not None and st["gate"].dim() == 2 else gate
    ry = torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) if st["case"]["after"] else 1.0
    n = y * ry
    x = x + st["scale"] * gate * n * wa
    out = {"x": x.to(dt), "h": (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * wb).to(dt)}
    if "d_h" not in st:
        return out
    rx = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    nx, dh = x * rx, st["d_h"].float()
    dn = dh * wb
    dx = st["d_x"].float() + rx * (dn - nx * (dn * nx).mean(-1, keepdim=True))
    dz = st["scale"] * gate * dx
    dn = dz * wa
    dy = ry * (dn - n * (dn * n).mean(-1, keepdim=True)) if st["case"]["after"] else dn
    out.update(dx=dx.to(dt), dy=dy.to(dt))
    if st["gate"] is not None:
        dgate = st["scale"] * dx * n * wa
        over = {"vector": (0, 1), "sequence": (1,), "element": ()}[st["case"]["gate"]]
        out["dgate"] = (dgate.sum(over) if over else dgate).view(st["gate"].shape).to(dt)
    if st["w_before"] is not None:
        out["dw_before"] = (dh * nx).sum((0, 1))
    if st["w_after"] is not None:
        out["dw_after"] = (dz * n).sum((0, 1))
    return out


# ---- the framework's calls -------------------------------------------------------------------------------------


def _own(st):
    import paper_2307_14995_amd as ltn
    kind = st["case"]["kind"]
    if kind.startswith("norm"):
        a = dict(gate=st["gate"], w_after=st["w_after"], w_before=st["w_before"], scale=st["scale"], eps=EPS, after=st["case"]["after"])
        x, h = ltn.ltn_block_norm_fwd(st["x"], st["y"], **a)
        out = {"x": x, "h": h}
        if kind == "norm_train":
            dx, dy, dgate, dwa, dwb = ltn.ltn_block_norm_bwd(st["x"], st["y"], st["d_x"], st["d_h"], **a)
            out.update(dx=dx, dy=dy)
            out.update({n: t for n, t in (("dgate", dgate), ("dw_after", dwa), ("dw_before", dwb)) if t is not None})
        return out
    args = [st[n] for n in ("q", "k", "v", "g", "beta")]
    if kind == "delta_decode":
        o = ltn.ltn_delta_decode_steps(*args[:3], st["kv"], *args[3:], scale=st["scale"])
        return {"o": o, "kv": st["kv"]}
    if kind == "delta_prefill":
        o, kv = ltn.ltn_delta_fwd(*args, kv_in=st.get("kv"), cu=st["cu"], scale=st["scale"], return_state=True)
        return {"o": o, "kv": kv}
    o = ltn.ltn_delta_fwd(*args, cu=st["cu"], scale=st["scale"])
    grads = ltn.ltn_delta_bwd(*args, st["d_o"], cu=st["cu"], scale=st["scale"])
    return {"o": o, **dict(zip(("dq", "dk", "dv", "dg", "dbeta"), grads))}


def run(st):
    if own:
        return _own(st)
    kind = st["case"]["kind"]
    if kind.startswith("norm"):
        return _plain_norm(st)
    return _plain_decode(st) if kind == "delta_decode" else _plain_delta(st, kind == "delta_train")


def work(case):
    """Bytes: each entry point's inputs read once and its outputs written once, with the fp32 states and gates.
    Operations: the recurrent form's products of 2 Dk Dv a token; forward three (read, correct, answer), gradients
    eight (the state again, and each of its two products' two derivatives)."""
    e = 4 if case["dtype"] == "fp32" else 2
    if case["kind"].startswith("norm"):
        unit = case["Bt"] * case["N"] * case["C"] * e
        element = case["gate"] == "element"
        if case["kind"] == "norm_infer":
            return {"bytes": (4 + element) * unit, "flops": 10 * unit // e}
        return {"bytes": (10 + 3 * element) * unit, "flops": 35 * unit // e}
    Bt, Hk, H, N, Dk, Dv = (case[n] for n in ("Bt", "Hk", "H", "N", "Dk", "Dv"))
    rows = Bt * N
    qk, vo, gates = 2 * rows * Hk * Dk * e, rows * H * Dv * e, rows * H
    state = (case["seqs"] or Bt) * H * Dk * Dv * 4
    product = 2 * Dk * Dv * rows * H
    if case["kind"] == "delta_train":
        return {"bytes": (qk + 2 * vo + 8 * gates) + (2 * qk + 3 * vo + 8 * gates + 2 * gates * e), "flops": 11 * product}
    states = 2 if case["kind"] == "delta_decode" or case["state_in"] else 1
    return {"bytes": qk + 2 * vo + 8 * gates + states * state, "flops": 3 * product}


# ---- 64 bits, from the definitions -----------------------------------------------------------------------------


def _exact_tokens(q, k, v, g, beta, scale, S, do=None):
    """The recurrence token by token on [B, H, N, D]: outputs, last state, and with `do` all gradients.  States are
    kept at every 64th token and formed again between."""
    N, every = q.shape[2], 64
    o, kept = torch.empty_like(v), []

    def step(S, t):
        A = torch.exp(g[:, :, t])[..., None, None] * S
        z = v[:, :, t] - (k[:, :, t].unsqueeze(-2) @ A).squeeze(-2)
        return A, z, torch.addcmul(A, k[:, :, t, :, None], (beta[:, :, t, None] * z)[..., None, :])

    for t in range(N):
        if t % every == 0:
            kept.append(S)
        S = step(S, t)[2]
        o[:, :, t] = scale * (q[:, :, t].unsqueeze(-2) @ S).squeeze(-2)
    if do is None:
        return o, S
    dS = torch.zeros_like(S)
    d = {"dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v), "dg": torch.empty_like(g), "dbeta": torch.empty_like(g)}
    for first in reversed(range(0, N, every)):
        S, seen = kept[first // every], []
        for t in range(first, min(N, first + every)):
            A, z, S = step(S, t)
            seen.append((A, z, S))
        for t in reversed(range(first, min(N, first + every))):
            A, z, S = seen[t - first]
            kt, b = k[:, :, t], beta[:, :, t, None]
            d["dq"][:, :, t] = scale * (S @ do[:, :, t, :, None]).squeeze(-1)
            dS = torch.addcmul(dS, q[:, :, t, :, None], scale * do[:, :, t, None, :])
            du = (kt.unsqueeze(-2) @ dS).squeeze(-2)
            d["dbeta"][:, :, t] = (du * z).sum(-1)
            dz = b * du
            d["dv"][:, :, t] = dz
            d["dk"][:, :, t] = (dS @ (b * z)[..., None] - A @ dz[..., None]).squeeze(-1)
            dS = torch.addcmul(dS, kt[..., None], dz[..., None, :], value=-1)
            d["dg"][:, :, t] = (dS * A).sum((-1, -2))
            dS = torch.exp(g[:, :, t])[..., None, None] * dS
    return o, d


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"].startswith("norm"):
        names = [n for n in ("x", "y", "gate", "w_after", "w_before") if st[n] is not None]
        d = {n: st[n].double().requires_grad_(case["kind"] == "norm_train") for n in names}

        def norm(t, w):
            t = t / (t.pow(2).mean(-1, keepdim=True) + EPS).sqrt()
            return t if w is None else t * w

        y = norm(d["y"], d.get("w_after")) if case["after"] else d["y"]
        if "gate" in d:
            y = y * (d["gate"][:, None] if d["gate"].dim() == 2 else d["gate"])
        x = d["x"] + st["scale"] * y
        h = norm(x, d.get("w_before"))
        out = {"x": x.detach(), "h": h.detach()}
        if case["kind"] == "norm_train":
            grads = torch.autograd.grad((x, h), [d[n] for n in names], (st["d_x"].double(), st["d_h"].double()))
            out.update({"dw" + n[1:] if n[0] == "w" else "d" + n: t for n, t in zip(names, grads)})
        return out
    H = case["H"]
    q, k = (st[n].double().repeat_interleave(H // case["Hk"], dim=1) for n in ("q", "k"))
    v, g, beta = (st[n].double() for n in ("v", "g", "beta"))
    do = st["d_o"].double() if "d_o" in st else None
    cu = [0, case["N"]] if st["cu"] is None else st["cu"].tolist()
    parts, states = [], []
    for i in range(len(cu) - 1):
        at = slice(cu[i], cu[i + 1])
        which = slice(None) if st["cu"] is None else slice(i, i + 1)
        S = st["kv"][which].double() if "kv" in st else v.new_zeros((case["Bt"], H, case["Dk"], case["Dv"]))
        if cu[i] == cu[i + 1]:
            states.append(S)
            continue
        o, rest = _exact_tokens(q[:, :, at], k[:, :, at], v[:, :, at], g[:, :, at], beta[:, :, at], st["scale"], S, None if do is None else do[:, :, at])
        parts.append({"o": o} if do is None else {"o": o, **rest})
        states.append(rest)
    out = {n: torch.cat([p[n] for p in parts], 2) for n in parts[0]}
    if do is None:
        out["kv"] = torch.cat(states)
    for n in ("dq", "dk"):
        if n in out:
            out[n] = out[n].unflatten(1, (case["Hk"], -1)).sum(2)
    return out

"""What the operators of a pre-norm block of gated delta attention are measured at: linear attention
with the gated delta rule (forward, backward, single token), layer norm with the residual sum before
it (forward, backward) and rotary positions with several axes.

A case names the operation ("fwd", "bwd", "step", "norm", "norm_bwd", "rotary"), the type and the
sizes.  H are the value heads, Hk the heads of queries and keys (H / Hk value heads share one).
"bthd" is the layout a projection leaves ([B, T, heads, channels] in memory), "bhtd" the one with the
heads outside.  With own false `run` computes the plain torch form, in 32 bits (triangular inverses in
64) and rounded once; with own true it calls the library.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
BASE = 10000.0
BLOCK = 64      # tokens of a block of the plain form


def _delta(name, op, dtype, B, H, Hk, T, dk, dv, layout="bthd", **more):
    return dict(name=name, op=op, dtype=dtype, B=B, H=H, Hk=Hk, T=T, dk=dk, dv=dv, layout=layout, **more)


def _norm(name, op, dtype, B, T, D, residual, affine):
    return dict(name=name, op=op, dtype=dtype, B=B, T=T, D=D, residual=residual, affine=affine)


def _rotary(name, dtype, B, H, Hk, T, D, sections, frames, layout="bthd", **more):
    return dict(name=name, op="rotary", dtype=dtype, B=B, H=H, Hk=Hk, T=T, D=D, sections=sections, frames=frames,
                layout=layout, **more)


def listed():
    return [
        # forward of a training batch
        _delta("fwd_bf16_b8h16_t4k", "fwd", "bf16", 8, 16, 16, 4096, 128, 128, lengths=False, state=True),
        # prefill of one long prompt
        _delta("fwd_bf16_h16_t32k", "fwd", "bf16", 1, 16, 16, 32768, 128, 128, lengths=False, state=True),
        # float32 prefill of a few prompts of different, odd lengths; two value heads to a key, sizes that no tile divides
        _delta("fwd_f32_ragged", "fwd", "f32", 3, 6, 3, 1003, 88, 74, lengths=True, state=False),
        # backward of the training batch
        _delta("bwd_bf16_b8h16_t4k", "bwd", "bf16", 8, 16, 16, 4096, 128, 128, lengths=False, state=True),
        # float32 backward of short odd sequences of different lengths, three value heads to a key
        _delta("bwd_f32_ragged", "bwd", "f32", 2, 6, 2, 509, 72, 58, "bhtd", lengths=True, state=True),
        # decode: one token for 16384 heads (1 GiB of states)
        _delta("step_f32_b512h32", "step", "f32", 512, 32, 32, 1, 128, 128),
        # decode of a few sequences with bf16 activations, where launches count
        _delta("step_bf16_b4h16", "step", "bf16", 4, 16, 8, 1, 128, 128),
        # the residual sum and the norm before a layer of the training batch
        _norm("norm_bf16_b8t4k_d2048", "norm", "bf16", 8, 4096, 2048, True, True),
        # a norm of few rows of an odd width, where launches count
        _norm("norm_f32_rows33_d1001", "norm", "f32", 1, 33, 1001, False, True),
        # the training batch's backward, with the gradient that comes along the residual stream
        _norm("norm_bwd_bf16_b8t4k_d2048", "norm_bwd", "bf16", 8, 4096, 2048, True, True),
        # queries and keys of video tokens: 8 frames of 32 x 32 patches, pairs in runs for time, height and width
        _rotary("rotary_bf16_video", "bf16", 4, 16, 16, 8192, 128, "16,24,24", 8, cyclic=False, interleaved=False, inverse=False),
        # one new token of 32 sequences after their images, pairs dealt to the axes in turn, half of the channels
        _rotary("rotary_f32_decode", "f32", 32, 16, 4, 1, 128, "12,10,10", 1, cyclic=True, interleaved=True, inverse=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _heads(rng, most):
    """Value heads and key heads that divide them."""
    H = rng.randint(1, max(1, min(32, most)))
    return H, rng.choice([H, H] + [n for n in range(1, H + 1) if H % n == 0])


def draw(rng):
    op = rng.choice(["fwd", "fwd", "fwd", "bwd", "bwd", "step", "norm", "norm_bwd", "rotary"])
    dtype = rng.choice(["f32", "bf16"])
    layout = rng.choice(["bthd", "bhtd"])
    if op in ("norm", "norm_bwd"):      # elements of the listed training batch at most, half of that in float32
        D = rng.choice([64 * _log_int(rng, 1, 128), _log_int(rng, 32, 8192)])
        rows = _log_int(rng, 1, (1 << (26 if dtype == "bf16" else 25)) // D)
        B = rng.choice([1, 1, 2, 4])
        case = _norm("", op, dtype, B, max(1, rows // B), D, rng.random() < 0.5, rng.random() < 0.8)
    elif op == "rotary":
        D = rng.choice([64, 128, 128, 256, rng.randint(8, 256)])
        H, Hk = _heads(rng, 32)
        most = (1 << 27) // (2 * D) // (2 if dtype == "f32" else 1)
        T = _log_int(rng, 1, min(16384, max(1, most // H)))
        axes = rng.randint(2, min(4, D // 2))
        cut = sorted(rng.sample(range(1, D // 2 + 1), axes))
        sections = [b - a for a, b in zip([0] + cut, cut)]
        case = _rotary("", dtype, _log_int(rng, 1, max(1, min(64, most // (T * H)))), H, Hk, T, D, ",".join(map(str, sections)),
                       rng.randint(1, 16), layout, cyclic=rng.random() < 0.5, interleaved=rng.random() < 0.5,
                       inverse=rng.random() < 0.5)
    else:
        dk, dv = (rng.choice([32, 64, 128, 128, 256, rng.randint(8, 256)]) for _ in range(2))
        H, Hk = _heads(rng, 32)
        if op == "step":                # at most the states of the listed decode
            B = _log_int(rng, 1, max(1, min(512, (1 << 28) // (H * dk * dv))))
            case = _delta("", op, dtype, B, H, Hk, 1, dk, dv, layout)
        else:                           # tokens x heads x channels of the listed training batch at most, half of that in float32
            most = (1 << 27) // (dk + dv) // (2 if dtype == "f32" else 1) // (2 if op == "bwd" else 1)
            T = rng.choice([_log_int(rng, 1, 32768), 64 * _log_int(rng, 1, 64)])
            H, Hk = _heads(rng, most // T)
            B = _log_int(rng, 1, max(1, min(64, most // (T * H))))
            case = _delta("", op, dtype, B, H, Hk, T, dk, dv, layout, lengths=rng.random() < 0.4, state=rng.random() < 0.6)
    del case["name"]
    return case


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, dt = case["op"], {"f32": torch.float32, "bf16": torch.bfloat16}[case["dtype"]]
    f32 = dict(device="cuda", dtype=torch.float32)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, **f32)

    s = dict(case=case)
    if op in ("norm", "norm_bwd"):
        B, T, D = case["B"], case["T"], case["D"]
        s.update(x=(normal(B, T, D) + 0.1).to(dt), weight=None, bias=None, residual=None, dtotal=None)
        if case["affine"]:
            s.update(weight=1.0 + 0.2 * normal(D), bias=0.1 * normal(D))
        if op == "norm_bwd":
            s["dy"] = normal(B, T, D).to(dt)
        if case["residual"]:            # the stream that the sum goes on as, or its gradient
            s["residual" if op == "norm" else "dtotal"] = (2.0 * normal(B, T, D)).to(dt)
        return s

    B, T, H, Hk = case["B"], case["T"], case["H"], case["Hk"]

    def heads(n, D, unit=False):        # [B, n, T, D] in the case's memory layout; unit: of length 1
        bhtd = case["layout"] == "bhtd"
        x = normal(*((B, n, T, D) if bhtd else (B, T, n, D)))
        if unit:
            x = x / x.square().sum(-1, keepdim=True).sqrt()
        return x.to(dt) if bhtd else x.to(dt).transpose(1, 2)

    if op == "rotary":
        sections = tuple(int(n) for n in case["sections"].split(","))
        pairs, D = sum(sections), case["D"]
        span = T + 64                   # the positions a program keeps tables for
        angle = torch.arange(span, device="cuda", dtype=torch.float64)[:, None] * \
            BASE ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)
        # time, height and width of each token (and its place in the frame, where there is a fourth axis), after some text
        frame = -(-T // case["frames"])
        wide = max(1, math.isqrt(frame))
        t = torch.arange(T, device="cuda")
        grid = torch.stack([t // frame, t % frame // wide, t % frame % wide, t % frame])[:len(sections)]
        text = torch.randint(0, 64, (B, 1), generator=gen, device="cuda")
        s.update(q=heads(H, D), k=heads(Hk, D), cos=angle.cos().float(), sin=angle.sin().float(), sections=sections,
                 positions=(grid[:, None] + text).to(torch.int32))
        return s

    dk, dv = case["dk"], case["dv"]
    # memories of 4 to 4096 tokens, the heads' horizons over the powers of two, and each token's own factor on the rate
    reach = 2.0 ** (2.0 + 10.0 * torch.arange(H, **f32) / max(H - 1, 1))
    g = -(normal(B, T, H) * 0.5).exp() / reach
    beta = torch.sigmoid(1.5 * normal(B, T, H))
    s.update(q=heads(Hk, dk, True), k=heads(Hk, dk, True), v=heads(H, dv), log_decay=g.transpose(1, 2), beta=beta.transpose(1, 2),
             scale=dk ** -0.5)
    if op == "step":
        s.update({x: s[x][:, :, 0] for x in ("q", "k", "v", "log_decay", "beta")})
        s["S"] = normal(B, H, dk, dv)
        return s
    s["S0"] = normal(B, H, dk, dv) if case["state"] else None
    s["lengths"] = None
    if case["lengths"]:
        s["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device="cuda").to(torch.int32)
    if op == "bwd":
        s["dO"] = heads(H, dv)
        s["dS_T"] = normal(B, H, dk, dv) if case["state"] else None
    return s


# ------------------------------------------------------------------ plain forms

def _t(x):
    return x.transpose(-1, -2).contiguous()


def _blocks(s, names):
    """The tokens in 32 bits and blocks [blocks, B, H, BLOCK, ...], queries and keys once for each value head; nothing is
    read, written or forgotten past a sequence's length."""
    case = s["case"]
    B, H, T = case["B"], case["H"], case["T"]
    there = torch.ones(B, T, device="cuda", dtype=torch.bool)
    if s["lengths"] is not None:
        there = torch.arange(T, device="cuda") < s["lengths"][:, None]
    n = -(-T // BLOCK)
    out = {}
    for name in names:
        x = s[name].float()
        x = x.unsqueeze(-1) if x.dim() == 3 else x
        x = torch.where(there[:, None, :, None], x, 0.0).repeat_interleave(H // x.shape[1], dim=1)
        x = torch.nn.functional.pad(x, (0, 0, 0, n * BLOCK - T))
        out[name] = x.reshape(B, H, n, BLOCK, -1).permute(2, 0, 1, 3, 4).contiguous()
    return out, there


def _factors(x):
    """What a block needs apart from the state: decays from its start and to its end, D_ij = decay from j to i (j <= i),
    the inverse of I + beta_i D_ij k_i . k_j (j < i)."""
    G = x["log_decay"].double().cumsum(-2)
    i = torch.arange(BLOCK, device="cuda")
    low = i[:, None] >= i
    D = torch.where(low, (G - _t(G)).clamp(max=0.0).exp(), 0.0)
    A = x["beta"].double() * D * torch.matmul(x["k"], _t(x["k"])).double()
    A = torch.where(i[:, None] > i, -A, 0.0)
    inv = torch.eye(BLOCK, device="cuda", dtype=torch.float64) + A      # the sum of A's powers, by doubling: A^64 = 0
    for _ in range(5):
        A = torch.matmul(A, A)
        inv = inv + torch.matmul(inv, A)
    e, b = G.exp().float(), (G[..., -1:, :] - G).exp().float()
    return e, b, D.float(), inv.float()


def _forward(s, x):
    """Outputs [blocks, ...], errors u_i / beta_i, states before each block and the last state."""
    e, b, D, inv = _factors(x)
    q, k, v, beta = x["q"], x["k"], x["v"], x["beta"]
    P = torch.matmul(q, _t(k)) * D
    kb, ke, qe = _t(k * b), k * e, q * e
    S = torch.zeros(*q.shape[1:3], q.shape[-1], v.shape[-1], device="cuda") if s["S0"] is None else s["S0"]
    o, u, states = [], [], []
    for c in range(q.shape[0]):
        states.append(S)
        u.append(torch.matmul(inv[c], beta[c] * (v[c] - torch.matmul(ke[c], S))))
        o.append(torch.matmul(qe[c], S) + torch.matmul(P[c], u[c]))
        S = e[c][..., -1:, :] * S + torch.matmul(kb[c], u[c])
    return torch.stack(o), torch.stack(u), torch.stack(states), S


def _tokens(x, T):
    """Blocks back to [B, H, T, ...]."""
    n, B, H, C, D = x.shape
    return x.permute(1, 2, 0, 3, 4).reshape(B, H, n * C, D)[:, :, :T]


def _plain_fwd(s):
    x, there = _blocks(s, ("q", "k", "v", "log_decay", "beta"))
    o, _, _, S = _forward(s, x)
    o = torch.where(there[:, None, :, None], s["scale"] * _tokens(o, s["case"]["T"]), 0.0)
    return {"o": o.to(s["v"].dtype), "S_T": S}


def _plain_bwd(s):
    case, c0 = s["case"], s["scale"]
    x, there = _blocks(s, ("q", "k", "v", "log_decay", "beta", "dO"))
    e, b, D, inv = _factors(x)
    q, k, v, beta, dO = x["q"], x["k"], x["v"], x["beta"], c0 * x["dO"]
    _, u, S, S_T = _forward(s, x)
    qk = torch.matmul(q, _t(k))
    back, local = _t(inv), torch.matmul(_t(qk * D), dO)
    kb, qe, ke = k * b, _t(q * e), _t(k * e * beta)
    G = torch.zeros_like(S_T) if s["dS_T"] is None else s["dS_T"]
    du, ends = [None] * q.shape[0], [None] * q.shape[0]
    for c in range(q.shape[0] - 1, -1, -1):         # G: dL/d(the state after block c); du: dL/d(beta (v - what the state holds))
        ends[c] = G
        du[c] = torch.matmul(back[c], local[c] + torch.matmul(kb[c], G))
        G = e[c][..., -1:, :] * G + torch.matmul(qe[c], dO[c]) - torch.matmul(ke[c], du[c])
    du, ends = torch.stack(du), torch.stack(ends)
    dv = beta * du
    W, M = torch.matmul(dO, _t(u)) * D, torch.matmul(dv, _t(u)) * D
    i = torch.arange(BLOCK, device="cuda")
    M = torch.where(i[:, None] > i, M, 0.0)
    dq = e * torch.matmul(dO, _t(S)) + torch.matmul(W, k)
    dk = b * torch.matmul(u, _t(ends)) + torch.matmul(_t(W), q) - e * torch.matmul(dv, _t(S)) - torch.matmul(M, k) - \
        torch.matmul(_t(M), k)
    # the error v - what the state holds, where beta may be 0: inv's columns by beta are its rows' by beta
    held = v - e * torch.matmul(k, S) - torch.where(i[:, None] > i, D * torch.matmul(k, _t(k)), 0.0) @ u
    dbeta = (du * held).sum(-1, keepdim=True)
    # a decay scales what the outputs from its token on read and what their writes cancel, and the block's last state
    dG = (q * dq).sum(-1, keepdim=True) - (v * dv).sum(-1, keepdim=True)
    after = torch.cat((S[1:], S_T[None]))
    dG[..., -1, 0] += (after * ends).sum((-1, -2))
    dg = dG.flip(-2).cumsum(-2).flip(-2)
    B, H, Hk, T, dt = case["B"], case["H"], case["Hk"], case["T"], s["q"].dtype
    out = {}
    for name, y in (("dq", dq), ("dk", dk), ("dv", dv), ("dlog_decay", dg), ("dbeta", dbeta)):
        y = torch.where(there[:, None, :, None], _tokens(y, T), 0.0)
        if name in ("dq", "dk"):
            y = y.reshape(B, Hk, H // Hk, T, -1).sum(2)
        out[name] = y.to(dt) if name in ("dq", "dk", "dv") else y[..., 0]
    return out | {"dS0": G}


def _plain_step(s):
    r = s["case"]["H"] // s["case"]["Hk"]
    q, k = (s[x].float().repeat_interleave(r, dim=1)[..., None, :] for x in "qk")
    S = s["S"] * s["log_decay"].exp()[..., None, None]
    u = s["beta"][..., None, None] * (s["v"].float()[..., None, :] - torch.matmul(k, S))
    S = S + k[..., 0, :, None] * u
    s["S"].copy_(S)
    return {"o": (s["scale"] * torch.matmul(q, S)[..., 0, :]).to(s["v"].dtype), "S": s["S"]}


def _normalised(x):
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    return x * r, r


def _plain_norm(s):
    x, total = s["x"].float(), None
    if s["residual"] is not None:       # the stream goes on rounded, and is what is normalised
        total = (x + s["residual"].float()).to(s["x"].dtype)
        x = total.float()
    y, _ = _normalised(x)
    if s["weight"] is not None:
        y = y * s["weight"] + s["bias"]
    return {"y": y.to(s["x"].dtype), "total": total}


def _plain_norm_bwd(s):
    xn, r = _normalised(s["x"].float())
    dy = s["dy"].float()
    g = dy if s["weight"] is None else dy * s["weight"]
    dx = r * (g - g.mean(-1, keepdim=True) - xn * (g * xn).mean(-1, keepdim=True))
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].float()
    none = s["weight"] is None
    return {"dx": dx.to(s["x"].dtype), "dweight": None if none else (dy * xn).sum((0, 1)), "dbias": None if none else dy.sum((0, 1))}


def _axis_of_pair(sections, cyclic):
    """The axis that each pair follows: runs of pairs, or dealt in turn to the axes that lack some."""
    if not cyclic:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    return [a for i in range(max(sections)) for a, n in enumerate(sections) if i < n]


def _plain_rotary(s):
    case = s["case"]
    R = 2 * sum(s["sections"])
    axis = torch.tensor(_axis_of_pair(s["sections"], case["cyclic"]), device="cuda")
    at = s["positions"].long()[axis].permute(1, 2, 0)                                   # [B, T, R / 2]
    pair = torch.arange(R // 2, device="cuda")
    c, n = s["cos"][at, pair][:, None], s["sin"][at, pair][:, None]
    n = -n if case["inverse"] else n

    def turn(x):
        y = x.float()
        a, b = (y[..., 0:R:2], y[..., 1:R:2]) if case["interleaved"] else (y[..., :R // 2], y[..., R // 2:R])
        u, w = a * c - b * n, a * n + b * c
        r = torch.stack((u, w), -1).flatten(-2) if case["interleaved"] else torch.cat((u, w), -1)
        return torch.cat((r, y[..., R:]), -1).to(x.dtype)
    return {"q": turn(s["q"]), "k": turn(s["k"])}


# ------------------------------------------------------------------ the library's calls

def _own(s):
    from paper_2607_11897_amd import sfda
    case = s["case"]
    op = case["op"]
    if op == "fwd":
        o, S_T = sfda.delta_attn_fwd(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["S0"], scale=s["scale"],
                                     lengths=s["lengths"])
        return {"o": o, "S_T": S_T}
    if op == "bwd":
        return sfda.delta_attn_bwd(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["S0"], s["dO"], s["dS_T"],
                                   scale=s["scale"], lengths=s["lengths"])
    if op == "step":
        o = sfda.delta_attn_step(s["q"], s["k"], s["v"], s["log_decay"], s["beta"], s["S"], scale=s["scale"])
        return {"o": o, "S": s["S"]}
    if op == "norm":
        y, total = sfda.layer_norm(s["x"], s["weight"], s["bias"], s["residual"], eps=EPS)
        return {"y": y, "total": total}
    if op == "norm_bwd":
        return sfda.layer_norm_bwd(s["dy"], s["x"], s["weight"], s["bias"], s["dtotal"], eps=EPS)
    q, k = sfda.rotary_axes(s["q"], s["k"], s["cos"], s["sin"], s["positions"], s["sections"], cyclic=case["cyclic"],
                            interleaved=case["interleaved"], inverse=case["inverse"])
    return {"q": q, "k": k}


_PLAIN = {"fwd": _plain_fwd, "bwd": _plain_bwd, "step": _plain_step, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd,
          "rotary": _plain_rotary}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ 64 bits

def _sweep(s):
    """The inputs in 64 bits, tokens first, with a key and a query for each value head, and the lengths."""
    case = s["case"]
    r = case["H"] // case["Hk"]
    x = {name: s[name].double().repeat_interleave(r, dim=1) if name in "qk" else s[name].double()
         for name in ("q", "k", "v", "log_decay", "beta", "dO") if name in s}
    x = {name: y.movedim(2, 0).contiguous() for name, y in x.items()}
    n = torch.full((case["B"],), case["T"], device="cuda") if s["lengths"] is None else s["lengths"].long()
    S = torch.zeros(case["B"], case["H"], case["dk"], case["dv"], device="cuda", dtype=torch.float64)
    return x, n, S if s["S0"] is None else s["S0"].double()


def _write(x, t, S):
    """The decayed state, what it lacks of the value, and the state after token t."""
    k = x["k"][t].unsqueeze(-1)
    S = S * x["log_decay"][t].exp()[..., None, None]
    lack = x["v"][t] - (S * k).sum(-2)
    return S, lack, S + k * (x["beta"][t].unsqueeze(-1) * lack).unsqueeze(-2)


def _exact_fwd(s):
    x, n, S = _sweep(s)
    o = torch.zeros_like(x["v"])
    for t in range(s["case"]["T"]):
        on = (t < n)[:, None, None, None]
        S = torch.where(on, _write(x, t, S)[2], S)
        o[t] = torch.where(on[..., 0], (S * x["q"][t].unsqueeze(-1)).sum(-2), 0.0)
    return {"o": (s["scale"] * o).movedim(0, 2), "S_T": S}


def _exact_bwd(s):
    case, c = s["case"], s["scale"]
    x, n, S = _sweep(s)
    T, step = case["T"], 64
    starts = []
    for t in range(T):                  # a state kept for every 64 tokens, the others made again from it
        if t % step == 0:
            starts.append(S)
        S = torch.where((t < n)[:, None, None, None], _write(x, t, S)[2], S)
    U = torch.zeros_like(S) if s["dS_T"] is None else s["dS_T"].double()
    out = {"d" + name: torch.zeros_like(x[name]) for name in ("q", "k", "v", "log_decay", "beta")}
    for first in range((T - 1) // step * step, -1, -step):
        states = [starts[first // step]]
        for t in range(first, min(first + step, T)):
            states.append(torch.where((t < n)[:, None, None, None], _write(x, t, states[-1])[2], states[-1]))
        for t in range(min(first + step, T) - 1, first - 1, -1):
            on = (t < n)[:, None, None, None]
            q, k, beta, dO = x["q"][t].unsqueeze(-1), x["k"][t].unsqueeze(-1), x["beta"][t].unsqueeze(-1), x["dO"][t]
            kept, lack, after = _write(x, t, states[t - first])
            V = U + c * q * dO.unsqueeze(-2)                    # dL/dS_t
            du = (V * k).sum(-2)
            dv = beta * du
            dkept = V - k * dv.unsqueeze(-2)
            put = dict(dq=c * (after * dO.unsqueeze(-2)).sum(-1), dv=dv, dbeta=(du * lack).sum(-1),
                       dk=(V * (beta * lack).unsqueeze(-2)).sum(-1) - (kept * dv.unsqueeze(-2)).sum(-1),
                       dlog_decay=(dkept * kept).sum((-1, -2)))
            for name, y in put.items():
                out[name][t] = torch.where(on.reshape(-1, *[1] * (y.dim() - 1)), y, 0.0)
            U = torch.where(on, dkept * x["log_decay"][t].exp()[..., None, None], U)
        del states
    out = {name: y.movedim(0, 2) for name, y in out.items()}
    for name in ("dq", "dk"):           # shared heads get the sum of their value heads' gradients
        out[name] = out[name].reshape(case["B"], case["Hk"], -1, T, case["dk"]).sum(2)
    return out | {"dS0": U}


def _exact_step(s):
    r = s["case"]["H"] // s["case"]["Hk"]
    x = {name: s[name].double().repeat_interleave(r, dim=1) if name in "qk" else s[name].double()
         for name in ("q", "k", "v", "log_decay", "beta")}
    _, _, S = _write({name: y[None] for name, y in x.items()}, 0, s["S"].double())
    return {"o": s["scale"] * (S * x["q"].unsqueeze(-1)).sum(-2), "S": S}


def _exact_norm(s, grad):
    # (the sum of two values of the type is taken in 32 bits and rounded: that is what the stream goes on as)
    x = s["x"] if s["residual"] is None else s["x"] + s["residual"]
    leaf = {name: y.double().requires_grad_(grad) for name, y in (("x", x), ("weight", s["weight"]), ("bias", s["bias"]))
            if y is not None}
    var, mean = torch.var_mean(leaf["x"], -1, correction=0, keepdim=True)
    y = (leaf["x"] - mean) / torch.sqrt(var + EPS)
    if "weight" in leaf:
        y = y * leaf["weight"] + leaf["bias"]
    if not grad:
        return {"y": y, "total": None if s["residual"] is None else x.double()}
    y.backward(s["dy"].double())
    dx = leaf["x"].grad if s["dtotal"] is None else leaf["x"].grad + s["dtotal"].double()
    return {"dx": dx, "dweight": leaf["weight"].grad if "weight" in leaf else None,
            "dbias": leaf["bias"].grad if "bias" in leaf else None}


def _exact_rotary(s):
    case = s["case"]
    left, order = list(s["sections"]), []
    while case["cyclic"] and any(left):
        for a in range(len(left)):
            if left[a]:
                left[a] -= 1
                order.append(a)
    order = order or sum(([a] * m for a, m in enumerate(left)), [])
    R = 2 * len(order)
    turn = torch.complex(s["cos"].double(), s["sin"].double())
    turn = torch.stack([turn[s["positions"][a].long(), i] for i, a in enumerate(order)], -1).unsqueeze(1)
    turn = turn.conj() if case["inverse"] else turn

    def one(x):
        x = x.double().clone()
        first, second = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x
    return {"q": one(s["q"]), "k": one(s["k"])}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("norm", "norm_bwd"):
        return _exact_norm(s, op == "norm_bwd")
    return {"fwd": _exact_fwd, "bwd": _exact_bwd, "step": _exact_step, "rotary": _exact_rotary}[op](s)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    B, T, op = case["B"], case["T"], case["op"]
    if op in ("norm", "norm_bwd"):
        n = B * T * case["D"]
        wide = (4 if case["residual"] else 2) if op == "norm" else (4 if case["residual"] else 3)
        return {"bytes": n * e * wide + (16 if op == "norm_bwd" else 8) * case["D"], "flops": n * (8 if op == "norm" else 16)}
    H, Hk = case["H"], case["Hk"]
    if op == "rotary":                  # q and k read and written, one value of each table for a token and pair; 6 flops a pair
        pairs = sum(int(n) for n in case["sections"].split(","))
        return {"bytes": 2 * B * (H + Hk) * T * case["D"] * e + B * T * 4 * len(case["sections"].split(",")) + 8 * T * pairs,
                "flops": 6 * B * (H + Hk) * T * pairs}
    dk, dv = case["dk"], case["dv"]
    state, rows = 4 * B * H * dk * dv, B * T
    # decay, what the state holds for the key, write and readout of the recurrence
    flops = 7 * rows * H * dk * dv
    if op == "step":
        return {"bytes": 2 * state + rows * (e * (2 * Hk * dk + 2 * H * dv) + 8 * H), "flops": flops}
    states = state * (2 if case["state"] else 1)
    if op == "fwd":
        return {"bytes": rows * (e * (2 * Hk * dk + 2 * H * dv) + 8 * H) + states, "flops": flops}
    # q, k, v, dO read, dq, dk, dv written, the scalars and theirs, S0, dS_T and dS0; both states' recurrences, five products more
    return {"bytes": rows * (e * (4 * Hk * dk + 3 * H * dv) + 16 * H) + states + (state if case["state"] else 0),
            "flops": 2 * flops + 10 * rows * H * dk * dv}

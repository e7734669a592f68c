"""GPU parity of the gated delta block's operators with their float64 oracle.

Error measure: max |x - ref| / max |ref| over a whole tensor.  Bars, from the arithmetic:
  * float32 sums (states of both types, float32 outputs and gradients, gradients of decays, strengths and weights): products to
    2^-22 and a few hundred to a few thousand terms of either sign in float32 (2^-24 each), errors growing like the square root of their
    number, and the block's inverse, whose error a system of a condition below 100 multiplies: 2e-5.
  * bfloat16 outputs and gradients: 2^-8 of the result's own rounding, and the operands of the products that give them
    rounded to bfloat16 (the state or its gradient, the scores, the writes): errors of up to 2^-8 of each of many terms of either sign,
    whose sum stays below their largest result's rounding, for each of the three or four products that make up a result: 2e-2.
  * layer norm in bfloat16: its own rounding, 4e-3 (2^-8); rotary positions as rotary's.
Every output lies between canary words, and rows that a call does not own keep theirs."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_util import ensure_built, rel_err
from oracle import delta as O
from test_gpu_layer import Buf, dev, dt, f32, stored, turned

pytestmark = pytest.mark.gpu
SUM = 2e-5
ATTN, NORM = {"f32": SUM, "bf16": 2e-2}, {"f32": SUM, "bf16": 4e-3}
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return ensure_built()


def say(*a):
    print("[case]", *a, flush=True)


# --------------------------------------------------------------------------- gated delta rule

def attn(seed, B, H, Hk, T, dk, dv, dtype, state=True, lengths=None, grads=False):
    """Keys of length 1, decays from a token's memory to none at all, with a reset and an undecayed run, strengths from 0 to 1."""
    rng = np.random.Generator(np.random.PCG64(seed))

    def unit(*shape):
        x = rng.standard_normal(shape)
        return stored_as(x / np.linalg.norm(x, axis=-1, keepdims=True), dtype)
    x = dict(q=unit(B, Hk, T, dk), k=unit(B, Hk, T, dk), v=stored(rng, (B, H, T, dv), dtype))
    g = -np.exp(rng.uniform(-7, 0.5, (B, H, 1)) + 0.5 * rng.standard_normal((B, H, T)))
    beta = rng.random((B, H, T))
    if T >= 8:
        g[:, 0, T // 2] = -np.inf
        g[:, -1, : T // 3] = 0.0
        beta[:, 0, 3], beta[:, -1, 5] = 0.0, 1.0
    x["log_decay"], x["beta"] = (y.astype(np.float32).astype(np.float64) for y in (g, beta))
    x["S0"] = stored(rng, (B, H, dk, dv), "f32") if state else None
    if grads:
        x["dO"] = stored(rng, (B, H, T, dv), dtype)
        x["dS_T"] = stored(rng, (B, H, dk, dv), "f32") if state else None
    x["lengths"] = None if lengths is None else np.asarray(lengths, np.int32)
    return x


def stored_as(x, dtype):
    import torch
    return torch.from_numpy(x).to(dt(dtype)).double().numpy()


def tokens(x, heads_inside):
    """[B,H,T] float32 on the device, as [B,T,H] in memory or not."""
    y = f32(x)
    return y.transpose(1, 2).contiguous().transpose(1, 2) if heads_inside else y


def run_fwd(x, dtype, layout, scale, poison=None, **more):
    import torch
    from paper_2607_11897_amd import sfda
    B, H, T, dv = x["v"].shape
    b = {n: Buf(x[n].shape, dt(dtype), layout, x[n]) for n in "qkv"}
    g, be = (tokens(x[n], layout == "bthd") for n in ("log_decay", "beta"))
    if poison is not None:
        for i, n in enumerate(np.clip(x["lengths"], 0, T)):
            for t in b.values():
                t.t[i, :, n:] = poison
            g[i, :, n:] = poison
            be[i, :, n:] = poison
    o = Buf(x["v"].shape, dt(dtype), layout)
    S = Buf((B, H, x["q"].shape[-1], dv), torch.float32)
    sfda.delta_attn_fwd(b["q"].t, b["k"].t, b["v"].t, g, be, f32(x["S0"]), scale=scale, lengths=dev(x["lengths"]), o=o.t, S_T=S.t, **more)
    torch.cuda.synchronize()
    o.check("o")
    S.check("S_T")
    return o.numpy(), S.numpy()


def names(x, *more):
    return {n: x[n] for n in ("q", "k", "v", "log_decay", "beta", "S0", "lengths") + more}


CASES = [  # B, H, Hk, T, dk, dv, dtype, layout, state
    (2, 2, 2, 1, 16, 8, "f32", "bhtd", True), (2, 4, 2, 1, 128, 128, "bf16", "bthd", True), (1, 1, 1, 0, 8, 8, "f32", "bhtd", True),
    (1, 3, 1, 0, 8, 8, "bf16", "bhtd", False), (2, 3, 3, 31, 1, 1, "f32", "bhtd", True), (2, 3, 1, 33, 3, 5, "f32", "padded", True),
    (1, 4, 4, 64, 64, 64, "f32", "bthd", False), (2, 3, 3, 97, 65, 66, "f32", "bhtd", True), (1, 2, 1, 130, 256, 256, "f32", "bthd", True),
    (1, 6, 3, 65, 129, 130, "f32", "padded", True), (1, 2, 2, 200, 128, 128, "f32", "bthd", True),
    (3, 3, 1, 63, 7, 9, "bf16", "padded", True), (2, 2, 2, 64, 32, 16, "bf16", "bthd", True), (2, 3, 3, 1, 1, 1, "bf16", "bhtd", True),
    (1, 4, 2, 65, 64, 64, "bf16", "bhtd", False), (2, 3, 3, 200, 128, 128, "bf16", "bthd", True), (1, 3, 1, 129, 88, 74, "bf16", "bthd", True),
    (1, 2, 2, 190, 256, 250, "bf16", "padded", True), (1, 1, 1, 700, 96, 160, "bf16", "bhtd", True),
]


@pytest.mark.parametrize("B,H,Hk,T,dk,dv,dtype,layout,state", CASES)
def test_fwd(B, H, Hk, T, dk, dv, dtype, layout, state):
    say("fwd", B, H, Hk, T, dk, dv, dtype, layout)
    x = attn(T + dk, B, H, Hk, T, dk, dv, dtype, state)
    o, S = run_fwd(x, dtype, layout, dk ** -0.5)
    ro, rS = O.delta_attn(**names(x), scale=dk ** -0.5)
    assert rel_err(o, ro) <= ATTN[dtype] and rel_err(S, rS) <= SUM


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("poison", [float("nan"), INF])
def test_fwd_lengths(dtype, poison):
    say("lengths", dtype, poison)
    B, H, Hk, T, dk, dv = 6, 4, 2, 150, 40, 24
    x = attn(9, B, H, Hk, T, dk, dv, dtype, True, [150, 0, -3, 999, 64, 33])
    o, S = run_fwd(x, dtype, "bthd", 0.5, poison)
    ro, rS = O.delta_attn(**names(x), scale=0.5)
    assert rel_err(o, ro) <= ATTN[dtype] and rel_err(S, rS) <= SUM
    assert np.array_equal(S[1], x["S0"][1]) and np.array_equal(S[2], x["S0"][2])
    for i, n in enumerate((150, 0, 0, 150, 64, 33)):
        assert not o[i, :, n:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv,Hk", [(128, 128, 3), (1, 1, 1), (37, 70, 3), (64, 256, 1), (256, 3, 3)])
def test_step(dtype, dk, dv, Hk):
    import torch
    from paper_2607_11897_amd import sfda
    say("step", dtype, dk, dv)
    B, H, T = 2, 3, 4
    x = attn(dk, B, H, Hk, T, dk, dv, dtype)
    x["log_decay"][0, 0, 1], x["beta"][0, 1, 2] = -np.inf, 0.0
    b = {n: Buf(x[n].shape, dt(dtype), "bthd", x[n]) for n in "qkv"}
    g, be = (tokens(x[n], True) for n in ("log_decay", "beta"))
    S = Buf((B, H, dk, dv), torch.float32, values=x["S0"])
    out = []
    for t in range(T):
        o = Buf((B, H, 1, dv), dt(dtype), "bthd")
        sfda.delta_attn_step(b["q"].t[:, :, t], b["k"].t[:, :, t], b["v"].t[:, :, t], g[:, :, t], be[:, :, t], S.t, scale=0.5, o=o.t[:, :, 0])
        o.check("o")
        out.append(o.numpy())
    torch.cuda.synchronize()
    S.check("S")
    ro, rS = O.delta_attn(**names(x), scale=0.5)
    o = np.concatenate(out, 2)
    assert rel_err(o, ro) <= (SUM if dtype == "f32" else 4e-3) and rel_err(S.numpy(), rS) <= SUM


# --------------------------------------------------------------------------- layer norm

ROWS = [  # B, T, D, dtype, layout
    (1, 1, 1, "f32", "bhtd"), (2, 5, 7, "f32", "padded"), (1, 33, 1001, "f32", "bhtd"), (3, 7, 64, "bf16", "bhtd"), (1, 9, 2048, "bf16", "bhtd"),
    (2, 3, 4100, "bf16", "padded"), (1, 5, 8192, "bf16", "bhtd"), (1, 3, 8200, "f32", "bhtd"), (1, 2, 16384, "f32", "padded"),
    (1, 4, 16384, "bf16", "bhtd"), (1, 0, 8, "f32", "bhtd"), (1, 700, 130, "bf16", "padded"), (2, 600, 257, "f32", "bhtd"),
    (1, 1300, 520, "bf16", "bhtd"),
]


@pytest.mark.parametrize("B,T,D,dtype,layout", ROWS)
@pytest.mark.parametrize("residual,affine", [(False, True), (True, True), (True, False)])
def test_layer_norm(B, T, D, dtype, layout, residual, affine):
    import torch
    from paper_2607_11897_amd import sfda
    say("layer_norm", B, T, D, dtype, layout, residual, affine)
    rng = np.random.Generator(np.random.PCG64(D + T))
    x, r = stored(rng, (B, T, D), dtype) + 0.0, stored(rng, (B, T, D), dtype, 3.0)
    w, b = (1 + 0.3 * stored(rng, (D,), "f32"), stored(rng, (D,), "f32")) if affine else (None, None)
    w, b = (None if y is None else y.astype(np.float32).astype(np.float64) for y in (w, b))
    total = stored_as(x + r, dtype) if residual else x
    bx, br, y, t = Buf((B, T, D), dt(dtype), layout, x), Buf((B, T, D), dt(dtype), layout, r), Buf((B, T, D), dt(dtype), layout), Buf((B, T, D), dt(dtype), layout)
    got = sfda.layer_norm(bx.t, f32(w), f32(b), br.t if residual else None, eps=1e-3, y=y.t, total=t.t if residual else None)
    torch.cuda.synchronize()
    y.check("y")
    t.check("total")
    assert (got[1] is None) == (not residual)
    ref = O.layer_norm(total, w, b, 1e-3)
    assert rel_err(y.numpy(), ref) <= NORM[dtype]
    if residual:
        assert np.array_equal(t.numpy(), total)
    # backward, in place of dy and of dtotal too
    dy, d2 = stored(rng, (B, T, D), dtype), stored(rng, (B, T, D), dtype)
    ref = O.layer_norm_backward(dy, total, w, b, d2 if residual else None, 1e-3)
    for place in ("new", "dy", "dtotal")[: 3 if residual else 2]:
        bt, bdy, bd2 = (Buf((B, T, D), dt(dtype), layout, z) for z in (total, dy, d2))
        dx = {"new": Buf((B, T, D), dt(dtype), layout), "dy": bdy, "dtotal": bd2}[place]
        g = sfda.layer_norm_bwd(bdy.t, bt.t, f32(w), f32(b), bd2.t if residual else None, eps=1e-3, dx=dx.t)
        torch.cuda.synchronize()
        dx.check("dx")
        assert rel_err(dx.numpy(), ref["dx"]) <= NORM[dtype], place
        for n in ("dweight", "dbias"):
            assert (g[n] is None) == (not affine)
            if affine:
                assert rel_err(g[n].double().cpu().numpy(), ref[n]) <= SUM, n


def test_layer_norm_in_place():
    import torch
    from paper_2607_11897_amd import sfda
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, r = (torch.randn(3, 50, 200, generator=gen, device="cuda") for _ in range(2))
    y, t = sfda.layer_norm(x, residual=r)
    x1, r1 = x.clone(), r.clone()
    y1, t1 = sfda.layer_norm(x1, residual=r1, total=r1)
    assert t1 is r1 and torch.equal(t1, t) and torch.equal(y1, y)
    x2 = x.clone()
    y2, t2 = sfda.layer_norm(x2, residual=r, total=x2)
    assert torch.equal(x2, t) and torch.equal(y2, y)
    y3, _ = sfda.layer_norm(x)
    assert torch.equal(sfda.layer_norm(x1, y=x1)[0], y3)


# --------------------------------------------------------------------------- rotary positions with several axes

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved,inverse,cyclic", [(False, False, False), (True, False, True), (False, True, True), (True, True, False)])
@pytest.mark.parametrize("B,Hq,Hk,T,D,sections,layout", [
    (2, 3, 1, 5, 16, (3, 2, 3), "bhtd"), (1, 4, 4, 17, 128, (16, 24, 24), "bthd"), (2, 2, 2, 9, 90, (10, 0, 13, 12), "padded"), (1, 2, 1, 3, 6, (1,), "bhtd"),
    (3, 5, 2, 1, 72, (12, 20), "bthd"), (1, 1, 1, 2, 300, (40, 41, 42, 27), "bhtd"), (2, 1, 0, 4, 8, (1, 1, 1, 1), "bhtd"),
])
def test_rotary_axes(dtype, interleaved, inverse, cyclic, B, Hq, Hk, T, D, sections, layout):
    import torch
    from paper_2607_11897_amd import sfda
    say("rotary_axes", dtype, interleaved, inverse, cyclic, B, Hq, Hk, T, D, sections, layout)
    rng = np.random.Generator(np.random.PCG64(D + T))
    half, P, A = sum(sections), 50, len(sections)
    cos, sin = sfda.rotary_tables(P, 2 * half)
    q, k = stored(rng, (B, Hq, T, D), dtype), stored(rng, (B, max(Hk, 1), T, D), dtype)
    for bits, shape in ((np.int32, (A, B, T)), (np.int64, (A, T))):
        pos = rng.integers(0, P, shape).astype(bits)
        bq, bk = Buf(q.shape, dt(dtype), layout, q), Buf(k.shape, dt(dtype), layout, k)
        oq, ok = Buf(q.shape, dt(dtype), layout), Buf(k.shape, dt(dtype), layout)
        args = dict(cyclic=cyclic, interleaved=interleaved, inverse=inverse)
        sfda.rotary_axes(bq.t, bk.t if Hk else None, cos, sin, dev(pos), sections, q_out=oq.t, k_out=ok.t if Hk else None, **args)
        torch.cuda.synchronize()
        c, s = (t.double().cpu().numpy() for t in (cos, sin))
        for x, o in ((q, oq), (k, ok))[: 2 if Hk else 1]:
            o.check("out")
            assert turned(o.numpy(), O.rotary_axes(x, c, s, pos, sections, **args), dtype)
        sfda.rotary_axes(bq.t, None, cos, sin, dev(pos), sections, q_out=bq.t, **args)         # in place
        assert torch.equal(bq.t, oq.t)


def test_rotary_axes_positions_outside():
    import torch
    from paper_2607_11897_amd import sfda
    cos, sin = sfda.rotary_tables(4, 8)
    q = torch.ones(1, 1, 2, 10, device="cuda")
    pos = torch.tensor([[0, 4], [-1, 3]], dtype=torch.int32, device="cuda")
    o, _ = sfda.rotary_axes(q, None, cos, sin, pos, (1, 3))
    bad = torch.isnan(o[0, 0])
    assert bad[0].tolist() == [False, True, True, True] * 2 + [False] * 2 and bad[1].tolist() == [True, False, False, False] * 2 + [False] * 2


# --------------------------------------------------------------------------- gated delta rule, backward

def run_bwd(x, dtype, layout, scale, poison=None, **more):
    import torch
    from paper_2607_11897_amd import sfda
    B, H, T, dv = x["v"].shape
    b = {n: Buf(x[n].shape, dt(dtype), layout, x[n]) for n in ("q", "k", "v", "dO")}
    g, be = (tokens(x[n], layout == "bthd") for n in ("log_decay", "beta"))
    if poison is not None:
        for i, n in enumerate(np.clip(x["lengths"], 0, T)):
            for t in b.values():
                t.t[i, :, n:] = poison
            g[i, :, n:] = poison
            be[i, :, n:] = poison
    out = {n: Buf(x[n[1:]].shape, dt(dtype), layout) for n in ("dq", "dk", "dv")}
    got = sfda.delta_attn_bwd(b["q"].t, b["k"].t, b["v"].t, g, be, f32(x["S0"]), b["dO"].t, f32(x["dS_T"]), scale=scale,
                              lengths=dev(x["lengths"]), **{n: y.t for n, y in out.items()}, **more)
    torch.cuda.synchronize()
    for n, y in out.items():
        y.check(n)
    return {n: y.double().cpu().numpy() for n, y in got.items()}


def check_bwd(got, ref, dtype):
    for n, y in ref.items():
        bar = ATTN[dtype] if n in ("dq", "dk", "dv") else SUM
        assert rel_err(got[n], y) <= bar, (n, rel_err(got[n], y))


@pytest.mark.parametrize("B,H,Hk,T,dk,dv,dtype,layout,state", CASES)
def test_bwd(B, H, Hk, T, dk, dv, dtype, layout, state):
    say("bwd", B, H, Hk, T, dk, dv, dtype, layout)
    x = attn(T + dk, B, H, Hk, T, dk, dv, dtype, state, grads=True)
    got = run_bwd(x, dtype, layout, dk ** -0.5)
    check_bwd(got, O.delta_attn_backward(**names(x, "dO", "dS_T"), scale=dk ** -0.5), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("poison", [float("nan"), INF])
def test_bwd_lengths(dtype, poison):
    say("bwd lengths", dtype, poison)
    x = attn(9, 6, 4, 2, 150, 40, 24, dtype, True, [150, 0, -3, 999, 64, 33], grads=True)
    got = run_bwd(x, dtype, "bthd", 0.5, poison)
    check_bwd(got, O.delta_attn_backward(**names(x, "dO", "dS_T"), scale=0.5), dtype)
    assert np.array_equal(got["dS0"][1], x["dS_T"][1])
    for i, n in enumerate((150, 0, 0, 150, 64, 33)):
        for name in ("dq", "dk", "dv", "dlog_decay", "dbeta"):
            assert not got[name][i, :, n:].any(), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_bwd_in_passes(dtype):
    """Groups of heads, as many as the workspace holds: the same results, bit by bit."""
    import torch
    from paper_2607_11897_amd import sfda
    say("passes", dtype)
    B, H, Hk, T, dk, dv = 2, 6, 3, 100, 33, 70
    x = attn(4, B, H, Hk, T, dk, dv, dtype, grads=True)
    ref = run_bwd(x, dtype, "bhtd", 0.3)
    least = sfda.delta_attn_bwd_workspace_bytes(1, H // Hk, 1, T, dk, dv, dtype)
    for n in (1, 2, 5):
        got = run_bwd(x, dtype, "bhtd", 0.3, workspace=torch.full((n * least,), 255, dtype=torch.uint8, device="cuda"))
        for name in ref:
            assert np.array_equal(got[name], ref[name]), (n, name)
    with pytest.raises(sfda.SfdaError, match="SHAPE"):
        run_bwd(x, dtype, "bhtd", 0.3, workspace=torch.empty(least - 16, dtype=torch.uint8, device="cuda"))


def test_bwd_against_differences():
    """float32 gradients against central differences of the library's own forward, on a loss that one token, decay or strength moves."""
    import torch
    from paper_2607_11897_amd import sfda
    say("differences")
    x = attn(12, 1, 2, 1, 40, 8, 6, "f32", grads=True)
    t = {n: f32(x[n]) for n in ("q", "k", "v", "log_decay", "beta", "S0")}
    t["log_decay"][0, 0, 20] = -0.4
    dO, dS = f32(x["dO"]), f32(x["dS_T"])

    def loss(**kw):
        o, S = sfda.delta_attn_fwd(**kw, scale=0.6)
        return (o.double() * dO).sum() + (S.double() * dS).sum()
    got = sfda.delta_attn_bwd(**t, dO=dO, dS_T=dS, scale=0.6)
    rng = np.random.default_rng(0)
    for name, y in t.items():
        d = torch.from_numpy(rng.standard_normal(tuple(y.shape))).to("cuda")
        d = (d / d.norm()).float()
        h = 1e-2
        up, down = loss(**{**t, name: y + h * d}), loss(**{**t, name: y - h * d})
        want, have = float(up - down) / (2 * h), float((got["d" + name].double() * d).sum())
        # off by h^2 / 6 of the third derivative along a direction of length 1, some tens of the loss's scale, and by the
        # forward's rounding, 2^-22 of a loss of some tens over h
        scale = float(got["d" + name].double().norm())
        assert abs(want - have) <= 2e-2 * scale, (name, want, have)


@pytest.mark.parametrize("B,H,Hk,T,dk,dv,dtype,lengths", [
    (1, 1, 1, 3000, 64, 64, "f32", None), (1, 2, 1, 4000, 96, 70, "f32", None), (1, 2, 2, 2113, 128, 128, "bf16", None),
    (2, 2, 1, 3001, 37, 50, "bf16", [3001, 1203]), (3, 1, 1, 3999, 80, 12, "f32", [0, 3999, 64]), (1, 1, 1, 2500, 200, 130, "bf16", None),
    (2, 1, 1, 2048, 100, 66, "bf16", [5, 2047]),
])
def test_fwd_segments(B, H, Hk, T, dk, dv, dtype, lengths):
    """Sequences long enough, and heads few enough, that they are cut into segments."""
    from paper_2607_11897_amd import sfda
    say("segments", B, H, Hk, T, dk, dv, dtype, lengths)
    whole = sfda.delta_attn_fwd_workspace_bytes(B, 512, T, dk, dv, dtype) // 512
    assert sfda.delta_attn_fwd_workspace_bytes(B, H, T, dk, dv, dtype) > H * whole
    x = attn(T, B, H, Hk, T, dk, dv, dtype, True, lengths)
    o, S = run_fwd(x, dtype, "bthd", dk ** -0.5, float("nan") if lengths else None)
    ro, rS = O.delta_attn(**names(x), scale=dk ** -0.5)
    assert rel_err(o, ro) <= ATTN[dtype] and rel_err(S, rS) <= SUM
    for i, n in enumerate(lengths or ()):
        assert not o[i, :, n:].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_fwd_segments_in_place(dtype):
    """S_T in S0's memory: the last segments, empty ones among them, write what the first ones start from."""
    from paper_2607_11897_amd import sfda
    B, H, T, dk, dv = 2, 12, 4500, 64, 64
    say("segments in place", dtype)
    whole = sfda.delta_attn_fwd_workspace_bytes(B, 512, T, dk, dv, dtype) // 512
    assert sfda.delta_attn_fwd_workspace_bytes(B, H, T, dk, dv, dtype) > H * whole
    x = attn(5, B, H, H, T, dk, dv, dtype, True, [3, T - 1])
    a = [dev(x[n]).to(dt(dtype)) for n in "qkv"] + [f32(x[n]) for n in ("log_decay", "beta")]
    S = f32(x["S0"])
    o, want = sfda.delta_attn_fwd(*a, S, lengths=dev(x["lengths"]))
    o2, have = sfda.delta_attn_fwd(*a, S, lengths=dev(x["lengths"]), S_T=S)
    assert have.data_ptr() == S.data_ptr() and want.equal(S) and o.equal(o2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,Hk,T,dk,dv", [(9, 16, 16, 200, 128, 128), (4, 16, 4, 131, 64, 72), (3, 8, 8, 97, 200, 256)])
def test_many_heads(B, H, Hk, T, dk, dv, dtype):
    """More workgroups than compute units, forward and backward, against the recurrence."""
    say("many heads", B, H, Hk, T, dk, dv, dtype)
    x = attn(71 + T, B, H, Hk, T, dk, dv, dtype, grads=True)
    scale = dk ** -0.5
    o, S = run_fwd(x, dtype, "bthd", scale)
    ro, rS = O.delta_attn(**names(x), scale=scale)
    assert rel_err(o, ro) <= ATTN[dtype] and rel_err(S, rS) <= SUM
    check_bwd(run_bwd(x, dtype, "bthd", scale), O.delta_attn_backward(**names(x, "dO", "dS_T"), scale=scale), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_broadcast_inputs(dtype):
    """Inputs whose batches, heads or tokens lie in one place: the gradients are those of every element by itself."""
    import torch
    from paper_2607_11897_amd import sfda
    say("broadcast", dtype)
    B, H, Hk, T, dk, dv = 3, 4, 2, 70, 48, 40
    gen = torch.Generator(device="cuda").manual_seed(6)
    unit = lambda *s: torch.nn.functional.normalize(torch.randn(*s, generator=gen, device="cuda"), dim=-1).to(dt(dtype))  # noqa: E731
    q, k = unit(1, Hk, T, dk).expand(B, -1, -1, -1), unit(B, 1, T, dk).expand(-1, Hk, -1, -1)
    v, dO = (torch.randn(B, H, 1, dv, generator=gen, device="cuda").to(dt(dtype)).expand(-1, -1, T, -1) for _ in range(2))
    g, beta = torch.full((1, 1, 1), -0.05, device="cuda").expand(B, H, T), torch.rand(1, H, 1, generator=gen, device="cuda").expand(B, -1, T)
    wide = [x.contiguous() for x in (q, k, v, g, beta)]
    for a, b in zip(sfda.delta_attn_fwd(q, k, v, g, beta, scale=0.3), sfda.delta_attn_fwd(*wide, scale=0.3)):
        assert torch.equal(a, b)
    a, b = sfda.delta_attn_bwd(q, k, v, g, beta, None, dO, scale=0.3), sfda.delta_attn_bwd(*wide, None, dO.contiguous(), scale=0.3)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_non_finite_values_stay_in_their_heads_and_after_their_blocks():
    import torch
    from paper_2607_11897_amd import sfda
    say("non finite")
    B, H, T, d = 2, 3, 256, 32
    gen = torch.Generator(device="cuda").manual_seed(7)
    for dtype, block in ((torch.float32, 32), (torch.bfloat16, 64)):
        q, k = (torch.nn.functional.normalize(torch.randn(B, H, T, d, generator=gen, device="cuda"), dim=-1).to(dtype) for _ in range(2))
        v = torch.randn(B, H, T, d, generator=gen, device="cuda").to(dtype)
        g, beta = -torch.rand(B, H, T, generator=gen, device="cuda"), torch.rand(B, H, T, generator=gen, device="cuda")
        want, _ = sfda.delta_attn_fwd(q, k, v, g, beta)
        for name in ("q", "k", "v", "g", "beta"):
            for bad in (float("nan"), INF):
                x = dict(q=q, k=k, v=v, g=g, beta=beta)
                x[name] = x[name].clone()
                x[name][1, 2, 130] = bad
                o, S = sfda.delta_attn_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"])
                assert torch.equal(o[0], want[0]) and torch.equal(o[1, :2], want[1, :2])
                assert torch.equal(o[1, 2, : 130 // block * block], want[1, 2, : 130 // block * block])
                assert not torch.isfinite(o[1, 2, 130]).all(), (name, bad)


def calls(gen, dtype):
    """Every operator once, on tensors that a graph may hold: (inputs, call)."""
    import torch
    from paper_2607_11897_amd import sfda
    B, H, Hk, T, dk, dv = 2, 4, 2, 150, 64, 72

    def rand(*s, to=dt(dtype)):
        return torch.randn(*s, generator=gen, device="cuda").to(to)
    f = torch.float32
    cos, sin = sfda.rotary_tables(200, 32)
    x = dict(q=rand(B, Hk, T, dk) / 8, k=rand(B, Hk, T, dk) / 8, v=rand(B, H, T, dv), dO=rand(B, H, T, dv), g=-rand(B, H, T, to=f).abs(),
             beta=torch.sigmoid(rand(B, H, T, to=f)), S0=rand(B, H, dk, dv, to=f), dS=rand(B, H, dk, dv, to=f), x=rand(B, T, 300), r=rand(B, T, 300),
             w=rand(300, to=f), b=rand(300, to=f), at=torch.randint(0, 200, (3, B, T), generator=gen, device="cuda", dtype=torch.int32),
             long=rand(1, 1, 4000, dk) / 8, lv=rand(1, 1, 4000, dv), lg=-rand(1, 1, 4000, to=f).abs(), lb=torch.sigmoid(rand(1, 1, 4000, to=f)))

    def call(stream=None):
        s = dict(stream=stream)
        out = list(sfda.delta_attn_fwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], scale=0.5, **s))
        out += list(sfda.delta_attn_fwd(x["long"], x["long"], x["lv"], x["lg"], x["lb"], **s))          # in segments
        out += list(sfda.delta_attn_bwd(x["q"], x["k"], x["v"], x["g"], x["beta"], x["S0"], x["dO"], x["dS"], scale=0.5, **s).values())
        y, t = sfda.layer_norm(x["x"], x["w"], x["b"], x["r"], **s)
        out += [y, t, *sfda.layer_norm_bwd(x["x"], t, x["w"], x["b"], x["r"], **s).values()]
        out += list(sfda.rotary_axes(x["q"], x["k"], cos, sin, x["at"], (6, 5, 5), cyclic=True, **s))
        return out
    return x, call


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_replayed_graphs(dtype):
    """Captured, and replayed several times on new inputs with eager calls and synchronisations between: the eager results, bit by bit."""
    import torch
    say("graph", dtype)
    gen = torch.Generator(device="cuda").manual_seed(8)
    x, call = calls(gen, dtype)
    call()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                      # two graphs whose workspaces come from one pool of their own each
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        graphs.append((graph, out))
    for turn in range(4):
        for n in ("q", "v", "dO", "x", "S0", "lv"):
            x[n].copy_(x[n].flip(-1) * (1.0 + 0.125 * turn))
        for graph, _ in graphs:
            graph.replay()
        want = call()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert len(out) == len(want)
            for a, b in zip(out, want):
                assert torch.equal(a, b), turn


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_other_streams(dtype):
    """Two streams at once, each with tensors of its own, against the current one."""
    import torch
    say("streams", dtype)
    gen = torch.Generator(device="cuda").manual_seed(9)
    jobs = [calls(gen, dtype)[1] for _ in range(2)]
    want = [job() for job in jobs]
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream() for _ in jobs]
    for _ in range(3):
        got = [job(stream=s) for job, s in zip(jobs, sides)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            for p, q in zip(a, b):
                assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lds_poison(dtype):
    """On the LDS-poison build, whose scans and gradients fill their whole LDS with NaN words at entry: the normal build's results, bit
    by bit.  Channels that fill their padded width and that do not, blocks that are whole and that are not, segments."""
    import os
    import torch
    from paper_2607_11897_amd import build, sfda
    if not os.path.exists(build.POISON_LIB):
        build.build(verbose=False, poison=True, out=build.POISON_LIB)
    for B, H, Hk, T, dk, dv, lengths in ((2, 2, 1, 75, 128, 128, None), (3, 1, 1, 130, 40, 24, [130, 0, 7]), (1, 2, 2, 97, 37, 101, None),
                                         (2, 1, 1, 150, 256, 192, [1, 149]), (1, 2, 1, 33, 3, 2, None), (1, 1, 1, 4000, 64, 64, None)):
        say("poison", dtype, B, H, Hk, T, dk, dv, lengths)
        x = attn(T, B, H, Hk, T, dk, dv, dtype, True, lengths, grads=True)

        def outputs():
            return [*run_fwd(x, dtype, "bthd", 0.5), *run_bwd(x, dtype, "bthd", 0.5).values()]
        want = outputs()
        with sfda.library(build.POISON_LIB):
            got = outputs()
            torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert np.isfinite(a).all() and np.array_equal(a, b)


def test_offsets_past_32_bits():
    """Rows so far apart that the last ones lie past 2^31 elements (4 GiB): the results of packed rows, bit by bit."""
    import torch
    from paper_2607_11897_amd import sfda
    B, H, T, d, apart = 1, 2, 135, 64, (16 << 20) - 1024       # (64 rows within 2^31 bytes)
    say("offsets", apart)
    mem = torch.empty((T - 1) * apart + 8192, dtype=torch.bfloat16, device="cuda")
    assert (T - 1) * apart > 1 << 31

    def spread(slot, x=None, columns=H * d, rows=T):
        t = mem.as_strided((B, rows, columns), (0, apart, 1), slot * 512)
        if x is not None:
            t.copy_(x.transpose(1, 2).reshape(B, rows, columns) if x.dim() == 4 else x)
        return t.view(B, rows, H, d).transpose(1, 2) if columns == H * d else t
    x = attn(3, B, H, H, T, d, d, "bf16", True, grads=True)
    q, k, v, dO = (dev(x[n]).to(torch.bfloat16) for n in ("q", "k", "v", "dO"))
    g, be, S0, dS = (f32(x[n]) for n in ("log_decay", "beta", "S0", "dS_T"))
    far = [spread(i, t) for i, t in enumerate((q, k, v, dO))]
    o, S = sfda.delta_attn_fwd(q, k, v, g, be, S0)
    of, Sf = sfda.delta_attn_fwd(*far[:3], g, be, S0, o=spread(4))
    assert o.equal(of) and S.equal(Sf)
    r = sfda.delta_attn_bwd(q, k, v, g, be, S0, dO, dS)
    f = sfda.delta_attn_bwd(*far[:3], g, be, S0, far[3], dS, dq=spread(4), dk=spread(5), dv=spread(6))
    assert all(r[n].equal(f[n]) for n in r)
    rows = torch.randn(B, T, 200, device="cuda").to(torch.bfloat16)
    more = torch.randn(B, T, 200, device="cuda").to(torch.bfloat16)
    w = torch.randn(200, device="cuda")
    y, t = sfda.layer_norm(rows, w, None, more)
    yf, tf = sfda.layer_norm(spread(0, rows, 200), w, None, spread(1, more, 200), y=spread(2, None, 200), total=spread(3, None, 200))
    assert y.equal(yf) and t.equal(tf)
    r = sfda.layer_norm_bwd(rows, t, w, None, more)
    f = sfda.layer_norm_bwd(spread(0, None, 200), tf, w, None, spread(1, None, 200), dx=spread(4, None, 200))
    assert r["dx"].equal(f["dx"]) and r["dweight"].equal(f["dweight"])


def test_more_heads_than_a_launch_takes():
    """8193 sequences of 32 heads: the results of each half of the sequences, bit by bit, and the recurrence's for the last ones."""
    import torch
    from paper_2607_11897_amd import sfda
    say("many sequences")
    B, H, T, dk, dv = 8193, 32, 3, 5, 4
    x = attn(21, B, H, H, T, dk, dv, "f32", grads=True)
    q, k, v, g, be, S0, dO, dS = (f32(x[n]) for n in ("q", "k", "v", "log_decay", "beta", "S0", "dO", "dS_T"))
    last = {n: None if x[n] is None else x[n][-2:] for n in x}
    halves = (slice(0, B // 2), slice(B // 2, B))
    S, parts = S0.clone(), [S0[h].clone() for h in halves]
    for t in range(T):
        o = sfda.delta_attn_step(q[:, :, t], k[:, :, t], v[:, :, t], g[:, :, t], be[:, :, t], S)
        for h, p in zip(halves, parts):
            assert torch.equal(o[h], sfda.delta_attn_step(q[h, :, t], k[h, :, t], v[h, :, t], g[h, :, t], be[h, :, t], p))
    assert torch.equal(S, torch.cat(parts))
    assert rel_err(S[-2:].double().cpu().numpy(), O.delta_attn(**names(last))[1]) <= SUM
    got = sfda.delta_attn_bwd(q, k, v, g, be, S0, dO, dS)
    for h in halves:
        half = sfda.delta_attn_bwd(*(t[h] for t in (q, k, v, g, be, S0, dO, dS)))
        for n in got:
            assert torch.equal(got[n][h], half[n]), n
    check_bwd({n: y[-2:].double().cpu().numpy() for n, y in got.items()}, O.delta_attn_backward(**names(last, "dO", "dS_T")), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,Hk,T,dk,dv,lengths", [(2, 6, 3, 100, 33, 70, None), (2, 3, 1, 2500, 64, 64, [3, 2499]), (1, 2, 1, 0, 8, 8, None)])
def test_fwd_in_passes(dtype, B, H, Hk, T, dk, dv, lengths):
    """Groups of heads, as many as the workspace holds, in segments too and with S_T in S0's memory: the same results, bit by bit."""
    import torch
    from paper_2607_11897_amd import sfda
    say("fwd passes", dtype, T)
    x = attn(4, B, H, Hk, T, dk, dv, dtype, True, lengths)
    o, S = run_fwd(x, dtype, "bthd", 0.3)
    whole = sfda.delta_attn_fwd_workspace_bytes(B, H, T, dk, dv, dtype)
    one = whole // (B * H)
    assert whole == one * B * H and (T < 1000) == (one == sfda.delta_attn_fwd_workspace_bytes(B, 4096, T, dk, dv, dtype) // (4096 * B))
    for n in (1, 2, 5):
        again = run_fwd(x, dtype, "bthd", 0.3, workspace=torch.full((n * one + 15,), 255, dtype=torch.uint8, device="cuda"))
        assert np.array_equal(again[0], o) and np.array_equal(again[1], S), n
    if T > 0:
        with pytest.raises(sfda.SfdaError, match="SHAPE"):
            run_fwd(x, dtype, "bthd", 0.3, workspace=torch.empty(one - 16, dtype=torch.uint8, device="cuda"))
        t = [dev(x[n]).to(dt(dtype)) for n in "qkv"] + [f32(x[n]) for n in ("log_decay", "beta", "S0")]
        room = torch.empty(2 * one, dtype=torch.uint8, device="cuda")
        o2, S2 = sfda.delta_attn_fwd(*t, scale=0.3, lengths=dev(x["lengths"]), S_T=t[-1], workspace=room)
        assert np.array_equal(o2.double().cpu().numpy(), o) and np.array_equal(t[-1].double().cpu().numpy(), S) and S2 is t[-1]


def test_fwd_of_more_heads_than_a_launch_takes():
    """8193 sequences of 32 heads: the results of each half of the sequences, bit by bit."""
    import torch
    from paper_2607_11897_amd import sfda
    say("many sequences forward")
    B, H, T, dk, dv = 8193, 32, 3, 5, 4
    x = attn(22, B, H, H, T, dk, dv, "f32")
    t = [f32(x[n]) for n in ("q", "k", "v", "log_decay", "beta", "S0")]
    o, S = sfda.delta_attn_fwd(*t)
    for h in (slice(0, B // 2), slice(B // 2, B)):
        for a, b in zip((o, S), sfda.delta_attn_fwd(*(y[h] for y in t))):
            assert torch.equal(a[h], b)


def directions(y, gen):
    """Six of them, of entries of size 1: a derivative along one is of the gradient's norm, and an input's gradient that were zero, or off by a
    third, would stand out along all but a hundredth of them."""
    import torch
    return [torch.randn(y.shape, generator=gen, device=y.device) for _ in range(6)]


@pytest.mark.parametrize("H,Hk", [(2, 1), (3, 3)])
def test_bwd_against_differences_along_many_directions(H, Hk):
    """float32 gradients against central differences, each bar in units of what is compared.  The loss is linear in q, v and S0: with
    steps of 1 a difference is off by the forward's rounding alone, 2^-22 in sums of a few thousand terms: 1e-3 of the gradient.  Keys,
    decays and strengths, steps of 1e-3: h^2 / 6 of a third derivative, in which 40 tokens' steps of 3e-3 of a key meet, 3e-4 of
    the gradient; the rounding, 1e-6 of the loss over h, 1e-3 of it at a loss of the gradient's size: 1e-2."""
    import torch
    from paper_2607_11897_amd import sfda
    say("many directions", H, Hk)
    x = attn(13, 1, H, Hk, 40, 8, 6, "f32", grads=True)
    t = {n: f32(x[n]) for n in ("q", "k", "v", "log_decay", "beta", "S0")}
    t["log_decay"][0, 0, 20] = -0.4         # (no reset: its difference is not a number)
    dO, dS = f32(x["dO"]), f32(x["dS_T"])
    gen = torch.Generator(device="cuda").manual_seed(1)

    def loss(**kw):
        o, S = sfda.delta_attn_fwd(**kw, scale=0.6)
        return float((o.double() * dO).sum() + (S.double() * dS).sum())
    got = sfda.delta_attn_bwd(**t, dO=dO, dS_T=dS, scale=0.6)
    for name, y in t.items():
        g = got["d" + name].double()
        h, bar = (1.0, 1e-3) if name in ("q", "v", "S0") else (1e-3, 1e-2)
        for d in directions(y, gen):
            up, down = y + h * d, y - h * d         # (the steps that the inputs hold)
            want = loss(**{**t, name: up}) - loss(**{**t, name: down})
            have = float((g * (up.double() - down.double())).sum())
            assert abs(want - have) <= bar * 2 * h * float(g.norm()), (name, want, have)

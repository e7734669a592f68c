"""GPU parity of the operators around the attention with their float64 oracle.

Error measure: max |x - ref| / max |ref| over a whole tensor.  Bars, from the arithmetic:
  * element-wise results (rotary): float32 two products and a sum of at most sqrt(2) max|x|, 3 roundings of
    2^-24: 4e-7; bfloat16 one rounding more, of up to 2^-8 of the element itself (spacing 2^-7 in [1, 2)).
  * float32 sums (decay attention, states of both types, norm's float32 results and weight gradients): a
    few hundred to a few thousand terms of either sign, errors of 2^-24 each growing like the square root of their
    number: 2e-5.
  * bfloat16 results: up to 2^-8 of the result's own rounding, and for the decay attention the scores and the state rounded
    as operands: errors of up to 2^-8 of each of many terms, of either sign, whose sum stays below their largest result's
    rounding: 1e-2 in all; the norm has only its own rounding, 4e-3 (2^-8).
Every output lies between canary words, and rows that a call does not own keep theirs."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_util import ensure_built, rel_err
from oracle import layer as O

pytestmark = pytest.mark.gpu
CANARY = -12288.0
SUM = 2e-5
ATTN, NORM = {"f32": SUM, "bf16": 1e-2}, {"f32": SUM, "bf16": 4e-3}


@pytest.fixture(scope="module", autouse=True)
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return ensure_built()


def say(*a):
    print("[case]", *a, flush=True)


def turned(x, ref, dtype):
    """Whether x is ref to float32, and for bfloat16 one rounding of each element more."""
    return bool(np.all(np.abs(x - ref) <= (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0) + 4e-7 * np.max(np.abs(ref), initial=0.0)))


def dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


class Buf:
    """A tensor of `shape` (an attention's [B, H, T, D], or [B, T, C]) in a canary-filled buffer.  layouts: "bhtd"
    contiguous; "bthd" heads inside; "padded" rows 3 elements longer and the buffer off its alignment by an element."""

    def __init__(self, shape, dtype, layout="bhtd", values=None):
        import torch
        self.n = [int(s) for s in shape]
        order = list(range(len(shape)))
        if layout == "bthd" and len(shape) == 4:
            order = [0, 2, 1, 3]
        pad, off = (3, 129) if layout == "padded" else (0, 128)
        mem = [self.n[i] for i in order]
        size = int(np.prod(mem[:-1])) * (mem[-1] + pad)
        self.flat = torch.full((size + off + 128,), CANARY, dtype=dtype, device="cuda")
        rows = self.flat[off:off + size].view(*mem[:-1], mem[-1] + pad)[..., :mem[-1]]
        self.t = rows.permute(*np.argsort(order).tolist())
        if values is not None:
            self.t.copy_(torch.from_numpy(np.asarray(values, np.float32)).to("cuda"))

    def numpy(self):
        return self.t.float().cpu().numpy().astype(np.float64)

    def check(self, what):
        """Nothing outside the tensor was written."""
        keep = self.t.clone()
        self.t.fill_(CANARY)
        assert bool((self.flat == CANARY).all()), what
        self.t.copy_(keep)


def stored(rng, shape, dtype, scale=1.0):
    """Values that the type holds, as float64."""
    import torch
    return torch.from_numpy(scale * rng.standard_normal(shape)).to(dt(dtype)).double().numpy()


def slopes(H):
    """Decays from 2 tokens' memory to none at all, and the two ends."""
    g = np.log1p(-(2.0 ** -np.linspace(1, 9, H))).astype(np.float32)
    if H >= 3:
        g[0], g[-1] = -np.inf, 0.0
    return g


# --------------------------------------------------------------------------- decay attention

def attn(seed, B, H, T, dk, dv, dtype, state=True, lengths=None, grads=False):
    rng = np.random.Generator(np.random.PCG64(seed))
    x = dict(q=stored(rng, (B, H, T, dk), dtype), k=stored(rng, (B, H, T, dk), dtype), v=stored(rng, (B, H, T, dv), dtype))
    x["S0"] = stored(rng, (B, H, dk, dv), "f32") if state else None
    if grads:
        x["dO"] = stored(rng, (B, H, T, dv), dtype)
        x["dS_T"] = stored(rng, (B, H, dk, dv), "f32") if state else None
    x["g"] = slopes(H)
    x["lengths"] = None if lengths is None else np.asarray(lengths, np.int32)
    return x


def dev(a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def f32(a):
    return None if a is None else dev(np.asarray(a, np.float32))


def run_fwd(x, dtype, layout, scale, poison=None, workspace=None):
    """o and S_T of the library for the inputs x; poison: what the tokens past a length hold."""
    import torch
    from paper_2607_11897_amd import sfda
    B, H, T, dk = x["q"].shape
    b = {n: Buf(x[n].shape, dt(dtype), layout, x[n]) for n in "qkv"}
    if poison is not None:
        for i, n in enumerate(np.clip(x["lengths"], 0, T)):
            for t in b.values():
                t.t[i, :, n:] = poison
    o = Buf(x["v"].shape, dt(dtype), layout)
    S = Buf((B, H, dk, x["v"].shape[-1]), torch.float32)
    sfda.decay_attn_fwd(b["q"].t, b["k"].t, b["v"].t, f32(x["g"]), f32(x["S0"]), scale=scale, lengths=dev(x["lengths"]), o=o.t, S_T=S.t,
                        workspace=workspace)
    torch.cuda.synchronize()
    o.check("o")
    S.check("S_T")
    return o.numpy(), S.numpy()


FWD = [  # B, H, T, dk, dv, dtype, layout, state
    (2, 3, 1, 16, 8, "f32", "bhtd", True), (2, 3, 1, 128, 128, "bf16", "bthd", True), (1, 1, 0, 8, 8, "f32", "bhtd", True),
    (1, 3, 0, 8, 8, "bf16", "bhtd", False), (2, 3, 31, 1, 1, "f32", "bhtd", True), (2, 3, 33, 3, 5, "f32", "padded", True),
    (1, 4, 64, 64, 64, "f32", "bthd", False), (2, 3, 97, 65, 66, "f32", "bhtd", True), (1, 2, 130, 256, 256, "f32", "bthd", True),
    (1, 3, 65, 129, 130, "f32", "padded", True), (3, 3, 63, 7, 9, "bf16", "padded", True), (2, 3, 64, 32, 16, "bf16", "bthd", True),
    (1, 4, 65, 64, 64, "bf16", "bhtd", False), (2, 3, 200, 128, 128, "bf16", "bthd", True), (1, 3, 129, 88, 74, "bf16", "bthd", True),
    (1, 2, 191, 200, 250, "bf16", "padded", True), (1, 2, 128, 256, 256, "bf16", "bthd", True), (2, 3, 66, 1, 2, "bf16", "bhtd", True),
    # segments: few heads, long sequences
    (1, 3, 1000, 128, 128, "bf16", "bthd", True), (1, 3, 1537, 33, 70, "f32", "bhtd", True), (1, 1, 2048, 64, 64, "bf16", "bthd", False),
]


@pytest.mark.parametrize("B,H,T,dk,dv,dtype,layout,state", FWD)
def test_decay_attn_fwd(B, H, T, dk, dv, dtype, layout, state):
    say("decay_attn_fwd", B, H, T, dk, dv, dtype, layout, state)
    x = attn(1 + T, B, H, T, dk, dv, dtype, state)
    scale = dk ** -0.5
    o_ref, S_ref = O.decay_attn(x["q"], x["k"], x["v"], x["g"], x["S0"], scale)
    o, S = run_fwd(x, dtype, layout, scale)
    eo, es = rel_err(o, o_ref), rel_err(S, S_ref)
    say("err(o)", eo, "err(S_T)", es)
    assert eo <= ATTN[dtype] and es <= SUM


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,lengths", [(70, [70, 0, 1, 64, 65, -3, 1000]), (700, [700, 0, 1, 256, 511, 513, 2])])
def test_decay_attn_lengths(dtype, T, lengths):
    """Sequences of their own lengths; what lies past them is NaN and does not reach any result."""
    say("decay_attn_fwd lengths", dtype, T, lengths)
    x = attn(5, len(lengths), 3, T, 40, 24, dtype, True, lengths)
    o_ref, S_ref = O.decay_attn(x["q"], x["k"], x["v"], x["g"], x["S0"], 0.5, x["lengths"])
    o, S = run_fwd(x, dtype, "bthd", 0.5, poison=float("nan"))
    assert rel_err(o, o_ref) <= ATTN[dtype] and rel_err(S, S_ref) <= SUM
    for i, n in enumerate(np.clip(lengths, 0, T)):
        assert not o[i, :, n:].any()
    assert np.array_equal(S[1], x["S0"][1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decay_attn_segments_agree_and_resume(dtype):
    """One scan, segments and two calls joined by their state give the same results up to rounding; in place too."""
    import torch
    from paper_2607_11897_amd import sfda
    say("decay_attn_fwd segments", dtype)
    B, H, T, dk, dv = 1, 3, 900, 48, 72
    x = attn(9, B, H, T, dk, dv, dtype)
    assert sfda.decay_attn_fwd_workspace_bytes(B, H, T, dk, dv, dtype) > 0
    a = run_fwd(x, dtype, "bhtd", 1.0)
    b = run_fwd(x, dtype, "bhtd", 1.0, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert rel_err(a[0], b[0]) <= ATTN[dtype] and rel_err(a[1], b[1]) <= SUM
    q, k, v = (f32(x[n]).to(dt(dtype)) for n in "qkv")
    S = f32(x["S0"])
    parts = []
    for lo, hi in ((0, 333), (333, 334), (334, 900)):
        o, out = sfda.decay_attn_fwd(q[:, :, lo:hi], k[:, :, lo:hi], v[:, :, lo:hi], f32(x["g"]), S, S_T=S)
        assert out is S
        parts.append(o)
    torch.cuda.synchronize()
    assert rel_err(torch.cat(parts, 2).double().cpu().numpy(), b[0]) <= ATTN[dtype] and rel_err(S.double().cpu().numpy(), b[1]) <= SUM
    again = run_fwd(x, dtype, "bhtd", 1.0)
    assert np.array_equal(a[0], again[0]) and np.array_equal(a[1], again[1])


def test_decay_attn_shared_heads_and_no_state():
    """Keys and values shared by heads as a view of stride 0, and no final state."""
    import torch
    from paper_2607_11897_amd import sfda
    say("decay_attn_fwd shared heads")
    x = attn(11, 2, 4, 100, 32, 32, "f32", False)
    x["k"][:], x["v"][:] = x["k"][:, :1], x["v"][:, :1]
    q, k, v = (f32(x[n]) for n in "qkv")
    o, S = sfda.decay_attn_fwd(q, k[:, :1].expand_as(q), v[:, :1].expand_as(v), f32(x["g"]), want_state=False)
    torch.cuda.synchronize()
    assert S is None and rel_err(o.double().cpu().numpy(), O.decay_attn(x["q"], x["k"], x["v"], x["g"])[0]) <= SUM


def test_decay_attn_long_memory():
    """A decay so slow that thousands of blocks add up: the blocks' decay keeps more than float32."""
    import torch
    from paper_2607_11897_amd import sfda
    say("decay_attn_fwd long memory")
    T, g = 200000, np.array([-1e-6, -3e-5], np.float32)
    rng = np.random.Generator(np.random.PCG64(3))
    S0 = stored(rng, (1, 2, 4, 4), "f32")
    z = torch.zeros(1, 2, T, 4, device="cuda")
    for ws in (None, torch.empty(4, dtype=torch.uint8, device="cuda")):
        _, S = sfda.decay_attn_fwd(z, z, z, f32(g), f32(S0), workspace=ws)
        torch.cuda.synchronize()
        want = np.exp(T * g.astype(np.float64))[None, :, None, None] * S0
        assert rel_err(S.double().cpu().numpy(), want) <= SUM


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decay_attn_not_finite(dtype):
    """A token that is not finite leaves the earlier blocks, the other heads and the other sequences alone."""
    say("decay_attn_fwd NaN", dtype)
    x = attn(13, 2, 3, 256, 32, 32, dtype)
    clean = run_fwd(x, dtype, "bhtd", 1.0)
    x["v"][1, 1, 150, 3] = np.nan
    o, S = run_fwd(x, dtype, "bhtd", 1.0)
    assert np.isnan(o[1, 1, 150:, 3]).all() and np.isnan(S[1, 1, :, 3]).all()
    o[1, 1, 128:, :], S[1, 1] = clean[0][1, 1, 128:], clean[1][1, 1]
    assert np.array_equal(o, clean[0]) and np.array_equal(S, clean[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name,at", [("v", 3), ("k", 5)])
def test_decay_attn_infinite(dtype, name, at):
    """An infinite value or key: its column, or with a key every column, of the later blocks is not finite, nor its column or row of
    S_T.  The earlier blocks, the other heads and sequences and, with a value, the other columns keep their results."""
    say("decay_attn_fwd inf", dtype, name)
    x = attn(15, 2, 3, 256, 32, 32, dtype)
    x["g"][1] = -0.01
    clean = run_fwd(x, dtype, "bhtd", 1.0)
    x[name][1, 1, 150, at] = np.inf
    o, S = run_fwd(x, dtype, "bhtd", 1.0)
    hit = [at] if name == "v" else list(range(32))
    assert not np.isfinite(o[1, 1, 192:, hit]).any()
    assert not np.isfinite(S[1, 1][:, hit] if name == "v" else S[1, 1, at]).any()
    o[1, 1, 128:, hit] = clean[0][1, 1, 128:, hit]
    if name == "v":
        S[1, 1][:, hit] = clean[1][1, 1][:, hit]
    else:
        S[1, 1, at] = clean[1][1, 1, at]
    assert np.array_equal(o, clean[0]) and np.array_equal(S, clean[1])


def run_bwd(x, dtype, layout, scale, want_dS0=True, poison=None):
    import torch
    from paper_2607_11897_amd import sfda
    T = x["q"].shape[2]
    b = {n: Buf(x[n].shape, dt(dtype), layout, x[n]) for n in ("q", "k", "v", "dO")}
    if poison is not None:
        for i, n in enumerate(np.clip(x["lengths"], 0, T)):
            for t in b.values():
                t.t[i, :, n:] = poison
    out = {n: Buf(x[n[1:]].shape, dt(dtype), layout) for n in ("dq", "dk", "dv")}
    got = sfda.decay_attn_bwd(b["q"].t, b["k"].t, b["v"].t, f32(x["g"]), f32(x["S0"]), b["dO"].t, f32(x["dS_T"]), scale=scale,
                              lengths=dev(x["lengths"]), want_dS0=want_dS0, **{n: t.t for n, t in out.items()})
    torch.cuda.synchronize()
    for n, t in out.items():
        t.check(n)
    r = {n: t.numpy() for n, t in out.items()}
    r["dS0"] = None if got["dS0"] is None else got["dS0"].double().cpu().numpy()
    return r


BWD = [(2, 3, 1, 16, 8, "f32", "bhtd", True, None), (2, 3, 1, 128, 128, "bf16", "bthd", True, None),
       (1, 3, 33, 3, 5, "f32", "padded", True, None), (1, 3, 97, 65, 130, "f32", "bthd", False, None),
       (1, 3, 70, 256, 40, "f32", "bhtd", True, None), (2, 3, 63, 7, 9, "bf16", "padded", True, None),
       (2, 3, 130, 128, 64, "bf16", "bthd", True, None), (1, 3, 129, 88, 74, "bf16", "bthd", False, None),
       (1, 2, 130, 250, 256, "bf16", "bhtd", True, None), (1, 3, 0, 8, 8, "bf16", "bhtd", True, None),
       (1, 3, 900, 64, 33, "f32", "bhtd", True, None), (1, 3, 1100, 128, 128, "bf16", "bthd", True, None),
       (5, 3, 70, 40, 24, "f32", "bthd", True, [70, 0, 1, 33, 64]), (5, 3, 140, 40, 24, "bf16", "bhtd", True, [140, 0, 1, 64, 129]),
       (3, 3, 800, 40, 24, "bf16", "bthd", True, [800, 300, 0]), (3, 3, 800, 16, 80, "f32", "bthd", True, [513, 800, 257])]


@pytest.mark.parametrize("B,H,T,dk,dv,dtype,layout,state,lengths", BWD)
def test_decay_attn_bwd(B, H, T, dk, dv, dtype, layout, state, lengths):
    say("decay_attn_bwd", B, H, T, dk, dv, dtype, layout, state, lengths)
    x = attn(21 + T, B, H, T, dk, dv, dtype, state, lengths, grads=True)
    scale = dk ** -0.5
    ref = O.decay_attn_backward(x["q"], x["k"], x["v"], x["g"], x["S0"], x["dO"], x["dS_T"], scale, x["lengths"])
    got = run_bwd(x, dtype, layout, scale, poison=float("nan") if lengths is not None else None)
    err = {n: rel_err(got[n], ref[n]) for n in ref}
    say(err)
    assert all(err[n] <= ATTN[dtype] for n in ("dq", "dk", "dv")) and err["dS0"] <= SUM
    if lengths is not None:
        for i, n in enumerate(lengths):
            assert not any(got[m][i, :, n:].any() for m in ("dq", "dk", "dv"))


# states of more than 128 and of at most 64 channels, one launch each: more heads than compute units; segments
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,T,dk,dv", [(16, 16, 70, 24, 150), (1, 8, 700, 40, 200), (20, 13, 5, 129, 60)])
def test_decay_attn_bwd_in_two_launches(B, H, T, dk, dv, dtype):
    test_decay_attn_bwd(B, H, T, dk, dv, dtype, "bthd", True, None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(128, 64), (33, 74)])
@pytest.mark.parametrize("stride", [1, 1 << 24, (1 << 26) + 8, 1 << 40])
def test_decay_attn_one_token_of_any_stride(dtype, dk, dv, stride):
    """One token: the stride of the tokens is whatever the caller's view has, and reaches no address."""
    import torch
    from paper_2607_11897_amd import sfda
    say("decay_attn one token", dtype, dk, dv, stride)
    x = attn(17, 2, 3, 1, dk, dv, dtype, True, grads=True)

    def far(t):
        st = t.stride()
        return t.as_strided(t.shape, (st[0], st[1], stride, st[3]), t.storage_offset())
    b = {n: Buf(x[n].shape, dt(dtype), "bhtd", x[n]) for n in ("q", "k", "v", "dO")}
    out = {n: Buf(x[m].shape, dt(dtype), "bhtd") for n, m in (("o", "v"), ("dq", "q"), ("dk", "k"), ("dv", "v"))}
    i, w = {n: far(t.t) for n, t in b.items()}, {n: far(t.t) for n, t in out.items()}
    _, S = sfda.decay_attn_fwd(i["q"], i["k"], i["v"], f32(x["g"]), f32(x["S0"]), scale=0.5, o=w["o"])
    got = sfda.decay_attn_bwd(i["q"], i["k"], i["v"], f32(x["g"]), f32(x["S0"]), i["dO"], f32(x["dS_T"]), scale=0.5,
                              **{n: w[n] for n in ("dq", "dk", "dv")})
    torch.cuda.synchronize()
    for n, t in out.items():
        t.check(n)
    o, S_ref = O.decay_attn(x["q"], x["k"], x["v"], x["g"], x["S0"], 0.5)
    ref = O.decay_attn_backward(x["q"], x["k"], x["v"], x["g"], x["S0"], x["dO"], x["dS_T"], 0.5) | dict(o=o)
    assert all(rel_err(out[n].numpy(), ref[n]) <= ATTN[dtype] for n in out)
    assert rel_err(S.double().cpu().numpy(), S_ref) <= SUM and rel_err(got["dS0"].double().cpu().numpy(), ref["dS0"]) <= SUM


def by_token(x, scale):
    """The recurrence and its reverse sweep in float64, all heads at a time: o, S_T, dq, dk, dv, dS0."""
    import torch
    q, k, v, dO = (dev(x[n]) for n in ("q", "k", "v", "dO"))
    T, c = q.shape[2], scale
    lam = torch.exp(dev(x["g"].astype(np.float64)))[None, :, None, None]
    n = torch.full((q.shape[0],), T, device="cuda") if x["lengths"] is None else dev(np.clip(x["lengths"], 0, T))
    o, dq, dk, dv = (torch.zeros_like(t) for t in (v, q, k, v))
    S, G = dev(x["S0"]), dev(x["dS_T"])
    for t in range(T):
        on = (t < n)[:, None, None, None]
        S = torch.where(on, lam * S + k[:, :, t, :, None] * v[:, :, t, None, :], S)
        o[:, :, t] = torch.where(on[..., 0], c * (S * q[:, :, t, :, None]).sum(2), 0.0)
        dq[:, :, t] = torch.where(on[..., 0], c * (S * dO[:, :, t, None, :]).sum(3), 0.0)
    for t in range(T - 1, -1, -1):
        on = (t < n)[:, None, None, None]
        U = G + c * q[:, :, t, :, None] * dO[:, :, t, None, :]
        dk[:, :, t] = torch.where(on[..., 0], (U * v[:, :, t, None, :]).sum(3), 0.0)
        dv[:, :, t] = torch.where(on[..., 0], (U * k[:, :, t, :, None]).sum(2), 0.0)
        G = torch.where(on, lam * U, G)
    torch.cuda.synchronize()
    return {m: t.cpu().numpy() for m, t in (("o", o), ("S_T", S), ("dq", dq), ("dk", dk), ("dv", dv), ("dS0", G))}


# (more workgroups than compute units, so that a block's state has one buffer, and several blocks a sequence; few heads, so
# that sequences are cut, into segments of several blocks, and lengths that end inside them)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,T,dk,dv,cut,lengths", [
    (9, 16, 300, 128, 128, False, None), (9, 16, 260, 126, 127, False, None), (9, 16, 200, 128, 64, False, [200, 0, 1, 64, 65, 127, 128, 129, 199]),
    (12, 16, 131, 64, 72, False, None), (5, 16, 150, 256, 200, False, None),
    (4, 4, 4001, 128, 128, True, [4001, 1900, 300, 0]), (2, 8, 3900, 88, 74, True, [3900, 2477]), (1, 3, 6000, 200, 256, True, None)])
def test_decay_attn_many_blocks(B, H, T, dk, dv, cut, lengths, dtype):
    from paper_2607_11897_amd import sfda
    say("decay_attn many blocks", B, H, T, dk, dv, cut, lengths, dtype)
    for f, states in ((sfda.decay_attn_fwd_workspace_bytes, 1), (sfda.decay_attn_bwd_workspace_bytes, 3)):
        segments = f(B, H, T, dk, dv, dtype) // (4 * states * B * H * dk * dv)
        assert (1 < segments <= T // 128) if cut else segments == 0
    x = attn(61 + T, B, H, T, dk, dv, dtype, True, lengths, grads=True)
    scale = dk ** -0.5
    ref = by_token(x, scale)
    poison = float("nan") if lengths is not None else None
    o, S = run_fwd(x, dtype, "bthd", scale, poison)
    got = run_bwd(x, dtype, "bthd", scale, poison=poison) | dict(o=o, S_T=S)
    err = {m: rel_err(got[m], ref[m]) for m in ref}
    say(err)
    assert all(err[m] <= (SUM if m in ("S_T", "dS0") else ATTN[dtype]) for m in ref)
    for i, n in enumerate(lengths or []):
        assert not any(got[m][i, :, n:].any() for m in ("o", "dq", "dk", "dv"))


def test_decay_attn_bwd_against_differences():
    """Directional differences of the GPU's own forward in float32."""
    import torch
    from paper_2607_11897_amd import sfda
    say("decay_attn_bwd differences")
    x = attn(31, 2, 3, 75, 24, 20, "f32", grads=True)
    got = run_bwd(x, "f32", "bhtd", 0.5)
    g = f32(x["g"])

    def loss(y):
        o, S = sfda.decay_attn_fwd(f32(y["q"]), f32(y["k"]), f32(y["v"]), g, f32(y["S0"]), scale=0.5)
        return float((o.double() * f32(x["dO"])).sum() + (S.double() * f32(x["dS_T"])).sum())
    rng = np.random.Generator(np.random.PCG64(1))
    h = 0.05            # o is bilinear in (q, k) and (q, v): central differences have no error of their own in one of them
    for name in ("q", "k", "v", "S0"):
        d = rng.standard_normal(x[name].shape)
        up, down = (loss(x | {name: x[name] + s * h * d}) for s in (1, -1))
        want = float((got["d" + name] * d).sum())
        # sums of float32 errors of 2^-24 of values of the size of `size`, over the step
        size = np.sqrt(sum(np.sum(got["d" + n] ** 2) for n in ("q", "k", "v", "S0")))
        assert abs((up - down) / (2 * h) - want) <= 1e-3 * size, name


@pytest.mark.parametrize("B,H,dk,dv,dtype,strided", [(2, 3, 128, 128, "f32", False), (2, 3, 128, 128, "bf16", True), (1, 3, 1, 1, "f32", False),
                                                     (3, 2, 33, 17, "bf16", True), (1, 3, 256, 256, "f32", True), (2, 3, 7, 130, "f32", True),
                                                     (1, 4, 64, 66, "bf16", False), (40, 16, 16, 32, "bf16", False)])
def test_decay_attn_step(B, H, dk, dv, dtype, strided):
    import torch
    from paper_2607_11897_amd import sfda
    say("decay_attn_step", B, H, dk, dv, dtype, strided)
    x = attn(41 + dk, B, H, 6, dk, dv, dtype)
    S = Buf((B, H, dk, dv), torch.float32, "bhtd", x["S0"])
    b = {n: Buf(x[n].shape, dt(dtype), "padded" if strided else "bhtd", x[n]) for n in "qkv"}
    o = Buf(x["v"].shape, dt(dtype), "padded" if strided else "bhtd")
    for t in range(6):
        sfda.decay_attn_step(b["q"].t[:, :, t], b["k"].t[:, :, t], b["v"].t[:, :, t], f32(x["g"]), S.t, scale=0.5, o=o.t[:, :, t])
    torch.cuda.synchronize()
    S.check("S")
    o.check("o")
    o_ref, S_ref = O.decay_attn(x["q"], x["k"], x["v"], x["g"], x["S0"], 0.5)
    assert rel_err(S.numpy(), S_ref) <= SUM and rel_err(o.numpy(), o_ref) <= NORM[dtype]


# --------------------------------------------------------------------------- rotary

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,Hq,Hk,T,D,rot,layout,inter", [(2, 3, 1, 5, 128, 128, "bthd", False), (2, 4, 4, 7, 64, 32, "bhtd", True),
                                                          (1, 5, 0, 1, 128, 128, "bhtd", False), (3, 2, 3, 9, 33, 10, "padded", False),
                                                          (3, 1, 6, 9, 37, 26, "padded", True), (1, 1, 1, 64, 2, 2, "bhtd", True),
                                                          (1, 7, 2, 3, 256, 250, "bthd", False), (2, 1, 1, 0, 16, 8, "bhtd", False)])
def test_rotary(B, Hq, Hk, T, D, rot, layout, inter, dtype):
    import torch
    from paper_2607_11897_amd import sfda
    say("rotary", B, Hq, Hk, T, D, rot, layout, inter, dtype)
    rng = np.random.Generator(np.random.PCG64(D + T))
    P = 80
    cos, sin = sfda.rotary_tables(P, rot)
    c, s = cos.double().cpu().numpy(), sin.double().cpu().numpy()
    q, k = stored(rng, (B, Hq, T, D), dtype), stored(rng, (B, Hk, T, D), dtype)
    each = rng.integers(0, P, (B, T))
    for positions, at, kw in ((None, np.arange(T) + 11, dict(offset=11)), (dev(each), each, {}), (dev(each.astype(np.int32)), each, dict(inverse=True)),
                              (dev(each[0].astype(np.int32)), each[0], {})):
        bq, bk, oq, ok = Buf(q.shape, dt(dtype), layout, q), Buf(k.shape, dt(dtype), layout, k), Buf(q.shape, dt(dtype), layout), Buf(k.shape, dt(dtype), layout)
        inv = kw.get("inverse", False)
        sfda.rotary(bq.t, bk.t if Hk else None, cos, sin, positions, interleaved=inter, q_out=oq.t, k_out=ok.t if Hk else None, **kw)
        torch.cuda.synchronize()
        oq.check("q")
        assert turned(oq.numpy(), O.rotary(q, c, s, at, inter, inv), dtype)
        assert np.array_equal(oq.numpy()[..., rot:], q[..., rot:])
        if Hk:
            ok.check("k")
            assert turned(ok.numpy(), O.rotary(k, c, s, at, inter, inv), dtype)
            sfda.rotary(bq.t, bk.t, cos, sin, positions, interleaved=inter, q_out=bq.t, k_out=bk.t, **kw)      # in place
            torch.cuda.synchronize()
            assert np.array_equal(bq.numpy(), oq.numpy()) and np.array_equal(bk.numpy(), ok.numpy())
            bq.check("q in place")


def test_rotary_packed_and_out_of_range():
    """Queries and keys as slices of one projection, turned in place; positions without a row of the tables give NaN."""
    import torch
    from paper_2607_11897_amd import sfda
    say("rotary packed")
    rng = np.random.Generator(np.random.PCG64(2))
    x = stored(rng, (2, 6, 3, 4, 32), "bf16")           # [B, T, (q, k, v), H, D]
    buf = dev(x.astype(np.float32)).to(torch.bfloat16)
    q, k = buf[:, :, 0].transpose(1, 2), buf[:, :, 1].transpose(1, 2)
    cos, sin = sfda.rotary_tables(16, 32)
    sfda.rotary(q, k, cos, sin, q_out=q, k_out=k)
    torch.cuda.synchronize()
    c, s = cos.double().cpu().numpy(), sin.double().cpu().numpy()
    for i, t in enumerate((q, k)):
        assert turned(t.double().cpu().numpy(), O.rotary(x[:, :, i].transpose(0, 2, 1, 3), c, s, np.arange(6)), "bf16")
    assert np.array_equal(buf[:, :, 2].double().cpu().numpy(), x[:, :, 2])
    with pytest.raises(sfda.SfdaError, match="SFDA_ERR_ALIAS"):
        sfda.rotary(q, k, cos, sin, q_out=k, k_out=q)
    y = torch.randn(1, 2, 4, 32, device="cuda")
    got, _ = sfda.rotary(y, None, cos[:, :8].contiguous(), sin[:, :8].contiguous(), dev(np.array([0, -1, 16, 15], np.int64)))
    torch.cuda.synchronize()
    bad = torch.isnan(got).cpu().numpy()
    assert bad[:, :, 1:3, :16].all() and not bad[:, :, [0, 3]].any() and not bad[..., 16:].any()
    with pytest.raises(sfda.SfdaError, match="SFDA_ERR_SHAPE"):
        sfda.rotary(y, None, cos, sin, offset=13)


# --------------------------------------------------------------------------- group norm

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,T,D,layout,gate,act,affine", [
    (2, 3, 17, 128, "bhtd", True, "silu", True), (2, 3, 17, 64, "bthd", False, "silu", True), (1, 1, 1, 1, "bhtd", False, "none", True),
    (2, 5, 33, 37, "padded", True, "silu", True), (1, 2, 70, 256, "bthd", True, "none", False), (1, 3, 9, 2048, "bhtd", True, "silu", True),
    (1, 2, 9, 1030, "padded", False, "silu", True), (2, 1, 300, 7, "bthd", False, "none", True), (0, 2, 3, 8, "bhtd", True, "silu", True),
    (1, 2, 0, 8, "bhtd", True, "silu", True), (1, 2, 40, 520, "bthd", True, "silu", True)])
def test_group_norm(B, H, T, D, layout, gate, act, affine, dtype):
    import torch
    from paper_2607_11897_amd import sfda
    say("group_norm", B, H, T, D, layout, gate, act, affine, dtype)
    rng = np.random.Generator(np.random.PCG64(D + T))
    x = stored(rng, (B, H, T, D), dtype, 2.0) + 0.5
    x = torch.from_numpy(x).to(dt(dtype)).double().numpy()
    z = stored(rng, (B, T, H * D), dtype) if gate else None
    dy = stored(rng, (B, T, H * D), dtype)
    w, b = ((1 + 0.3 * rng.standard_normal(H * D)).astype(np.float32), rng.standard_normal(H * D).astype(np.float32)) if affine else (None, None)
    lay = "padded" if layout == "padded" else "bhtd"
    bx, bz, bdy = Buf(x.shape, dt(dtype), layout, x), Buf(dy.shape, dt(dtype), lay, z), Buf(dy.shape, dt(dtype), lay, dy)
    y, dx, dz = Buf(dy.shape, dt(dtype), lay), Buf(x.shape, dt(dtype), layout), Buf(dy.shape, dt(dtype), lay)
    zt = bz.t if gate else None
    sfda.group_norm(bx.t, f32(w), f32(b), zt, activation=act, eps=1e-3, y=y.t)
    got = sfda.group_norm_bwd(bdy.t, bx.t, f32(w), f32(b), zt, activation=act, eps=1e-3, dx=dx.t, dgate=dz.t if gate else None)
    torch.cuda.synchronize()
    for t, what in ((y, "y"), (dx, "dx"), (dz, "dgate")):
        t.check(what)
    assert rel_err(y.numpy(), O.group_norm(x, w, b, z, act, 1e-3)) <= NORM[dtype]
    ref = O.group_norm_backward(dy, x, w, b, z, act, 1e-3)
    if D > 1:           # (one channel: x^ is 0 and dx cancels to it)
        assert rel_err(dx.numpy(), ref["dx"]) <= NORM[dtype]
    if gate:
        assert rel_err(dz.numpy(), ref["dgate"]) <= NORM[dtype]
    for name in ("dweight", "dbias"):
        assert (got[name] is None) == (not affine)
        if affine and D > 1:
            assert rel_err(got[name].double().cpu().numpy(), ref[name]) <= SUM


def test_group_norm_extremes():
    """A constant group (no variance), gates far out on both sides, one group that is not finite."""
    import torch
    from paper_2607_11897_amd import sfda
    say("group_norm extremes")
    x = torch.randn(1, 4, 6, 32, device="cuda")
    x[0, 0] = 3.0
    z = torch.full((1, 6, 128), -200.0, device="cuda")
    z[:, 3:] = 200.0
    z[:, 0] = -float("inf")
    y = sfda.group_norm(x, gate=z, activation="silu")
    assert not y[0, :, :32].any() and torch.isfinite(y).all() and not y[:, :3].any()
    g = sfda.group_norm_bwd(torch.ones_like(z), x, gate=z, activation="silu")
    torch.cuda.synchronize()
    assert torch.isfinite(g["dx"]).all() and torch.isfinite(g["dgate"]).all()
    clean = sfda.group_norm(x, activation="silu")
    x[0, 2, 1, 5] = float("nan")
    dirty = sfda.group_norm(x, activation="silu")
    torch.cuda.synchronize()
    at = torch.isnan(dirty).nonzero().cpu().numpy()
    assert set(map(tuple, at[:, :2])) == {(0, 1)} and set(at[:, 2]) == set(range(64, 96))
    assert torch.equal(torch.nan_to_num(dirty)[0, 2:], clean[0, 2:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,T,D,gate,act", [(1, 2, 1, 128, True, "silu"), (1, 3, 5, 64, False, "silu"), (2, 1, 3, 8, True, "none"),
                                              (1, 1, 40, 2048, False, "none"), (3, 2, 70, 33, True, "silu")])
def test_group_norm_without_eps(B, H, T, D, gate, act, dtype):
    """eps = 0 where every group has a variance: lanes that have no row add nothing to the weights' gradients."""
    import torch
    from paper_2607_11897_amd import sfda
    say("group_norm eps 0", B, H, T, D, gate, act, dtype)
    rng = np.random.Generator(np.random.PCG64(D + T))
    x, dy = stored(rng, (B, H, T, D), dtype), stored(rng, (B, T, H * D), dtype)
    z = stored(rng, dy.shape, dtype) if gate else None
    w, b = (1 + 0.3 * rng.standard_normal(H * D)).astype(np.float32), rng.standard_normal(H * D).astype(np.float32)
    X, Y = f32(x).to(dt(dtype)), f32(dy).to(dt(dtype))
    Z = f32(z).to(dt(dtype)) if gate else None
    y = sfda.group_norm(X, f32(w), f32(b), Z, activation=act, eps=0.0)
    got = sfda.group_norm_bwd(Y, X, f32(w), f32(b), Z, activation=act, eps=0.0)
    torch.cuda.synchronize()
    assert rel_err(y.double().cpu().numpy(), O.group_norm(x, w, b, z, act, 0.0)) <= NORM[dtype]
    ref = O.group_norm_backward(dy, x, w, b, z, act, 0.0)
    for name in ("dx", "dgate", "dweight", "dbias"):
        if got[name] is not None:
            bar = SUM if name in ("dweight", "dbias") else NORM[dtype]
            assert rel_err(got[name].double().cpu().numpy(), ref[name]) <= bar, name


def test_group_norm_subnormal_variance():
    """eps = 0 and values of 2^-65: the variance is a subnormal of 19 bits (its sum's terms are rounded to multiples of 2^-149,
    2^-20 of it), the results are ordinary numbers; dx is some 2^65."""
    import torch
    from paper_2607_11897_amd import sfda
    say("group_norm subnormal variance")
    rng = np.random.Generator(np.random.PCG64(6))
    x, dy = stored(rng, (2, 3, 21, 128), "f32"), stored(rng, (2, 21, 384), "f32")
    x = np.asarray(x, np.float32) * np.float32(2.0 ** -65)
    w = (1 + 0.3 * rng.standard_normal(384)).astype(np.float32)
    y = sfda.group_norm(f32(x), f32(w), eps=0.0)
    got = sfda.group_norm_bwd(f32(dy), f32(x), f32(w), eps=0.0)
    torch.cuda.synchronize()
    assert rel_err(y.double().cpu().numpy(), O.group_norm(x, w, eps=0.0)) <= SUM
    ref = O.group_norm_backward(dy, x, w, eps=0.0)
    assert all(rel_err(got[n].double().cpu().numpy(), ref[n]) <= SUM for n in ("dx", "dweight"))


def test_group_norm_bwd_many_channels():
    """2^29 channels in all: more sums of weight gradients than one launch has places for.  One token: dweight = dy x^, dbias = dy."""
    import torch
    from paper_2607_11897_amd import sfda
    say("group_norm_bwd 2^29 channels")
    H, D = 1 << 18, 2048
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(1, H, 1, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    dy = torch.randn(1, 1, H * D, generator=gen, device="cuda", dtype=torch.bfloat16)
    w = torch.ones(H * D, device="cuda")
    got = sfda.group_norm_bwd(dy, x, w, w)
    torch.cuda.synchronize()
    del w
    assert torch.equal(got["dbias"], dy.view(-1).float())
    for lo in range(0, H, H // 16):
        rows = slice(lo, lo + H // 16)
        f = x[0, rows, 0].double()
        f = (f - f.mean(-1, keepdim=True)) / (f.var(-1, unbiased=False, keepdim=True) + 1e-5).sqrt()
        want = f * dy.view(H, D)[rows].double()
        assert float((got["dweight"].view(H, D)[rows].double() - want).abs().max()) <= SUM * float(want.abs().max())


# --------------------------------------------------------------------------- streams and graphs

def test_other_stream_and_graph():
    """On a stream given by the caller, and captured into a graph that is replayed between eager work."""
    import torch
    from paper_2607_11897_amd import sfda
    say("stream and graph")
    x = attn(51, 2, 3, 700, 32, 48, "bf16")
    q, k, v = (f32(x[n]).to(torch.bfloat16) for n in "qkv")
    g, S0 = f32(x["g"]), f32(x["S0"])
    cos, sin = sfda.rotary_tables(700, 32)

    def layer(stream=None):
        a, b = sfda.rotary(q, k, cos, sin, stream=stream)
        o, S = sfda.decay_attn_fwd(a, b, v, g, S0, stream=stream)
        return o, S, sfda.group_norm(o, activation="silu", stream=stream)
    want = layer()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = layer(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer()
    for i in range(3):
        q.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        eager = layer()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, held)), i

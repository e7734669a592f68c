"""Refusals of the gated delta block's operators: the C entry points' argument checks (no pointer is dereferenced, nothing is
launched) and the binding's (CPU only)."""
from __future__ import annotations

import ctypes

import pytest

from gpu_util import ensure_built

A = 1 << 28


@pytest.fixture(scope="module")
def lib():
    return ensure_built()


def arr(*x, t=ctypes.c_longlong):
    return (t * len(x))(*x)


def fwd(lib, **kw):
    a = dict(q=A, k=2 * A, v=3 * A, g=4 * A, b=5 * A, n=None, S0=6 * A, o=7 * A, S_T=8 * A, B=1, H=4, Hk=2, T=8, dk=16, dv=8, strides=None, dt=0,
             ws=9 * A, nws=1 << 24) | kw
    return lib.sfda_delta_attn_fwd(*(a[x] for x in ("q", "k", "v", "g", "b", "n", "S0", "o", "S_T", "B", "H", "Hk", "T", "dk", "dv")), 1.0,
                                   a["strides"], a["dt"], a["ws"], a["nws"], None)


def bwd(lib, **kw):
    a = dict(q=A, k=2 * A, v=3 * A, g=4 * A, b=5 * A, n=None, S0=6 * A, dO=7 * A, dS_T=8 * A, dq=9 * A, dk_=10 * A, dv_=11 * A, dg=12 * A,
             db=13 * A, dS0=14 * A, B=1, H=4, Hk=2, T=8, dk=16, dv=8, strides=None, dt=0, ws=15 * A, nws=1 << 27) | kw
    return lib.sfda_delta_attn_bwd(*(a[x] for x in ("q", "k", "v", "g", "b", "n", "S0", "dO", "dS_T", "dq", "dk_", "dv_", "dg", "db", "dS0", "B",
                                                   "H", "Hk", "T", "dk", "dv")), 1.0, a["strides"], a["dt"], a["ws"], a["nws"], None)


def test_delta_attn_fwd(lib):
    assert fwd(lib, dt=2) == 4
    for bad in (dict(B=-1), dict(H=-1), dict(Hk=-1), dict(Hk=3), dict(Hk=0), dict(H=2, Hk=4), dict(T=-1), dict(dk=0), dict(dk=257), dict(dv=0),
                dict(dv=257), dict(B=1 << 20, H=1 << 10, Hk=1), dict(T=(1 << 31) - 1), dict(B=1 << 10, T=1 << 28), dict(nws=16)):
        assert fwd(lib, **bad) == 2, bad
        assert bad == dict(nws=16) or bwd(lib, **bad) == 2, bad
    for name in ("q", "k", "v", "g", "b", "o", "ws"):
        assert fwd(lib, **{name: None}) == 1, name
    assert fwd(lib, q=A + 2) == 5 and fwd(lib, g=4 * A + 1) == 5 and fwd(lib, b=5 * A + 2) == 5 and fwd(lib, S_T=8 * A + 2) == 5
    assert fwd(lib, ws=9 * A + 4) == 5 and fwd(lib, n=10 * A + 2) == 5
    # o over inputs, S_T partly over S0 and over o, the workspace over an input and an output
    for bad in (dict(o=A), dict(o=3 * A + 4), dict(o=4 * A), dict(o=5 * A), dict(S_T=6 * A + 16), dict(S_T=7 * A), dict(ws=2 * A), dict(ws=7 * A)):
        assert fwd(lib, **bad) == 6, bad
    assert fwd(lib, B=0, q=None) == 0 and fwd(lib, H=0, Hk=0, q=None) == 0


def test_delta_attn_strides(lib):
    # [B, T, heads, D] of q, k, v, log_decay, beta, o
    s = [8 * 2 * 16, 16, 2 * 16] * 2 + [8 * 4 * 8, 8, 4 * 8] + [8 * 4, 1, 4] * 2 + [8 * 4 * 8, 8, 4 * 8]
    for at, value, want in ((2, -1, 2), (0, 1 << 50, 2), (11, 1 << 62, 2), (16, 0, 6), (17, 24, 6), (5, 1 << 30, 2)):
        bad = list(s)
        bad[at] = value
        assert fwd(lib, strides=arr(*bad), B=2) == want, (at, value)
    t = list(s)
    t[9:12] = [0, 0, 0]                     # one log decay for all tokens is fine: its refusal comes from the workspace
    assert fwd(lib, strides=arr(*t), nws=0) == 2
    # o in the slice of a buffer behind v, one element into it
    p = s[:6] + [8 * 2 * 32, 8, 2 * 32] + s[9:15] + [8 * 2 * 32, 8, 2 * 32]
    assert fwd(lib, strides=arr(*p), o=3 * A + 31 * 4) == 6


def test_delta_attn_bwd(lib):
    assert bwd(lib, dt=-1) == 4
    for name in ("q", "k", "v", "g", "b", "dO", "dq", "dk_", "dv_", "dg", "db", "ws"):
        assert bwd(lib, **{name: None}) == 1, name
    for bad in (dict(dq=A), dict(dk_=9 * A), dict(dv_=7 * A), dict(dg=4 * A), dict(db=12 * A), dict(dS0=8 * A), dict(ws=9 * A), dict(ws=A)):
        assert bwd(lib, **bad) == 6, bad
    assert bwd(lib, dv_=11 * A + 2) == 5 and bwd(lib, ws=15 * A + 8) == 5 and bwd(lib, dg=12 * A + 2) == 5
    least = lib.sfda_delta_attn_bwd_workspace_bytes(1, 2, 1, 8, 16, 8, 0)
    assert bwd(lib, nws=least - 1) == 2 and bwd(lib, nws=0) == 2
    assert bwd(lib, H=0, Hk=0) == 0 and bwd(lib, B=0) == 0


def test_delta_attn_step(lib):
    def step(q=A, k=2 * A, v=3 * A, g=4 * A, b=5 * A, S=6 * A, o=7 * A, B=1, H=4, Hk=2, dk=16, dv=8, dt=0):
        return lib.sfda_delta_attn_step(q, k, v, g, b, S, o, B, H, Hk, dk, dv, 1.0, None, dt, None)
    assert step(dt=7) == 4
    for bad in (dict(dk=0), dict(dv=300), dict(B=-1), dict(Hk=3), dict(Hk=0)):
        assert step(**bad) == 2, bad
    for name in ("q", "k", "v", "g", "b", "S", "o"):
        assert step(**{name: None}) == 1, name
    assert step(S=A) == 6 and step(o=6 * A) == 6 and step(S=5 * A) == 6 and step(S=6 * A + 1) == 5 and step(B=0) == 0


def test_workspaces(lib):
    f, b = lib.sfda_delta_attn_fwd_workspace_bytes, lib.sfda_delta_attn_bwd_workspace_bytes
    assert f(0, 1, 64, 8, 8, 0) == 0 and f(1, 1, 0, 8, 8, 0) == 0 and f(1, 1, 64, 257, 8, 0) == 0 and f(1, 1, 64, 8, 8, 2) == 0 and f(-1, 1, 64, 8, 8, 0) == 0
    assert f(1, 2, 64, 8, 8, 0) == 2 * f(1, 1, 64, 8, 8, 0) > 0
    assert b(1, 4, 3, 64, 8, 8, 0) == 0 and b(2, 4, 2, 64, 8, 8, 1) > b(1, 2, 1, 64, 8, 8, 1) > 0
    # few heads over a long sequence: room for the segments' states
    assert f(1, 1, 1 << 15, 128, 128, 1) > f(1, 512, 1 << 15, 128, 128, 1) // 512
    M, N = (1 << 31) - 1, 1 << 30
    for B, H in ((M, M), (N, N), (1 << 22, N)):
        assert f(B, H, 4096, 16, 8, 0) == 0 and b(B, H, 1, 4096, 16, 8, 1) == 0
    g = lib.sfda_layer_norm_bwd_workspace_bytes
    assert g(2, 5, 16, 0) >= 2 * 16 * 4 and g(2, 5, 16385, 0) == 0 and g(2, 5, 16, 9) == 0 and g(0, 5, 16, 0) > 0


def test_more_heads_than_a_launch_takes(lib):
    """262144 heads: what is refused is the missing pointer behind the sizes.  A head that no launch takes is refused for its length,
    and its workspace, which 64 bits do not count, is 0."""
    z = ctypes.c_void_p(None)
    assert lib.sfda_delta_attn_step(z, 2 * A, 3 * A, 4 * A, 5 * A, 6 * A, 7 * A, 8192, 32, 32, 4, 4, 1.0, None, 0, None) == 1
    many = dict(B=8192, H=32, Hk=32, T=64, dk=4, dv=4, q=None)
    assert bwd(lib, **many) == 1 and bwd(lib, **(many | dict(H=64, Hk=1))) == 1
    assert bwd(lib, B=1, H=600000, Hk=1, T=64, dk=4, dv=4, q=None) == 2
    b = lib.sfda_delta_attn_bwd_workspace_bytes
    for Hk in (1, 600000):
        assert b(1, 600000, Hk, (1 << 31) - 1025, 256, 256, 0) == 0
    # forward: passes over as many heads as a launch takes, or as the workspace holds
    assert fwd(lib, **(many | dict(nws=1 << 40))) == 1 and fwd(lib, B=1, H=600000, Hk=1, T=64, dk=4, dv=4, q=None) == 1
    assert fwd(lib, T=(1 << 31) - 1025, nws=1 << 60, q=None) == 2
    one = lib.sfda_delta_attn_fwd_workspace_bytes(1, 4, 8, 16, 8, 0) // 4
    assert fwd(lib, nws=one - 1) == 2 and fwd(lib, nws=one, q=None) == 1
    assert b(8192, 32, 32, 64, 4, 4, 1) >= 200000 * b(1, 1, 1, 64, 4, 4, 1) - (200000 << 6)


def norm(lib, **kw):
    a = dict(x=A, w=2 * A, b=3 * A, r=4 * A, y=5 * A, t=6 * A, B=1, T=8, D=16, eps=1e-5, strides=None, dt=0) | kw
    return lib.sfda_layer_norm(*(a[x] for x in ("x", "w", "b", "r", "y", "t", "B", "T", "D")), a["eps"], a["strides"], a["dt"], None)


def norm_bwd(lib, **kw):
    a = dict(dy=A, x=2 * A, w=3 * A, d=4 * A, dx=5 * A, dw=6 * A, db=7 * A, B=1, T=8, D=16, eps=1e-5, strides=None, dt=0, ws=8 * A, nws=1 << 24) | kw
    return lib.sfda_layer_norm_bwd(*(a[x] for x in ("dy", "x", "w", "d", "dx", "dw", "db", "B", "T", "D")), a["eps"], a["strides"], a["dt"], a["ws"],
                                   a["nws"], None)


def test_layer_norm(lib):
    for f in (norm, norm_bwd):
        assert f(lib, dt=3) == 4
        for bad in (dict(D=0), dict(D=16385), dict(eps=-1.0), dict(eps=float("nan")), dict(T=-1), dict(B=-1)):
            assert f(lib, **bad) == 2, (f, bad)
    for name in ("x", "y", "t"):
        assert norm(lib, **{name: None}) == 1, name
    for bad in (dict(y=A), dict(y=4 * A), dict(y=6 * A), dict(t=A + 64), dict(t=2 * A), dict(y=3 * A)):
        assert norm(lib, **bad) == 6, bad
    # the stream in place with other strides; rows of y that lie in one place
    assert norm(lib, t=4 * A, strides=arr(128, 16, 128, 16, 128, 16, 256, 32)) == 6 and norm(lib, strides=arr(128, 16, 128, 16, 128, 0, 128, 16)) == 6
    assert norm(lib, x=A + 2) == 5 and norm(lib, w=2 * A + 1) == 5 and norm(lib, T=0, x=None) == 0 and norm(lib, B=0) == 0
    for name in ("dy", "x", "dx", "ws"):
        assert norm_bwd(lib, **{name: None}) == 1, name
    for bad in (dict(dx=2 * A), dict(dx=A + 4), dict(dw=7 * A), dict(ws=5 * A), dict(db=3 * A)):
        assert norm_bwd(lib, **bad) == 6, bad
    assert norm_bwd(lib, nws=16) == 2 and norm_bwd(lib, T=0, dw=None, db=None) == 0


def rot(lib, **kw):
    a = dict(q=A, k=2 * A, cos=3 * A, sin=4 * A, pos=7 * A, bits=32, astride=8, pstride=0, sections=(2, 1, 1), axes=None, qo=5 * A, ko=6 * A, B=1,
             Hq=2, Hk=2, T=8, D=16, P=32, strides=None, dt=0) | kw
    n = a["axes"] if a["axes"] is not None else len(a["sections"])
    s = None if a["sections"] is None else arr(*a["sections"], t=ctypes.c_int)
    return lib.sfda_rotary_axes(a["q"], a["k"], a["cos"], a["sin"], a["pos"], a["bits"], a["astride"], a["pstride"], s, n, 0, a["qo"], a["ko"],
                                a["B"], a["Hq"], a["Hk"], a["T"], a["D"], a["P"], 0, 0, a["strides"], a["dt"], None)


def test_rotary_axes(lib):
    assert rot(lib, dt=2) == 4
    for bad in (dict(sections=(0, 0)), dict(sections=(9,)), dict(sections=(4, 5)), dict(sections=(-1, 3)), dict(sections=(1,) * 5), dict(axes=0),
                dict(bits=16), dict(astride=-1), dict(pstride=-1), dict(T=-1), dict(P=0), dict(D=5000), dict(sections=((1 << 31) - 1, 2)),
                dict(astride=1 << 62, B=2)):
        assert rot(lib, **bad) == 2, bad
    for name in ("q", "cos", "sin", "pos", "qo", "ko"):
        assert rot(lib, **{name: None}) == 1, name
    assert rot(lib, sections=None, axes=3) == 1
    assert rot(lib, pos=7 * A + 2) == 5 and rot(lib, pos=7 * A + 4, bits=64) == 5 and rot(lib, qo=2 * A) == 6 and rot(lib, qo=7 * A) == 6
    assert rot(lib, T=0) == 0 and rot(lib, B=0, q=None) == 0


def test_binding(lib):
    import torch
    from paper_2607_11897_amd import sfda
    B, H, Hk, T, dk, dv = 1, 4, 2, 8, 16, 8
    q, k, v = torch.zeros(B, Hk, T, dk), torch.zeros(B, Hk, T, dk), torch.zeros(B, H, T, dv)
    g = torch.zeros(B, H, T)
    for call, error, match in (
            (lambda: sfda.delta_attn_fwd(q, k, v, g, g), ValueError, "GPU tensor"),
            (lambda: sfda.delta_attn_fwd(q, k, v[:, :3], g, g), ValueError, "multiple"),
            (lambda: sfda.delta_attn_fwd(q[:, :0], k[:, :0], v, g, g), ValueError, "multiple"),
            (lambda: sfda.delta_attn_fwd(q, k, v, g[:, :2], g), ValueError, "shape"),
            (lambda: sfda.delta_attn_fwd(q, k, v, g, g[..., :4]), ValueError, "shape"),
            (lambda: sfda.delta_attn_fwd(q, k, v, g.bfloat16(), g), TypeError, "log_decay must be float32"),
            (lambda: sfda.delta_attn_fwd(q, k, v, g, g.double()), TypeError, "beta must be float32"),
            (lambda: sfda.delta_attn_fwd(q, k.bfloat16(), v, g, g), TypeError, "k must be"),
            (lambda: sfda.delta_attn_fwd(q, k, v, g, g, lengths=torch.zeros(B, dtype=torch.int64)), TypeError, "lengths must be int32"),
            (lambda: sfda.delta_attn_bwd(q, k, v, g, g, None, q), ValueError, "shape"),
            (lambda: sfda.delta_attn_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], g[..., 0], g[..., 0], torch.zeros(B, H, dk, dv + 1)), ValueError, "shape"),
            (lambda: sfda.layer_norm(q), ValueError, "3 dimensions"),
            (lambda: sfda.layer_norm(q[0], weight=torch.zeros(dk + 1)), ValueError, "shape"),
            (lambda: sfda.layer_norm(q[0], residual=q[0].bfloat16()), TypeError, "residual must be"),
            (lambda: sfda.layer_norm_bwd(q[0], k[0, :1]), ValueError, "shape"),
            (lambda: sfda.rotary_axes(q, k, torch.zeros(9, 4), torch.zeros(9, 4), torch.zeros(2, T, dtype=torch.int32), (1, 2)), ValueError, "add up"),
            (lambda: sfda.rotary_axes(q, k, torch.zeros(9, 4), torch.zeros(9, 4), torch.zeros(2, T), (2, 2)), TypeError, "positions"),
            (lambda: sfda.rotary_axes(q, k, torch.zeros(9, 4), torch.zeros(9, 4), torch.zeros(3, T, dtype=torch.int32), (2, 2)), ValueError, "shape")):
        with pytest.raises(error, match=match):
            call()

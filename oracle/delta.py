"""The operators of a block of gated delta attention from their definitions, in float64 numpy: linear attention with the gated
delta rule (forward and backward), layer norm with the residual sum before it (forward and backward), rotary positions
with several axes."""
from __future__ import annotations

import numpy as np

from .layer import _lengths, _pairs


def _shared(x, H):
    """Queries or keys [B,Hk,...], once for each value head."""
    return np.repeat(np.asarray(x, np.float64), H // x.shape[1], axis=1)


def delta_attn(q, k, v, log_decay, beta, S0=None, scale=1.0, lengths=None):
    """S_t = a_t S_(t-1) + k_t u_t^T, u_t = beta_t (v_t - a_t S_(t-1)^T k_t), o_t = scale S_t^T q_t: (o, S at each length)."""
    v, a, beta = np.asarray(v, np.float64), np.exp(np.asarray(log_decay, np.float64)), np.asarray(beta, np.float64)
    B, H, T, dv = v.shape
    q, k = _shared(q, H), _shared(k, H)
    n = _lengths(lengths, B, T)
    o = np.zeros((B, H, T, dv))
    S = np.zeros((B, H, k.shape[-1], dv)) if S0 is None else np.asarray(S0, np.float64).copy()
    for b in range(B):
        for t in range(n[b]):
            S[b] *= a[b, :, t, None, None]
            u = beta[b, :, t, None] * (v[b, :, t] - np.einsum("hkv,hk->hv", S[b], k[b, :, t]))
            S[b] += k[b, :, t, :, None] * u[:, None]
            o[b, :, t] = scale * np.einsum("hkv,hk->hv", S[b], q[b, :, t])
    return o, S


def delta_attn_backward(q, k, v, log_decay, beta, S0, dO, dS_T=None, scale=1.0, lengths=None):
    """Gradients of L through delta_attn by the reverse sweep over its tokens."""
    Hk = np.shape(q)[1]
    v, dO, beta = (np.asarray(x, np.float64) for x in (v, dO, beta))
    a = np.exp(np.asarray(log_decay, np.float64))
    B, H, T, dv_ = v.shape
    q, k = _shared(q, H), _shared(k, H)
    dk_ = k.shape[-1]
    n = _lengths(lengths, B, T)
    zero = np.zeros((B, H, dk_, dv_))
    dS0 = zero.copy() if dS_T is None else np.asarray(dS_T, np.float64).copy()
    dq, dk, dv, dg, db = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros((B, H, T)), np.zeros((B, H, T))
    for b in range(B):
        S = [zero[b] if S0 is None else np.asarray(S0[b], np.float64)]
        for t in range(n[b]):
            held = S[-1] * a[b, :, t, None, None]
            u = beta[b, :, t, None] * (v[b, :, t] - np.einsum("hkv,hk->hv", held, k[b, :, t]))
            S.append(held + k[b, :, t, :, None] * u[:, None])
        U = dS0[b]
        for t in range(n[b] - 1, -1, -1):
            kt, held = k[b, :, t], S[t] * a[b, :, t, None, None]
            lack = v[b, :, t] - np.einsum("hkv,hk->hv", held, kt)
            dq[b, :, t] = scale * np.einsum("hkv,hv->hk", S[t + 1], dO[b, :, t])
            U = U + scale * q[b, :, t, :, None] * dO[b, :, t, None]
            du = np.einsum("hkv,hk->hv", U, kt)
            db[b, :, t] = (du * lack).sum(-1)
            dv[b, :, t] = beta[b, :, t, None] * du
            dk[b, :, t] = np.einsum("hkv,hv->hk", U, beta[b, :, t, None] * lack) - np.einsum("hkv,hv->hk", held, dv[b, :, t])
            U = U - kt[:, :, None] * dv[b, :, t, None]
            dg[b, :, t] = (U * held).sum((-1, -2))
            U = U * a[b, :, t, None, None]
        dS0[b] = U
    dq, dk = (x.reshape(B, Hk, H // Hk, T, dk_).sum(2) for x in (dq, dk))
    return dict(dq=dq, dk=dk, dv=dv, dlog_decay=dg, dbeta=db, dS0=dS0)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """x [B,T,D] (the total) -> y."""
    return _normal(x, eps)[0] * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)


def _normal(x, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(-1, keepdims=True)
    std = np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    return (x - mean) / std, std


def layer_norm_backward(dy, x, weight=None, bias=None, dtotal=None, eps=1e-5):
    xn, std = _normal(x, eps)
    dy = np.asarray(dy, np.float64)
    g = dy * (1.0 if weight is None else weight)
    dx = (g - g.mean(-1, keepdims=True) - xn * (g * xn).mean(-1, keepdims=True)) / std
    return dict(dx=dx if dtotal is None else dx + dtotal, dweight=None if weight is None else (dy * xn).sum((0, 1)),
                dbias=None if bias is None else dy.sum((0, 1)))


def axis_of_pair(sections, cyclic=False):
    """The axis that each pair follows: in runs, or dealt in turn to the axes that lack some."""
    if not cyclic:
        return np.repeat(np.arange(len(sections)), sections)
    return np.array([a for i in range(max(sections)) for a, n in enumerate(sections) if i < n])


def rotary_axes(x, cos, sin, positions, sections, cyclic=False, interleaved=False, inverse=False):
    """x [B,H,T,D] turned by the tables' rows positions[axis of the pair], positions [A,T] or [A,B,T]."""
    x = np.asarray(x, np.float64)
    half = cos.shape[1]
    a, b = _pairs(x.shape[-1], 2 * half, interleaved)
    at = np.asarray(positions)
    at = np.broadcast_to(at if at.ndim == 3 else at[:, None], (len(sections), x.shape[0], x.shape[2]))
    rows = at[axis_of_pair(sections, cyclic)].transpose(1, 2, 0)
    c, s = (np.asarray(t, np.float64)[rows, np.arange(half)][:, None] for t in (cos, sin))
    if inverse:
        s = -s
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y

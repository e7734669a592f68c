"""The operators around the attention from their definitions, in float64 numpy: rotary positions,
linear attention with one decay for each head (forward and backward), group norm with an activation
or a gate (forward and backward)."""
from __future__ import annotations

import numpy as np


def _pairs(D, rot, interleaved):
    """The channels (a, b) of each pair."""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotary(x, cos, sin, positions, interleaved=False, inverse=False):
    """x [B,H,T,D] turned by the rows `positions` [T] or [B,T] of cos, sin [P, rot/2]."""
    x = np.asarray(x, np.float64)
    a, b = _pairs(x.shape[-1], 2 * cos.shape[1], interleaved)
    at = np.broadcast_to(np.asarray(positions), (x.shape[0], x.shape[2]))
    c, s = (np.asarray(t, np.float64)[at][:, None] for t in (cos, sin))
    if inverse:
        s = -s
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def _lengths(lengths, B, T):
    return np.full(B, T) if lengths is None else np.clip(np.asarray(lengths), 0, T)


def decay_attn(q, k, v, log_decay, S0=None, scale=1.0, lengths=None):
    """S_t = exp(log_decay) S_(t-1) + k_t v_t^T, o_t = scale S_t^T q_t: (o, S at each sequence's length)."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    B, H, T, dk = q.shape
    dv = v.shape[-1]
    lam = np.exp(np.asarray(log_decay, np.float64))
    n = _lengths(lengths, B, T)
    o = np.zeros((B, H, T, dv))
    S = np.zeros((B, H, dk, dv)) if S0 is None else np.asarray(S0, np.float64).copy()
    for b in range(B):
        for h in range(H):
            for t in range(n[b]):
                S[b, h] = lam[h] * S[b, h] + np.outer(k[b, h, t], v[b, h, t])
                o[b, h, t] = scale * (q[b, h, t] @ S[b, h])
    return o, S


def decay_attn_backward(q, k, v, log_decay, S0, dO, dS_T=None, scale=1.0, lengths=None):
    """Gradients of L through decay_attn by the reverse sweep over its tokens."""
    q, k, v, dO = (np.asarray(x, np.float64) for x in (q, k, v, dO))
    B, H, T, dk_ = q.shape
    lam = np.exp(np.asarray(log_decay, np.float64))
    n = _lengths(lengths, B, T)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    zero = np.zeros((B, H, dk_, v.shape[-1]))
    dS0 = zero.copy() if dS_T is None else np.asarray(dS_T, np.float64).copy()
    for b in range(B):
        for h in range(H):
            S = zero[b, h] if S0 is None else np.asarray(S0[b, h], np.float64)
            for t in range(n[b]):
                S = lam[h] * S + np.outer(k[b, h, t], v[b, h, t])
                dq[b, h, t] = scale * (S @ dO[b, h, t])
            G = dS0[b, h]                                   # dL/dS_t
            for t in range(n[b] - 1, -1, -1):
                G = G + scale * np.outer(q[b, h, t], dO[b, h, t])
                dk[b, h, t] = G @ v[b, h, t]
                dv[b, h, t] = G.T @ k[b, h, t]
                G = lam[h] * G
            dS0[b, h] = G
    return dict(dq=dq, dk=dk, dv=dv, dS0=dS0)


def _act(z, activation):
    if activation == "none":
        return z, np.ones_like(z)
    s = 1.0 / (1.0 + np.exp(-z))
    return z * s, s * (1.0 + z * (1.0 - s))


def group_norm(x, weight=None, bias=None, gate=None, activation="none", eps=1e-5):
    """x [B,H,T,D] -> [B,T,H*D]: n = x^ weight + bias, act(n) or n act(gate)."""
    n, _, _ = _normal(x, weight, bias, eps)
    if gate is None:
        return _act(n, activation)[0]
    return n * _act(np.asarray(gate, np.float64), activation)[0]


def _normal(x, weight, bias, eps):
    x = np.asarray(x, np.float64)
    B, H, T, D = x.shape
    mean = x.mean(-1, keepdims=True)
    std = np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    xn = ((x - mean) / std).transpose(0, 2, 1, 3).reshape(B, T, H * D)
    n = xn * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)
    return n, xn, std


def group_norm_backward(dy, x, weight=None, bias=None, gate=None, activation="none", eps=1e-5):
    B, H, T, D = np.shape(x)
    dy = np.asarray(dy, np.float64)
    n, xn, std = _normal(x, weight, bias, eps)
    f, df = _act(n if gate is None else np.asarray(gate, np.float64), activation)
    dn = dy * (df if gate is None else f)
    g = (dn * (1.0 if weight is None else weight)).reshape(B, T, H, D).transpose(0, 2, 1, 3)
    y = xn.reshape(B, T, H, D).transpose(0, 2, 1, 3)
    dx = (g - g.mean(-1, keepdims=True) - y * (g * y).mean(-1, keepdims=True)) / std
    return dict(dx=dx, dgate=None if gate is None else dy * n * df,
                dweight=None if weight is None else (dn * xn).sum((0, 1)), dbias=None if bias is None else dn.sum((0, 1)))

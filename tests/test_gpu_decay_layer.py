"""The layer of examples/decay_layer.py: its operators together, against the same layer in plain float64 torch, decoding
against whole sequences, and training."""
from __future__ import annotations

import os
import sys

import pytest

from gpu_util import ROOT, ensure_built

sys.path.insert(0, os.path.join(ROOT, "examples"))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return ensure_built()


def plain(layer, w, x):
    """The layer with autograd, token by token."""
    import torch
    B, T, _ = x.shape
    H, R = layer.heads, layer.dk
    q, k, v = (x @ w[n] for n in ("wq", "wk", "wv"))
    q, k, v = (t.view(B, T, H, -1).transpose(1, 2) for t in (q, k, v))
    c, s = layer.cos[:T].double(), layer.sin[:T].double()

    def turn(t):
        a, b = t[..., :R // 2], t[..., R // 2:]
        return torch.cat((a * c - b * s, a * s + b * c), -1)
    q, k = turn(q), turn(k)
    S = torch.zeros(B, H, layer.dk, layer.dv, dtype=torch.float64, device=x.device)
    o = []
    for t in range(T):
        S = torch.exp(layer.log_decay.double())[:, None, None] * S + k[:, :, t, :, None] * v[:, :, t, None, :]
        o.append(layer.scale * (S * q[:, :, t, :, None]).sum(2))
    o = torch.stack(o, 2)
    o = (o - o.mean(-1, keepdim=True)) / (o.var(-1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    n = o.transpose(1, 2).reshape(B, T, -1) * w["norm_w"] + w["norm_b"]
    g = x @ w["wg"]
    return (n * g * torch.sigmoid(g)) @ w["wo"]


def test_gradients_match_autograd():
    """float32: every sum is of a few hundred float32 terms (2e-5 of the largest, as each operator's own bar), through
    three products and the norm's division: 2e-4."""
    import torch
    from decay_layer import DecayLayer
    layer = DecayLayer(64, 3, 32, 48, dtype=torch.float32, seed=3)
    x = torch.randn(2, 70, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    dy = torch.randn(2, 70, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    y, _, kept = layer.forward(x)
    grads, dx = layer.backward(dy, kept)
    w = {n: t.double().requires_grad_() for n, t in layer.weights.items()}
    x64 = x.double().requires_grad_()
    ref = plain(layer, w, x64)
    ref.backward(dy.double())

    def err(a, b):
        return float((a.double() - b).abs().max() / b.abs().max())
    assert err(y, ref.detach()) <= 2e-4
    assert err(dx, x64.grad) <= 2e-4
    for n, t in w.items():
        assert err(grads[n], t.grad) <= 2e-4, n


@pytest.mark.parametrize("dtype,bar", [("float32", 1e-4), ("bfloat16", 5e-2)])
def test_decoding_continues_prompts(dtype, bar):
    """Tokens after prompts of different lengths give what the whole sequences give (bfloat16: every activation is rounded
    to 2^-8 on both sides, some of them differently: a handful of such roundings)."""
    import torch
    from decay_layer import decode
    one, whole = decode(B=3, T=150, new=5, dtype=getattr(torch, dtype))
    assert float((one.float() - whole.float()).abs().max()) <= bar * float(whole.float().abs().max())


def test_training_learns():
    from decay_layer import train
    losses = train(steps=25)
    assert losses[-1] < 0.9 * losses[0] and all(b < 1.5 * losses[0] for b in losses)


def test_training_learns_to_remember():
    """The wanted outputs have variance 1 and say nothing about their own tokens' inputs: without memory zeros are best, a loss of
    about 1.  Weights that only shrink the output, or gradients of queries, keys or values that are wrong, stay there."""
    from decay_layer import train
    losses = train()
    assert sum(losses[-10:]) / 10 < 0.7 and all(b < 1.5 * losses[0] for b in losses)

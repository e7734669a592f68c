"""The block of examples/delta_block.py: its operators together, against the same block in plain float64 torch with autograd, against
differences, and decoding against whole sequences."""
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


def plain(block, w, x, stream, at):
    """The block with autograd, token by token: y and the new stream."""
    import torch
    import torch.nn.functional as F
    B, T, _ = x.shape
    H, Hk = block.heads, block.key_heads
    total = x + stream
    h = (total - total.mean(-1, keepdim=True)) / (total.var(-1, unbiased=False, keepdim=True) + 1e-5).sqrt() * w["ln_w"] + w["ln_b"]
    q, k, v = ((h @ w[n]).view(B, T, -1, d).transpose(1, 2) for n, d in (("wq", block.dk), ("wk", block.dk), ("wv", block.dv)))
    q, k = (t * torch.rsqrt(t.square().sum(-1, keepdim=True) + 1e-6) for t in (q, k))
    axis = torch.tensor([a for a, n in enumerate(block.sections) for _ in range(n)], device=x.device)
    R = len(axis)
    c, s = (t.double()[at.long()[axis].T, torch.arange(R, device=x.device)] for t in (block.cos, block.sin))

    def turn(t):
        a, b = t[..., :R], t[..., R:2 * R]
        return torch.cat((a * c - b * s, a * s + b * c, t[..., 2 * R:]), -1)
    q, k = (turn(t).repeat_interleave(H // Hk, dim=1) for t in (q, k))
    decay = torch.exp(-w["a"].exp() * F.softplus(h @ w["wa"])).transpose(1, 2)
    beta = torch.sigmoid(h @ w["wb"]).transpose(1, 2)
    S, o = torch.zeros(B, H, block.dk, block.dv, dtype=torch.float64, device=x.device), []
    for t in range(T):
        S = S * decay[:, :, t, None, None]
        u = beta[:, :, t, None] * (v[:, :, t] - (S * k[:, :, t, :, None]).sum(2))
        S = S + k[:, :, t, :, None] * u[:, :, None]
        o.append(block.scale * (S * q[:, :, t, :, None]).sum(2))
    o = torch.stack(o, 2)
    o = (o - o.mean(-1, keepdim=True)) / (o.var(-1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    n = o.transpose(1, 2).reshape(B, T, -1) * w["norm_w"] + w["norm_b"]
    g = h @ w["wg"]
    return (n * g * torch.sigmoid(g)) @ w["wo"], total


def test_gradients_match_autograd():
    """float32: every sum is of a few hundred float32 terms (2e-5 of the largest, as each operator's own bar), through
    four products and two norms' divisions, of which that of small outputs multiplies errors by up to a few: 5e-4."""
    import torch
    from delta_block import DeltaBlock, video
    block = DeltaBlock(64, 4, 2, 64, 40, (8, 12, 10), dtype=torch.float32, seed=3)
    at = video(3, 5, 5)
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, stream, dy, ds = (torch.randn(2, at.shape[1], 64, device="cuda", generator=gen) for _ in range(4))
    y, total, _, kept = block.forward(x, stream, at)
    grads, dx = block.backward(dy, ds, kept)
    w = {n: t.double().requires_grad_() for n, t in block.weights.items()}
    x64 = x.double().requires_grad_()
    ref, stream64 = plain(block, w, x64, stream.double(), at)
    ((ref * dy).sum() + (stream64 * ds).sum()).backward()

    def off(a, b):
        return float((a.double() - b).abs().max() / b.abs().max())
    assert off(y, ref.detach()) <= 5e-4 and off(total, stream64.detach()) <= 1e-6
    for n, t in w.items():
        assert off(grads[n], t.grad) <= 5e-4, n
    assert off(dx, x64.grad) <= 5e-4


def test_gradients_match_differences():
    """A central difference is off by h^2 / 6 of the third derivative along the direction (steps of 0.05 x 0.02 of the weights) and by
    the float32 losses' rounding over h: within a hundredth of a derivative of the size of the gradients' product with it."""
    from delta_block import difference
    got, want = difference()
    assert abs(got - want) <= 1e-2 * max(abs(got), abs(want))


def test_decoding_matches_whole_sequences():
    """bfloat16: outputs of the attention 2e-2 off each way, as its own bar, divided by the norm and through a product whose terms
    have either sign: 6e-2 of the largest."""
    from delta_block import decode
    one, whole = decode()
    assert float((one.float() - whole.float()).abs().max()) <= 6e-2 * float(whole.float().abs().max())

"""A layer of linear attention with one decay for each head, from the library's operators: rotary positions,
the attention, the head-wise norm with its gate.  For training (forward and the gradients of all its weights), for
prompts of different lengths and for single tokens.  Projections are torch products.

    python examples/decay_layer.py

runs all three: some steps of training on a task that needs memory, then prompts and decoding.
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_11897_amd import sfda  # noqa: E402

EPS = 1e-5


class DecayLayer:
    """y = Wo (norm(attention(rotary(Wq x), rotary(Wk x), Wv x)) * silu(Wg x)).  Head h remembers about 2^(3 + 9 h / (H - 1))
    tokens."""

    def __init__(self, width: int, heads: int, dk: int, dv: int, positions: int = 4096, dtype=torch.bfloat16, device="cuda", seed: int = 0):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.dk, self.dv, self.scale = heads, dk, dv, dk ** -0.5
        shapes = dict(wq=(width, heads * dk), wk=(width, heads * dk), wv=(width, heads * dv), wg=(width, heads * dv), wo=(heads * dv, width))
        self.weights = {n: (torch.randn(s, generator=gen, device=device) / math.sqrt(s[0])).to(dtype) for n, s in shapes.items()}
        self.weights["norm_w"] = torch.ones(heads * dv, device=device)
        self.weights["norm_b"] = torch.zeros(heads * dv, device=device)
        reach = 2.0 ** (3.0 + 9.0 * torch.arange(heads, device=device) / max(heads - 1, 1))
        self.log_decay = torch.log1p(-1.0 / reach).float()
        self.cos, self.sin = sfda.rotary_tables(positions, dk, device=device)

    def _split(self, x, d):
        """[B, T, H d] -> [B, H, T, d], a view."""
        return x.view(*x.shape[:2], self.heads, d).transpose(1, 2)

    def forward(self, x, state=None, lengths=None, offset: int = 0):
        """x [B, T, width] -> (y, state after each sequence's last token, what backward needs)."""
        w = self.weights
        q, k, v = self._split(x @ w["wq"], self.dk), self._split(x @ w["wk"], self.dk), self._split(x @ w["wv"], self.dv)
        gate = x @ w["wg"]
        sfda.rotary(q, k, self.cos, self.sin, offset=offset, q_out=q, k_out=k)          # in place
        o, after = sfda.decay_attn_fwd(q, k, v, self.log_decay, state, scale=self.scale, lengths=lengths)
        h = sfda.group_norm(o, w["norm_w"], w["norm_b"], gate, activation="silu", eps=EPS)
        return h @ w["wo"], after, (x, q, k, v, gate, o, h, state, lengths, offset)

    def backward(self, dy, kept):
        """Gradients of the weights and of x, given dy = dL/dy."""
        w = self.weights
        x, q, k, v, gate, o, h, state, lengths, offset = kept
        B, T, _ = x.shape
        flat = lambda t: t.reshape(B * T, -1)  # noqa: E731
        g = {"wo": flat(h).T @ flat(dy)}
        n = sfda.group_norm_bwd(dy @ w["wo"].T, o, w["norm_w"], w["norm_b"], gate, activation="silu", eps=EPS)
        g["norm_w"], g["norm_b"] = n["dweight"], n["dbias"]
        # gradients straight into the projections' layout
        dq, dk, dv = (torch.empty(B, T, self.heads * d, dtype=x.dtype, device=x.device) for d in (self.dk, self.dk, self.dv))
        a, b, c = self._split(dq, self.dk), self._split(dk, self.dk), self._split(dv, self.dv)
        sfda.decay_attn_bwd(q, k, v, self.log_decay, state, n["dx"], scale=self.scale, lengths=lengths, want_dS0=False, dq=a, dk=b, dv=c)
        sfda.rotary(a, b, self.cos, self.sin, offset=offset, inverse=True, q_out=a, k_out=b)
        dx = 0
        for name, t in (("wq", dq), ("wk", dk), ("wv", dv), ("wg", n["dgate"])):
            g[name] = flat(x).T @ flat(t)
            dx = dx + t @ w[name].T
        return g, dx

    def step(self, x, state, positions):
        """One token of every sequence: x [B, width], positions [B] (int32); the state is updated in place."""
        w = self.weights
        B = x.shape[0]
        q, k, v = (t.view(B, self.heads, 1, -1) for t in (x @ w["wq"], x @ w["wk"], x @ w["wv"]))
        sfda.rotary(q, k, self.cos, self.sin, positions.view(B, 1), q_out=q, k_out=k)
        o = sfda.decay_attn_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], self.log_decay, state, scale=self.scale)
        h = sfda.group_norm(o.unsqueeze(2), w["norm_w"], w["norm_b"], (x @ w["wg"]).view(B, 1, -1), activation="silu", eps=EPS)
        return h[:, 0] @ w["wo"]


def train(steps: int = 120, B: int = 4, T: int = 192, width: int = 16, heads: int = 4, lag: int = 3, rate: float = 3e-2):
    """Adam on y_t = x_(t - lag) with new random x at every step: the losses.  Channel 0 of x is a constant, of which queries and keys
    that depend on the position only can be made; the others are what has to be remembered.  As x_t says nothing about x_(t - lag), a
    layer that carries nothing from token to token reaches 1 - lag / T at best, with zeros; a loss well below that is memory."""
    layer = DecayLayer(width, heads, 32, 32, dtype=torch.float32)
    gen = torch.Generator(device="cuda").manual_seed(1)
    moments = {n: (torch.zeros_like(w), torch.zeros_like(w)) for n, w in layer.weights.items()}
    losses = []
    for i in range(1, steps + 1):
        x = torch.randn(B, T, width, generator=gen, device="cuda")
        x[..., 0] = 2.0
        want = torch.roll(x, lag, 1)
        want[:, :lag] = 0
        y, _, kept = layer.forward(x)
        off = y - want
        off[..., 0] = 0
        count = off[..., 1:].numel()
        losses.append(float(off.square().sum() / count))
        grads, _ = layer.backward(off * (2.0 / count), kept)
        for name, g in grads.items():
            m, v = moments[name]
            m.mul_(0.9).add_(g, alpha=0.1)
            v.mul_(0.99).addcmul_(g, g, value=0.01)
            layer.weights[name] -= rate * (m / (1 - 0.9 ** i)) / ((v / (1 - 0.99 ** i)).sqrt() + 1e-8)
    return losses


def decode(B: int = 3, T: int = 300, new: int = 8, width: int = 256, heads: int = 4, dtype=torch.bfloat16):
    """Prompts of different lengths, then new tokens one by one: the outputs of both ways, token by token and the whole
    sequences at once, [B, new, width] each."""
    layer = DecayLayer(width, heads, 128, 128, dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(B, T + new, width, generator=gen, device="cuda").to(dtype)
    lengths = torch.tensor([T - 37 * b for b in range(B)], dtype=torch.int32, device="cuda")
    prompts = x[:, :T].contiguous()
    _, state, _ = layer.forward(prompts, lengths=lengths)
    at, one = lengths.clone(), []
    for _ in range(new):
        token = x[torch.arange(B, device="cuda"), at.long()]
        one.append(layer.step(token, state, at))
        at += 1
    whole, _, _ = layer.forward(x)
    rows = lengths.long()[:, None] + torch.arange(new, device="cuda")
    return torch.stack(one, 1), whole[torch.arange(B, device="cuda")[:, None], rows]


def main():
    losses = train()
    print("training: loss %.4f -> %.4f in %d steps (zeros: about 1)" % (losses[0], losses[-1], len(losses)))
    one, whole = decode()
    print("decoding: largest difference from the whole sequences %.2g of %.2g" % (float((one - whole).abs().max()), float(whole.abs().max())))


if __name__ == "__main__":
    main()

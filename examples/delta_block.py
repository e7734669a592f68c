"""A pre-norm block of gated delta attention, from the library's operators: the residual sum and the layer norm, rotary positions
with several axes (video tokens, or one axis for text), the gated delta rule with keys of length 1, the head-wise norm with its gate.
For training (forward and the gradients of all its weights), for prompts of different lengths and for single tokens. Projections are
torch products.

    python examples/delta_block.py

runs all three on random tokens: gradients against differences, then prompts and decoding.
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_11897_amd import sfda  # noqa: E402

EPS = 1e-5


class DeltaBlock:
    """stream' = stream + x;  h = LN(stream');  y = Wo (norm(delta(rotary(|Wq h|), rotary(|Wk h|), Wv h, g, beta)) * silu(Wg h)), with
    log decays g = -exp(a) softplus(Wa h) and strengths beta = sigmoid(Wb h); value heads share key heads in groups."""

    def __init__(self, width: int, heads: int, key_heads: int, dk: int, dv: int, sections=(16, 24, 24), positions: int = 4096,
                 dtype=torch.bfloat16, device="cuda", seed: int = 0):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.heads, self.key_heads, self.dk, self.dv, self.sections, self.scale = heads, key_heads, dk, dv, tuple(sections), dk ** -0.5
        shapes = dict(wq=(width, key_heads * dk), wk=(width, key_heads * dk), wv=(width, heads * dv), wg=(width, heads * dv),
                      wa=(width, heads), wb=(width, heads), wo=(heads * dv, width))
        self.weights = {n: (torch.randn(s, generator=gen, device=device) / math.sqrt(s[0])).to(dtype) for n, s in shapes.items()}
        f32 = dict(device=device, dtype=torch.float32)
        self.weights.update(ln_w=torch.ones(width, **f32), ln_b=torch.zeros(width, **f32), norm_w=torch.ones(heads * dv, **f32),
                            norm_b=torch.zeros(heads * dv, **f32), a=-torch.linspace(0, 6, heads, **f32))
        self.cos, self.sin = sfda.rotary_tables(positions, 2 * sum(self.sections), device=device)

    def _split(self, x, d):
        """[B, T, n d] -> [B, n, T, d], a view."""
        return x.view(*x.shape[:2], -1, d).transpose(1, 2)

    def _unit(self, x):
        """Heads of length 1, and what their gradient needs."""
        r = torch.rsqrt(x.float().square().sum(-1, keepdim=True) + 1e-6)
        return (x.float() * r).to(x.dtype), r

    @staticmethod
    def _unit_grad(dy, x, r):
        y, dy = x.float() * r, dy.float()
        return (r * (dy - y * (dy * y).sum(-1, keepdim=True))).to(x.dtype)

    def forward(self, x, stream, positions, state=None, lengths=None):
        """x, stream [B, T, width], positions [axes, T] or [axes, B, T] -> (y, stream', state after each sequence's last token,
        what backward needs)."""
        w = self.weights
        h, total = sfda.layer_norm(x, w["ln_w"], w["ln_b"], stream, eps=EPS)
        q0, k0, v = self._split(h @ w["wq"], self.dk), self._split(h @ w["wk"], self.dk), self._split(h @ w["wv"], self.dv)
        (q, rq), (k, rk) = self._unit(q0), self._unit(k0)
        sfda.rotary_axes(q, k, self.cos, self.sin, positions, self.sections, q_out=q, k_out=k)      # in place
        za, zb = (h @ w["wa"]).float(), (h @ w["wb"]).float()
        g, beta = -w["a"].exp() * torch.nn.functional.softplus(za), torch.sigmoid(zb)               # [B, T, heads]
        gate = h @ w["wg"]
        o, after = sfda.delta_attn_fwd(q, k, v, g.transpose(1, 2), beta.transpose(1, 2), state, scale=self.scale, lengths=lengths)
        n = sfda.group_norm(o, w["norm_w"], w["norm_b"], gate, activation="silu", eps=EPS)
        return n @ w["wo"], total, after, (total, h, q0, k0, rq, rk, q, k, v, za, g, beta, gate, o, n, positions, state, lengths)

    def backward(self, dy, dstream, kept):
        """Gradients of the weights, and of x (which is that of the stream too), given dL/dy and dL/dstream'."""
        w = self.weights
        total, h, q0, k0, rq, rk, q, k, v, za, g, beta, gate, o, n, positions, state, lengths = kept
        flat = lambda t: t.reshape(-1, t.shape[-1])  # noqa: E731
        grads = {"wo": flat(n).T @ flat(dy)}
        d = sfda.group_norm_bwd(dy @ w["wo"].T, o, w["norm_w"], w["norm_b"], gate, activation="silu", eps=EPS)
        grads["norm_w"], grads["norm_b"] = d["dweight"], d["dbias"]
        a = sfda.delta_attn_bwd(q, k, v, g.transpose(1, 2), beta.transpose(1, 2), state, d["dx"], scale=self.scale, lengths=lengths,
                                want_dS0=False)
        dq, dk = sfda.rotary_axes(a["dq"], a["dk"], self.cos, self.sin, positions, self.sections, inverse=True, q_out=a["dq"],
                                  k_out=a["dk"])
        dq, dk = self._unit_grad(dq, q0, rq), self._unit_grad(dk, k0, rk)
        dg, db = a["dlog_decay"].transpose(1, 2), a["dbeta"].transpose(1, 2)
        grads["a"] = (dg * g).sum((0, 1))
        dza, dzb = -dg * w["a"].exp() * torch.sigmoid(za), db * beta * (1 - beta)
        dh = 0
        for name, t in (("wq", dq), ("wk", dk), ("wv", a["dv"]), ("wg", d["dgate"]), ("wa", dza.to(h.dtype)), ("wb", dzb.to(h.dtype))):
            t = t.transpose(1, 2).flatten(2) if t.dim() == 4 else t
            grads[name] = flat(h).T @ flat(t)
            dh = dh + t @ w[name].T
        e = sfda.layer_norm_bwd(dh, total, w["ln_w"], w["ln_b"], dstream, eps=EPS)
        grads["ln_w"], grads["ln_b"] = e["dweight"], e["dbias"]
        return grads, e["dx"]

    def step(self, x, stream, positions, state):
        """One token of every sequence: x, stream [B, width], positions [axes, B]; the state is updated in place."""
        w = self.weights
        B = x.shape[0]
        h, total = sfda.layer_norm(x.unsqueeze(1), w["ln_w"], w["ln_b"], stream.unsqueeze(1), eps=EPS)
        q, k, v = self._split(h @ w["wq"], self.dk), self._split(h @ w["wk"], self.dk), self._split(h @ w["wv"], self.dv)
        (q, _), (k, _) = self._unit(q), self._unit(k)
        q, k = sfda.rotary_axes(q, k, self.cos, self.sin, positions.unsqueeze(-1), self.sections)
        g = -w["a"].exp() * torch.nn.functional.softplus((h @ w["wa"]).float())
        o = sfda.delta_attn_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], g[:, 0], torch.sigmoid((h @ w["wb"]).float())[:, 0], state,
                                 scale=self.scale)
        n = sfda.group_norm(o.unsqueeze(2), w["norm_w"], w["norm_b"], h @ w["wg"], activation="silu", eps=EPS)
        return (n @ w["wo"])[:, 0], total[:, 0]


def video(frames: int, rows: int, columns: int, device="cuda"):
    """Time, row and column of each of frames * rows * columns tokens: [3, T]."""
    t = torch.arange(frames * rows * columns, device=device, dtype=torch.int32)
    return torch.stack((t // (rows * columns), t // columns % rows, t % columns))


def difference(width: int = 96, seed: int = 1):
    """The derivative along a random direction of all weights, by the gradients and by differences: float32, one video."""
    block = DeltaBlock(width, 4, 2, 64, 48, (8, 12, 12), dtype=torch.float32, seed=seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    at = video(3, 5, 6)
    x, stream, dy, ds = (torch.randn(2, at.shape[1], width, generator=gen, device="cuda") for _ in range(4))
    y, total, _, kept = block.forward(x, stream, at)
    grads, _ = block.backward(dy, ds, kept)
    start = {n: t.clone() for n, t in block.weights.items()}
    way = {n: torch.randn(t.shape, generator=gen, device="cuda") * 0.02 for n, t in start.items()}
    h, side = 0.05, []
    for s in (h, -h):
        block.weights = {n: t + s * way[n] for n, t in start.items()}
        y, total, _, _ = block.forward(x, stream, at)
        side.append(float((y.double() * dy).sum() + (total.double() * ds).sum()))
    return float(sum((grads[n].double() * way[n]).sum() for n in way)), (side[0] - side[1]) / (2 * h)


def decode(B: int = 3, T: int = 300, new: int = 8, width: int = 256, dtype=torch.bfloat16):
    """Prompts of different lengths, then new tokens one by one: the outputs of both ways, token by token and the whole
    sequences at once, [B, new, width] each."""
    block = DeltaBlock(width, 4, 2, 128, 128, (32, 16, 16), dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, stream = (torch.randn(B, T + new, width, generator=gen, device="cuda").to(dtype) for _ in range(2))
    at = torch.arange(T + new, device="cuda", dtype=torch.int32).expand(3, -1).contiguous()         # text: the same on all axes
    lengths = torch.tensor([T - 37 * b for b in range(B)], dtype=torch.int32, device="cuda")
    _, _, state, _ = block.forward(x[:, :T], stream[:, :T], at[:, :T].contiguous(), lengths=lengths)
    rows, every, one = lengths.long(), torch.arange(B, device="cuda"), []
    for _ in range(new):
        y, _ = block.step(x[every, rows], stream[every, rows], rows.to(torch.int32).expand(3, -1).contiguous(), state)
        one.append(y)
        rows = rows + 1
    whole, _, _, _ = block.forward(x, stream, at)
    return torch.stack(one, 1), whole[every[:, None], lengths.long()[:, None] + torch.arange(new, device="cuda")]


def main():
    got, want = difference()
    print("gradients: along a random direction %.6g, by differences %.6g" % (got, want))
    one, whole = decode()
    print("decoding: largest difference from the whole sequences %.2g of %.2g" % (float((one - whole).abs().max()), float(whole.abs().max())))


if __name__ == "__main__":
    main()

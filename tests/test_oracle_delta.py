"""The float64 oracle of the gated delta block's operators, against what pins it: differences, an undecayed solve, single tokens,
autograd's gradients (CPU only)."""
from __future__ import annotations

import numpy as np
import pytest

from oracle import delta as O
from oracle import layer as OL


def inputs(seed, B=2, H=4, Hk=2, T=5, dk=3, dv=4):
    r = np.random.default_rng(seed)
    k = r.standard_normal((B, Hk, T, dk))
    return dict(q=r.standard_normal((B, Hk, T, dk)), k=k / np.linalg.norm(k, axis=-1, keepdims=True), v=r.standard_normal((B, H, T, dv)),
                log_decay=-r.random((B, H, T)), beta=r.random((B, H, T)), S0=r.standard_normal((B, H, dk, dv)))


def test_without_erasure_it_is_decay_attention():
    """Keys that are orthogonal to all others and states see nothing to erase."""
    r = np.random.default_rng(0)
    T = 4
    k = np.eye(T)[None, None]
    q, v = r.standard_normal((1, 1, T, T)), r.standard_normal((1, 1, T, 3))
    g = np.full((1, 1, T), -0.3)
    o, S = O.delta_attn(q, k, v, g, np.ones((1, 1, T)), scale=0.5)
    o2, S2 = OL.decay_attn(q, k, v, np.array([-0.3]), scale=0.5)
    assert np.allclose(o, o2, atol=1e-14) and np.allclose(S, S2, atol=1e-14)


def test_a_key_of_length_one_is_answered_with_its_value():
    x = inputs(1, T=7)
    x["beta"][:] = 1.0
    o, S = O.delta_attn(x["k"], x["k"], x["v"], x["log_decay"], x["beta"], x["S0"])
    assert np.allclose(o, x["v"], atol=1e-13)


@pytest.mark.parametrize("lengths", [None, [3, 0], [-2, 9]])
def test_backward_against_differences(lengths):
    x = inputs(2)
    r = np.random.default_rng(3)
    dO, dS = r.standard_normal(x["v"].shape), r.standard_normal(x["S0"].shape)

    def loss(y):
        o, S = O.delta_attn(**y, scale=0.7, lengths=lengths)
        return (o * dO).sum() + (S * dS).sum()
    got = O.delta_attn_backward(**{n: x[n] for n in ("q", "k", "v", "log_decay", "beta", "S0")}, dO=dO, dS_T=dS, scale=0.7, lengths=lengths)
    h = 1e-5
    for name in x:
        for at in [tuple(r.integers(0, s) for s in x[name].shape) for _ in range(12)]:
            up, down = ({n: y.copy() for n, y in x.items()} for _ in range(2))
            up[name][at] += h
            down[name][at] -= h
            d = (loss(up) - loss(down)) / (2 * h)
            # (a central difference is off by h^2 / 6 of a third derivative of some hundreds, and by rounding: 1e-16 of the loss over h)
            assert abs(got["d" + name][at] - d) < 1e-6, (name, at)


@pytest.mark.parametrize("affine", [False, True])
def test_layer_norm(affine):
    import torch
    r = np.random.default_rng(4)
    x, dy, dt = (r.standard_normal((2, 3, 7)) for _ in range(3))
    w, b = (r.standard_normal(7), r.standard_normal(7)) if affine else (None, None)
    leaf = {n: torch.tensor(y, requires_grad=True) for n, y in (("x", x), ("w", w), ("b", b)) if y is not None}
    y = torch.nn.functional.layer_norm(leaf["x"], (7,), leaf.get("w"), leaf.get("b"), 1e-5)
    assert np.allclose(O.layer_norm(x, w, b), y.detach().numpy(), atol=1e-13)
    (y * torch.tensor(dy)).sum().backward()
    got = O.layer_norm_backward(dy, x, w, b, dt)
    assert np.allclose(got["dx"], leaf["x"].grad.numpy() + dt, atol=1e-12)
    if affine:
        assert np.allclose(got["dweight"], leaf["w"].grad.numpy(), atol=1e-12) and np.allclose(got["dbias"], leaf["b"].grad.numpy(), atol=1e-12)


def test_rotary_axes():
    r = np.random.default_rng(5)
    x = r.standard_normal((2, 3, 4, 14))
    c, s = np.cos(r.standard_normal((9, 6))), np.sin(r.standard_normal((9, 6)))
    assert list(O.axis_of_pair((3, 1, 2), True)) == [0, 1, 2, 0, 2, 0] and list(O.axis_of_pair((1, 0, 2))) == [0, 2, 2]
    at = r.integers(0, 9, (4,))
    for cyclic in (False, True):        # the same position on all axes is one position
        y = O.rotary_axes(x, c, s, np.stack([at] * 3), (3, 1, 2), cyclic)
        assert np.allclose(y, OL.rotary(x, c, s, at))
    # an axis' pairs turn as its own positions say
    p = r.integers(0, 9, (3, 2, 4))
    y = O.rotary_axes(x, c, s, p, (3, 1, 2), interleaved=True)
    for a, chans in ((0, slice(0, 6)), (1, slice(6, 8)), (2, slice(8, 12))):
        assert np.allclose(y[..., chans], OL.rotary(x, c, s, p[a], True)[..., chans])

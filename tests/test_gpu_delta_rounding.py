"""What the gated delta rule's results lose beside their own rounding, for keys that are alike and strengths up to 2: there the terms
of an output alternate and cancel, and what each of them lost counts for more than in a sum of independent ones.

Bars, from the arithmetic:
  * bfloat16 outputs and gradients (root mean square): an operand in two bfloat16 parts is off by 2^-16 of itself at most (one part: 2^-8).
    With terms of up to 50 times the result in root mean square, sums are off by 8e-4 of it, under a half of the 0.0017 that
    rounding the result itself leaves, and errors that do not depend on each other add in squares: 1.1 times that rounding's.
  * float32 results, states of both types, gradients of decays, strengths and start states (largest error over the largest value, as
    everywhere): entries of the block's inverse are strengths times products of reflections, 2 at most, so that errors of its
    entries before (2^-24 of up to 2, in sums of 128 and then of 64 terms) reach a result as sums over pairs of tokens, 64^2 / 2 terms of
    either sign: 2^-24 x 4 x sqrt(2048) x 4 = 4.3e-5, 5e-5 with the sums of the products after it."""
from __future__ import annotations

import numpy as np
import pytest

from gpu_util import ensure_built, rel_err
from oracle import delta as O
from test_gpu_delta import names, run_bwd, run_fwd, say, stored_as
from test_gpu_layer import stored

pytestmark = pytest.mark.gpu
SUM = 5e-5
OWN = 1.1


@pytest.fixture(scope="module", autouse=True)
def lib():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return ensure_built()


def alike(seed, B, H, Hk, T, dk, dv, dtype, cosine, low, high, state, decay=0.0):
    """Keys and queries of length 1 around one direction of each key head, `cosine` between two of them; strengths of low to high."""
    rng = np.random.Generator(np.random.PCG64(seed))

    def unit(x):
        return x / np.linalg.norm(x, axis=-1, keepdims=True)
    common = unit(rng.standard_normal((B, Hk, 1, dk)))

    def around():
        return stored_as(unit(cosine ** 0.5 * common + (1 - cosine) ** 0.5 * unit(rng.standard_normal((B, Hk, T, dk)))), dtype)
    x = dict(q=around(), k=around(), v=stored(rng, (B, H, T, dv), dtype), log_decay=-decay * rng.random((B, H, T)),
             beta=low + (high - low) * rng.random((B, H, T)))
    for n in ("log_decay", "beta"):
        x[n] = x[n].astype(np.float32).astype(np.float64)
    x["S0"] = stored(rng, (B, H, dk, dv), "f32") if state else None
    x["dO"] = stored(rng, (B, H, T, dv), dtype)
    x["dS_T"] = stored(rng, (B, H, dk, dv), "f32") if state else None
    x["lengths"] = None
    return x


def off(x, ref):
    """Root mean square of the error, and of what rounding the reference leaves, over the reference's."""
    size = np.sqrt(np.mean(ref ** 2))
    return np.sqrt(np.mean((x - ref) ** 2)) / size, np.sqrt(np.mean((stored_as(ref, "bf16") - ref) ** 2)) / size


def close(name, x, ref, dtype, rounded):
    if dtype == "bf16" and rounded:
        error, own = off(x, ref)
        print("  %s %.5f of %.5f" % (name, error, own), flush=True)
        return error <= OWN * own
    print("  %s %.2e" % (name, rel_err(x, ref)), flush=True)
    return rel_err(x, ref) <= SUM


KEYS = [(0.0, 0.0, 1.0, 0.1), (0.8, 0.0, 1.0, 0.0), (0.8, 1.0, 2.0, 0.0), (0.98, 1.0, 2.0, 0.0), (0.98, 1.0, 2.0, 0.2)]
SIZES = [(1, 4, 2, 192, 128, 128, False), (1, 2, 2, 200, 128, 128, True), (2, 2, 1, 130, 64, 40, True), (1, 2, 1, 150, 200, 72, False),
         (1, 2, 2, 128, 256, 256, True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cosine,low,high,decay", KEYS)
@pytest.mark.parametrize("B,H,Hk,T,dk,dv,state", SIZES)
def test_fwd_of_keys_that_are_alike(B, H, Hk, T, dk, dv, state, cosine, low, high, decay, dtype):
    say("alike fwd", B, H, Hk, T, dk, dv, state, cosine, low, high, decay, dtype)
    x = alike(T + dk, B, H, Hk, T, dk, dv, dtype, cosine, low, high, state, decay)
    scale = dk ** -0.5
    o, S = run_fwd(x, dtype, "bthd", scale)
    ro, rS = O.delta_attn(**names(x), scale=scale)
    good = [close("o", o, ro, dtype, True), close("S_T", S, rS, dtype, False)]
    assert all(good)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cosine,low,high,decay", KEYS)
@pytest.mark.parametrize("B,H,Hk,T,dk,dv,state", SIZES)
def test_bwd_of_keys_that_are_alike(B, H, Hk, T, dk, dv, state, cosine, low, high, decay, dtype):
    say("alike bwd", B, H, Hk, T, dk, dv, state, cosine, low, high, decay, dtype)
    x = alike(T + dk, B, H, Hk, T, dk, dv, dtype, cosine, low, high, state, decay)
    scale = dk ** -0.5
    got = run_bwd(x, dtype, "bthd", scale)
    ref = O.delta_attn_backward(**names(x, "dO", "dS_T"), scale=scale)
    good = [close(n, got[n], y, dtype, n in ("dq", "dk", "dv")) for n, y in ref.items()]
    assert all(good)


def test_fwd_segments_of_keys_that_are_alike():
    """A sequence cut into segments; its results too.  Sixteen times the tokens of the others: decays keep what a block lost from adding
    up over more of them."""
    from paper_2607_11897_amd import sfda
    B, H, T, d = 1, 1, 2500, 128
    whole = sfda.delta_attn_fwd_workspace_bytes(B, 512, T, d, d, "bf16") // 512
    assert sfda.delta_attn_fwd_workspace_bytes(B, H, T, d, d, "bf16") > H * whole
    x = alike(5, B, H, H, T, d, d, "bf16", 0.9, 1.0, 2.0, True, 0.02)
    say("alike segments")
    o, S = run_fwd(x, "bf16", "bthd", d ** -0.5)
    ro, rS = O.delta_attn(**names(x), scale=d ** -0.5)
    good = [close("o", o, ro, "bf16", True), close("S_T", S, rS, "bf16", False)]
    assert all(good)

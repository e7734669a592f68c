"""Decay attention on the LDS-poison debug build (libsfda_poison.so), whose scan fills its whole LDS with NaN words at
entry: what the scan reads it has written, so the outputs are the normal build's, bit by bit.  Channels that fill their padded
width and that do not, blocks and segments that are whole and that are not, sequences without a token."""
from __future__ import annotations

import os

import pytest

from gpu_util import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import torch
    from paper_2607_11897_amd import build
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    ensure_built()
    if not os.path.exists(build.POISON_LIB):
        build.build(verbose=False, poison=True, out=build.POISON_LIB)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,T,dk,dv,lengths", [
    (2, 3, 64, 64, 64, None), (2, 2, 75, 128, 128, None), (3, 1, 130, 40, 24, [130, 0, 7]), (1, 2, 97, 37, 101, None),
    (2, 1, 150, 256, 192, [1, 149]), (1, 2, 33, 3, 2, None), (1, 1, 1500, 128, 70, None), (1, 2, 1024, 128, 128, None),
])
def test_scan_under_poison(dtype, B, H, T, dk, dv, lengths):
    import torch
    from paper_2607_11897_amd import build, sfda
    print("[case]", dtype, B, H, T, dk, dv, lengths, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(B + T + dk)
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
    q, k, v, d = (torch.randn(B, H, T, D, generator=gen, device="cuda").to(dt) for D in (dk, dk, dv, dv))
    S0, dS = (torch.randn(B, H, dk, dv, generator=gen, device="cuda") for _ in range(2))
    g = -torch.rand(H, generator=gen, device="cuda")
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")

    def outputs():
        fwd = sfda.decay_attn_fwd(q, k, v, g, S0, lengths=n)
        bwd = sfda.decay_attn_bwd(q, k, v, g, S0, d, dS, lengths=n)
        torch.cuda.synchronize()
        return [x for x in (*fwd, *bwd.values()) if x is not None]

    want = outputs()
    with sfda.library(build.POISON_LIB):
        got = outputs()
    assert len(want) == len(got) == 6
    for a, b in zip(want, got):
        assert torch.isfinite(a).all() and torch.equal(a, b)

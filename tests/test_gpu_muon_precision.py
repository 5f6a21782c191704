"""How far the orthogonalised matrices may be off, in absolute figures.

Held against the fp64 iteration, errors as 2-norms relative to the result's.  Factors of
22 bits lose what test_gpu_muon.py allows (four times an fp32 iteration's error and
2^-20), or 1e-4 on updates that are nearly of low rank, where an fp32 iteration itself
loses 2e-5 to 6e-5.

A bf16 result v = bf16(k) of a kernel value k that is off by at most d from the exact u:
the distance to the nearest bf16 value changes by at most |k - u|, so
|v - u| <= |bf16(k) - k| + |k - u| <= |bf16(u) - u| + 2 |k - u|, and norms follow.
"""
import numpy as np
import pytest

from oracle import operators_oracle as oo
from tests.test_gpu_muon import allowed, f64, off

pytestmark = pytest.mark.gpu
LOW_RANK = 1e-4


def _say(msg):
    print(msg, flush=True)


def update(rng, r, c, rank, noise):
    """`rank` directions and noise of that share of their size (rank 0: noise alone)."""
    u = rng.standard_normal((r, c)) * (noise if rank else 1.0)
    return u + rng.standard_normal((r, rank)) @ rng.standard_normal((rank, c)) if rank else u


def workspace(n):
    import torch
    return torch.empty(n, dtype=torch.uint8, device="cuda").fill_(255)


def check_bf16(x, out, steps=5, low=False):
    import torch
    u = f64(x)
    ref = oo.newton_schulz(u, steps, eps=np.float64(np.float32(1e-7)))
    rounded = torch.from_numpy(ref).to(torch.bfloat16).double().numpy()
    d = max(allowed(u, ref, "f32", steps), LOW_RANK if low else 0.0) + 32 * 2.0 ** -22
    e, tol = off(f64(out), ref), off(rounded, ref) + 2 * d
    _say(f"      {u.shape} steps={steps}: off {e:.3e} of {tol:.3e}")
    assert e <= tol


@pytest.mark.parametrize("r,c,rank,noise", [
    (512, 512, 0, 1.0), (512, 2048, 0, 1.0), (100, 1000, 0, 1.0), (1030, 260, 16, 1.0),
    (256, 1024, 16, 1e-2), (512, 512, 16, 1e-3), (1024, 64, 1, 1e-3), (70, 90, 2, 1e-2)],
    ids=lambda v: str(v))
def test_orthogonalize_bf16_is_the_rounded_definition(r, c, rank, noise):
    """bf16 is how the matrices are held; the products carry 22 bits."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say(f"[gpu] orthogonalize bf16 {r} x {c} rank={rank} noise={noise}")
    x = torch.from_numpy(update(np.random.default_rng(r + c), r, c, rank, noise)).to(torch.bfloat16).cuda()
    out = torch.empty_like(x)
    part = [pb.ortho_tensor(x, out)]
    pb.pblock_orthogonalize(part, "bf16", workspace(pb.pblock_orthogonalize_workspace_bytes(part, "bf16")))
    check_bf16(x, out, low=noise < 1.0)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6])
def test_orthogonalize_bf16_steps_in_both_tiles(steps):
    """Wide and square matrices in large and small tiles, an even and an odd number of
    steps, in place and apart; twice over one workspace."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say(f"[gpu] orthogonalize bf16 chains, steps={steps}")
    rng = np.random.default_rng(steps)
    for shapes in ([(1200, 3000), (1100, 1200)], [(130, 600), (200, 150)]):
        xs = [torch.from_numpy(rng.standard_normal(s)).to(torch.bfloat16).cuda() for s in shapes]
        outs = [torch.full_like(x, 7.0) for x in xs]
        part = [pb.ortho_tensor(x, o) for x, o in zip(xs, outs)]
        ws = workspace(pb.pblock_orthogonalize_workspace_bytes(part, "bf16"))
        pb.pblock_orthogonalize(part, "bf16", ws, steps)
        for x, o in zip(xs, outs):
            check_bf16(x, o, steps)
        keep = [x.clone() for x in xs]
        pb.pblock_orthogonalize([pb.ortho_tensor(x, x) for x in xs], "bf16", ws, steps)
        assert all(torch.equal(x, o) for x, o in zip(xs, outs))
        assert not any(torch.equal(x, k) for x, k in zip(xs, keep))

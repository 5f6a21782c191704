"""Sines and cosines of the rotary positions, which the pairs (1, 0) return, to fp32's own
precision: the angle within its turn is not rounded to fp32 first.

The fp32 sine and cosine of the angle's leading 24 bits are off by at most a step of the
values from 1/2 to 1 (2^-24), the correction for the bits behind it by the rounding of one
sum (2^-25) and less than 2^-40: 2^-24 + 2^-25.  An angle rounded to fp32 is off by up to
2^-25 of half a turn, pi 2^-25 more.  (Positions stay below 2^22, where the angle in fp64
is good to 2^-53 of 2^22 turns.)
"""
import numpy as np
import pytest

from oracle import operators_oracle as oo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_angles_keep_fp32_precision(interleaved, backward):
    import torch
    from paper_2402_15627_amd import pblock as pb
    print(f"[gpu] rope angles adjacent={interleaved} backward={backward}", flush=True)
    tokens, d = 4000, 128
    pos = np.random.default_rng(1).integers(0, 1 << 22, tokens)
    x = torch.zeros(tokens, d, device="cuda")
    first = slice(0, d, 2) if interleaved else slice(0, d // 2)
    second = slice(1, d, 2) if interleaved else slice(d // 2, d)
    x[:, first] = 1.0
    y = torch.empty_like(x)
    fn = pb.pblock_rope_backward if backward else pb.pblock_rope_forward
    fn(pb.rope_config(d, interleaved=interleaved, dtype="f32"), [pb.rope_tensor(x, d, 1, y, d)], tokens,
       positions=torch.from_numpy(pos).cuda())
    angle = pos[:, None].astype(np.float64) * oo.rope_frequencies(d, 10000.0)[None, :]
    y = y.double().cpu().numpy()
    e = np.concatenate([y[:, first] - np.cos(angle),
                        y[:, second] - (-np.sin(angle) if backward else np.sin(angle))])
    print(f"      off {np.abs(e).max():.2e} at most, {np.sqrt(np.mean(e * e)):.2e} rms", flush=True)
    assert np.abs(e).max() <= 2.0 ** -24 + 2.0 ** -25 + 2.0 ** -40

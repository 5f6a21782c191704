"""AdamW step on the GPU with values far from one and with gradients that are not finite:
weights, copies, both states, their codes and scales.

Tolerances as in test_gpu_adamw.  Where g^2 is below 2^-126 the second moment's terms are
multiples of 2^-149: v is off by three halves of that more (a product, a product with 1 -
beta2, a sum), which sqrt(v c2) + eps = eps (1e-8) and more does not show in the weight.  The
codes of sqrt(v) then follow from a root that is off by what 2^-149 is under it.  (At 1e-22
squares are below 2^-149: v is 0.)"""
import numpy as np
import pytest

from oracle import score_oracle as so
from tests.test_gpu_adamw import F, HYPER, check, expected, make, tensor

pytestmark = pytest.mark.gpu


def zeros_and(scale, e4m3, n=2000):
    """States of zero and gradients of a size, a seventh of them zero."""
    t = make(n, 4, e4m3)
    t["g"].mul_(scale / 1e-3)
    t["g"][::7] = 0.0
    for k in ("m", "v") if not e4m3 else ("m", "r", "m_scale", "r_scale"):
        t[k].zero_()
    return t


@pytest.mark.parametrize("scale", [1e-15, 1e-12, 1e12, 1e15, 1e18])
@pytest.mark.parametrize("e4m3", [False, True])
def test_everything_that_a_step_writes(scale, e4m3):
    """(1e18: g^2 to 1e37, sqrt(v c2) beyond the fast path's range.)"""
    import torch
    from paper_2402_15627_amd import pblock as pb
    t = zeros_and(scale, e4m3)
    e = expected(t, **HYPER)
    pb.pblock_adamw_step(pb.adamw_config(**HYPER), [tensor(pb, t)])
    torch.cuda.synchronize()
    check(t, e)


@pytest.mark.parametrize("scale", [1e-19, 1e-22])
@pytest.mark.parametrize("e4m3", [False, True])
def test_squares_below_the_smallest_number(scale, e4m3):
    import torch
    from paper_2402_15627_amd import pblock as pb
    t = zeros_and(scale, e4m3)
    e = expected(t, **HYPER)
    pb.pblock_adamw_step(pb.adamw_config(**HYPER), [tensor(pb, t)])
    torch.cuda.synchronize()
    w = t["w"].double().cpu().numpy()
    assert (abs(w - e["w"]) <= 12 * F * e["a_u"] + 3 * F * (abs(e["w0"]) + abs(e["w"]))).all()
    assert torch.equal(t["copy"], t["w"].to(t["copy"].dtype))
    least = 2.0 ** -149
    if not e4m3:
        assert (abs(t["m"].double().cpu().numpy() - e["m"]) <= 4 * F * e["a_m"] + least).all()
        assert (abs(t["v"].double().cpu().numpy() - e["v"]) <= 5 * F * e["v"] + 1.5 * least).all()
        return
    n = len(w)
    bits = so.random_bits(t["seed"] & (2 ** 64 - 1), n)
    root = np.sqrt(e["v"])
    # of v +- 1.5 least
    err = np.maximum(np.sqrt(e["v"] + 1.5 * least) - root, root - np.sqrt(np.maximum(e["v"] - 1.5 * least, 0.0)))
    for key, x, part, off in (("m", e["m"], bits >> np.uint64(16), 4 * F * e["a_m"] + least),
                              ("r", root, bits & np.uint64(0xffff), err + 4 * F * root)):
        got, scale_of = t[key].cpu().numpy(), t[key + "_scale"].double().cpu().numpy()
        per = np.repeat(scale_of, 256)[:n]
        for k in range(len(scale_of)):
            block = slice(256 * k, 256 * k + 256)
            top = max(abs(x[block]).max() / 448, 2.0 ** -126)
            assert abs(scale_of[k] - top) <= off[block].max() / 448 + 3 * F * top
        assert (per >= 2.0 ** -126).all()
        value = abs(so.from_e4m3(got, t[key + "_scale"].cpu().numpy()))
        # a code is one of the two beside the value: an eighth of it, or 2^-9 scales
        assert (abs(value - abs(x)) <= off + abs(x) / 8 * (1 + 8 * F) + 2.0 ** -9 * per).all()
        assert not got[::7].any()  # (zero gradients, zero states)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_block_with_a_gradient_that_is_not_finite_is_lost_as_a_whole(value):
    """Both of its states, and no other block's."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    t, u = make(1000, 3, True), make(1000, 3, True)
    t["g"][300] = value
    for x in (t, u):
        pb.pblock_adamw_step(pb.adamw_config(**HYPER), [tensor(pb, x)])
    torch.cuda.synchronize()
    for key in ("m", "r"):
        scales = t[key + "_scale"]
        assert not torch.isfinite(scales[1]) and torch.isfinite(scales[[0, 2, 3]]).all()
        back = t[key].view(torch.float8_e4m3fn).float() * scales.repeat_interleave(256)[:1000]
        assert not torch.isfinite(back[256:512]).any()
        same = torch.ones(1000, dtype=torch.bool, device="cuda")
        same[256:512] = False
        assert torch.equal(t[key][same], u[key][same])


@pytest.mark.parametrize("odd", [1e-22, 1e19])
@pytest.mark.parametrize("e4m3", [False, True])
def test_neighbours_of_a_value_far_from_one(odd, e4m3):
    """A value in each block of 256 that takes the general root and quotient: the others keep
    the bits that they have without it. (2^25 elements, whose new weights are the update
    itself.)"""
    import torch
    from paper_2402_15627_amd import pblock as pb
    n, g = 1 << 25, torch.Generator(device="cuda").manual_seed(8)
    rnd = lambda std: torch.empty(n, device="cuda").normal_(std=std, generator=g)  # noqa: E731
    grad, m, v = rnd(1e-3), rnd(3e-4), rnd(5e-4).square()
    runs = []
    for k in range(2):
        t = dict(w=torch.zeros(n, device="cuda"), g=grad.clone(), copy=torch.zeros(n, dtype=torch.bfloat16, device="cuda"))
        if e4m3:
            codes = torch.zeros(n, dtype=torch.uint8, device="cuda")
            t.update(m=codes, r=codes.clone(), m_scale=torch.ones(n // 256, device="cuda"),
                     r_scale=torch.ones(n // 256, device="cuda"), decay=0.1, seed=1)
        else:
            t.update(m=m.clone(), v=v.clone(), decay=0.1, seed=0)
            t["m"][100::256], t["v"][100::256] = 0.0, 0.0
        if k:
            t["g"][100::256] = odd
        pb.pblock_adamw_step(pb.adamw_config(**HYPER), [tensor(pb, t)])
        runs.append(t)
    torch.cuda.synchronize()
    others = torch.ones(n, dtype=torch.bool, device="cuda")
    others[100::256] = False
    for k in ("w", "copy") if e4m3 else ("w", "copy", "m", "v"):
        assert torch.equal(runs[0][k][others], runs[1][k][others]), k

"""Gradients of capped scores that are all 3 to 8 caps large, where 1 - tanh^2 is a small
difference: dq and dk against the fp64 oracle.

Tolerances as in test_gpu_score_attn (bf16 products) and test_gpu_score_products, with the
cap's slope: its logarithm moves by 2 tanh for each unit of x = u / cap, so an error of u by
r (as there, absolute) is 2 r / cap of the slope, and the exponential's argument 2 |x| log2 e,
x itself and the quotient's parts round by 2^-24 each: (8 |x| + 16) 2^-24."""
import numpy as np
import pytest

from tests.test_gpu_score_attn import F, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "bf16_products"])
@pytest.mark.parametrize("bias", [dict(), dict(slopes=True), dict(buckets=8, max_distance=20)])
@pytest.mark.parametrize("at", [3.5, 5.5, 7.5])
def test_gradients_of_scores_near_their_cap(kind, bias, at):
    import torch
    print(kind, bias, at, flush=True)
    d = 64
    c = Case(dtype="f32" if kind == "f32" else "bf16", seq=150, heads=2, d=d, cap=16.0 / at, **bias)
    if kind == "bf16_products":
        c.cfg.products = c.pb.PB_BF16
    g = torch.Generator(device="cuda").manual_seed(3)
    for x, mean in ((c.q, 2.0), (c.k, 1.0)):  # q.k / 8: 16, of either sign by the query
        x.copy_(mean + 0.2 * torch.empty(x.shape, device="cuda").normal_(generator=g))
    c.q[::3] *= -1.0
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    r = c.oracle()
    x = abs(np.einsum("bqhd,bkhd->bhqk", c.numpy(c.q), c.numpy(c.k, True))) / 8 / (16.0 / at)
    assert at - 1.5 <= x.min() and x.max() <= at + 1.5
    h = F if kind == "f32" else 2.0 ** -8
    rel = F * (d + 8) * float(r["a_s"].max()) + F * 150
    slope = 2 * rel * at / 16.0 + F * (8 * (at + 1.5) + 16)
    factors = h * h if kind == "bf16" else h  # P and dS rounded before their products
    term = h if kind == "bf16_products" else F if kind == "f32" else 0.0  # o in the row term
    for n, got in (("dq", c.numpy(c.dq)), ("dk", c.numpy(c.dk, True))):
        tol = h * abs(r[n]) + (factors + 2 * rel + slope) * r["a_" + n] + (term + 2 * rel) * r["e_" + n]
        off = abs(got - r[n])
        assert (off <= 1.02 * tol).all(), (n, float((off / tol).max()))
        print(n, "%.2e" % (np.linalg.norm(off) / np.linalg.norm(r[n])), flush=True)
        if kind != "bf16_products":  # (there the row term's rounding is more than the slopes')
            assert np.linalg.norm(off) <= (1e-4 if kind == "f32" else 2e-3) * np.linalg.norm(r[n]), n

"""The fp32 bias table's gradient, and dq with it, where a row's terms nearly cancel.

o and lse are the exact ones rounded to fp32, so the row term and P each bring a rounding
that the row's other terms do not share; a table's entry adds them up over rows.  Formed from
the products themselves they drop out, and what is left are the products' own sums: chains of
up to 32 matrix instructions' roundings, 2^-25 rms each of partial sums that grow to the
whole (sqrt(32 / 3) of them, 1e-7 of q.k and of dO.v each), which a difference of two terms
of one size doubles, the exponential's 2^-24 and the entry's own sum: 8 2^-24 (4.8e-7) in
norm."""
import numpy as np
import pytest

from tests.test_gpu_score_attn import F, Case

pytestmark = pytest.mark.gpu

CASES = {
    "rows_of_two": dict(seq=1000, heads=4, kv_heads=1, window=2, buckets=8, max_distance=300),
    "rows_of_two_prefix": dict(seq=700, heads=4, kv_heads=1, window=2, buckets=8, max_distance=300, prefix=[90]),
    "short": dict(batch=20, seq=3, heads=8, kv_heads=2, buckets=32, max_distance=128, cap=20.0, d=128),
    "both_ways": dict(seq=300, heads=2, causal=False, window=3, buckets=16, max_distance=50, d=96),
    "long": dict(seq=600, heads=2, buckets=16, max_distance=60),
}


@pytest.mark.parametrize("name", CASES)
def test_the_tables_gradient_keeps_its_bits(name):
    import torch
    print(name, flush=True)
    c = Case(dtype="f32", **CASES[name])
    r = c.oracle()
    b, sq, _, h, _, d = c.shape
    c.o.copy_(torch.from_numpy(r["o"].reshape(b * sq, h * d)).float())
    c.lse.copy_(torch.from_numpy(r["lse"]).float())
    c.backward()
    torch.cuda.synchronize()
    c.check(r, ("dq", "dk", "dv", "dtable"))
    for n, got in (("dtable", c.dtable.double().cpu().numpy()), ("dq", c.numpy(c.dq))):
        off = np.linalg.norm(got - r[n]) / np.linalg.norm(r[n])
        print(n, "%.2e" % off, flush=True)
        assert off <= 8 * F, (n, off)

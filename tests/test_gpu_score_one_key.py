"""Attention with terms in its scores where no query sees two keys: P is 1 whatever the
scores are, so dq, dk and dtable are exactly 0 (a difference of two roundings would be all
that they hold), and dv is d_o, summed over the heads that share a key head."""
import numpy as np
import pytest

from tests.test_gpu_score_attn import Case

pytestmark = pytest.mark.gpu

ONE = {
    "window": dict(seq=300, heads=2, window=1),
    "window_both_ways": dict(batch=2, seq=70, heads=4, kv_heads=2, window=1, causal=False, cap=3.0),
    "token": dict(batch=3, seq=1, heads=4, kv_heads=1, d=96),
    "token_prefix": dict(batch=2, seq=1, heads=2, prefix=[1, 0]),
    "docs": dict(seq=200, heads=2, window=1, docs=[3, 50, 190], d=128),
    "slopes": dict(seq=90, heads=2, window=1, slopes=True),
    "table": dict(seq=90, heads=2, window=1, buckets=8, max_distance=20),
    "table_both_ways": dict(seq=90, heads=2, window=1, causal=False, buckets=8, max_distance=20, d=128),
    "few_queries": dict(seq=900, seq_q=5, heads=2, window=1),
}


@pytest.mark.parametrize("kind", ["f32", "bf16", "bf16_products"])
@pytest.mark.parametrize("name", ONE)
def test_gradients_of_scores_are_zero(name, kind):
    import torch
    print(name, kind, flush=True)
    c = Case(dtype="f32" if kind == "f32" else "bf16", **ONE[name])
    if kind == "bf16_products":
        c.cfg.products = c.pb.PB_BF16
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    assert not c.dq.any() and not c.dk.any()
    assert c.dtable is None or not c.dtable.any()
    r = c.oracle()
    c.check(r, ("dv",))
    assert np.abs(r["dq"]).max(initial=0.0) == 0.0


def test_a_prefix_adds_keys():
    """window 1 beside a prefix: queries see its keys too."""
    import torch
    for dtype in ("f32", "bf16"):
        c = Case(dtype=dtype, seq=60, heads=2, window=1, prefix=[4])
        c.run()
        assert c.dq.any() and c.dk.any()
        torch.cuda.synchronize()

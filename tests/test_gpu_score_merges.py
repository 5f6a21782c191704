"""Attention with terms in its scores where blocks are cut into chunks and a value behind
the mask is not finite in one feature only: the rows whose parts it enters are computed
again, each by one wave as a whole, so that every run gives the same bits.

Tolerance: rows computed again are fp32 sums of unrounded factors, the others have the
products' (16 bits of P and dS by default, 8 with products "bf16") and both one rounding of
the result; test_gpu_score_attn's tolerances hold either."""
import pytest

from tests.test_gpu_score_attn import Case

pytestmark = pytest.mark.gpu

# the last tokens belong to no document
CUT = {
    "rows": dict(seq=1500, heads=2, docs=[0, 1450]),
    "rows_cap": dict(seq=1300, heads=2, docs=[0, 1250], cap=8.0, slopes=True),
    "shared": dict(seq=1500, heads=4, kv_heads=1, docs=[0, 700, 1450], prefix=[64, 10]),
    "token": dict(batch=2, seq=3000, seq_q=1, heads=8, kv_heads=2, docs=[0, 3000, 3010, 6000], prefix=[0, 0, 0]),
    "few_queries": dict(seq=4000, seq_q=70, heads=2, docs=[10, 4000]),
    "many_shared": dict(seq=300, heads=11, kv_heads=1, docs=[0, 270]),
    "table": dict(seq=1300, heads=3, kv_heads=1, docs=[0, 1250], buckets=32, max_distance=128),
}


@pytest.mark.parametrize("products", ["f32", "bf16"])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("name", CUT)
def test_rows_computed_again_are_whole_and_repeat(name, d, products):
    import torch
    print(name, d, products, flush=True)
    spec = dict(CUT[name], d=d)
    c = Case(**spec)
    c.cfg.products = c.pb.PB_F32 if products == "f32" else c.pb.PB_BF16
    batch, seq_q, seq, heads, kv_heads, _ = c.shape
    see = c.see.any(axis=1).reshape(-1)  # keys that any query sees
    asks = c.see.any(axis=2).reshape(-1)
    r = c.oracle()  # (what see hides is not read)
    hidden_k, hidden_q = ~torch.from_numpy(see), ~torch.from_numpy(asks)
    for x, where, heads_ in ((c.k, hidden_k, kv_heads), (c.v, hidden_k, kv_heads), (c.q, hidden_q, heads),
                             (c.d_o, hidden_q, heads)):
        rows = where.nonzero()[:, 0].cuda()
        for head in range(heads_):
            x[rows, head * d + 37] = float("nan")
            x[rows, head * d + d - 1] = float("inf")
    first = None
    for run in range(3):
        for x in (c.o, c.dq, c.dk, c.dv, c.lse):
            x.fill_(7.0)
        c.forward()
        c.backward()
        torch.cuda.synchronize()
        got = [x.clone() for x in (c.o, c.lse, c.dq, c.dk, c.dv)]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, got)), run
        first = got
    c.check(r, ("o", "lse"))
    c.check(r, ("dq", "dk", "dv"))


def test_every_case_is_cut():
    """(or the merges would not run)"""
    for name, spec in CUT.items():
        c = Case(**dict(spec, d=96))
        pb = c.pb
        sizes = [pb.pblock_score_attn_workspace_bytes(c.cfg, m) for m in
                 (pb.ATTN_WS_FORWARD, pb.ATTN_WS_BACKWARD_MIN, pb.ATTN_WS_BACKWARD)]
        # (eleven heads are eleven sets, whose parts are merged whatever the workspace)
        assert sizes[0] > 0 or sizes[2] > sizes[1] or name == "many_shared", name

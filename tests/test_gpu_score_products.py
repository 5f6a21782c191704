"""Attention with terms in its scores on bf16 tensors: how far results are off with each
kind of products.

products "f32", per element (h, f, r, a_*, e_* as in test_gpu_score_attn): a result's own
rounding h |x|; P and its gradient as a bf16 value and its remainder, h^2 of the sums'
magnitudes; fp32's r of them, twice for dq and dk (scores enter P and dP - delta); and the
row term, formed from unrounded values, 2 r of sum |d_o| (|o| + sum P |v|).  In norm the
result's rounding alone stays: the others are below a fiftieth of it each, and a sum of
squares over some thousand roundings varies by a few hundredths, so 1.1 of what rounding
the exact values gives.

products "bf16": the tolerances of test_gpu_score_attn.
"""
import numpy as np
import pytest

from tests.test_gpu_score_attn import CASES, F, Case
from tests.test_gpu_score_attn_more import SPLIT

pytestmark = pytest.mark.gpu
H = 2.0 ** -8


def tolerances(c, r):
    d, seq = c.shape[-1], c.shape[2]
    rel = F * (d + 8) * float(r["a_s"].max(initial=0.0)) + F * seq
    return dict(o=H * abs(r["o"]) + (H * H + rel) * r["a_o"],
                dv=H * abs(r["dv"]) + (H * H + rel) * r["a_dv"],
                dq=H * abs(r["dq"]) + (H * H + 2 * rel) * r["a_dq"] + 2 * rel * r["e_dq"],
                dk=H * abs(r["dk"]) + (H * H + 2 * rel) * r["a_dk"] + 2 * rel * r["e_dk"])


def results(c):
    return dict(o=c.numpy(c.o), dq=c.numpy(c.dq), dk=c.numpy(c.dk, True), dv=c.numpy(c.dv, True))


def rounded(x):
    import torch
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


def check(c, r, norms=True):
    tol = tolerances(c, r)
    for n, got in results(c).items():
        off = abs(got - r[n])
        assert (off <= 1.02 * tol[n] + 1e-30).all(), (n, float((off - tol[n]).max()))
        if norms:
            once = np.linalg.norm(rounded(r[n]) - r[n])
            assert np.linalg.norm(got - r[n]) <= 1.1 * once, (n, np.linalg.norm(got - r[n]) / once)


PRECISE = {
    "rows_of_two": dict(seq=600, heads=2, window=2),
    "rows_of_four": dict(seq=600, heads=2, window=4, d=96),
    "window": dict(seq=500, heads=2, window=16, cap=20.0, d=128),
    "short": dict(batch=30, seq=7, heads=4, kv_heads=2),
    "documents": dict(seq=500, heads=2, docs=[0, 3, 60, 61, 350, 490], prefix=[0, 5, 1, 100, 0]),
    "cap": dict(seq=400, heads=2, cap=3.0, d=96),
    "slopes": dict(seq=400, heads=4, kv_heads=1, slopes=True, d=128),
    "both_ways": dict(seq=300, heads=2, causal=False, slopes=True, cap=6.0, d=128),
    "table": dict(seq=400, heads=3, buckets=32, max_distance=100, d=128),
    "table_cap": dict(seq=300, heads=2, buckets=16, max_distance=60, cap=4.0, d=96),
    "table_shared": dict(batch=2, seq=200, heads=4, kv_heads=1, buckets=16, max_distance=60, causal=False),
    "many_shared": dict(seq=150, heads=22, kv_heads=2, window=40),
    "last_queries": dict(batch=2, seq=300, seq_q=90, heads=4, kv_heads=2, cap=9.0),
}


@pytest.mark.parametrize("name", PRECISE)
def test_results_are_off_by_their_own_rounding(name):
    import torch
    print(name, flush=True)
    c = Case(**PRECISE[name])
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    check(c, c.oracle())


@pytest.mark.parametrize("name", SPLIT)
def test_split_results_too(name):
    """Blocks in chunks, the row term's among them, and whole."""
    import torch
    print(name, flush=True)
    c = Case(**SPLIT[name])
    r = c.oracle()
    for split, mode in ((True, c.pb.ATTN_WS_BACKWARD), (False, c.pb.ATTN_WS_BACKWARD_MIN)):
        c.forward(split=split)
        c.backward(mode)
        torch.cuda.synchronize()
        check(c, r, norms=name != "token")


@pytest.mark.parametrize("bias", [dict(), dict(slopes=True), dict(buckets=4, max_distance=9)])
def test_rows_of_one_key_have_no_gradient_of_scores(bias):
    """P is 1, dP - delta 0: what is left is fp32's."""
    import torch
    print(bias, flush=True)
    c = Case(seq=300, heads=2, window=1, **bias)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    r = c.oracle()
    assert not r["dq"].any() and not r["dk"].any()
    check(c, r, norms=False)
    assert torch.equal(c.o, c.v)


def narrow(**spec):
    c = Case(**spec)
    c.cfg.products = c.pb.PB_BF16
    return c


@pytest.mark.parametrize("name", CASES)
def test_bf16_products(name):
    print(name, flush=True)
    narrow(**CASES[name]).run()


@pytest.mark.parametrize("name", SPLIT)
def test_bf16_products_split_and_whole(name):
    import torch
    print(name, flush=True)
    c = narrow(**SPLIT[name])
    r = c.oracle()
    for split, mode in ((True, c.pb.ATTN_WS_BACKWARD), (False, c.pb.ATTN_WS_BACKWARD_MIN)):
        first = None
        for _ in range(2):
            c.forward(split=split)
            c.backward(mode)
            torch.cuda.synchronize()
            got = [x.clone() for x in (c.o, c.lse, c.dq, c.dk, c.dv)]
            assert first is None or all(torch.equal(x, y) for x, y in zip(first, got))
            first = got
        c.check(r, ("o", "lse"))
        c.check(r, ("dq", "dk", "dv", "dtable"))


@pytest.mark.parametrize("heads,kv_heads", [(16, 1), (11, 1), (24, 2), (14, 2)])
@pytest.mark.parametrize("table", [False, True])
def test_bf16_products_of_many_shared_heads(heads, kv_heads, table):
    print(heads, kv_heads, table, flush=True)
    more = dict(buckets=8, max_distance=30) if table else dict(slopes=True)
    narrow(seq=90, heads=heads, kv_heads=kv_heads, **more).run()


def test_fp32_tensors_have_one_kind():
    import torch
    c = Case(dtype="f32", seq=200, heads=2, cap=5.0)
    outs = lambda: [x.clone() for x in (c.o, c.lse, c.dq, c.dk, c.dv)]  # noqa: E731
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    want = outs()
    c.cfg.products = c.pb.PB_BF16
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs(), want))

"""Attention with terms in its scores on the GPU, beyond sizes: what masks hide, split and
whole runs, streams, graphs, long strides, many shared heads, masks of the lowest value,
differences.  Tolerances as in test_gpu_score_attn."""
import numpy as np
import pytest

from tests.test_gpu_score_attn import Case

pytestmark = pytest.mark.gpu

HIDDEN = {
    # a document's values are another's masked places, in the same tiles and blocks
    "second_document": (dict(seq=150, heads=2, docs=[0, 70, 150], cap=4.0), slice(70, 150)),
    "first_document": (dict(seq=150, heads=4, kv_heads=2, docs=[0, 40, 150], slopes=True), slice(0, 40)),
    "padding": (dict(seq=200, heads=2, docs=[10, 133], buckets=8, max_distance=30), None),
    "padding_windows": (dict(seq=200, heads=2, docs=[0, 133], window=20, d=128), None),
    "small_chunks": (dict(seq=1500, heads=1, docs=[0, 1450], d=128, buckets=32, max_distance=100), None),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("name", HIDDEN)
def test_what_a_mask_hides_enters_nothing(name, value, dtype):
    """Tokens of another document, or of none, hold infinities and NaN in every tensor:
    the others' results are those without them."""
    import torch
    spec, tokens = HIDDEN[name]
    print(name, value, dtype, flush=True)
    c = Case(dtype=dtype, **spec)
    seq = spec["seq"]
    away = torch.ones(seq, dtype=torch.bool, device="cuda")
    if tokens is None:
        away[spec["docs"][0]:spec["docs"][-1]] = False
    else:
        away[:] = False
        away[tokens] = True
    for x in (c.q, c.k, c.v, c.d_o):
        x[away] = 0.0
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    want = {n: getattr(c, n)[~away].clone() for n in ("o", "dq", "dk", "dv")}
    lse, dtable = c.lse[:, :, ~away].clone(), None if c.dtable is None else c.dtable.clone()
    for x in (c.q, c.k, c.v, c.d_o):
        x[away] = value
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    h = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for n, w in want.items():
        got = getattr(c, n)[~away].double()
        w = w.double()
        assert torch.isfinite(got).all(), n
        # rows that were computed again by the definition differ by roundings: P and dS of
        # the products (h of terms up to the largest), the row term's and the result's
        assert (got - w).abs().max() <= 16 * h * max(1.0, float(w.abs().max())), n
    assert torch.allclose(c.lse[:, :, ~away], lse, rtol=1e-5, atol=1e-5)
    if dtable is not None and tokens is None:
        assert torch.isfinite(c.dtable).all()
        assert (c.dtable - dtable).abs().max() <= 1e-4 * dtable.abs().max()
    if tokens is None:  # tokens of no document: empty rows
        assert not c.o[away].any() and not c.dq[away].any() and not c.dk[away].any() and not c.dv[away].any()
        assert bool((c.lse[:, :, away] == -float("inf")).all())


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_later_token_enters_no_earlier_one(value):
    """Causal: keys and values ahead of a query, in its own tile, hold no finite value."""
    import torch
    for d, heads, kv in ((64, 2, 2), (128, 4, 1)):
        c = Case(seq=100, heads=heads, kv_heads=kv, d=d)
        c.forward()
        torch.cuda.synchronize()
        o, lse = c.o.clone(), c.lse.clone()
        c.k[77] = value
        c.v[77] = value
        c.forward()
        torch.cuda.synchronize()
        assert torch.isfinite(c.o[:77]).all()
        assert (c.o[:77].float() - o[:77].float()).abs().max() <= 4 * 2.0 ** -8 * o.float().abs().max()
        assert torch.allclose(c.lse[:, :, :77], lse[:, :, :77], rtol=1e-5, atol=1e-5)
        assert not torch.isfinite(c.o[77:].float()).all(1).any()


SPLIT = {
    "token": dict(batch=2, seq=3000, seq_q=1, heads=8, kv_heads=2, d=128, slopes=True),
    "rows": dict(seq=1200, heads=2, d=128, cap=20.0),
    "rows_docs": dict(seq=1500, heads=4, kv_heads=1, docs=[0, 1000, 1003, 1499], prefix=[100, 1, 0], d=64),
    "table": dict(seq=1300, heads=2, kv_heads=1, d=96, buckets=32, max_distance=128),
    "table_both": dict(seq=1000, heads=2, causal=False, d=64, buckets=16, max_distance=50),
    "few_queries": dict(seq=4000, seq_q=70, heads=2, d=128, buckets=32, max_distance=128),
}


@pytest.mark.parametrize("name", SPLIT)
def test_split_and_whole_runs(name):
    """With the workspace for splitting and without: both within the tolerances, and each
    the same bits when run again."""
    import torch
    print(name, flush=True)
    c = Case(**SPLIT[name])
    pb = c.pb
    r = c.oracle()
    assert pb.pblock_score_attn_workspace_bytes(c.cfg, pb.ATTN_WS_FORWARD) > 0
    modes = (pb.ATTN_WS_BACKWARD, pb.ATTN_WS_BACKWARD_MIN)
    sizes = [pb.pblock_score_attn_workspace_bytes(c.cfg, m) for m in modes]
    assert sizes[0] > sizes[1] or name == "token"  # (one query's keys stay one workgroup's)
    for split, mode in ((True, modes[0]), (False, modes[1])):
        c.forward(split=split)
        torch.cuda.synchronize()
        c.check(r, ("o", "lse"))
        c.backward(mode)
        torch.cuda.synchronize()
        c.check(r, ("dq", "dk", "dv", "dtable"))
        first = [x.clone() for x in (c.o, c.lse, c.dq, c.dk, c.dv)] + ([c.dtable.clone()] if c.dtable is not None else [])
        c.forward(split=split)
        c.backward(mode)
        torch.cuda.synchronize()
        again = [c.o, c.lse, c.dq, c.dk, c.dv] + ([c.dtable] if c.dtable is not None else [])
        assert all(torch.equal(x, y) for x, y in zip(first, again))


@pytest.mark.parametrize("heads,kv_heads", [(16, 1), (11, 1), (24, 2), (22, 2), (14, 2)])
@pytest.mark.parametrize("table", [False, True])
def test_many_heads_share_a_key_head(heads, kv_heads, table):
    """More heads than a block of rows holds, and numbers that no power of two divides."""
    print(heads, kv_heads, table, flush=True)
    more = dict(buckets=8, max_distance=30) if table else dict(slopes=True)
    Case(seq=90, heads=heads, kv_heads=kv_heads, **more).run()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lowest", ["finfo", "-inf"])
def test_a_table_of_the_lowest_value_masks(dtype, lowest):
    """Buckets of the type's lowest value are not seen; rows that see no other are empty."""
    import torch
    low = torch.finfo(torch.float32).min if lowest == "finfo" else -float("inf")
    c = Case(dtype=dtype, seq=80, heads=2, buckets=4, max_distance=8)
    c.t["table"][0] = low  # distance 0: row 0 sees nothing then
    c.t["table"][3, 1] = low  # and far keys in head 1
    c.terms["table"] = np.where(c.t["table"].cpu().numpy() < -1e38, -np.inf, c.t["table"].double().cpu().numpy())
    c.forward()
    torch.cuda.synchronize()
    r = c.oracle()
    c.check(r, ("o", "lse"))
    assert not c.o[0].any() and bool((c.lse[0, :, 0] == -float("inf")).all())
    c.backward()
    torch.cuda.synchronize()
    c.check(r, ("dq", "dk", "dv", "dtable"))
    assert not c.dtable[0].any() and not c.dtable[3, 1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_graph_replays(dtype):
    """A captured forward and backward, replayed among eager work, gives the eager bits;
    two graphs have workspaces of their own."""
    import torch
    cases = [Case(dtype=dtype, seed=s, seq=700, heads=4, kv_heads=2, buckets=16, max_distance=60,
                  docs=[0, 500, 690], prefix=[30, 0]) for s in (1, 2)]
    ws = [(c.ws(c.pb.ATTN_WS_FORWARD), c.ws(c.pb.ATTN_WS_BACKWARD)) for c in cases]
    outs = lambda c: [c.o, c.lse, c.dq, c.dk, c.dv, c.dtable]  # noqa: E731
    want, graphs = [], []
    for c, w in zip(cases, ws):
        c.forward(ws=w[0])
        c.backward(ws=w[1])
        torch.cuda.synchronize()
        want.append([x.clone() for x in outs(c)])
    for c, w in zip(cases, ws):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.forward(ws=w[0])
            c.backward(ws=w[1])
        graphs.append(g)
    for k in range(3):
        for c in cases:
            for x in outs(c):
                x.fill_(3.0 + k)
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert all(torch.equal(x, y) for x, y in zip(outs(c), w)), k


def test_two_streams_at_once():
    import torch
    cases = [Case(seed=s, seq=900, heads=4, d=128, cap=10.0) for s in (1, 2)]
    want = []
    for c in cases:
        c.forward()
        c.backward()
        torch.cuda.synchronize()
        want.append([x.clone() for x in (c.o, c.lse, c.dq, c.dk, c.dv)])
        for x in (c.o, c.lse, c.dq, c.dk, c.dv):
            x.zero_()
    ws = [(c.ws(c.pb.ATTN_WS_FORWARD), c.ws(c.pb.ATTN_WS_BACKWARD)) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        for c, s, w in zip(cases, streams, ws):
            c.forward(stream=s, ws=w[0])
            c.backward(stream=s, ws=w[1])
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert all(torch.equal(x, y) for x, y in zip((c.o, c.lse, c.dq, c.dk, c.dv), w))


@pytest.mark.parametrize("seq_q", [1, 300])
def test_rows_that_pass_32_bits(seq_q):
    """Keys 4 GB of stride apart and more: the last of them 4.7 GB behind the first."""
    import torch
    c = Case(seq=300, seq_q=seq_q, heads=2, d=64)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    want = [x.clone() for x in (c.o, c.dq, c.dk, c.dv)]
    ld = (1 << 23) - 8
    far = torch.empty(300 * ld, dtype=torch.bfloat16, device="cuda").view(300, ld)
    far[:, :128], far[:, 128:256] = c.k, c.v
    c.k, c.v = far[:, :128], far[:, 128:256]
    c.dk, c.dv = far[:, 256:384], far[:, 384:512]
    for x in (c.o, c.dq, c.dk, c.dv):
        x.zero_()
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((c.o, c.dq, c.dk, c.dv), want))


def test_gradients_against_differences():
    """fp32: sum(o d_o) along random directions of every input, by central differences of
    fp64 sums of the fp32 results (steps of 2^-6; the third derivative's share and the
    roundings stay below 2e-3 of each)."""
    import torch
    c = Case(dtype="f32", seq=60, heads=4, kv_heads=2, buckets=8, max_distance=20, cap=6.0, q_std=1.0,
             docs=[0, 25, 60], prefix=[5, 3])
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    grads = dict(q=c.dq.clone(), k=c.dk.clone(), v=c.dv.clone(), table=c.dtable.clone())
    at = dict(q=c.q, k=c.k, v=c.v, table=c.t["table"])
    g = torch.Generator(device="cuda").manual_seed(5)
    for name, x in at.items():
        u = torch.empty(x.shape, device="cuda").normal_(generator=g)
        x0, f = x.clone(), []
        for step in (2.0 ** -6, -(2.0 ** -6)):
            x.copy_(x0 + step * u)
            c.forward()
            torch.cuda.synchronize()
            f.append(float((c.o.double() * c.d_o.double()).sum()))
        x.copy_(x0)
        num, got = (f[0] - f[1]) * 2.0 ** 5, float((grads[name].double() * u.double()).sum())
        size = float((grads[name].double() * u.double()).norm())
        assert abs(num - got) <= 2e-3 * max(abs(got), size), (name, num, got)


def test_dtable_is_left_out_where_it_is_not_asked_for():
    import torch
    c = Case(seq=200, heads=2, buckets=16, max_distance=40)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    want = [x.clone() for x in (c.dq, c.dk, c.dv)]
    c.dtable.fill_(7.0)
    keep, c.dtable = c.dtable, None
    c.backward()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((c.dq, c.dk, c.dv), want)) and bool((keep == 7.0).all())


def test_unsorted_offsets_touch_nothing_outside():
    """Offsets in no order: any result, but finite inputs' results are finite and nothing
    beside the outputs is written."""
    import torch
    c = Case(seq=200, heads=2, docs=[0, 100, 200])
    c.t["docs"].copy_(torch.tensor([150, 20, 1 << 30], dtype=torch.int32))
    c.t["prefix"] = torch.tensor([-(1 << 31), (1 << 31) - 1], dtype=torch.int32, device="cuda")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    for n, x in c.full.items():
        assert bool((x[:, -c.pad:] == 7.0).all()), n
    assert torch.isfinite(c.o.float()).all() and torch.isfinite(c.dk.float()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bias", [dict(), dict(slopes=True), dict(buckets=8, max_distance=20)])
@pytest.mark.parametrize("cap", [2.0 ** -12, 2.0 ** -6, 1.0, 2.0 ** 99])
def test_caps_to_the_bounds(dtype, bias, cap):
    """From scores that are all at the cap to those far below it.  (Where 1 - tanh^2 is
    next to nothing, its rounding, 2^-24 of 1, is all there is of dq and dk: they are only
    finite there.)"""
    import torch
    print(dtype, bias, cap, flush=True)
    c = Case(dtype=dtype, seq=100, heads=2, kv_heads=1, cap=cap * 64 ** -0.5, **bias)
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    r = c.oracle()
    c.check(r, ("o", "lse"))
    c.check(r, ("dv", "dtable") + (("dq", "dk") if cap > 1 else ()))
    assert bool(torch.isfinite(c.dq).all()) and bool(torch.isfinite(c.dk).all())


@pytest.mark.parametrize("what", [
    dict(seq=600, heads=4, kv_heads=1, docs=[0, 250, 251, 599], prefix=[40, 0, 300], cap=5.0),
    dict(seq=530, heads=2, kv_heads=1, d=96, buckets=32, max_distance=200),
    dict(seq=530, heads=2, kv_heads=1, buckets=64, max_distance=200, d=128),
    dict(seq=900, seq_q=3, heads=4, kv_heads=2, slopes=True, causal=False)])
def test_long_rows_in_fp32(what):
    """Rows of 32 tiles and more: backward workgroups of eight waves (with 64 buckets, of
    four)."""
    print(what, flush=True)
    Case(dtype="f32", **what).run()

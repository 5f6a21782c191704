"""Refusals, sizes and borders of attention with terms in its scores and of the AdamW
step, on a machine without a GPU: every call below fails a host check (or has nothing
to launch), so its pointers are never read."""
import ctypes

import pytest
import torch

from oracle import score_oracle as so
from paper_2402_15627_amd import pblock as pb

FAKE = 1 << 40
GAP = 1 << 32
OK, BAD, UNSUPPORTED, SMALL = 0, 1, 2, 3
INF, NAN = float("inf"), float("nan")


def config(**over):
    cfg = pb.score_attn_config(2, 40, 40, 4, 2, 64, buckets=over.pop("buckets", 0),
                               max_distance=over.pop("max_distance", 0))
    for k, v in over.items():
        setattr(cfg, k, v)
    return cfg


def call(backward=False, terms=None, **over):
    names = ["q", "ld_q", "k", "v", "ld_kv", "o", "ld_o"] + (["d_o", "ld_do"] if backward else []) + ["lse"]
    names += ["dq", "ld_dq", "dk", "dv", "ld_dkv", "dtable"] if backward else []
    names += ["ws", "ws_bytes"]
    a = {}
    for i, n in enumerate(names):
        a[n] = 512 if n.startswith("ld") else FAKE + i * GAP
    a["dtable"] = None if backward else a.pop("dtable", None)
    if not backward:
        a.pop("dtable")
    a["ws_bytes"] = 1 << 30
    cfg = config(**{k: v for k, v in over.items() if k not in a})
    a.update({k: v for k, v in over.items() if k in a})
    t = pb.ScoreTerms(**(terms or {}))
    fn = "pblock_score_attn_backward" if backward else "pblock_score_attn_forward"
    return getattr(pb.load_library(), fn)(ctypes.byref(cfg), ctypes.byref(t), *a.values(), None)


BUCKETS = dict(buckets=8, max_distance=20)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("over,status", [
    (dict(batch=0), BAD), (dict(seq_q=0), BAD), (dict(seq_k=0), BAD), (dict(seq_q=41), BAD),
    (dict(heads=0), BAD), (dict(kv_heads=0), BAD), (dict(kv_heads=3), BAD), (dict(head_dim=80), UNSUPPORTED),
    (dict(causal=2), BAD), (dict(window=0), BAD), (dict(scale=0.0), BAD), (dict(scale=NAN), BAD),
    (dict(scale=INF), BAD), (dict(cap=-1.0), BAD), (dict(cap=NAN), BAD), (dict(cap=INF), BAD),
    (dict(cap=1e-9), BAD), (dict(dtype=7), BAD), (dict(cap=0.125 / 4100), BAD), (dict(cap=2.0 ** 101), BAD),
    (dict(cap=1.0, scale=2.0 ** -121), BAD),
    (dict(buckets=8, max_distance=4), BAD), (dict(buckets=1, max_distance=9), BAD),
    (dict(buckets=65, max_distance=99), BAD), (dict(buckets=8, max_distance=1 << 21), BAD),
    (dict(buckets=8, max_distance=20, causal=0), BAD),  # buckets without a table
    (dict(batch=1 << 20, seq_k=1 << 12, seq_q=1), UNSUPPORTED),
    (dict(batch=1 << 14, seq_k=1 << 13, seq_q=1 << 13), UNSUPPORTED),
    (dict(batch=1 << 22, seq_k=1, seq_q=1, heads=1, kv_heads=1), UNSUPPORTED),
    (dict(q=None), BAD), (dict(q=FAKE + 8), BAD), (dict(k=None), BAD), (dict(v=FAKE + 2), BAD),
    (dict(o=None), BAD), (dict(lse=None), BAD), (dict(lse=FAKE + 2), BAD),
    (dict(ld_q=255), BAD), (dict(ld_q=260), BAD), (dict(ld_kv=127), BAD), (dict(ld_o=256 + 4), BAD),
    (dict(ld_q=1 << 24), UNSUPPORTED), (dict(ws=FAKE + 128), BAD),
])
def test_refusals(backward, over, status):
    assert call(backward, **over) == status
    assert pb.pblock_last_error() != ""


@pytest.mark.parametrize("over,status", [
    (dict(d_o=None), BAD), (dict(dq=FAKE + 4), BAD), (dict(dk=None), BAD), (dict(dv=None), BAD),
    (dict(ld_dq=8), BAD), (dict(ld_dkv=8), BAD), (dict(ld_do=100), BAD), (dict(dtable=FAKE + 100 * GAP), BAD),
    (dict(ws_bytes=0), SMALL), (dict(ws=None), BAD)])
def test_backward_refusals(over, status):
    assert call(True, **over) == status


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("terms,over", [
    (dict(docs=FAKE + 2, n_docs=1), {}), (dict(docs=FAKE, n_docs=-1), {}), (dict(prefix=FAKE + 1), {}),
    (dict(slopes=FAKE + 2), {}), (dict(table=FAKE + 200 * GAP), {}), (dict(), BUCKETS),
    (dict(slopes=FAKE + 200 * GAP, table=FAKE + 201 * GAP), BUCKETS), (dict(table=FAKE + 2), BUCKETS)])
def test_refusals_of_terms(backward, terms, over):
    assert call(backward, terms, **over) == BAD


@pytest.mark.parametrize("names", [("q", "o"), ("k", "o"), ("v", "o"), ("lse", "o"), ("lse", "q"), ("ws", "o"),
                                   ("ws", "k")])
def test_forward_refuses_shared_memory(names):
    at = FAKE + 50 * GAP
    assert call(False, **{n: at for n in names}) == BAD
    assert "overlap" in pb.pblock_last_error()


@pytest.mark.parametrize("names", [("q", "dq"), ("k", "dk"), ("dk", "dv"), ("d_o", "dq"), ("o", "dv"),
                                   ("lse", "dq"), ("ws", "dq"), ("ws", "d_o"), ("dq", "dk")])
def test_backward_refuses_shared_memory(names):
    at = FAKE + 50 * GAP
    assert call(True, **{n: at for n in names}) == BAD
    assert "overlap" in pb.pblock_last_error()


def test_terms_may_not_be_written():
    at = FAKE + 50 * GAP
    for n in ("docs", "prefix", "slopes"):
        assert call(False, {n: at, "n_docs": 1}, lse=at) == BAD
    assert call(False, dict(table=at), lse=at, **BUCKETS) == BAD
    assert call(True, dict(table=at), dtable=at, **BUCKETS) == BAD


def test_null_arguments():
    lib = pb.load_library()
    assert lib.pblock_score_attn_borders(None, None) == BAD
    assert lib.pblock_score_attn_workspace_bytes(None, 0) == 0
    assert lib.pblock_score_attn_forward(None, None, None, 0, None, None, 0, None, 0, None, None, 0, None) == BAD


@pytest.mark.parametrize("causal", [True, False])
def test_borders_are_the_oracles(causal):
    for buckets in (2, 4, 6, 8, 10, 16, 32, 48, 64):
        side = buckets if causal else buckets // 2
        if side < 2:
            continue
        for far in (side // 2 + 1, side, 63, 64, 77, 128, 300, 512, 1000, 1024, 4096, 9999, 65536, 1 << 20):
            if far <= side // 2:
                continue
            cfg = pb.score_attn_config(1, 1, 1, 1, 1, 64, causal, buckets=buckets, max_distance=far)
            assert pb.pblock_score_attn_borders(cfg) == so.bucket_borders(buckets, far, causal), (buckets, far)
    with pytest.raises(pb.PblockError):
        pb.pblock_score_attn_borders(pb.score_attn_config(1, 1, 1, 1, 1, 64))


def test_workspaces():
    size = pb.pblock_score_attn_workspace_bytes
    few = pb.score_attn_config(1, 1, 8192, 8, 8, 128)
    assert size(few, pb.ATTN_WS_FORWARD) >= 2 * 8 * 129 * 4
    many = pb.score_attn_config(8, 4096, 4096, 16, 16, 128)
    assert size(many, pb.ATTN_WS_FORWARD) == 0
    for cfg in (few, many, pb.score_attn_config(1, 300, 300, 22, 2, 64, buckets=32, max_distance=99)):
        small, full = size(cfg, pb.ATTN_WS_BACKWARD_MIN), size(cfg, pb.ATTN_WS_BACKWARD)
        assert 0 < small <= full and small % 256 == 0
        assert size(cfg, 9) == 0
    assert size(pb.score_attn_config(0, 1, 1, 1, 1, 64), pb.ATTN_WS_BACKWARD) == 0
    assert size(pb.score_attn_config(1, 9, 9, 2, 2, 64, dtype="f32"), pb.ATTN_WS_FORWARD) == 0


def test_binding_checks_tensors():
    cfg = pb.score_attn_config(1, 4, 4, 2, 1, 64)
    x = lambda w, dt=torch.bfloat16: torch.zeros(4, w, dtype=dt)  # noqa: E731
    lse = torch.zeros(1, 2, 4)
    call = lambda q, k, v, o, **t: pb.pblock_score_attn_forward(cfg, q, k, v, o, lse, **t)  # noqa: E731
    with pytest.raises(ValueError, match="q is torch.float32"):
        call(x(128, torch.float32), x(64), x(64), x(128))
    with pytest.raises(ValueError, match=r"q is \(4, 64\)"):
        call(x(64), x(64), x(64), x(128))
    with pytest.raises(ValueError, match="not on a GPU"):
        call(x(128), x(64), x(64), x(128))
    with pytest.raises(ValueError, match="rows are not contiguous"):
        call(x(128).t().contiguous().t(), x(64), x(64), x(128))
    with pytest.raises(ValueError, match="docs is empty"):
        pb._ScoreCall(cfg).terms(torch.zeros(0, dtype=torch.int32), None, None, None)


# ------------------------------------------------------------ AdamW step
def adam(tensors, copy_dtype=0, n=None, **over):
    cfg = pb.adamw_config(1e-3)
    for k, v in over.items():
        setattr(cfg, k, v)
    arr = (pb.AdamwTensor * max(len(tensors), 1))(*tensors)
    return pb.load_library().pblock_adamw_step(ctypes.byref(cfg), len(tensors) if n is None else n, arr,
                                               copy_dtype, None)


def one(at=FAKE, numel=10, **over):
    t = pb.AdamwTensor(at, at + GAP, at + 2 * GAP, at + 3 * GAP, at + 4 * GAP, at + 5 * GAP, None, numel, 0, 0.1)
    for k, v in over.items():
        setattr(t, k, v)
    return t


@pytest.mark.parametrize("state", [0, 1])
@pytest.mark.parametrize("over,status", [
    (dict(lr=NAN), BAD), (dict(lr=INF), BAD), (dict(beta1=1.0), BAD), (dict(beta1=-0.1), BAD),
    (dict(beta2=1.0), BAD), (dict(beta2=NAN), BAD), (dict(eps=0.0), BAD), (dict(eps=INF), BAD),
    (dict(grad_scale=NAN), BAD), (dict(step=0), BAD), (dict(bias_correction=2), BAD), (dict(n=0), BAD),
    (dict(n=1025), BAD), (dict(copy_dtype=3), BAD)])
def test_adamw_refusals(state, over, status):
    assert adam([one()], state=state, **over) == status
    assert pb.pblock_last_error() != ""


@pytest.mark.parametrize("state", [0, 1])
@pytest.mark.parametrize("over,status", [
    (dict(param=None), BAD), (dict(grad=None), BAD), (dict(exp_avg=None), BAD), (dict(exp_avg_sq=None), BAD),
    (dict(param=FAKE + 2), BAD), (dict(grad=FAKE + GAP + 1), BAD), (dict(param_copy=FAKE + 9 * GAP + 1), BAD),
    (dict(weight_decay=-1.0), BAD), (dict(weight_decay=NAN), BAD), (dict(numel=1 << 34), UNSUPPORTED),
    (dict(numel=(1 << 34) - 1023), UNSUPPORTED),
    # shared memory: with another array, and by the end of one
    (dict(grad=FAKE), BAD), (dict(exp_avg=FAKE), BAD), (dict(param_copy=FAKE), BAD),
    (dict(param=FAKE + GAP - 4), BAD), (dict(exp_avg_sq=FAKE + 2 * GAP), BAD)])
def test_adamw_refuses_tensors(state, over, status):
    assert adam([one(), one(FAKE + 100 * GAP, **over)] if "weight_decay" in over else [one(**over)],
                state=state) == status


def test_adamw_states_and_scales():
    assert adam([one(exp_avg=FAKE + 2 * GAP + 1)], state=0) == BAD
    assert adam([one(avg_scale=None)], state=1) == BAD
    assert adam([one(sq_scale=FAKE + 2)], state=1) == BAD
    assert adam([one(sq_scale=FAKE + 4 * GAP)], state=1) == BAD
    assert adam([one()], state=2) == BAD
    # the scales of 300 elements are two: 8 bytes
    assert adam([one(numel=300, sq_scale=FAKE + 4 * GAP + 4)], state=1) == BAD


def test_adamw_refuses_the_same_tensor_twice_and_takes_none():
    assert adam([one(), one()]) == BAD and "overlaps" in pb.pblock_last_error()
    a, b = one(), one(FAKE + 100 * GAP)
    b.exp_avg = a.exp_avg
    assert adam([a, b]) == BAD
    b = one(FAKE + 100 * GAP)
    b.grad = a.param + 36  # the last element of another tensor's weights
    assert adam([a, b]) == BAD
    nothing = pb.AdamwTensor(None, None, None, None, None, None, None, 0, 0, 0.0)
    for state in (0, 1):
        assert adam([nothing] * 5, state=state) == OK
    assert pb.load_library().pblock_adamw_step(None, 1, None, 0, None) == BAD


def test_adamw_binding():
    x = torch.zeros(300)
    codes, scales = torch.zeros(300, dtype=torch.float8_e4m3fn), torch.zeros(2)
    with pytest.raises(ValueError, match="need avg_scale"):
        pb.adamw_tensor(x, x, codes, codes)
    with pytest.raises(ValueError, match="have no scales"):
        pb.adamw_tensor(x, x, x, x, avg_scale=scales, sq_scale=scales)
    with pytest.raises(ValueError, match="param is torch.float64"):
        pb.adamw_tensor(x.double(), x, x, x)
    with pytest.raises(ValueError, match="not on a GPU"):
        pb.adamw_tensor(x, x, x, x)
    with pytest.raises(ValueError, match="no tensors"):
        pb.AdamwTensors([])

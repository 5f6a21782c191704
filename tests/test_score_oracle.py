"""Pins of oracle/score_oracle.py: buckets against the logarithm, masks by hand,
attention against torch autograd of an independent form in float64 and central
differences, the step against torch's AdamW, e4m3 against torch's type; and mistakes
that a pin catches."""
import math

import numpy as np
import pytest
import torch

from oracle import pblock_oracle as po
from oracle import score_oracle as so

RNG = np.random.default_rng


@pytest.mark.parametrize("buckets,max_distance,causal", [
    (32, 128, True), (32, 128, False), (16, 64, True), (64, 1024, True), (64, 64, True), (2, 5, True),
    (4, 100, False), (8, 100000, True), (10, 77, True), (32, 300, False)])
def test_buckets_follow_the_logarithm(buckets, max_distance, causal):
    n = buckets if causal else buckets // 2
    e = n // 2
    first = so.bucket_borders(buckets, max_distance, causal)
    assert len(first) == n and first == sorted(first) and first[:e + 1] == list(range(e + 1))
    for d in list(range(0, 400)) + [999, 5000, 99999, 100000, 10 ** 7]:
        b = so.bucket(d, buckets, max_distance, causal)
        assert 0 <= b < n
        if d < e:
            assert b == d
        elif d >= max_distance:
            assert b == n - 1
        else:
            x = e + (n - e) * math.log(d / e) / math.log(max_distance / e)
            if abs(x - round(x)) > 1e-9:
                assert b == min(int(x), n - 1)
            else:  # a border in whole numbers
                assert b == min(round(x), n - 1)
        back = so.bucket(-d, buckets, max_distance, causal)
        assert back == (0 if causal else b + (n if d else 0))


def test_visible_by_hand():
    m = so.visible(1, 4, 4, True, 2)[0].astype(int).tolist()
    assert m == [[1, 0, 0, 0], [1, 1, 0, 0], [0, 1, 1, 0], [0, 0, 1, 1]]
    m = so.visible(1, 4, 4, False, 2)[0].astype(int).tolist()
    assert m == [[1, 1, 0, 0], [1, 1, 1, 0], [0, 1, 1, 1], [0, 0, 1, 1]]
    # two documents, token 0 and the last in none, a prefix of two in the second
    m = so.visible(1, 6, 6, True, 1, docs=[1, 2, 5], prefix=[0, 2])[0].astype(int).tolist()
    assert m == [[0] * 6, [0, 1, 0, 0, 0, 0], [0, 0, 1, 1, 0, 0], [0, 0, 1, 1, 0, 0], [0, 0, 1, 1, 1, 0],
                 [0] * 6]
    # a document that runs over the end of a batch row is cut there
    m = so.visible(2, 1, 3, True, 9, docs=[0, 2, 6])
    assert m.astype(int).tolist() == [[[0, 0, 1]], [[1, 1, 1]]]
    assert np.array_equal(so.visible(1, 2, 5, True, 3)[0], so.visible(1, 5, 5, True, 3)[0][3:])


def independent(q, k, v, see, scale, cap, slopes, table, ids, dist):
    """Attention by torch, a head at a time, its own formulas."""
    out, lse = [], []
    heads, group = q.shape[2], q.shape[2] // k.shape[2]
    for h in range(heads):
        s = torch.einsum("bqd,bkd->bqk", q[:, :, h], k[:, :, h // group]) * scale
        if cap:
            e = torch.exp(-2 * s / cap)
            s = cap * (1 - e) / (1 + e)
        if slopes is not None:
            s = s - slopes[h] * dist.abs()
        if table is not None:
            s = s + table[:, h][ids]
        s = s.masked_fill(~see, -math.inf)
        lse.append(torch.logsumexp(s, 2))
        out.append(torch.einsum("bqk,bkd->bqd", torch.nan_to_num(torch.softmax(s, 2)), v[:, :, h // group]))
    return torch.stack(out, 2), torch.stack(lse, 1)


@pytest.mark.parametrize("cap,bias,causal,docs", [
    (0.0, None, True, None), (2.0, None, True, [0, 4, 9, 14]), (0.0, "slopes", False, None),
    (1.5, "slopes", True, [2, 9, 13]), (0.0, "table", True, None), (3.0, "table", False, [0, 5, 14])])
def test_attention_against_autograd(cap, bias, causal, docs):
    r = RNG(3)
    b, sq, sk, h, kv, d = 2, 5, 7, 4, 2, 6
    q, g = r.standard_normal((b, sq, h, d)) * 2, r.standard_normal((b, sq, h, d))
    k, v = r.standard_normal((b, sk, kv, d)), r.standard_normal((b, sk, kv, d))
    see = so.visible(b, sq, sk, causal, 4, docs, None if docs is None else [3] * (len(docs) - 1))
    terms = dict(cap=cap, causal=causal)
    if bias == "slopes":
        terms["slopes"] = r.random(h)
    if bias == "table":
        terms.update(table=r.standard_normal((8, h)), max_distance=9)
    out = so.attention(q, k, v, see, 0.3, d_o=g, **terms)
    t = lambda x: torch.tensor(x, requires_grad=True)  # noqa: E731
    tq, tk, tv = t(q), t(k), t(v)
    dist = torch.arange(sk - sq, sk)[:, None] - torch.arange(sk)[None]
    table = t(terms["table"]) if bias == "table" else None
    ids = None if table is None else torch.tensor(
        [[so.bucket(int(x), 8, 9, causal) for x in row] for row in dist])
    slopes = torch.tensor(terms["slopes"]) if bias == "slopes" else None
    o, lse = independent(tq, tk, tv, torch.tensor(see), 0.3, cap, slopes, table, ids, dist)
    np.testing.assert_allclose(out["o"], o.detach().numpy(), atol=1e-12)
    np.testing.assert_allclose(out["lse"], lse.detach().numpy(), atol=1e-12)
    # autograd through rows of -inf gives NaN: leave them out of the loss
    live = torch.tensor(see.any(2))
    o, _ = independent(tq, tk, tv, torch.tensor(see) | ~live[:, :, None], 0.3, cap, slopes, table, ids, dist)
    (o * torch.tensor(g) * live[:, :, None, None]).sum().backward()
    for name, x in (("dq", tq), ("dk", tk), ("dv", tv)):
        np.testing.assert_allclose(out[name], x.grad.numpy(), atol=1e-11)
    if table is not None:
        np.testing.assert_allclose(out["dtable"], table.grad.numpy(), atol=1e-11)


def test_gradients_against_differences():
    r = RNG(4)
    b, s, h, kv, d = 1, 6, 2, 1, 3
    x = dict(q=r.standard_normal((b, s, h, d)), k=r.standard_normal((b, s, kv, d)),
             v=r.standard_normal((b, s, kv, d)), table=r.standard_normal((4, h)))
    g = r.standard_normal((b, s, h, d))
    see = so.visible(b, s, s, True, 5, docs=[0, 4, 6])
    call = lambda y, **more: so.attention(y["q"], y["k"], y["v"], see, 0.7, table=y["table"],  # noqa: E731
                                          max_distance=4, cap=1.0, **more)
    out = call(x, d_o=g)
    for name, got in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("table", "dtable")):
        num = np.zeros_like(x[name])
        for i in np.ndindex(x[name].shape):
            f = []
            for step in (1e-6, -1e-6):
                y = dict(x, **{name: x[name].copy()})
                y[name][i] += step
                f.append(float((call(y)[0] * g).sum()))
            num[i] = (f[0] - f[1]) / 2e-6
        np.testing.assert_allclose(out[got], num, atol=1e-8)


def test_plain_scores_are_the_block_attention():
    r = RNG(5)
    q, k, v = (r.standard_normal((1, 9, 1, 8)) for _ in range(3))
    o, lse = so.attention(q, k, v, so.visible(1, 9, 9, True, 4), 8 ** -0.5)
    want = po.swa_head_forward(q[0, :, 0], k[0, :, 0], v[0, :, 0], 4)
    np.testing.assert_allclose(o[0, :, 0], want[0], atol=1e-13)


def test_masked_values_are_not_read_and_empty_rows_are_empty():
    r = RNG(6)
    q, k, v, g = (r.standard_normal((1, 6, 1, 4)) for _ in range(4))
    see = so.visible(1, 6, 6, True, 6, docs=[1, 4])
    a = so.attention(q, k, v, see, 0.5, d_o=g)
    for x in (k, v, q, g):
        x[0, 4:] = np.nan
        x[0, :1] = np.inf
    b = so.attention(q, k, v, see, 0.5, d_o=g)
    for n in ("o", "lse", "dq", "dk", "dv"):
        np.testing.assert_array_equal(a[n], b[n])
    assert (b["lse"][0, 0, 4:] == -np.inf).all() and not b["o"][0, 4:].any() and not b["dk"][0, 4:].any()


def test_the_table_gradient_sums_to_zero_over_all_buckets():
    """A constant added to every bucket changes no probability."""
    r = RNG(7)
    q, k, v, g = (r.standard_normal((1, 12, 2, 4)) for _ in range(4))
    out = so.attention(q, k, v, so.visible(1, 12, 12, True, 12), 0.5, d_o=g, table=r.standard_normal((6, 2)),
                       max_distance=8)
    assert np.abs(out["dtable"].sum(0)).max() < 1e-12 and np.abs(out["dtable"]).max() > 1e-2


# ------------------------------------------------------------ AdamW step
def test_step_is_adamw():
    r = RNG(8)
    w, m, v = r.standard_normal(50), np.zeros(50), np.zeros(50)
    p = torch.tensor(w.copy(), requires_grad=True)
    opt = torch.optim.AdamW([p], lr=0.01, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
    for step in range(1, 6):
        g = r.standard_normal(50)
        p.grad = torch.tensor(0.5 * g)
        opt.step()
        w, m, v = so.adamw(w, g, m, v, 0.01, 0.9, 0.95, 1e-8, step, 0.1, 0.5)
        np.testing.assert_allclose(w, p.detach().numpy(), rtol=1e-12)
    state = opt.state[p]
    np.testing.assert_allclose(m, state["exp_avg"].numpy(), rtol=1e-12)
    np.testing.assert_allclose(v, state["exp_avg_sq"].numpy(), rtol=1e-12)
    # without bias correction the first step is (1 - b1) g / (sqrt((1 - b2) g^2) + eps)
    one, _, _ = so.adamw(np.zeros(1), np.ones(1), np.zeros(1), np.zeros(1), 1.0, 0.9, 0.75, 1e-3, 1,
                         bias_correction=False)
    np.testing.assert_allclose(one, -0.1 / 0.501, rtol=1e-12)


def test_codes_are_torchs_type():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn)
    np.testing.assert_array_equal(so.e4m3_values(), codes.double().numpy())
    c, s = so.to_e4m3(np.array([-448.0, 1.0, 0.0, 2.0 ** -9]), np.zeros(4))
    assert s[0] == 1.0 and c.tolist() == [254, 56, 0, 1]
    np.testing.assert_array_equal(so.from_e4m3(c, s), [-448.0, 1.0, 0.0, 2.0 ** -9])


def test_rounding_is_even_handed_over_its_random_numbers():
    x = np.concatenate([[448.0], np.full(255, 1.03), [448.0], np.full(255, 2.0 ** -10)])
    bits = (np.arange(512) * 257) % 65536
    c, s = so.to_e4m3(x, bits)
    v = so.from_e4m3(c, s)
    assert set(v[1:256]) == {1.0, 1.125} and abs(v[1:256].mean() - 1.03) < 2e-3
    assert set(v[257:]) == {0.0, 2.0 ** -9} and abs(v[257:].mean() - 2.0 ** -10) < 2e-5
    kept, _ = so.to_e4m3(x, bits, keep=True)
    assert (so.from_e4m3(kept, s)[257:] == 2.0 ** -9).all()


def test_random_bits_are_spread():
    a, b = so.random_bits(12345, 20000), so.random_bits(12346, 20000)
    for x in (a, b):
        for part in (x >> np.uint64(16), x & np.uint64(0xffff)):
            f = part.astype(float) / 65536
            assert abs(f.mean() - 0.5) < 5 / math.sqrt(12 * 20000)
            assert abs(np.corrcoef(f[1:], f[:-1])[0, 1]) < 5 / math.sqrt(20000)
            assert np.histogram(f, 16, (0, 1))[0].std() < 5 * math.sqrt(20000 / 16)
    assert abs(np.corrcoef(a.astype(float), b.astype(float))[0, 1]) < 5 / math.sqrt(20000)
    assert len(np.intersect1d(a, b)) < 10


# -------------------------------------------------- mistakes that a pin catches
def plant(monkeypatch, name, fn):
    monkeypatch.setattr(so, name, fn)


@pytest.mark.parametrize("what", ["bias_under_cap", "no_slope", "bucket_of_magnitude", "window_off_by_one"])
def test_planted_mistakes_are_caught(monkeypatch, what):
    scores, visible, bucket = so.scores, so.visible, so.bucket
    if what == "bias_under_cap":
        def wrong(dot, h, dist, scale, cap=0.0, slopes=None, **more):
            s = scale * dot - (0 if slopes is None else slopes[h] * np.abs(dist))
            return scores(s / scale, h, dist, scale, cap, None, **more)
        plant(monkeypatch, "scores", wrong)
    elif what == "no_slope":
        plant(monkeypatch, "scores", lambda *a, **k: (scores(*a, **k)[0], np.ones_like(a[0])))
    elif what == "bucket_of_magnitude":
        plant(monkeypatch, "bucket", lambda d, n, m, causal: bucket(abs(d), n, m, causal))
    else:
        plant(monkeypatch, "visible", lambda b, q, k, causal, window, *a, **m: visible(
            b, q, k, causal, window + 1, *a, **m))
    pins = [lambda: test_attention_against_autograd(1.5, "slopes", True, [2, 9, 13]),
            lambda: test_gradients_against_differences(),
            lambda: test_buckets_follow_the_logarithm(32, 128, True), test_visible_by_hand]
    caught = 0
    for pin in pins:
        try:
            pin()
        except AssertionError:
            caught += 1
    assert caught

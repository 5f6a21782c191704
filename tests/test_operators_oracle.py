"""Pins of oracle/operators_oracle.py: gradients against central differences, the
rotation as complex numbers, torch's RMS norm and its autograd, and the
Newton-Schulz iteration as its polynomial on the singular values; and mistakes that
each pin catches."""
import math

import numpy as np
import pytest
import torch

from oracle import operators_oracle as oo

RNG = np.random.default_rng


def central(f, x, h=1e-6):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        p, q = x.copy(), x.copy()
        p[i] += h
        q[i] -= h
        g[i] = (f(p) - f(q)) / (2 * h)
    return g


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("scaling", ["plain", "linear", "by_parts"])
def test_rope_turns_pairs_and_its_gradient_is_the_transpose(interleaved, scaling):
    r = RNG(1)
    x, pos = r.standard_normal((3, 2, 10)), np.array([0, 7, -5])
    freq = oo.rope_frequencies(6, 100.0, scaling, 4.0, 64.0, 1.0, 8.0)
    y = oo.rope(x, pos, freq, interleaved, 1.5)
    first, second = (slice(0, 6, 2), slice(1, 6, 2)) if interleaved else (slice(0, 3), slice(3, 6))
    z = (x[..., first] + 1j * x[..., second]) * 1.5 * np.exp(1j * pos[:, None, None] * freq)
    np.testing.assert_allclose(y[..., first] + 1j * y[..., second], z, rtol=1e-13, atol=1e-13)
    np.testing.assert_array_equal(y[..., 6:], x[..., 6:])
    dy = r.standard_normal(x.shape)
    dx = oo.rope(dy, pos, freq, interleaved, 1.5, backward=True)
    num = central(lambda v: float(np.sum(dy * oo.rope(v, pos, freq, interleaved, 1.5))), x)
    np.testing.assert_allclose(dx, num, atol=1e-8)


def test_rope_scores_depend_on_distance_alone():
    r = RNG(2)
    q, k = r.standard_normal((1, 1, 8)), r.standard_normal((1, 1, 8))
    freq = oo.rope_frequencies(8, 10000.0)
    dot = [float(np.sum(oo.rope(q, [a], freq, False) * oo.rope(k, [b], freq, False)))
           for a, b in ((5, 2), (1005, 1002))]
    assert abs(dot[0] - dot[1]) < 1e-11


def test_rope_scaled_frequencies():
    plain = oo.rope_frequencies(64, 10000.0)
    np.testing.assert_allclose(oo.rope_frequencies(64, 10000.0, "linear", 8.0), plain / 8)
    parts = oo.rope_frequencies(64, 10000.0, "by_parts", 8.0, 4096.0)
    turns = 4096.0 * plain / (2 * math.pi)
    np.testing.assert_allclose(parts[turns >= 32], plain[turns >= 32])
    np.testing.assert_allclose(parts[turns <= 1], plain[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and np.all(parts[mid] < plain[mid]) and np.all(parts[mid] > plain[mid] / 8)


@pytest.mark.parametrize("resid", [False, True])
def test_rmsnorm_against_torch_and_differences(resid):
    r = RNG(3)
    x, g, dy, ds = (r.standard_normal(v) for v in ((4, 9), (9,), (4, 9), (4, 9)))
    res = r.standard_normal((4, 9)) if resid else None
    s, rstd, y = oo.rmsnorm(x, g, 1e-3, res)
    tx, tg = torch.tensor(x, requires_grad=True), torch.tensor(g, requires_grad=True)
    tr = torch.tensor(res, requires_grad=True) if resid else None
    ts = tx + tr if resid else tx
    ty = torch.nn.functional.rms_norm(ts, (9,), tg, 1e-3)
    np.testing.assert_allclose(y, ty.detach().numpy(), rtol=1e-12)
    ((ty * torch.tensor(dy)).sum() + (ts * torch.tensor(ds)).sum()).backward()
    dx, dg = oo.rmsnorm_backward(s, g, rstd, dy, ds)
    np.testing.assert_allclose(dx, tx.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(dg, tg.grad.numpy(), rtol=1e-10)
    if resid:
        np.testing.assert_allclose(dx, tr.grad.numpy(), rtol=1e-10, atol=1e-12)
    base = 0.0 if res is None else res
    num = central(lambda v: float(np.sum(dy * oo.rmsnorm(v, g, 1e-3, res)[2]) + np.sum(ds * (v + base))), x)
    np.testing.assert_allclose(dx, num, atol=1e-7)
    np.testing.assert_allclose(dg, central(lambda v: float(np.sum(dy * oo.rmsnorm(x, v, 1e-3, res)[2])), g),
                               atol=1e-8)


def test_e4m3_scales_by_loops():
    y = RNG(4).standard_normal((3, 75))
    y[1, 32:64] = 0.0
    s = oo.e4m3_scales(y, 32)
    for i in range(3):
        for k in range(3):
            most = max(abs(v) for v in y[i, 32 * k:32 * k + 32])
            assert s[i, k] == max(most / 448.0, 2.0 ** -126)
    np.testing.assert_array_equal(oo.e4m3_scales(y, 0)[:, 0], np.abs(y).max(1) / 448.0)


@pytest.mark.parametrize("shape", [(1, 1), (1, 6), (5, 5), (4, 9), (9, 4)])
@pytest.mark.parametrize("steps", [1, 5])
def test_newton_schulz_is_its_polynomial_on_the_singular_values(shape, steps):
    u = RNG(5).standard_normal(shape)
    p, s, q = np.linalg.svd(u, full_matrices=False)
    s = s / (math.sqrt(float(np.sum(s * s))) + 1e-7)
    a, b, c = oo.NS
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    np.testing.assert_allclose(oo.newton_schulz(u, steps), p @ np.diag(s) @ q, atol=1e-12)
    np.testing.assert_array_equal(oo.newton_schulz(np.zeros(shape)), np.zeros(shape))


def test_newton_schulz_stays_in_the_range_that_the_planes_are_scaled_for():
    """Over [0, 1]: X <= 1.2024, X X^T <= 1.446 and a + b s + c s^2 within [0.637, a], with
    the powers of two of the kernel's planes below fp16's largest number."""
    s = np.linspace(0, 1, 200001)
    a, b, c = oo.NS
    for _ in range(16):
        t = s * s
        poly = b * t + c * t * t
        assert s.max() <= 1.2024 and t.max() <= 1.446
        assert a + poly.min() >= 0.637 and poly.max() <= 1e-12
        s = np.abs(a * s + poly * s)
    assert 1.2024 * 32768 < 65504 and 1.446 * 32768 < 65504 and a * 16384 < 65504


def test_two_newton_schulz_steps_by_one_product_with_the_matrix():
    """X'' = (B' B) X with A' = (B A) B for A = X X^T, what pairs of steps compute, and
    the range of its further matrices: B A <= 1.446 and B' B <= 11.87."""
    x = RNG(6).standard_normal((7, 31))
    x /= np.linalg.norm(x) + 1e-7
    a, b, c = oo.NS
    poly = lambda t: a * np.eye(len(t)) + b * t + c * t @ t
    g = x @ x.T
    p = poly(g)
    q = poly(p @ g @ p)
    np.testing.assert_allclose(q @ p @ x, oo.newton_schulz(RNG(6).standard_normal((7, 31)), 2), atol=1e-12)
    s = np.linspace(0, 1, 200001)
    for _ in range(16):
        f = a + b * s ** 2 + c * s ** 4
        s1 = np.abs(f) * s
        f1 = a + b * s1 ** 2 + c * s1 ** 4
        assert (f * s * s).max() <= 1.446 and (f * f1).max() <= 11.87
        s = s1
    assert 1.446 * 32768 < 65504 and 11.87 * 4096 < 65504


@pytest.mark.parametrize("nesterov", [False, True])
def test_muon_step_by_hand(nesterov):
    """One row: the orthogonalised update is the unit row times the polynomial of 1."""
    w, g, m = np.array([[1.0, 2.0]]), np.array([[0.6, 0.8]]), np.array([[0.0, 0.0]])
    w2, m2, _ = oo.muon_step(w, g, m, 0.1, 0.5, nesterov, 0.2, 3.0, grad_scale=2.0, steps=1, eps=0.0)
    np.testing.assert_allclose(m2, 2 * g)
    np.testing.assert_allclose(w2, w * 0.98 - 0.3 * sum(oo.NS) * np.array([[0.6, 0.8]]))


MISTAKES = {
    "rope sign": lambda: np.allclose(oo.rope(np.ones((1, 1, 2)), [1], np.array([1.0]), False)[0, 0],
                                     [math.cos(1) + math.sin(1), math.cos(1) - math.sin(1)]),
    "mean without eps": lambda: np.allclose(oo.rmsnorm(np.full((1, 4), 1e-3), np.ones(4), 1.0)[2], 1.0),
    "sum for mean": lambda: np.allclose(oo.rmsnorm(np.ones((1, 4)), np.ones(4), 0.0)[2], 0.5),
    "cubic alone": lambda: np.allclose(oo.newton_schulz(np.ones((1, 1)), 1, 0.0), oo.NS[0] + oo.NS[1]),
}


@pytest.mark.parametrize("name", sorted(MISTAKES))
def test_mistakes_do_not_hold(name):
    assert not MISTAKES[name]()

"""Rotary positions, the root-mean-square norm and the Muon step in numpy float64,
from their definitions.  Takes arrays, imports nothing of the package."""
from __future__ import annotations

import math

import numpy as np

NS = (3.4445, -4.7750, 2.0315)


# ------------------------------------------------------- rotary positions
def rope_frequencies(rot_dim, base, scaling="plain", factor=1.0, orig_len=0.0, low=1.0, high=32.0):
    out = []
    for i in range(rot_dim // 2):
        f = base ** (-2.0 * i / rot_dim)
        if scaling == "linear":
            f = f / factor
        elif scaling == "by_parts":
            g = (orig_len * f / (2.0 * math.pi) - low) / (high - low)
            g = min(1.0, max(0.0, g))
            f = f * (g + (1.0 - g) / factor)
        out.append(f)
    return np.array(out)


def rope(x, positions, freq, interleaved, magnitude=1.0, backward=False):
    """x [tokens, heads, head_dim]; the leading 2 len(freq) elements turn."""
    x = np.asarray(x, np.float64)
    n = len(freq)
    y = x.copy()
    t = np.asarray(positions, np.float64)[:, None] * freq[None, :]
    c, s = magnitude * np.cos(t)[:, None, :], magnitude * np.sin(t)[:, None, :]
    if backward:
        s = -s
    first = slice(0, 2 * n, 2) if interleaved else slice(0, n)
    second = slice(1, 2 * n, 2) if interleaved else slice(n, 2 * n)
    a, b = x[..., first], x[..., second]
    y[..., first] = a * c - b * s
    y[..., second] = b * c + a * s
    return y


# ------------------------------------------------- root-mean-square norm
def rmsnorm(x, gamma, eps, resid=None):
    """(s, r, y) of the forward."""
    s = np.asarray(x, np.float64) + (0.0 if resid is None else np.asarray(resid, np.float64))
    r = 1.0 / np.sqrt(np.mean(s * s, axis=1) + eps)
    return s, r, s * r[:, None] * np.asarray(gamma, np.float64)


def rmsnorm_backward(s, gamma, r, dy, dsum=None):
    """(dx, dgamma)."""
    s, dy = np.asarray(s, np.float64), np.asarray(dy, np.float64)
    r = np.asarray(r, np.float64)[:, None]
    g = dy * np.asarray(gamma, np.float64)
    dx = r * g - s * r ** 3 * np.mean(g * s, axis=1, keepdims=True)
    if dsum is not None:
        dx = dx + np.asarray(dsum, np.float64)
    return dx, np.sum(dy * s * r, axis=0)


def e4m3_scales(y, group):
    """Scale of each group of columns (0: the row) before it is rounded to fp32."""
    rows, cols = y.shape
    g = group or cols
    out = np.empty((rows, -(-cols // g)))
    for k in range(out.shape[1]):
        out[:, k] = np.maximum(np.abs(y[:, k * g:(k + 1) * g]).max(axis=1) / 448.0, 2.0 ** -126)
    return out


# ------------------------------------------------------------- Muon step
def newton_schulz(u, steps=5, eps=1e-7, rnd=lambda v: v, dtype=np.float64):
    """The orthogonalised u; rnd rounds X, A and B as they are stored."""
    a, b, c = (dtype(v) for v in NS)
    x = np.asarray(u, np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = rnd((x / (math.sqrt(float(np.sum(x * x))) + eps)).astype(dtype))
    for _ in range(steps):
        gram = rnd(x @ x.T)
        poly = rnd(b * gram + c * (gram @ gram))
        x = rnd(a * x + poly @ x)
    return x.T if tall else x


def muon_step(w, g, m, lr, momentum, nesterov, weight_decay, scale, grad_scale=1.0, steps=5,
              eps=1e-7):
    """(w, m) after the step, and the orthogonalised update."""
    g = grad_scale * np.asarray(g, np.float64)
    m = momentum * np.asarray(m, np.float64) + g
    u = g + momentum * m if nesterov else m
    o = newton_schulz(u, steps, eps)
    w = np.asarray(w, np.float64)
    return w * (1.0 - lr * weight_decay) - lr * scale * o, m, o

"""Attention with terms in its scores and the AdamW step in numpy float64, from their
definitions.  Takes arrays, imports nothing of the package."""
from __future__ import annotations

import math

import numpy as np


# ------------------------------------------------------------- buckets
def bucket_borders(buckets, max_distance, causal):
    """First distance of each bucket of a side, in whole numbers."""
    n = buckets if causal else buckets // 2
    e = n // 2
    first = list(range(e + 1))
    for k in range(1, n - e):
        d = first[-1]
        while d ** (n - e) < max_distance ** k * e ** (n - e - k):
            d += 1
        first.append(d)
    return first


def bucket(distance, buckets, max_distance, causal):
    """Bucket of the distance query position - key position."""
    first = bucket_borders(buckets, max_distance, causal)
    d = max(distance, 0) if causal else abs(distance)
    b = max(i for i, f in enumerate(first) if f <= d)
    return b + (buckets // 2 if not causal and distance < 0 else 0)


# ---------------------------------------------------------------- masks
def visible(batch, seq_q, seq_k, causal, window, docs=None, prefix=None):
    """[batch, seq_q, seq_k]: docs, the offsets; one pair at a time."""
    out = np.zeros((batch, seq_q, seq_k), bool)
    docs = [b * seq_k for b in range(batch + 1)] if docs is None else list(docs)
    doc = np.full(batch * seq_k, -1)
    for d in range(len(docs) - 1):
        doc[max(docs[d], 0):max(docs[d + 1], 0)] = d
    for b in range(batch):
        for i in range(seq_q):
            p = i + seq_k - seq_q
            d = doc[b * seq_k + p]
            if d < 0:
                continue
            for j in range(seq_k):
                if doc[b * seq_k + j] != d:
                    continue
                ok = 0 <= p - j < window if causal else abs(p - j) < window
                if prefix is not None and b * seq_k + j < docs[d] + prefix[d]:
                    ok = True
                out[b, i, j] = ok
    return out


# ------------------------------------------------------------ attention
def scores(dot, h, dist, scale, cap=0.0, slopes=None, table=None, max_distance=0, causal=True):
    """Scores of the products q.k of head h at distances dist, and the cap's slope."""
    s = scale * dot
    slope = np.ones_like(s)
    if cap:
        t = np.tanh(s / cap)
        s, slope = cap * t, 1.0 - t * t
    if slopes is not None:
        s = s - slopes[h] * np.abs(dist)
    if table is not None:
        n = len(table)
        of = {d: bucket(d, n, max_distance, causal) for d in np.unique(dist)}
        s = s + np.vectorize(lambda d: table[of[d]][h])(dist)
    return s, slope


def attention(q, k, v, see, scale, d_o=None, **terms):
    """q, d_o [batch, seq_q, heads, d]; k, v [batch, seq_k, kv_heads, d]; see as visible()
    gives it.  (o, lse), or with d_o a dict of the gradients too.  Rows that see nothing:
    o 0, lse -inf.  What see hides is never read.  a_* : what the results' roundings grow
    with, the same sums over magnitudes."""
    batch, seq_q, heads, d = q.shape
    seq_k, kv_heads = k.shape[1], k.shape[2]
    group = heads // kv_heads
    dist = np.arange(seq_k - seq_q, seq_k)[:, None] - np.arange(seq_k)[None]
    r = dict(o=np.zeros(q.shape), lse=np.full((batch, heads, seq_q), -np.inf),
             a_o=np.zeros(q.shape), a_s=np.zeros((batch, heads, seq_q)))
    if d_o is not None:
        table = terms.get("table")
        r.update({n: np.zeros(x.shape) for n, x in (
            ("dq", q), ("dk", k), ("dv", v), ("a_dq", q), ("a_dk", k), ("a_dv", v), ("e_dq", q),
            ("e_dk", k))})
        if table is not None:
            r.update(dtable=np.zeros(np.shape(table)), a_dtable=np.zeros(np.shape(table)))
            n, md, causal = len(table), terms["max_distance"], terms.get("causal", True)
            of = {x: bucket(x, n, md, causal) for x in np.unique(dist)}
            ids = np.vectorize(of.get)(dist)
    for b in range(batch):
        for h in range(heads):
            g = h // group
            m = see[b]
            any_ = m.any(1)
            keys = m.any(0)  # (rows that nothing reads may hold anything)
            kk = np.where(keys[:, None], k[b, :, g], 0.0)
            vv = np.where(keys[:, None], v[b, :, g], 0.0)
            qq = np.where(any_[:, None], q[b, :, h], 0.0)
            s, slope = scores(qq @ kk.T, h, dist, scale, **terms)
            s = np.where(m, s, -np.inf)
            top = np.where(any_, s.max(1, initial=-np.inf), 0.0)
            top = np.where(np.isfinite(top), top, 0.0)
            p = np.exp(s - top[:, None])
            total = p.sum(1)
            live = total > 0
            p = p / np.where(live, total, 1.0)[:, None]
            r["o"][b, :, h] = p @ vv
            r["a_o"][b, :, h] = p @ np.abs(vv)
            with np.errstate(divide="ignore"):
                r["lse"][b, h] = top + np.log(total)
            mag = scale * (np.abs(qq) @ np.abs(kk).T)  # of the products' own sums
            finite = np.abs(np.where(np.isfinite(s), s, 0.0))  # (a bias of -inf masks)
            r["a_s"][b, h] = np.where(m, mag + finite, 0.0).max(1)
            if d_o is None:
                continue
            gg = np.where(any_[:, None], d_o[b, :, h], 0.0)
            dp = gg @ vv.T
            delta = (p * dp).sum(1, keepdims=True)
            dz = p * (dp - delta)
            du = dz * slope
            r["dv"][b, :, g] += p.T @ gg
            r["a_dv"][b, :, g] += p.T @ np.abs(gg)
            r["dq"][b, :, h] = scale * du @ kk
            r["a_dq"][b, :, h] = scale * np.abs(du) @ np.abs(kk)
            r["dk"][b, :, g] += scale * du.T @ qq
            r["a_dk"][b, :, g] += scale * np.abs(du).T @ np.abs(qq)
            # what an error of the row term by sum |d_o| (|o| + sum p |v|) gives
            err = (np.abs(gg) * (np.abs(r["o"][b, :, h]) + r["a_o"][b, :, h])).sum(1, keepdims=True)
            pe = p * slope * err
            r["e_dq"][b, :, h] = scale * pe @ np.abs(kk)
            r["e_dk"][b, :, g] += scale * pe.T @ np.abs(qq)
            if terms.get("table") is not None:
                # errors of the scores, of dP and of the row term, relative to 1
                a_dp = np.abs(gg) @ np.abs(vv).T
                a = p * ((mag + finite + 4) * (np.abs(dp) + np.abs(delta)) + a_dp
                         + (p * a_dp).sum(1, keepdims=True))
                for n in range(len(terms["table"])):
                    at = ids == n
                    r["dtable"][n, h] += dz[at].sum()
                    r["a_dtable"][n, h] += a[at].sum()
    return (r["o"], r["lse"]) if d_o is None else r


# ------------------------------------------------------------ AdamW step
BLOCK = 256


def random_bits(seed, n):
    """32 bits for each element's number below n."""
    word = 0xffffffff
    out = np.empty(n, np.uint64)
    for e in range(n):
        x = ((e & word) * 0x9E3779B1 + (seed & word)) & word
        x = ((x ^ (x >> 16)) * 0x6A09E667) & word
        x = (x + (e >> 32) * 0x9E3779B1 + (seed >> 32)) & word
        x = ((x ^ (x >> 15)) * 0xBB67AE85) & word
        out[e] = x ^ (x >> 16)
    return out


def e4m3_values():
    """The magnitudes of the codes 0 .. 126."""
    return np.array([(c % 8) * 2.0 ** -9 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7)
                     for c in range(127)])


def to_e4m3(x, bits, keep=False):
    """(codes, scales) of x; bits: 16 random ones each.  Below the quotient, or above
    where its place between the neighbours and bits / 2^16 add up to one."""
    grid = e4m3_values()
    codes = np.zeros(len(x), np.uint8)
    scales = np.empty(-(-len(x) // BLOCK), np.float32)
    for k in range(len(scales)):
        part = slice(k * BLOCK, (k + 1) * BLOCK)
        y = np.asarray(x[part], np.float64)
        scales[k] = max(np.abs(y).max() / 448.0, 2.0 ** -126)
        y = y / np.float64(scales[k])
        a = np.minimum(np.abs(y), 448.0)
        low = np.searchsorted(grid, a, side="right") - 1
        high = np.minimum(low + 1, 126)
        gap = np.where(high > low, grid[high] - grid[low], 1.0)
        c = np.where((a - grid[low]) / gap + bits[part] / 65536.0 >= 1.0, high, low)
        if keep:
            c = np.where((a > 0) & (c == 0), 1, c)
        codes[part] = c + np.where((y < 0) & (not keep), 128, 0)
    return codes, scales


def to_e4m3_of(x, err, bits, scale, keep=False):
    """For each element the codes that a value within err of x may get."""
    grid = e4m3_values()
    out = []
    for v, e, b, s in zip(np.abs(x), err, bits, scale):
        codes = set()
        for a in ((v - e) / s, v / s, (v + e) / s):
            a = min(max(a, 0.0), 448.0)
            low = int(np.searchsorted(grid, a, side="right")) - 1
            high = min(low + 1, 126)
            up = high > low and (a - grid[low]) / (grid[high] - grid[low]) + b / 65536.0 >= 1.0
            codes.add(high if up else low)
        out.append(codes)
    sign = np.where((np.asarray(x) < 0) & (not keep), 128, 0)
    return [{(max(c, 1) if keep and v > 0 else c) + int(g) for c in s}
            for s, g, v in zip(out, sign, np.abs(x))]


def from_e4m3(codes, scales):
    v = e4m3_values()[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    return v * np.repeat(scales.astype(np.float64), BLOCK)[:len(codes)]


def adamw(w, g, m, v, lr, beta1, beta2, eps, step, weight_decay=0.0, grad_scale=1.0,
          bias_correction=True):
    """(w, m, v) after the step."""
    w, g, m, v = (np.asarray(x, np.float64) for x in (w, g, m, v))
    g = grad_scale * g
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    c1 = 1.0 - beta1 ** step if bias_correction else 1.0
    c2 = 1.0 - beta2 ** step if bias_correction else 1.0
    return w - lr * weight_decay * w - lr * (m / c1) / (np.sqrt(v / c2) + eps), m, v

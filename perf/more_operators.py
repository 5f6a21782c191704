"""Attention with terms in its scores, and the AdamW step: what a training program
with packed documents and position biases runs next to the block calls.

A case is one pass as a program makes it:

  forward   attention whose scores are capped by a tanh, or get a bias by distance
            or by learned buckets, under a document, prefix or window mask, with
            key heads that query heads may share
  backward  its gradients (the bias table's among them), from what the forward kept
  adamw     the optimizer's step over many tensors, with states in 32 or 8 bits

``listed`` has the fixed cases, ``draw`` more of the same ranges, ``prepare``
what a program holds before the call, ``run`` the call (in elementary torch
operations, or where ``own`` is set through ``paper_2402_15627_amd.pblock``),
``work`` the bytes and operations it cannot do without, ``exact`` the outputs
from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
ADAMW = dict(lr=6e-5, beta1=0.9, beta2=0.95, eps=1e-8, step=100, grad_scale=0.5)
DECAY = 0.1
BLOCK = 256  # elements of a state that share a scale
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126


def _attn(name, kind, dtype, batch, seq, heads, kv_heads, head_dim, **more):
    """docs: lengths of the documents that lie one after another in the batch's
    tokens (none: each sequence is one); prefix: of each, the leading tokens that
    all of it sees. seq_q: the queries are the last ones of each sequence."""
    c = dict(kind=kind, dtype=dtype, batch=batch, seq=seq, seq_q=seq, heads=heads,
             kv_heads=kv_heads, head_dim=head_dim, causal=True, window=seq, cap=0.0, bias="none",
             buckets=0, max_distance=0, docs="", prefix="")
    c.update(more)
    return dict(c, name=name) if name else c


def _adamw(name, state, sizes):
    """sizes: elements, or elements * tensors, each tensor "@" elements into its storage."""
    c = dict(kind="adamw", dtype="f32", state=state, sizes=sizes)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token of four long contexts, bias by distance, eight key heads
        # for forty query heads: what an evaluation during training generates with.
        _attn("token_slopes", "forward", "bf16", 4, 8192, 40, 8, 128, seq_q=1, bias="slopes"),
        # Capped scores at the 175B tensor-parallel share.
        _attn("fwd_cap_175b_share", "forward", "bf16", 1, 2048, 12, 12, 128, cap=30.0),
        # A long row of packed documents with a bias by distance, the last 64
        # tokens padding: the largest forward.
        _attn("fwd_docs_slopes_8k", "forward", "bf16", 1, 8192, 16, 4, 128, window=4096,
              bias="slopes", docs="2731,1000,1,4096,300"),
        # Gradients with capped scores, packed documents and prefixes: the
        # largest backward.
        _attn("bwd_cap_docs_prefix", "backward", "bf16", 1, 4096, 16, 4, 128, cap=50.0,
              docs="1500,77,2519", prefix="300,0,1000"),
        # fp32, odd lengths, shared key heads, a prefix of each sequence.
        _attn("fwd_f32_ragged", "forward", "f32", 2, 333, 16, 4, 96, cap=20.0, bias="slopes",
              prefix="50,7"),
        # Short sequences that see both ways, with learned buckets.
        _attn("fwd_buckets_both_ways", "forward", "bf16", 8, 512, 8, 8, 64, causal=False,
              bias="buckets", buckets=32, max_distance=128),
        # Gradients, the table's among them, at the 13B width and window.
        _attn("bwd_buckets_13b", "backward", "bf16", 1, 2048, 40, 40, 128, window=512,
              bias="buckets", buckets=32, max_distance=128),
        # The smallest block's attention: launches and one chain of dependent work.
        _attn("bwd_buckets_f32_tiny", "backward", "f32", 1, 128, 4, 4, 64, window=64,
              bias="buckets", buckets=16, max_distance=64),
        # The biases, norm gains and bias tables of 24 layers at the 13B width.
        _adamw("adamw_vectors", "f32", "5120*72,35840*24,1280*24"),
        # The 175B share's weights as one step takes them, with their bf16 copies.
        _adamw("adamw_175b_share", "f32", "132120576,12288*3,10752,94371840"),
        # The same with states of 8 bits: the largest of these.
        _adamw("adamw_e4m3_175b_share", "e4m3", "132120576,12288*3,10752,94371840"),
        # Odd sizes from one element up, at odd places.
        _adamw("adamw_e4m3_ragged", "e4m3", "1,255,257@1,99999@3,1048577,65536@2"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("forward", "forward", "backward", "backward", "adamw"))
    if kind == "adamw":
        sizes, left = [], 100_000_000
        for _ in range(rng.choice((1, 2, 5, 12))):
            n = min(_log(rng, 1, 30_000_000), left)
            many = rng.choice((1, 1, 3, 20)) if n < 100_000 else 1
            if n < 1:
                break
            left -= n * many
            sizes.append("%d" % n + ("*%d" % many if many > 1 else "") +
                         ("@%d" % rng.randint(1, 7) if rng.random() < 0.25 else ""))
        return _adamw(None, rng.choice(("f32", "e4m3")), ",".join(sizes))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    head_dim = rng.choice((64, 96, 128, 128))
    kv_heads = _log(rng, 1, 16)
    heads = kv_heads * rng.choice((1, 1, 2, 4, 5, 8))
    batch = rng.choice((1, 1, 2, 3, 8))
    # scores as many as the largest listed cases have (fp32: an eighth)
    most = 2 ** 28 if kind == "backward" else 2 ** 30
    most = most // (heads * batch * (8 if dtype == "f32" else 1))
    seq = max(1, min(_log(rng, 1, 8192), int(math.sqrt(most))))
    c = dict(causal=rng.random() < 0.75)
    c["window"] = seq if rng.random() < 0.5 else _log(rng, 1, seq)
    if kind == "forward" and c["causal"] and rng.random() < 0.25:
        c["seq_q"] = 1 if rng.random() < 0.5 else rng.randint(1, seq)
    c["cap"] = rng.choice((0.0, 0.0, 20.0, 50.0))
    c["bias"] = rng.choice(("none", "slopes", "buckets", "buckets"))
    if c["bias"] == "buckets":
        c["buckets"] = rng.choice((8, 16, 32, 64))
        c["max_distance"] = rng.choice((64, 128, 128, 300, 1024))
    lengths = [seq] * batch
    if rng.random() < 0.5:
        lengths, left = [], batch * seq
        while left > 0 and len(lengths) < 60:
            lengths.append(min(_log(rng, 1, max(1, seq)), left))
            left -= lengths[-1]
        c["docs"] = ",".join(map(str, lengths))
    if rng.random() < 0.4:
        c["prefix"] = ",".join(str(rng.randint(0, n)) for n in lengths)
    return _attn(None, kind, dtype, batch, seq, heads, kv_heads, head_dim, **c)


def _ints(text):
    return [int(v) for v in text.split(",") if v]


def _sizes(c):
    out = []
    for t in c["sizes"].split(","):
        t, _, at = t.partition("@")
        n, _, many = t.partition("*")
        out += [(int(n), int(at) if at else 0)] * (int(many) if many else 1)
    return out


def _act(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _seeded(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return lambda *shape, std=1.0, mean=0.0: torch.empty(shape, device=DEV).normal_(mean, std, generator=g)


def _prepare_adamw(s, rnd, seed):
    s["tensors"] = []

    def at(x, off):
        """x's values, off elements into a storage of their own."""
        if not off:
            return x
        return torch.empty(x.numel() + off, dtype=x.dtype, device=DEV)[off:].copy_(x)

    for i, (n, off) in enumerate(_sizes(s)):
        t = dict(w=at(rnd(n, std=0.02), off), g=at(rnd(n, std=1e-3), off),
                 copy=at(torch.empty(n, dtype=torch.bfloat16, device=DEV), off),
                 decay=DECAY if n > 50000 else 0.0, seed=seed * 1000003 + i)
        m, r = rnd(n, std=2e-4), rnd(n, std=5e-4).abs() + 1e-5
        if s["state"] == "f32":
            t.update(m=at(m, off), v=at(r.square_(), off))
        else:
            # states as an earlier step left them: codes and a scale per block
            for key, x in (("m", m), ("r", r)):
                pad = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
                scale = (pad.abs().amax(1) / E4M3_MAX).clamp(min=SCALE_MIN)
                q = (pad / scale[:, None]).view(-1)[:n].to(torch.float8_e4m3fn)
                t[key], t[key + "_scale"] = at(q, off), scale
        s["tensors"].append(t)
    return s


def prepare(case, seed):
    c = case
    rnd = _seeded(seed)
    s = dict(c)
    if c["kind"] == "adamw":
        return _handles(_prepare_adamw(s, rnd, seed))
    act, d = _act(c), c["head_dim"]
    B, Sq, Sk, H, KV = c["batch"], c["seq_q"], c["seq"], c["heads"], c["kv_heads"]
    s["act"] = act

    def packed(rows, widths):
        """Column ranges of one matrix, as the in-projection's output has them."""
        z = rnd(rows, sum(widths) + 64).to(act)
        at = np.cumsum([0] + widths)
        return [z[:, a:b] for a, b in zip(at[:-1], at[1:])]

    if Sq == Sk:
        s["q"], s["k"], s["v"] = packed(B * Sk, [H * d, KV * d, KV * d])
    else:
        s["q"], = packed(B * Sq, [H * d])
        s["k"], s["v"] = packed(B * Sk, [KV * d, KV * d])
    s["q"].mul_(2.0)  # scores of a standard deviation of 2
    s["scale"] = 1.0 / math.sqrt(d)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s["docs"] = ints(np.cumsum([0] + _ints(c["docs"])).tolist()) if c["docs"] else None
    s["prefix"] = ints(_ints(c["prefix"])) if c["prefix"] else None
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device=DEV) / H) if c["bias"] == "slopes" else None
    s["table"] = rnd(c["buckets"], H, std=0.7) if c["bias"] == "buckets" else None
    new = lambda *shape, dtype=act: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    s["o"], s["lse"] = new(B * Sq, H * d), new(B, H, Sq, dtype=torch.float32)
    if c["kind"] == "backward":
        o, lse = _plain_forward(s)
        s["o"].copy_(o)
        s["lse"].copy_(lse)
        s["d_o"] = rnd(B * Sq, H * d).to(act)
        dz = new(B * Sk, (H + 2 * KV) * d)
        s["dq"], s["dk"], s["dv"] = dz[:, :H * d], dz[:, H * d:(H + KV) * d], dz[:, (H + KV) * d:]
        s["dtable"] = new(c["buckets"], H, dtype=torch.float32) if c["bias"] == "buckets" else None
    return _handles(s)


def _handles(s):
    """What a program of the library makes once and keeps: configurations and
    workspaces. Plain forms need none."""
    if not own:
        return s
    from paper_2402_15627_amd import pblock as pb
    if s["kind"] == "adamw":
        s["cfg"] = pb.adamw_config(**ADAMW)
        s["parts"] = pb.AdamwTensors(
            pb.adamw_tensor(t["w"], t["g"], t["m"], t["v"], t["copy"], t["decay"])
            if s["state"] == "f32" else
            pb.adamw_tensor(t["w"], t["g"], t["m"], t["r"], t["copy"], t["decay"], t["m_scale"],
                            t["r_scale"], t["seed"])
            for t in s["tensors"])
        return s
    s["cfg"] = pb.score_attn_config(s["batch"], s["seq_q"], s["seq"], s["heads"], s["kv_heads"],
                                    s["head_dim"], causal=s["causal"], window=s["window"],
                                    cap=s["cap"], buckets=s["buckets"],
                                    max_distance=s["max_distance"], dtype=s["dtype"])
    mode = pb.ATTN_WS_BACKWARD if s["kind"] == "backward" else pb.ATTN_WS_FORWARD
    n = pb.pblock_score_attn_workspace_bytes(s["cfg"], mode)
    s["ws"] = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------ the passes
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2402_15627_amd import pblock as pb
    if s["kind"] == "adamw":
        pb.pblock_adamw_step(s["cfg"], s["parts"], pb.PB_BF16)
        return _adamw_outputs(s)
    terms = dict(docs=s["docs"], prefix=s["prefix"], slopes=s["slopes"], table=s["table"])
    if s["kind"] == "forward":
        pb.pblock_score_attn_forward(s["cfg"], s["q"], s["k"], s["v"], s["o"], s["lse"],
                                     ws=s["ws"], **terms)
        return dict(o=s["o"], lse=s["lse"])
    pb.pblock_score_attn_backward(s["cfg"], s["q"], s["k"], s["v"], s["o"], s["d_o"], s["lse"],
                                  s["dq"], s["dk"], s["dv"], s["ws"], dtable=s["dtable"], **terms)
    return dict(dq=s["dq"], dk=s["dk"], dv=s["dv"], dtable=s["dtable"])


def _run_plain(s):
    if s["kind"] == "adamw":
        for t in s["tensors"]:
            _plain_adamw(s, t)
        return _adamw_outputs(s)
    if s["kind"] == "forward":
        o, lse = _plain_forward(s)
        s["o"].copy_(o)
        return dict(o=s["o"], lse=lse)
    return _plain_backward(s)


def _heads_first(x, B, S, KV, d):
    """[B S, heads d] -> [B KV, heads/KV S, d] in fp32."""
    x = x.float().reshape(B, S, KV, -1, d)
    return x.permute(0, 2, 3, 1, 4).reshape(B * KV, -1, d).contiguous()


def _tokens_first(x, B, S, KV, d):
    return x.view(B, KV, -1, S, d).permute(0, 3, 1, 2, 4).reshape(B * S, -1)


def _visible(s):
    """[B, Sq, Sk]: which keys each query sees."""
    B, Sq, Sk = s["batch"], s["seq_q"], s["seq"]
    j = torch.arange(Sk, device=DEV)
    p = j[Sk - Sq:, None]
    row = torch.arange(B, device=DEV)[:, None] * Sk
    if s["docs"] is None:
        first, end = torch.zeros((B, Sk), dtype=torch.long, device=DEV), torch.full((B, Sk), Sk, device=DEV)
        doc = torch.arange(B, device=DEV)[:, None].expand(B, Sk)
        inside = torch.ones((B, Sk), dtype=torch.bool, device=DEV)
    else:
        docs = s["docs"].long()
        n = docs.numel() - 1
        doc = torch.bucketize(row + j, docs, right=True) - 1
        inside = (doc >= 0) & (doc < n)
        doc = doc.clamp(0, max(n - 1, 0))
        first, end = docs[doc] - row, docs[doc + 1] - row
    pick = lambda x: x[:, Sk - Sq:, None]  # noqa: E731
    near = (p - j < s["window"]) & (p - j >= 0) if s["causal"] else (p - j).abs() < s["window"]
    if s["prefix"] is not None:
        near = near | (j < pick(first + s["prefix"].long()[doc]))
    return pick(inside) & (j >= pick(first)) & (j < pick(end)) & near


def _bucket(s, dist):
    """Bucket of each distance (query position minus key position). (Logarithms in
    64 bits: distances next to a border.)"""
    n = s["buckets"] if s["causal"] else s["buckets"] // 2
    d = dist.clamp(min=0) if s["causal"] else dist.abs()
    whole = n // 2
    far = torch.log(d.clamp(min=1).double() / whole) / math.log(s["max_distance"] / whole)
    far = whole + torch.floor(far * (n - whole) + 1e-9).long()
    b = torch.where(d < whole, d, far.clamp(max=n - 1))
    return b if s["causal"] else b + n * (dist < 0)


def _scores(s, q, k):
    """Scores [B, KV, G, Sq, Sk] before the mask, and what the cap's tanh gives."""
    B, Sq, Sk, H, KV = s["batch"], s["seq_q"], s["seq"], s["heads"], s["kv_heads"]
    x = torch.bmm(q, k.mT.contiguous()).mul_(s["scale"]).view(B, KV, H // KV, Sq, Sk)
    t = None
    if s["cap"] > 0:
        t = torch.tanh(x / s["cap"])
        x = t * s["cap"]
    j = torch.arange(Sk, device=DEV)
    dist = j[Sk - Sq:, None] - j
    if s["slopes"] is not None:
        x = x - s["slopes"].view(KV, -1, 1, 1) * dist.abs()
    if s["table"] is not None:
        x = x + s["table"][_bucket(s, dist)].permute(2, 0, 1).reshape(KV, -1, Sq, Sk)
    return x, t


def _plain_forward(s):
    B, Sq, Sk, H, KV, d = (s[n] for n in ("batch", "seq_q", "seq", "heads", "kv_heads", "head_dim"))
    q, k, v = _heads_first(s["q"], B, Sq, KV, d), _heads_first(s["k"], B, Sk, KV, d), _heads_first(s["v"], B, Sk, KV, d)
    x, _ = _scores(s, q, k)
    x = x.masked_fill(~_visible(s)[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - top.clamp(min=torch.finfo(torch.float32).min))
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(B * KV, -1, Sk), v).view(B, KV, -1, Sq, d) / total.clamp(min=1e-30)
    lse = (top + torch.log(total)).view(B, H, Sq)
    return _tokens_first(o, B, Sq, KV, d).to(s["act"]), lse


def _plain_backward(s):
    B, Sq, Sk, H, KV, d = (s[n] for n in ("batch", "seq_q", "seq", "heads", "kv_heads", "head_dim"))
    q, k, v = _heads_first(s["q"], B, Sq, KV, d), _heads_first(s["k"], B, Sk, KV, d), _heads_first(s["v"], B, Sk, KV, d)
    g = _heads_first(s["d_o"], B, Sq, KV, d)
    x, t = _scores(s, q, k)
    lse = s["lse"].view(B, KV, -1, Sq, 1)
    p = torch.exp(x - lse.clamp(min=torch.finfo(torch.float32).min))
    p = p.masked_fill(~_visible(s)[:, None, None], 0.0).view(B * KV, -1, Sk)
    dv = torch.bmm(p.mT.contiguous(), g)
    ds = torch.bmm(g, v.mT.contiguous())
    # (the row's term from unrounded values: what the forward kept is rounded, and
    # the table's gradient, sums over thousands of rows, shows it)
    ds = ds.sub_((p * ds).sum(-1, keepdim=True)).mul_(p)
    out = {}
    if s["table"] is not None:
        # sums along the diagonals (each one distance), in 64 bits: long sums
        rows = ds.view(B, H, Sq, Sk).sum(0, dtype=torch.float64).flip(1)
        rows = torch.nn.functional.pad(rows, (0, Sq)).view(H, -1)[:, :Sq * (Sk + Sq - 1)]
        by_distance = rows.view(H, Sq, Sk + Sq - 1).sum(1)
        bucket = _bucket(s, Sk - 1 - torch.arange(Sk + Sq - 1, device=DEV))
        of = torch.nn.functional.one_hot(bucket, s["buckets"]).double()
        out["dtable"] = (by_distance @ of).t().float()
    if t is not None:
        ds = ds * (1 - t * t).view_as(ds)
    dq, dk = torch.bmm(ds, k).mul_(s["scale"]), torch.bmm(ds.mT.contiguous(), q).mul_(s["scale"])
    for name, x, S in (("dq", dq, Sq), ("dk", dk, Sk), ("dv", dv, Sk)):
        out[name] = s[name].copy_(_tokens_first(x, B, S, KV, d))
    return out


def _adamw_outputs(s):
    names = ("w", "copy", "m", "v") if s["state"] == "f32" else ("w", "copy", "m", "m_scale", "r", "r_scale")
    if len(s["tensors"]) <= 8:
        return [{n: t[n] for n in names} for t in s["tensors"]]
    return {n: torch.cat([t[n] for t in s["tensors"]]) for n in names}


def _random(seed, n):
    """Of each element's number, 32 bits by two rounds of shifts and products."""
    low = 0xffffffff
    e = torch.arange(n, device=DEV)
    x = ((e & low) * 0x9E3779B1 + (seed & low)) & low
    x = ((x ^ (x >> 16)) * 0x6A09E667) & low
    x = (x + (((e >> 32) * 0x9E3779B1) & low) + ((seed >> 32) & low)) & low
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & low
    return x ^ (x >> 16)


def _to_e4m3(x, bits, keep):
    """Codes of x and their scales, rounded up where `bits` (16) say so: to either
    neighbour as often as it is near. keep: what is above zero stays so. (In 64
    bits: values next to a border.)"""
    n = x.numel()
    pad = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    scale = (pad.abs().amax(1) / E4M3_MAX).clamp(min=SCALE_MIN)
    y = (pad * (1.0 / scale)[:, None]).view(-1)[:n]
    a = y.abs().double()
    step = torch.exp2((torch.frexp(a).exponent - 1).clamp(min=-6) - 3.0)
    q = torch.floor(a / step + bits.double() / 65536) * step
    q = q.clamp(max=E4M3_MAX)
    if keep:
        q = torch.where(a > 0, q.clamp(min=2.0 ** -9), q)
    return (q * y.sign()).float().to(torch.float8_e4m3fn), scale


def _from_e4m3(q, scale):
    return q.float() * scale.repeat_interleave(BLOCK)[:q.numel()]


def _plain_adamw(s, t):
    f = lambda v: float(np.float32(v))  # noqa: E731
    b1, b2 = f(ADAMW["beta1"]), f(ADAMW["beta2"])
    c1, c2 = f(1 / (1 - b1 ** ADAMW["step"])), f(1 / (1 - b2 ** ADAMW["step"]))
    lr, eps = f(ADAMW["lr"]), f(ADAMW["eps"])
    if s["state"] == "f32":
        m, v = t["m"], t["v"]
    else:
        m, v = _from_e4m3(t["m"], t["m_scale"]), _from_e4m3(t["r"], t["r_scale"]).square()
    g = t["g"] * f(ADAMW["grad_scale"])
    m = m * b1 + g * (1 - b1)
    v = v * b2 + (g * g) * (1 - b2)
    u = (m * c1) / (torch.sqrt(v * c2) + eps)
    t["w"].copy_(t["w"] * f(1 - lr * f(t["decay"])) - u * lr)
    t["copy"].copy_(t["w"])
    if s["state"] == "f32":
        t["m"].copy_(m)
        t["v"].copy_(v)
        return
    bits = _random(t["seed"], m.numel())
    for name, x, part, keep in (("m", m, bits >> 16, False), ("r", torch.sqrt(v), bits & 0xffff, True)):
        q, scale = _to_e4m3(x, part, keep)
        t[name].copy_(q)
        t[name + "_scale"].copy_(scale)


# ----------------------------------------------------------- what it takes
def _pairs(c):
    """(query, key) pairs that are visible, of one head."""
    B, Sq, Sk = c["batch"], c["seq_q"], c["seq"]
    lengths = _ints(c["docs"]) if c["docs"] else [Sk] * B
    prefix = _ints(c["prefix"]) if c["prefix"] else [0] * len(lengths)
    total, at = 0, 0
    for n, pre in zip(lengths, prefix):
        for b in range(at // Sk, (at + n - 1) // Sk + 1) if n else ():
            # the document's part in sequence b, and its queries
            lo, hi = max(at, b * Sk) - b * Sk, min(at + n, (b + 1) * Sk) - b * Sk
            p = np.arange(max(lo, Sk - Sq), hi)
            known = at + pre - b * Sk
            first = np.maximum(p - c["window"] + 1, lo)
            last = p if c["causal"] else np.minimum(p + c["window"] - 1, hi - 1)
            end = min(max(known, lo), hi)  # of the prefix
            total += int((last - first + 1).sum())
            total += int((end - lo - np.maximum(0, np.minimum(end, last + 1) - np.maximum(lo, first))).sum())
        at += n
    return total


def work(case):
    c = case
    if c["kind"] == "adamw":
        n = sum(size for size, _ in _sizes(c))
        blocks = sum(-(-size // BLOCK) for size, _ in _sizes(c))
        # w, g, m, v read; w, m, v and the copy written
        return {"bytes": 30 * n if c["state"] == "f32" else 18 * n + 16 * blocks, "flops": 14 * n}
    e = 2 if c["dtype"] == "bf16" else 4
    q = c["batch"] * c["seq_q"] * c["heads"] * c["head_dim"] * e
    k = c["batch"] * c["seq"] * c["kv_heads"] * c["head_dim"] * e
    lse = 4 * c["batch"] * c["seq_q"] * c["heads"]
    flops = 2 * c["head_dim"] * c["heads"] * _pairs(c)
    if c["kind"] == "forward":
        return {"bytes": 2 * q + 2 * k + lse, "flops": 2 * flops}
    # q, o, d_o, k, v read, dq, dk, dv written; scores and four more products
    return {"bytes": 4 * q + 4 * k + lse, "flops": 5 * flops}


# ------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    c = dict(case)
    s = prepare(case, seed)
    if c["kind"] == "adamw":
        return _exact_adamw(c, s)
    return _exact_attn(c, s)


def _exact_borders(c):
    """First distance of each bucket, in whole numbers: d belongs to bucket whole + k
    or a later one where (d / whole)^logs >= (max_distance / whole)^k."""
    n = c["buckets"] if c["causal"] else c["buckets"] // 2
    whole = n // 2
    logs = n - whole
    first = list(range(whole + 1))
    for k in range(1, logs):
        d = first[-1]
        while d ** logs < c["max_distance"] ** k * whole ** (logs - k):
            d += 1
        first.append(d)
    return n, first


def _exact_attn(c, s):
    B, Sq, Sk, H, KV, d = (c[n] for n in ("batch", "seq_q", "seq", "heads", "kv_heads", "head_dim"))
    lengths = _ints(c["docs"]) if c["docs"] else [Sk] * B
    prefix = _ints(c["prefix"]) if c["prefix"] else [0] * len(lengths)
    doc = np.full(B * Sk, -1)
    known = np.zeros(B * Sk, dtype=bool)  # keys in their document's prefix
    at = 0
    for i, (n, pre) in enumerate(zip(lengths, prefix)):
        doc[at:at + n] = i
        known[at:at + min(pre, n)] = True
        at += n
    doc, known = torch.tensor(doc, device=DEV), torch.tensor(known, device=DEV)
    dist = torch.arange(Sk - Sq, Sk, device=DEV)[:, None] - torch.arange(Sk, device=DEV)[None]
    near = ((dist >= 0) if c["causal"] else (dist > -c["window"])) & (dist < c["window"])
    bucket = None
    if c["bias"] == "buckets":
        n, first = _exact_borders(c)
        of = lambda x: torch.searchsorted(torch.tensor(first, device=DEV), x, right=True) - 1  # noqa: E731
        bucket = of(dist.clamp(min=0)) if c["causal"] else torch.where(dist < 0, n + of(-dist.clamp(max=0)), of(dist.clamp(min=0)))
    double = lambda x, S: x.double().reshape(B, S, -1, d)  # noqa: E731
    q, k, v = double(s["q"], Sq), double(s["k"], Sk), double(s["v"], Sk)
    o, lse = torch.zeros_like(q), torch.empty((B, H, Sq), dtype=torch.float64, device=DEV)
    if c["kind"] == "backward":
        g = double(s["d_o"], Sq)
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        dtable = torch.zeros((max(1, c["buckets"]), H), dtype=torch.float64, device=DEV)
    for b in range(B):
        ids = doc[b * Sk:(b + 1) * Sk]
        sees = (ids[Sk - Sq:, None] == ids[None]) & (ids[None] >= 0)
        sees = sees & (near | known[None, b * Sk:(b + 1) * Sk])
        for h in range(H):
            kv = h // (H // KV)
            raw = (q[b, :, h] @ k[b, :, kv].t()) / math.sqrt(d)
            x = raw if not c["cap"] else c["cap"] * torch.tanh(raw / c["cap"])
            if c["bias"] == "slopes":
                x = x - float(s["slopes"][h]) * dist.abs()
            if bucket is not None:
                x = x + s["table"][:, h].double()[bucket]
            x = torch.where(sees, x, -math.inf)
            lse[b, h] = torch.logsumexp(x, 1)
            p = torch.where(sees, torch.exp(x - lse[b, h][:, None]), 0.0)
            o[b, :, h] = p @ v[b, :, kv]
            if c["kind"] == "forward":
                continue
            dv[b, :, kv] += p.t() @ g[b, :, h]
            dp = g[b, :, h] @ v[b, :, kv].t()
            dx = p * (dp - (p * dp).sum(1, keepdim=True))
            if bucket is not None:
                dtable[:, h].index_add_(0, bucket.reshape(-1), dx.reshape(-1))
            if c["cap"]:
                dx = dx / torch.cosh(raw / c["cap"]) ** 2
            dq[b, :, h] = dx @ k[b, :, kv] / math.sqrt(d)
            dk[b, :, kv] += dx.t() @ q[b, :, h] / math.sqrt(d)
    if c["kind"] == "forward":
        return dict(o=o.reshape(B * Sq, -1), lse=lse)
    return dict(dq=dq.reshape(B * Sq, -1), dk=dk.reshape(B * Sk, -1), dv=dv.reshape(B * Sk, -1),
                dtable=dtable if bucket is not None else None)


def _exact_adamw(c, s):
    f = lambda v: float(np.float32(v))  # noqa: E731
    b1, b2, lr = f(ADAMW["beta1"]), f(ADAMW["beta2"]), f(ADAMW["lr"])
    out = []
    for t in s["tensors"]:
        n = t["w"].numel()
        wide = lambda x: torch.repeat_interleave(x.double(), BLOCK)[:n]  # noqa: E731
        if c["state"] == "f32":
            m, v = t["m"].double(), t["v"].double()
        else:
            m = t["m"].float().double() * wide(t["m_scale"])
            v = (t["r"].float().double() * wide(t["r_scale"])) ** 2
        g = t["g"].double() * ADAMW["grad_scale"]
        m = b1 * m + (1 - b1) * g
        v = b2 * v + (1 - b2) * g * g
        mean, root = m / (1 - b1 ** ADAMW["step"]), (v / (1 - b2 ** ADAMW["step"])).sqrt()
        w = t["w"].double()
        w = w - lr * (mean / (root + f(ADAMW["eps"])) + f(t["decay"]) * w)
        one = dict(w=w, copy=w, m=m, v=v)
        if c["state"] != "f32":
            # the same random numbers, in numpy's unsigned words
            e = np.arange(n, dtype=np.uint64)
            word = np.uint64(0xffffffff)
            x = ((e & word) * np.uint64(0x9E3779B1) + np.uint64(t["seed"] & 0xffffffff)) & word
            x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x6A09E667)) & word
            x = (x + np.uint64(t["seed"] >> 32)) & word
            x = ((x ^ (x >> np.uint64(15))) * np.uint64(0xBB67AE85)) & word
            x = torch.from_numpy((x ^ (x >> np.uint64(16))).astype(np.int64)).to(DEV)
            one = dict(w=w, copy=w)
            for name, value, up in (("m", m, x // 65536), ("r", v.sqrt(), x % 65536)):
                blocks = -(-n // BLOCK)
                full = torch.zeros(blocks * BLOCK, dtype=torch.float64, device=DEV)
                full[:n] = value.abs()
                scale = torch.clamp(full.view(blocks, BLOCK).max(1).values / E4M3_MAX, min=SCALE_MIN)
                # (a scale is kept in 32 bits, and what is divided by is what is kept)
                a = full[:n] / wide(scale.float())
                grid = 2.0 ** torch.clamp(torch.floor(torch.log2(a.clamp(min=1e-300))), min=-6) / 8
                code = torch.clamp(torch.floor(a / grid + up / 65536.0) * grid, max=E4M3_MAX)
                if name == "r":
                    code = torch.where((a > 0) & (code == 0), 2.0 ** -9, code)
                one[name], one[name + "_scale"] = code * torch.sign(value), scale
        out.append(one)
    if len(out) <= 8:
        return out
    return {name: torch.cat([t[name] for t in out]) for name in out[0]}

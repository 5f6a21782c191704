"""What a block's training path needs around the block calls: rotary positions,
root-mean-square norm with the residual's addition, and the Muon step.

A case is one pass as a program makes it:

  rope      Q and K (or their gradients, ``backward``) of a packed in-projection
            output rotated by their positions
  rmsnorm   residual's addition and norm, ``mode`` forward, 8-bit output, or
            forward and backward
  ortho     the orthogonalisation of some matrices, bf16 or fp32
  muon      the optimizer step that uses it, over fp32 master weights

``listed`` has the fixed cases, ``draw`` more of the same ranges, ``prepare``
what a program holds before the call, ``run`` the call (in elementary torch
operations, or where ``own`` is set through ``paper_2402_15627_amd.pblock``),
``work`` the bytes and operations it cannot do without, ``exact`` the outputs
from the definitions in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
NS = (3.4445, -4.7750, 2.0315)
STEPS = 5
ORTHO_EPS = 1e-7
MUON = dict(lr=1e-3, momentum=0.95, grad_scale=0.5)
DECAY = 0.1
E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126


def _rope(name, dtype, tokens, seq, q_heads, k_heads, head_dim, rot_dim, interleaved, **more):
    c = dict(kind="rope", dtype=dtype, tokens=tokens, seq=seq, q_heads=q_heads, k_heads=k_heads,
             head_dim=head_dim, rot_dim=rot_dim, interleaved=interleaved, backward=False, far=0,
             base=10000.0, scaling="plain", factor=1.0, orig_len=0, magnitude=1.0)
    c.update(more)
    return dict(c, name=name) if name else c


def _rms(name, mode, dtype, rows, cols, resid=True, group=0):
    c = dict(kind="rmsnorm", mode=mode, dtype=dtype, rows=rows, cols=cols, resid=resid, group=group)
    return dict(c, name=name) if name else c


def _mats(name, kind, dtype, mats, **more):
    """mats: rows x columns, or rows x columns @ elements between rows."""
    c = dict(kind=kind, dtype=dtype, mats=mats, **more)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token of four sequences, far into a context that was stretched
        # to 16 times its trained length: a launch's latency.
        _rope("rope_token", "bf16", 4, 1, 40, 40, 128, 128, False, far=131072, base=500000.0,
              scaling="by_parts", factor=16.0, orig_len=8192, magnitude=1.2772588722239782),
        # Q and K of the 175B tensor-parallel share, in place in the packed
        # projection's rows, as training runs it.
        _rope("rope_175b_share", "bf16", 2048, 2048, 12, 12, 128, 128, False),
        # The gradients of a long sequence's Q and K: the largest; adjacent pairs.
        _rope("rope_long_bwd", "bf16", 8192, 8192, 40, 40, 128, 128, True, backward=True),
        # fp32, odd-length sequences, shared key heads, a quarter of each head
        # rotated.
        _rope("rope_f32_ragged", "f32", 666, 333, 16, 4, 96, 24, False, scaling="linear",
              factor=4.0),
        # One token's residual and norm between two layers.
        _rms("rms_token", "forward", "bf16", 1, 5120),
        # The 175B share's norm with its output in 8 bits, a scale per 128
        # columns, for what is sent or multiplied in 8 bits next.
        _rms("rms_q8_175b", "q8", "bf16", 2048, 12288, group=128),
        # Forward and backward over a long sequence at the 13B width: the largest.
        _rms("rms_step_8k", "step", "bf16", 8192, 5120),
        # Forward and backward, fp32, a width and a row count of no tile.
        _rms("rms_f32_ragged", "step", "f32", 675, 1999, resid=False),
        # The six matrices of the smallest block: launches and the chain of
        # dependent products count.
        _mats("muon_tiny", "muon", "f32", "256x256,256x256,256x256,1024x256,256x256@1280,256x1024@1280",
              nesterov=True),
        # The 175B share's matrices, Q, K, V and MLP-up rows of one weight and
        # attention-out and MLP-down columns of the other: the largest.
        _mats("muon_175b_share", "muon", "f32",
              "1536x12288,1536x12288,1536x12288,6144x12288,12288x1536@7680,12288x6144@7680",
              nesterov=True),
        # Updates held in bf16 by a program with its own optimizer: square and
        # tall matrices of a 13B-width block.
        _mats("ortho_13b", "ortho", "bf16", "5120x5120,5120x5120,20480x5120"),
        # Odd sizes, from a single row up, fp32.
        _mats("ortho_f32_ragged", "ortho", "f32", "1x777,333x1001,1999x675@700"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "rope", "rmsnorm", "rmsnorm", "muon", "ortho"))
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if kind == "rope":
        head_dim = rng.choice((64, 80, 96, 128, 128, 256))
        rot = head_dim if rng.random() < 0.6 else 2 * rng.randint(1, head_dim // 2)
        k_heads = _log(rng, 1, 24)
        q_heads = k_heads * rng.choice((1, 1, 2, 4))
        # as many elements as the largest listed case at most
        most = (8192 * 80 * 128) // ((q_heads + k_heads) * head_dim * (2 if dtype == "f32" else 1))
        batch = rng.choice((1, 1, 2, 3))
        seq = max(1, _log(rng, 1, min(8192, most)) // batch)
        scaling = rng.choice(("plain", "linear", "by_parts"))
        factor = 1.0 if scaling == "plain" else rng.choice((2.0, 4.0, 8.0, 32.0))
        return _rope(None, dtype, batch * seq, seq, q_heads, k_heads, head_dim, rot,
                     rng.random() < 0.5, backward=rng.random() < 0.5,
                     far=0 if rng.random() < 0.5 else _log(rng, 1000, 4_000_000),
                     base=rng.choice((10000.0, 500000.0, 1000000.0)), scaling=scaling,
                     factor=factor, orig_len=4096 if scaling == "by_parts" else 0,
                     magnitude=1.0 + 0.1 * math.log(factor) if scaling == "by_parts" else 1.0)
    if kind == "rmsnorm":
        mode = rng.choice(("forward", "q8", "step", "step"))
        cols = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            cols = max(64, cols // 64 * 64)
        most = min(8192, 8192 * 5120 // (cols * (2 if dtype == "f32" else 1)))
        return _rms(None, mode, dtype, _log(rng, 1, most), cols, rng.random() < 0.7,
                    rng.choice((0, 32, 64, 128)) if mode == "q8" else 0)
    mats = []
    for _ in range(rng.choice((1, 1, 2, 3, 6))):
        r, n = _log(rng, 16, 5120), _log(rng, 16, 8192)
        if rng.random() < 0.5:
            r, n = max(64, r // 64 * 64), max(64, n // 64 * 64)
        if rng.random() < 0.5:
            r, n = n, r
        mats.append("%dx%d" % (r, n) + ("@%d" % (n + 8 * rng.randint(1, 64)) if rng.random() < 0.3 else ""))
    if kind == "muon":
        return _mats(None, "muon", "f32", ",".join(mats), nesterov=rng.random() < 0.7)
    return _mats(None, "ortho", dtype, ",".join(mats))


def _act(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _shapes(c):
    out = []
    for t in c["mats"].split(","):
        size, _, ld = t.partition("@")
        r, n = (int(v) for v in size.split("x"))
        out.append((r, n, int(ld) if ld else n))
    return out


def _seeded(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return lambda *shape, std=1.0, mean=0.0: torch.empty(shape, device=DEV).normal_(mean, std, generator=g)


def _gradient(rnd, r, n, ld, std):
    """A few strong directions in noise, as a weight's gradient has."""
    k = min(16, r, n)
    x = rnd(r, k) @ rnd(k, n) * (std / math.sqrt(k)) + rnd(r, n, std=std)
    if ld == n:
        return x
    full = torch.zeros((r, ld), device=DEV)
    full[:, :n] = x
    return full[:, :n]


def prepare(case, seed):
    c = case
    rnd = _seeded(seed)
    act = _act(c)
    s = dict(c, act=act)
    if c["kind"] == "rope":
        d, T = c["head_dim"], c["tokens"]
        wide = (c["q_heads"] + 2 * c["k_heads"]) * d + 64  # Q | K | V and some of the MLP's columns
        s["z"] = rnd(T, wide).to(act)
        s["out"] = torch.empty((T, (c["q_heads"] + c["k_heads"]) * d), dtype=act, device=DEV)
        pos = torch.arange(T, device=DEV) % c["seq"]
        if c["far"]:
            batch = T // c["seq"]
            g = torch.Generator(device=DEV)
            g.manual_seed(seed + 1)
            first = torch.randint(c["far"] // 2, c["far"] + 1, (batch,), generator=g, device=DEV)
            pos = pos + first.repeat_interleave(c["seq"])
        s["pos"] = pos
    elif c["kind"] == "rmsnorm":
        T, H = c["rows"], c["cols"]
        s.update(x=rnd(T, H).to(act), gamma=rnd(H, std=0.1, mean=1.0).to(act),
                 resid=rnd(T, H, std=2.0).to(act) if c["resid"] else None)
        new = lambda *shape, dtype=act: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
        s["sum"] = new(T, H) if c["resid"] else None
        s["y"] = new(T, H) if c["mode"] != "q8" else None
        if c["mode"] == "q8":
            groups = -(-H // c["group"]) if c["group"] else 1
            s.update(q8=new(T, H, dtype=torch.float8_e4m3fn), scales=new(T, groups, dtype=torch.float32))
        if c["mode"] == "step":
            s.update(rstd=new(T, dtype=torch.float32), dy=rnd(T, H).to(act), dx=new(T, H),
                     dsum=rnd(T, H).to(act) if c["resid"] else None,
                     dgamma=new(H, dtype=torch.float32))
    else:
        mats = []
        for r, n, ld in _shapes(c):
            m = dict(g=_gradient(rnd, r, n, ld, 1e-3).to(act), rows=r, cols=n)
            if m["g"].stride(0) != ld:  # the cast packs its rows
                full = torch.zeros((r, ld), dtype=act, device=DEV)
                full[:, :n] = m["g"]
                m["g"] = full[:, :n]
            if c["kind"] == "muon":
                m["w"] = torch.empty((r, ld), device=DEV)[:, :n].copy_(rnd(r, n, std=0.02))
                m["m"] = _gradient(rnd, r, n, ld, 5e-3)
                m["copy"] = torch.empty((r, ld), dtype=torch.bfloat16, device=DEV)[:, :n]
                # the root mean square of a step is then 0.2 lr, whatever the shape
                m["scale"] = 0.2 * math.sqrt(max(r, n))
            else:
                m["out"] = torch.empty((r, n), dtype=act, device=DEV)
            mats.append(m)
        s["mats"] = mats
    return _handles(s)


def _handles(s):
    """What a program of the library makes once and keeps: configurations and
    workspaces. Plain forms need none."""
    if not own:
        return s
    from paper_2402_15627_amd import pblock as pb
    ws = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)  # noqa: E731
    if s["kind"] == "rope":
        s["cfg"] = pb.rope_config(s["head_dim"], s["rot_dim"], s["interleaved"], s["base"],
                                  s["scaling"], s["factor"], s["orig_len"],
                                  magnitude=s["magnitude"], dtype=s["dtype"])
        d, ld, q = s["head_dim"], s["z"].stride(0), s["q_heads"] * s["head_dim"]
        ld_out = s["out"].stride(0)
        s["parts"] = [pb.rope_tensor(s["z"], ld, s["q_heads"], s["out"], ld_out),
                      pb.rope_tensor(s["z"][:, q:], ld, s["k_heads"], s["out"][:, q:], ld_out)]
    elif s["kind"] == "rmsnorm":
        s["cfg"] = pb.rmsnorm_config(s["rows"], s["cols"], dtype=s["dtype"], group=s["group"])
        if s["mode"] == "step":
            s["ws"] = ws(pb.pblock_rmsnorm_workspace_bytes(s["cfg"]))
    elif s["kind"] == "muon":
        s["cfg"] = pb.muon_config(nesterov=s["nesterov"], steps=STEPS, eps=ORTHO_EPS, **MUON)
        s["parts"] = [pb.muon_tensor(m["w"], m["g"], m["m"], m["copy"], DECAY, m["scale"])
                      for m in s["mats"]]
        s["ws"] = ws(pb.pblock_muon_workspace_bytes(s["cfg"], s["parts"]))
    else:
        s["parts"] = [pb.ortho_tensor(m["g"], m["out"]) for m in s["mats"]]
        s["ws"] = ws(pb.pblock_orthogonalize_workspace_bytes(s["parts"], s["dtype"]))
    return s


# ------------------------------------------------------------ the passes
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2402_15627_amd import pblock as pb
    if s["kind"] == "rope":
        call = pb.pblock_rope_backward if s["backward"] else pb.pblock_rope_forward
        call(s["cfg"], s["parts"], s["tokens"], s["seq"], s["pos"] if s["far"] else None)
        return s["out"]
    if s["kind"] == "rmsnorm":
        pb.pblock_rmsnorm_forward(s["cfg"], s["x"], s["gamma"], s["y"], resid=s["resid"],
                                  sum_out=s["sum"], q8=s.get("q8"), scales=s.get("scales"),
                                  rstd=s.get("rstd"))
        if s["mode"] == "q8":
            return dict(sum=s["sum"], q8=s["q8"], scales=s["scales"])
        if s["mode"] == "forward":
            return dict(sum=s["sum"], y=s["y"])
        pb.pblock_rmsnorm_backward(s["cfg"], s["sum"] if s["resid"] is not None else s["x"],
                                   s["gamma"], s["rstd"], s["dy"], s["dx"], s["dgamma"], s["ws"],
                                   dsum=s["dsum"])
        return dict(sum=s["sum"], y=s["y"], dx=s["dx"], dgamma=s["dgamma"])
    if s["kind"] == "muon":
        pb.pblock_muon_step(s["cfg"], s["parts"], pb.PB_BF16, s["ws"])
        return [dict(w=m["w"], m=m["m"], copy=m["copy"]) for m in s["mats"]]
    pb.pblock_orthogonalize(s["parts"], s["dtype"], s["ws"], STEPS, ORTHO_EPS)
    return [m["out"] for m in s["mats"]]


def _run_plain(s):
    if s["kind"] == "rope":
        return _plain_rope(s)
    if s["kind"] == "rmsnorm":
        return _plain_rms(s)
    if s["kind"] == "muon":
        return [_plain_muon(s, m) for m in s["mats"]]
    return [_plain_ortho(m["g"].float()).to(s["act"]) for m in s["mats"]]


def _frequencies(s):
    """Angle of one position step for each pair, in 64 bits."""
    i = torch.arange(s["rot_dim"] // 2, dtype=torch.float64, device=DEV)
    f = torch.exp(i * (-2.0 * math.log(s["base"]) / s["rot_dim"]))
    if s["scaling"] == "linear":
        return f / s["factor"]
    if s["scaling"] == "by_parts":
        turns = s["orig_len"] * f / (2 * math.pi)
        keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
        return f * (keep + (1 - keep) / s["factor"])
    return f


def _plain_rope(s):
    """Angles of far positions in 64 bits, the rotation in 32."""
    T, d, r = s["tokens"], s["head_dim"], s["rot_dim"]
    angle = s["pos"].double()[:, None] * _frequencies(s)
    cos = (angle.cos() * s["magnitude"]).float()[:, None]
    sin = (angle.sin() * (-s["magnitude"] if s["backward"] else s["magnitude"])).float()[:, None]
    x = s["z"][:, :(s["q_heads"] + s["k_heads"]) * d].float().view(T, -1, d)
    if s["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    s["out"].view(T, -1, d).copy_(torch.cat([y, x[..., r:]], -1))
    return s["out"]


def _quantise(y, group):
    """e4m3 values and fp32 scales of y (64 bits: codes next to a border). A
    scale is a group's largest magnitude over 448."""
    T, H = y.shape
    g = group or H
    pad = torch.nn.functional.pad(y, (0, -H % g)).view(T, -1, g)
    scale = (pad.abs().amax(-1) / E4M3_MAX).clamp(min=SCALE_MIN).float()
    q = (pad / scale.double()[..., None]).view(T, -1)[:, :H]
    return q.to(torch.float8_e4m3fn), scale


def _plain_rms(s):
    wide = torch.float64 if s["mode"] == "q8" else torch.float32
    gamma = s["gamma"].to(wide)
    total = s["x"].to(wide)
    if s["resid"] is not None:
        total = total + s["resid"].to(wide)
    kept = total.to(s["act"])
    rstd = torch.rsqrt(total.square().mean(-1, keepdim=True) + 1e-5)
    y = total * rstd * gamma
    out = dict(sum=kept if s["resid"] is not None else None)
    if s["mode"] == "q8":
        q, scale = _quantise(y, s["group"])
        return dict(out, q8=q, scales=scale)
    out["y"] = y.to(s["act"])
    if s["mode"] == "forward":
        return out
    dy = s["dy"].float()
    xhat = kept.float() * rstd
    g = dy * gamma
    dx = rstd * (g - xhat * (g * xhat).mean(-1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    # (a sum over thousands of rows, in 64 bits)
    dgamma = (dy * xhat).sum(0, dtype=torch.float64).float()
    return dict(out, dx=dx.to(s["act"]), dgamma=dgamma)


def _plain_ortho(u):
    a, b, c = NS
    x = u.mT if u.shape[0] > u.shape[1] else u
    # (the norm of millions of elements in 64 bits)
    norm = x.square().sum(dtype=torch.float64).sqrt()
    x = x / (norm + ORTHO_EPS).float()
    for _ in range(STEPS):
        gram = x @ x.mT
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.mT if u.shape[0] > u.shape[1] else x


def _plain_muon(s, m):
    lr, mu = MUON["lr"], MUON["momentum"]
    g = m["g"] * MUON["grad_scale"]
    m["m"].mul_(mu).add_(g)
    u = g + mu * m["m"] if s["nesterov"] else m["m"]
    m["w"].mul_(1 - lr * DECAY).sub_(_plain_ortho(u), alpha=lr * m["scale"])
    m["copy"].copy_(m["w"])
    return dict(w=m["w"], m=m["m"], copy=m["copy"])


# ----------------------------------------------------------- what it takes
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "rope":
        n = c["tokens"] * (c["q_heads"] + c["k_heads"]) * c["head_dim"]
        rotated = n // c["head_dim"] * c["rot_dim"]
        return {"bytes": 2 * n * e + (8 * c["tokens"] if c["far"] else 0), "flops": 3 * rotated}
    if c["kind"] == "rmsnorm":
        n, H = c["rows"] * c["cols"], c["cols"]
        forward = (1 + 2 * c["resid"]) * n * e + H * e  # x, and the residual and the sum
        if c["mode"] == "q8":
            groups = -(-H // c["group"]) if c["group"] else 1
            return {"bytes": forward + n + 4 * c["rows"] * groups, "flops": 6 * n}
        forward += n * e
        if c["mode"] == "forward":
            return {"bytes": forward, "flops": 5 * n}
        backward = (3 + c["resid"]) * n * e + H * e + 4 * H + 8 * c["rows"]
        return {"bytes": forward + backward, "flops": 16 * n}
    total = {"bytes": 0, "flops": 0}
    for r, n, _ in _shapes(c):
        m, w = min(r, n), max(r, n)
        # X X^T and A A are symmetric: half of each is enough
        total["flops"] += STEPS * (m * (m + 1) * w + m * m * (m + 1) + 2 * m * m * w)
        # g, M and W read, M, W and the bf16 copy written; or in and out
        total["bytes"] += r * n * (22 if c["kind"] == "muon" else 2 * e)
    return total


# ------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    c = dict(case)
    s = prepare(case, seed)
    if c["kind"] == "rope":
        return _exact_rope(c, s)
    if c["kind"] == "rmsnorm":
        return _exact_rms(c, s)
    out = []
    for m in s["mats"]:
        g = m["g"].double()
        if c["kind"] == "ortho":
            out.append(_exact_polar(g))
            continue
        g = MUON["grad_scale"] * g
        mom = MUON["momentum"] * m["m"].double() + g
        u = _exact_polar(g + MUON["momentum"] * mom if c["nesterov"] else mom)
        w = m["w"].double()
        w = w - MUON["lr"] * (DECAY * w + m["scale"] * u)
        out.append(dict(w=w, m=mom, copy=w))
    return out


def _exact_polar(u):
    """X <- (a I + b X X^T + c (X X^T)^2) X, from U / |U|."""
    a, b, c = NS
    tall = u.size(0) > u.size(1)
    x = u / (torch.sqrt((u * u).sum()) + ORTHO_EPS)
    for _ in range(STEPS):
        left = x.t() if tall else x
        gram = left @ left.t()
        poly = b * gram
        poly += c * (gram @ gram)
        poly.diagonal().add_(a)
        x = x @ poly if tall else poly @ x
    return x


def _exact_rope(c, s):
    """Each pair as a complex number times m e^(i angle)."""
    d, r, heads = c["head_dim"], c["rot_dim"], c["q_heads"] + c["k_heads"]
    freq = []
    for i in range(r // 2):
        f = c["base"] ** (-2.0 * i / r)
        if c["scaling"] == "linear":
            f /= c["factor"]
        if c["scaling"] == "by_parts":
            g = min(1.0, max(0.0, (c["orig_len"] * f / (2 * math.pi) - 1.0) / 31.0))
            f *= g + (1.0 - g) / c["factor"]
        freq.append(f)
    phi = s["pos"].double()[:, None, None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(phi, c["magnitude"]), -phi if c["backward"] else phi)
    x = s["z"][:, :heads * d].double().reshape(c["tokens"], heads, d)
    y = x.clone()
    first, second = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    turned = torch.complex(x[..., first], x[..., second]) * turn
    y[..., first], y[..., second] = turned.real, turned.imag
    return y.reshape(c["tokens"], heads * d)


def _exact_rms(c, s):
    x, gamma = s["x"].double(), s["gamma"].double()
    if s["resid"] is not None:
        x = x + s["resid"].double()
    r = 1.0 / torch.sqrt((x * x).sum(1, keepdim=True) / c["cols"] + 1e-5)
    y = x * r * gamma
    out = dict(sum=x if s["resid"] is not None else None)
    if c["mode"] == "q8":
        g = c["group"] or c["cols"]
        scales = torch.empty((c["rows"], -(-c["cols"] // g)), dtype=torch.float64, device=DEV)
        codes = torch.empty_like(y)
        for k in range(scales.shape[1]):
            part = y[:, k * g:(k + 1) * g]
            scales[:, k] = torch.clamp(part.abs().max(1).values / E4M3_MAX, min=SCALE_MIN)
            # (a scale is kept in 32 bits, and what is divided by is what is kept)
            codes[:, k * g:(k + 1) * g] = part / scales[:, k:k + 1].float().double()
        return dict(out, q8=codes.to(torch.float8_e4m3fn).double(), scales=scales)
    out["y"] = y
    if c["mode"] == "forward":
        return out
    # the gradient at the sum that is kept, with the forward's 1 / rms
    kept = x.to(s["act"]).double()
    dy = s["dy"].double()
    weighted = dy * gamma
    dx = r * weighted - kept * r ** 3 * ((weighted * kept).sum(1, keepdim=True) / c["cols"])
    if s["dsum"] is not None:
        dx = dx + s["dsum"].double()
    return dict(out, dx=dx, dgamma=(dy * kept * r).sum(0))

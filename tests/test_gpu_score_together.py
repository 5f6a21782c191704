"""Attention with terms in its scores and the AdamW step as a training step uses them: a
block over packed documents with a learned position bias and capped scores, built from
the library's calls, its backward with the bias table's gradient, and one AdamW step
over everything it learns, against torch autograd and the oracle in float64.

    h = rmsnorm(x);  Z = h W_in^T + b_in = [Q | K | V | U]
    y = x + [attention(Q, K, V) | GeLU(U)] W_out^T + b_out

The projections run through the pipelined calls with one rank.  Tolerances are the
block's own, normwise: 2e-2 for bf16 and 1e-5 for fp32 (the table's gradient in fp32,
sums of thousands of terms of either sign, 2e-5); weights after the step by the oracle's
step on the gradients that the block gave, 12 2^-24 of the update and 3 2^-24 of the
weight.
"""
import math

import numpy as np
import pytest

from oracle import score_oracle as so
from tests.parity_util import TOL, normwise

pytestmark = pytest.mark.gpu

B, S, H, NH, D, F = 2, 192, 256, 4, 64, 320
A, T = NH * D, B * S
N_IN, K_OUT = 3 * A + F, A + F
DOCS, PREFIX = [0, 100, 130, 192, 300, 377], [20, 0, 62, 5, 0]  # the last 7 tokens: padding
CAP, BUCKETS, FAR = 4.0, 16, 60
STEP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1)


def f64(t):
    return t.detach().double().cpu().numpy()


def reference(t):
    """y, and the gradients of sum(y dy), by autograd of the definition in float64."""
    import torch
    p = {k: t[k].double().requires_grad_(k != "dy") for k in t}
    h = p["x"] * torch.rsqrt(p["x"].square().mean(1, keepdim=True) + float(np.float32(1e-5))) * p["gamma"]
    z = h @ p["w_in"].t() + p["b_in"]
    q, k, v = (z[:, i * A:(i + 1) * A].reshape(B, S, NH, D) for i in range(3))
    see = torch.from_numpy(so.visible(B, S, S, True, S, DOCS, PREFIX)).cuda()
    live = see.any(2)
    i = np.arange(S)
    of = {d: so.bucket(d, BUCKETS, FAR, True) for d in range(-S, S)}
    ids = torch.tensor([[of[a - b] for b in i] for a in i], device="cuda")
    o = []
    for b in range(B):
        for m in range(NH):
            s = CAP * torch.tanh(q[b, :, m] @ k[b, :, m].t().contiguous() / math.sqrt(D) / CAP)
            s = (s + p["table"][:, m][ids]).masked_fill(~(see[b] | ~live[b][:, None]), -math.inf)
            o.append((torch.softmax(s, 1) @ v[b, :, m]) * live[b][:, None])
    o = torch.stack(o).view(B, NH, S, D).transpose(1, 2).reshape(T, A)
    g = torch.nn.functional.gelu(z[:, 3 * A:], approximate="tanh")
    y = p["x"] + torch.cat([o, g], 1) @ p["w_out"].t() + p["b_out"]
    (y * p["dy"]).sum().backward()
    return y, {k: x.grad for k, x in p.items() if k != "dy"}


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_biased_block_over_documents_and_adamw_step(dtype, e4m3):
    import torch
    from paper_2402_15627_amd import pblock as pb
    print(f"[gpu] scored block and AdamW {dtype} {e4m3}", flush=True)
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *s, std=1.0, mean=0.0: torch.empty(s, device="cuda").normal_(  # noqa: E731
        mean, std, generator=gen).to(act)
    t = dict(x=draw(T, H), gamma=draw(H, std=0.1, mean=1.0), w_in=draw(N_IN, H, std=0.06),
             b_in=draw(N_IN, std=0.06), w_out=draw(H, K_OUT, std=0.06), b_out=draw(H, std=0.06), dy=draw(T, H),
             table=draw(BUCKETS, NH).float())
    new = lambda *s, d=act: torch.empty(s, dtype=d, device="cuda")  # noqa: E731
    ws = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")  # noqa: E731
    cfg = pb.make_config(B, S, H, NH, D, F, S, dtype)
    norm = pb.rmsnorm_config(T, H, dtype=dtype)
    attn = pb.score_attn_config(B, S, S, NH, NH, D, cap=CAP, buckets=BUCKETS, max_distance=FAR, dtype=dtype)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    terms = dict(docs=ints(DOCS), prefix=ints(PREFIX), table=t["table"])
    main, comm = torch.cuda.current_stream(), [torch.cuda.Stream()]
    cols = lambda x, i: x[:, i * A:(i + 1) * A]  # noqa: E731

    # forward
    h, rstd = new(T, H), new(T, d=torch.float32)
    pb.pblock_rmsnorm_forward(norm, t["x"], t["gamma"], h, rstd=rstd)
    z, c, lse = new(T, N_IN), new(T, K_OUT), new(B, NH, S, d=torch.float32)
    part, y = new(T, H), new(T, H)
    with pb.TpContext(1) as ctx:
        pb.pblock_ag_in_proj(cfg, 1, 0, [h], h, t["w_in"], t["b_in"], z, c, 1, None, main, comm, ctx)
        pb.pblock_score_attn_forward(attn, cols(z, 0), cols(z, 1), cols(z, 2), cols(c, 0), lse,
                                     ws=ws(pb.pblock_score_attn_workspace_bytes(attn, pb.ATTN_WS_FORWARD)), **terms)
        pb.pblock_rs_out_proj(cfg, 1, 0, c, t["w_out"], part, [part], 1, None, main, comm, ctx)
        pb.pblock_rs_reduce(cfg, 1, [part], t["x"], t["b_out"], y)
        # backward
        d_o, dz, dh, dx = new(T, A), new(T, N_IN), new(T, H), new(T, H)
        dgamma, dtable = new(H, d=torch.float32), new(BUCKETS, NH, d=torch.float32)
        pb.pblock_ag_dc(cfg, 1, 0, [t["dy"]], t["dy"], t["w_out"], z, d_o, dz, 1, None, main, comm, ctx)
        pb.pblock_score_attn_backward(attn, cols(z, 0), cols(z, 1), cols(z, 2), cols(c, 0), d_o, lse, cols(dz, 0),
                                      cols(dz, 1), cols(dz, 2),
                                      ws(pb.pblock_score_attn_workspace_bytes(attn, pb.ATTN_WS_BACKWARD)),
                                      dtable=dtable, **terms)
        pb.pblock_rs_dh(cfg, 1, 0, dz, t["w_in"], dh, [dh], 1, None, main, comm, ctx)
        pb.pblock_rmsnorm_backward(norm, t["x"], t["gamma"], rstd, dh, dx, dgamma,
                                   ws(pb.pblock_rmsnorm_workspace_bytes(norm)), dsum=t["dy"])
        torch.cuda.synchronize()
    ref_y, ref = reference(t)
    grads = dict(w_in=dz.float().t() @ h.float(), w_out=t["dy"].float().t() @ c.float(),
                 b_in=dz.float().sum(0), b_out=t["dy"].float().sum(0), gamma=dgamma, table=dtable)
    got = dict(y=(y, ref_y), x=(dx, ref["x"]), **{k: (g, ref[k]) for k, g in grads.items()})
    for name, (a, b) in got.items():
        e = normwise(f64(a), f64(b))
        print(f"      {name} {e:.2e}", flush=True)
        assert e <= (2e-5 if name == "table" and dtype == "f32" else TOL[dtype]), name

    # one step over all that the block learns: matrices with decay, the others without
    parts, kept = [], []
    for i, (name, g) in enumerate(grads.items()):
        w, g = t[name].float().reshape(-1).clone(), g.reshape(-1).contiguous()
        n, decay = w.numel(), 0.1 if name.startswith("w_") else 0.0
        copy = torch.empty(n, dtype=act, device="cuda")
        if e4m3:
            m, v = (torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
            s = [torch.zeros(-(-n // pb.ADAMW_BLOCK), device="cuda") for _ in range(2)]
            parts.append(pb.adamw_tensor(w, g, m, v, copy, decay, *s, seed=i))
        else:
            m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
            parts.append(pb.adamw_tensor(w, g, m, v, copy, decay))
        kept.append((name, f64(w), w, f64(g), copy, decay))
    pb.pblock_adamw_step(pb.adamw_config(**STEP), pb.AdamwTensors(parts), pb.PB_BF16 if dtype == "bf16" else pb.PB_F32)
    torch.cuda.synchronize()
    hyper = {k: float(np.float32(x)) for k, x in STEP.items() if k != "step"}
    for name, w0, w, g, copy, decay in kept:
        want, m, _ = so.adamw(w0, g, np.zeros_like(w0), np.zeros_like(w0), step=1,
                              weight_decay=float(np.float32(decay)), **hyper)
        tol = 2.0 ** -24 * (12 * hyper["lr"] + 3 * (abs(w0) + abs(want)))
        assert (abs(f64(w) - want) <= tol).all(), name
        assert torch.equal(copy, w.to(act)), name

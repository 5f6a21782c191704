"""The operators as a training step uses them: a block with a root-mean-square norm and
rotary positions, built from the library's calls, its backward, and a Muon step on its
matrices, against torch autograd and the oracle in float64.

    h = rmsnorm(x + r);  Z = h W_in^T + b_in;  Q, K turned by their positions
    y = (x + r) + [SWAttn(Q, K, V) | GeLU(U)] W_out^T + b_out

The projections run through the pipelined calls with one rank.  Tolerances are the
block's own, normwise: 2e-2 for bf16 and 1e-5 for fp32 (weights after the step: the
update's error times its length, and the rounding of the weights).
"""
import math

import numpy as np
import pytest

from oracle import operators_oracle as oo
from tests.parity_util import TOL, normwise

pytestmark = pytest.mark.gpu

B, S, H, NH, D, F, W = 2, 192, 256, 4, 64, 320, 100
A, T = NH * D, B * S
N_IN, K_OUT = 3 * A + F, A + F
ROPE = dict(rot_dim=48, interleaved=False, base=10000.0, scaling="by_parts", factor=4.0, orig_len=64.0,
            magnitude=1.0 + 0.1 * math.log(4.0))


def f64(t):
    return t.detach().double().cpu().numpy()


def reference(t):
    """y, and the gradients of sum(y dy), by autograd of the definition in float64."""
    import torch
    p = {k: t[k].double().requires_grad_(k != "dy") for k in t}
    s = p["x"] + p["r"]
    h = s * torch.rsqrt(s.square().mean(1, keepdim=True) + float(np.float32(1e-5))) * p["gamma"]
    z = h @ p["w_in"].t() + p["b_in"]
    freq = torch.from_numpy(oo.rope_frequencies(ROPE["rot_dim"], ROPE["base"], "by_parts", 4.0, 64.0)).cuda()
    pos = (torch.arange(T, device="cuda") % S).double()[:, None, None] * freq
    c, sn, n = torch.cos(pos) * ROPE["magnitude"], torch.sin(pos) * ROPE["magnitude"], len(freq)

    def turn(x):
        x = x.reshape(T, NH, D)
        a, b = x[..., :n], x[..., n:2 * n]
        return torch.cat([a * c - b * sn, b * c + a * sn, x[..., 2 * n:]], -1)

    q, k, v = turn(z[:, :A]), turn(z[:, A:2 * A]), z[:, 2 * A:3 * A].reshape(T, NH, D)
    i = torch.arange(S, device="cuda")
    seen = (i[:, None] >= i) & (i[:, None] - i < W)
    o = []
    for b in range(B):
        rows = slice(b * S, (b + 1) * S)
        for m in range(NH):
            a = (q[rows, m] @ k[rows, m].t().contiguous() / math.sqrt(D)).masked_fill(~seen, -math.inf)
            o.append(torch.softmax(a, 1) @ v[rows, m])
    o = torch.stack(o).view(B, NH, S, D).transpose(1, 2).reshape(T, A)
    g = torch.nn.functional.gelu(z[:, 3 * A:], approximate="tanh")
    y = s + torch.cat([o, g], 1) @ p["w_out"].t() + p["b_out"]
    (y * p["dy"]).sum().backward()
    return y, {k: v.grad for k, v in p.items() if k != "dy"}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotary_rms_block_and_muon_step(dtype):
    import torch
    from paper_2402_15627_amd import pblock as pb
    print(f"[gpu] operators together {dtype}", flush=True)
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda *s, std=1.0, mean=0.0: torch.empty(s, device="cuda").normal_(  # noqa: E731
        mean, std, generator=gen).to(act)
    t = dict(x=draw(T, H), r=draw(T, H), gamma=draw(H, std=0.1, mean=1.0), w_in=draw(N_IN, H, std=0.06),
             b_in=draw(N_IN, std=0.06), w_out=draw(H, K_OUT, std=0.06), b_out=draw(H, std=0.06),
             dy=draw(T, H))
    new = lambda *s, d=act: torch.empty(s, dtype=d, device="cuda")  # noqa: E731
    ws = lambda n: torch.empty(max(n, 256), dtype=torch.uint8, device="cuda")  # noqa: E731
    cfg = pb.make_config(B, S, H, NH, D, F, W, dtype)
    norm, rope = pb.rmsnorm_config(T, H, dtype=dtype), pb.rope_config(D, dtype=dtype, **ROPE)
    main, comm = torch.cuda.current_stream(), [torch.cuda.Stream()]

    # forward
    s, h, rstd = new(T, H), new(T, H), new(T, d=torch.float32)
    pb.pblock_rmsnorm_forward(norm, t["x"], t["gamma"], h, t["r"], s, rstd=rstd)
    z, c, lse = new(T, N_IN), new(T, K_OUT), new(B, NH, S, d=torch.float32)
    part, y = new(T, H), new(T, H)
    with pb.TpContext(1) as ctx:
        pb.pblock_ag_in_proj(cfg, 1, 0, [h], h, t["w_in"], t["b_in"], z, c, 1, None, main, comm, ctx)
        pb.pblock_rope_forward(rope, [pb.rope_tensor(z, N_IN, NH), pb.rope_tensor(z[:, A:], N_IN, NH)], T, S)
        q, k, v = z, z[:, A:], z[:, 2 * A:]
        pb.pblock_swattn_forward(cfg, q, k, v, N_IN, c, K_OUT, lse)
        pb.pblock_rs_out_proj(cfg, 1, 0, c, t["w_out"], part, [part], 1, None, main, comm, ctx)
        pb.pblock_rs_reduce(cfg, 1, [part], s, t["b_out"], y)
        # backward
        d_o, dz, dh, dx = new(T, A), new(T, N_IN), new(T, H), new(T, H)
        dgamma = new(H, d=torch.float32)
        pb.pblock_ag_dc(cfg, 1, 0, [t["dy"]], t["dy"], t["w_out"], z, d_o, dz, 1, None, main, comm, ctx)
        pb.pblock_swattn_backward(cfg, q, k, v, N_IN, c, K_OUT, d_o, A, lse, dz, dz[:, A:], dz[:, 2 * A:],
                                  N_IN, ws(pb.pblock_swattn_workspace_bytes(cfg, pb.ATTN_WS_BACKWARD)))
        pb.pblock_rope_backward(rope, [pb.rope_tensor(dz, N_IN, NH), pb.rope_tensor(dz[:, A:], N_IN, NH)],
                                T, S)
        pb.pblock_rs_dh(cfg, 1, 0, dz, t["w_in"], dh, [dh], 1, None, main, comm, ctx)
        pb.pblock_rmsnorm_backward(norm, s, t["gamma"], rstd, dh, dx, dgamma,
                                   ws(pb.pblock_rmsnorm_workspace_bytes(norm)), dsum=t["dy"])
        torch.cuda.synchronize()
    ref_y, ref = reference(t)
    dw_in, dw_out = (dz.float().t() @ h.float()), (t["dy"].float().t() @ c.float())
    got = dict(y=(y, ref_y), dx=(dx, ref["x"]), dr=(dx, ref["r"]), dgamma=(dgamma, ref["gamma"]),
               dw_in=(dw_in, ref["w_in"]), dw_out=(dw_out, ref["w_out"]), db_in=(dz.float().sum(0), ref["b_in"]))
    for name, (a, b) in got.items():
        e = normwise(f64(a), f64(b))
        print(f"      {name} {e:.2e}", flush=True)
        assert e <= TOL[dtype], name

    # the step: Q, K, V and MLP-up rows of one weight, O and MLP-down columns of the other
    w_in, w_out = t["w_in"].float(), t["w_out"].float()
    m_in, m_out = torch.zeros_like(w_in), torch.zeros_like(w_out)
    c_in, c_out = torch.empty_like(t["w_in"]), torch.empty_like(t["w_out"])
    parts, named = [], []
    for sl in (slice(0, A), slice(A, 2 * A), slice(2 * A, 3 * A), slice(3 * A, N_IN)):
        named.append((w_in[sl], dw_in[sl], m_in[sl], c_in[sl]))
    for sl in (slice(0, A), slice(A, K_OUT)):
        named.append((w_out[:, sl], dw_out[:, sl], m_out[:, sl], c_out[:, sl]))
    before = [f64(n[0]) for n in named]
    lr, decay = 0.01, 0.1
    for w, g, m, cp in named:
        parts.append(pb.muon_tensor(w, g, m, cp, decay, 0.2 * max(w.shape) ** 0.5))
    step = pb.muon_config(lr)
    pb.pblock_muon_step(step, parts, pb.PB_BF16 if dtype == "bf16" else pb.PB_F32,
                        ws(pb.pblock_muon_workspace_bytes(step, parts)))
    torch.cuda.synchronize()
    lr = float(np.float32(lr))
    for (w, g, m, cp), w0 in zip(named, before):
        scale = float(np.float32(0.2 * max(w.shape) ** 0.5))
        rw, rm, o = oo.muon_step(w0, f64(g), np.zeros_like(w0), lr, float(np.float32(0.95)), True,
                                 float(np.float32(decay)), scale)
        # (2e-5: what the fp32 iteration itself loses on matrices of these sizes, fourfold)
        tol = 2e-5 * lr * scale * np.linalg.norm(o) + 2.0 ** -22 * np.linalg.norm(w0)
        assert np.linalg.norm(f64(w) - rw) <= tol
        assert normwise(f64(m), rm) <= 2.0 ** -23
        assert torch.equal(cp, w.to(act))

"""Rotary positions on the GPU against the fp64 oracle.

Tolerance per element: one rounding of the result to its type (half a step, eps / 2
of the value) and the fp32 arithmetic, relative to m (|x_a| + |x_b|): the angle in
turns is rounded to fp32 (2^-25 turns, 2^-22.3 as an angle), sine and cosine are good
to 2^-23, their product with m and the two products and the sum round once each
(2^-24): together below 2^-20.
"""
import numpy as np
import pytest

from oracle import operators_oracle as oo

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)


def torch_type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def run(dtype, tokens, heads, head_dim, rot, interleaved, positions=None, seq=None, pad=0, offset=0,
        in_place=False, backward=False, pad_out=0, stream=None, seed=0, **scaling):
    """heads: one count per tensor, packed side by side.  Returns (input, output, the
    output's padding) as numpy, and the call's oracle."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    act, d = torch_type(dtype), head_dim
    width = sum(heads) * d
    ld, ld_out = width + pad, (width + pad if in_place else width + pad_out)
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.empty(offset + tokens * ld, device="cuda").normal_(generator=g).to(act)
    x = flat[offset:].view(tokens, ld)
    x0 = x[:, :width].float().cpu().numpy().astype(np.float64).reshape(tokens, sum(heads), d)
    pad0 = x[:, width:].clone()
    if in_place:
        out = x
    else:
        out = torch.full((offset + tokens * ld_out,), 7.0, dtype=act, device="cuda")[offset:]
        out = out.view(tokens, ld_out)
    cfg = pb.rope_config(d, rot, interleaved, dtype=dtype, **scaling)
    parts, at = [], 0
    for h in heads:
        parts.append(pb.rope_tensor(x[:, at:], ld, h, None if in_place else out[:, at:],
                                    None if in_place else ld_out))
        at += h * d
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int64, device="cuda")
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    fn = pb.pblock_rope_backward if backward else pb.pblock_rope_forward
    fn(cfg, parts, tokens, seq, pos, stream)
    torch.cuda.synchronize()
    got = out[:, :width].float().cpu().numpy().astype(np.float64).reshape(x0.shape)
    want_pad = pad0 if in_place else torch.full_like(out[:, width:], 7.0)
    assert torch.equal(out[:, width:], want_pad)
    if not in_place:
        assert torch.equal(x[:, :width].float().cpu().double().view(x0.shape), torch.from_numpy(x0))
    p = np.arange(tokens) % (seq or tokens) if positions is None else np.asarray(positions)
    kw = {k: v for k, v in scaling.items() if k in ("factor", "orig_len", "scaling")}
    freq = oo.rope_frequencies(rot or d, scaling.get("base", 10000.0), **kw)
    m = scaling.get("magnitude", 1.0)
    ref = oo.rope(x0, p, freq, interleaved, m, backward)
    size = np.abs(x0)
    n = len(freq)
    a, b = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    both = size[..., a] + size[..., b]
    size[..., a] = size[..., b] = m * both
    half = torch.finfo(act).eps / 2
    tol = half * np.abs(ref) + 2.0 ** -20 * size
    tol[..., 2 * n:] = 0.0  # passed through
    bad = np.abs(got - ref) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[0], float((np.abs(got - ref) - tol).max()))
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,d,rot,pad,offset", [
    (1, (1,), 64, None, 0, 0),
    (1, (40, 40), 128, None, 0, 0),
    (33, (3, 1), 128, None, 64, 0),        # shared key heads; a packed row's other columns
    (65, (2, 2), 96, 32, 8, 8),            # a third of the head
    (7, (5,), 80, 80, 0, 0),
    (5, (3, 2), 6, 2, 1, 0),               # nothing aligned
    (9, (2,), 128, 124, 0, 0),             # aligned heads, an odd rotated part
    (9, (2,), 64, 64, 0, 1),               # a pointer off by one element
    (300, (9, 1, 2, 4), 64, 48, 0, 0),     # four tensors
    (3, (260,), 256, 256, 0, 0),           # more heads than a workgroup takes
    (11, (130,), 256, 2, 0, 0),
    (4100, (1,), 64, None, 0, 0),          # many tokens, few heads
])
def test_rope_matches_oracle(dtype, interleaved, tokens, heads, d, rot, pad, offset):
    _say(f"[gpu] rope {dtype} adjacent={interleaved} {tokens} x {heads} x {d} rot={rot}")
    for in_place in (False, True):
        for backward in (False, True):
            run(dtype, tokens, heads, d, rot, interleaved, pad=pad, offset=offset, in_place=in_place,
                backward=backward, pad_out=3 if pad % 8 else 16)


@pytest.mark.parametrize("scaling", [
    dict(scaling="linear", factor=4.0), dict(scaling="linear", factor=0.5),
    dict(scaling="by_parts", factor=16.0, orig_len=4096.0, magnitude=1.2772588722239782),
    dict(base=500000.0, magnitude=0.5)])
def test_rope_positions_and_scaled_frequencies(scaling):
    _say(f"[gpu] rope {scaling}")
    pos = [0, 1, 131071, 4_000_003, -17, 2**31 - 1, 5, 5]
    for dtype in ("bf16", "f32"):
        for backward in (False, True):
            # (the largest position's angle is good to 2^31 2^-53 turns)
            run(dtype, 8, (4, 2), 128, 64, False, positions=pos, backward=backward, **scaling)
    run("f32", 12, (2,), 64, None, True, seq=5, **scaling)


def test_rope_backward_undoes_forward_and_holds_against_differences():
    """<dy, R x> = <R^T dy, x>, and for a small change e of x, R (x + e) - R x against
    the same: the map is linear, so differences are exact up to rounding."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say("[gpu] rope adjoint")
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.empty(50, 6 * 128, device="cuda").normal_(generator=g) for _ in range(2))
    cfg = pb.rope_config(128, 96, True, magnitude=1.5, dtype="f32")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    pb.pblock_rope_forward(cfg, [pb.rope_tensor(x, 768, 6, y, 768)], 50)
    pb.pblock_rope_backward(cfg, [pb.rope_tensor(dy, 768, 6, dx, 768)], 50)
    lhs, rhs = (dy.double() * y.double()).sum(), (dx.double() * x.double()).sum()
    size = float((dy.double() * y.double()).abs().sum())
    assert abs(float(lhs - rhs)) <= 2.0 ** -20 * size
    e = torch.zeros_like(x)
    e[17, 300] = 1.0
    y2 = torch.empty_like(x)
    pb.pblock_rope_forward(cfg, [pb.rope_tensor(x + e, 768, 6, y2, 768)], 50)
    num = float((dy.double() * (y2.double() - y.double())).sum())
    assert abs(num - float(dx[17, 300])) <= 2.0 ** -19 * 16


def test_rope_infinities_stay_in_their_pair():
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say("[gpu] rope infinities")
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    x[1, 3], x[2, 40] = float("inf"), float("nan")
    y = torch.empty_like(x)
    pb.pblock_rope_forward(pb.rope_config(64), [pb.rope_tensor(x, 64, 1, y, 64)], 4)
    bad = (~torch.isfinite(y)).nonzero().tolist()
    assert bad == [[1, 3], [1, 35], [2, 8], [2, 40]]


def test_rope_offsets_past_32_bits():
    """Rows 2^16 elements apart: the last ones lie past 2^31 elements."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say("[gpu] rope, 2.3e9 elements")
    tokens, ld = 35000, 1 << 16
    x = torch.empty(tokens, ld, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    vals = torch.empty(tokens, 256, device="cuda").normal_(generator=g).to(torch.bfloat16)
    x[:, 1000:1256] = vals
    y = torch.empty(tokens, 256, dtype=torch.bfloat16, device="cuda")
    cfg = pb.rope_config(128)
    pb.pblock_rope_forward(cfg, [pb.rope_tensor(vals, 256, 2, y, 256)], tokens)
    pb.pblock_rope_forward(cfg, [pb.rope_tensor(x[:, 1000:], ld, 2)], tokens)
    assert torch.equal(x[:, 1000:1256], y)


def test_rope_on_another_stream_and_in_a_graph():
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say("[gpu] rope stream and graph")
    run("bf16", 70, (4, 4), 128, None, False, stream=torch.cuda.Stream())
    x = torch.randn(64, 512, device="cuda").to(torch.bfloat16)
    y, pos = torch.empty_like(x), torch.arange(64, device="cuda")
    cfg, part = pb.rope_config(128), [pb.rope_tensor(x, 512, 4, y, 512)]
    pb.pblock_rope_forward(cfg, part, 64, positions=pos)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pb.pblock_rope_forward(cfg, part, 64, positions=pos)
    for r in range(3):
        x.normal_()
        pos.add_(1000)
        pb.pblock_rope_forward(cfg, part, 64, positions=pos)
        want = y.clone()
        y.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), r

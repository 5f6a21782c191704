"""The root-mean-square norm on the GPU against the fp64 oracle.

Tolerances.  u: half a step of the type (eps / 2).  The row's sum of squares is a tree
of at most 32 terms a thread, six steps in a wave and up to 16 waves: below 2^6 fp32
roundings of a sum of positives, half of that in the root, then the division, the
root and two products: y is off by u and below 2^-18 of itself.  The backward's row
mean likewise, relative to the mean of the magnitudes; dgamma adds up rows one after
the other in a workgroup, then workgroups 16 at a time: ceil(rows / 512) + 48 + 4
roundings of the sum of magnitudes (rows that share a workgroup: 16 more).  The sum
x + resid is rounded to fp32 and to its type: u + 2^-24.
"""
import numpy as np
import pytest

from oracle import operators_oracle as oo

pytestmark = pytest.mark.gpu
EPS = np.float64(np.float32(1e-5))


def _say(msg):
    print(msg, flush=True)


def f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def make(dtype, rows, cols, seed=0, offset=0, resid=True):
    import torch
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(seed)

    def new(n, shape, mean=0.0, std=1.0):
        t = torch.empty(n + offset, device="cuda").normal_(mean, std, generator=g).to(act)
        return t[offset:].view(shape)

    n = rows * cols
    return dict(act=act, x=new(n, (rows, cols)), resid=new(n, (rows, cols), std=3.0) if resid else None,
                gamma=new(cols, (cols,), 1.0, 0.2), dy=new(n, (rows, cols)),
                dsum=new(n, (rows, cols)) if resid else None, half=torch.finfo(act).eps / 2)


SIZES = [(1, 1), (1, 8), (3, 5), (17, 16), (100, 64), (33, 128), (5, 136), (7, 1000), (4, 1024),
         (9, 1999), (600, 2048), (3, 4104), (530, 5120), (2, 8192), (6, 8200), (1, 12288), (5, 16384),
         (3, 16392), (2, 24577), (3, 32768)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", SIZES, ids=lambda v: str(v))
def test_rmsnorm_matches_oracle(dtype, rows, cols):
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say(f"[gpu] rmsnorm {dtype} {rows} x {cols}")
    for resid, offset in ((True, 0), (False, 0), (True, 1)):
        t = make(dtype, rows, cols, seed=cols, offset=offset, resid=resid)
        act, half = t["act"], t["half"]
        empty = lambda *s, d=act: torch.empty(offset + int(np.prod(s)), dtype=d,  # noqa: E731
                                              device="cuda")[offset:].view(s)
        y, total = empty(rows, cols), empty(rows, cols) if resid else None
        rstd, dx, dgamma = empty(rows, d=torch.float32), empty(rows, cols), empty(cols, d=torch.float32)
        cfg = pb.rmsnorm_config(rows, cols, dtype=dtype)
        pb.pblock_rmsnorm_forward(cfg, t["x"], t["gamma"], y, resid=t["resid"], sum_out=total, rstd=rstd)
        s = total if resid else t["x"]
        ws = torch.empty(max(1, pb.pblock_rmsnorm_workspace_bytes(cfg)), dtype=torch.uint8, device="cuda")
        pb.pblock_rmsnorm_backward(cfg, s, t["gamma"], rstd, t["dy"], dx, dgamma, ws, dsum=t["dsum"])
        torch.cuda.synchronize()
        rs, rr, ry = oo.rmsnorm(f64(t["x"]), f64(t["gamma"]), EPS, f64(t["resid"]) if resid else None)
        assert np.all(np.abs(f64(y) - ry) <= (half + 2.0 ** -18) * np.abs(ry))
        assert np.all(np.abs(f64(rstd) - rr) <= 2.0 ** -18 * rr)
        if resid:
            assert np.all(np.abs(f64(total) - rs) <= (half + 2.0 ** -24) * np.abs(rs))
        # the backward from what the forward kept
        sk, rk, dy, gm = f64(s), f64(rstd), f64(t["dy"]), f64(t["gamma"])
        ds = f64(t["dsum"]) if resid else np.zeros_like(sk)
        rdx, rdg = oo.rmsnorm_backward(sk, gm, rk, dy, ds)
        r1 = rk[:, None]
        size = np.abs(ds) + np.abs(r1 * dy * gm) + np.abs(sk * r1) * np.mean(
            np.abs(dy * gm * sk * r1), axis=1, keepdims=True) * r1
        assert np.all(np.abs(f64(dx) - rdx) <= half * np.abs(rdx) + 2.0 ** -18 * size)
        steps = -(-rows // 512) + 48 + 4 + 16
        assert np.all(np.abs(f64(dgamma) - rdg) <= steps * 2.0 ** -24 * np.sum(np.abs(dy * sk * r1), 0))


def codes_of(y, scales, group):
    """e4m3 codes of y over the scales that the kernel kept, through fp32 like a cast."""
    import torch
    cols = y.shape[1]
    g = group or cols
    wide = np.repeat(scales, g, axis=1)[:, :cols]
    return torch.from_numpy(y / wide).float().to(torch.float8_e4m3fn)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("rows,cols", [(1, 1), (4, 40), (33, 100), (5, 128), (3, 160), (70, 2048),
                                       (9, 1999), (3, 12288), (2, 12345), (2, 32768), (3, 32767)],
                         ids=lambda v: str(v))
def test_rmsnorm_codes_are_those_of_the_definition(dtype, group, rows, cols):
    """Scales are the definition's rounded to fp32 (the row's own rounding in fp64 moves
    them by less than a step: 2^-23); codes are then equal, all of them."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say(f"[gpu] rmsnorm e4m3 {dtype} {rows} x {cols} group={group}")
    t = make(dtype, rows, cols, seed=cols + group)
    if rows > 2:
        t["x"][1], t["resid"][1] = 0.0, 0.0  # a row of zeros
    cfg = pb.rmsnorm_config(rows, cols, dtype=dtype, group=group)
    groups = -(-cols // group) if group else 1
    q = torch.empty(rows, cols, dtype=torch.float8_e4m3fn, device="cuda")
    sc = torch.empty(rows, groups, device="cuda")
    y, total = torch.empty_like(t["x"]), torch.empty_like(t["x"])
    pb.pblock_rmsnorm_forward(cfg, t["x"], t["gamma"], y, t["resid"], total, q, sc)
    torch.cuda.synchronize()
    _, _, ry = oo.rmsnorm(f64(t["x"]), f64(t["gamma"]), EPS, f64(t["resid"]))
    ref = oo.e4m3_scales(ry, group)
    got = f64(sc)
    assert np.all(np.abs(got - ref) <= 2.0 ** -23 * ref)
    want = codes_of(ry, got, group)
    same = q.cpu().view(torch.uint8) == want.view(torch.uint8)
    zero = (q.cpu().float() == 0) & (want.float() == 0)
    assert bool((same | zero).all()), int((~(same | zero)).sum())
    # y beside the codes, once rounded from 64 bits (through fp32)
    assert np.all(np.abs(f64(y) - ry) <= (t["half"] + 2.0 ** -23) * np.abs(ry))


def test_rmsnorm_in_place():
    """sum over resid and y over x, dx over dy: the bits of separate buffers."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say("[gpu] rmsnorm in place")
    for rows, cols in ((37, 100), (5, 5120), (18, 64)):
        t = make("bf16", rows, cols)
        cfg = pb.rmsnorm_config(rows, cols)
        y, total, rstd = torch.empty_like(t["x"]), torch.empty_like(t["x"]), torch.empty(rows, device="cuda")
        pb.pblock_rmsnorm_forward(cfg, t["x"], t["gamma"], y, t["resid"], total, rstd=rstd)
        x2, r2 = t["x"].clone(), t["resid"].clone()
        pb.pblock_rmsnorm_forward(cfg, x2, t["gamma"], x2, r2, r2)
        assert torch.equal(x2, y) and torch.equal(r2, total)
        x3 = t["x"].clone()
        pb.pblock_rmsnorm_forward(cfg, x3, t["gamma"], y, t["resid"], x3)
        assert torch.equal(x3, total)
        ws = torch.empty(pb.pblock_rmsnorm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        dg, dg2, dx = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda"), torch.empty_like(y)
        args = lambda dy, out, g, ds: pb.pblock_rmsnorm_backward(  # noqa: E731
            cfg, total, t["gamma"], rstd, dy, out, g, ws, dsum=ds)
        args(t["dy"], dx, dg, t["dsum"])
        for which in ("dy", "dsum"):
            u = {k: t[k].clone() for k in ("dy", "dsum")}
            args(u["dy"], u[which], dg2, u["dsum"])
            assert torch.equal(u[which], dx) and torch.equal(dg2, dg), which


def test_rmsnorm_rows_apart():
    """A NaN, an infinity or values that fill the type's range stay in their row; without
    rows dgamma is zero; eps 0 on a row of zeros gives NaN there alone."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say("[gpu] rmsnorm rows apart")
    t = make("f32", 40, 72, resid=False)
    cfg = pb.rmsnorm_config(40, 72, dtype="f32")
    clean = torch.empty_like(t["x"])
    pb.pblock_rmsnorm_forward(cfg, t["x"], t["gamma"], clean)
    x = t["x"].clone()
    x[3, 5], x[17, 0], x[20] = float("nan"), float("inf"), 1e18
    y = torch.empty_like(x)
    pb.pblock_rmsnorm_forward(cfg, x, t["gamma"], y)
    keep = [i for i in range(40) if i not in (3, 17, 20)]
    assert torch.equal(y[keep], clean[keep]) and bool(torch.isnan(y[3]).all())
    assert bool(torch.isnan(y[17, 0])) and bool((y[17, 1:] == 0).all())
    np.testing.assert_allclose(f64(y[20]), f64(t["gamma"]), rtol=2.0 ** -18)
    x[0] = 0.0
    pb.pblock_rmsnorm_forward(pb.rmsnorm_config(40, 72, eps=0.0, dtype="f32"), x, t["gamma"], y)
    assert bool(torch.isnan(y[0]).all()) and bool(torch.isfinite(y[1]).all())
    dg = torch.full((72,), 5.0, device="cuda")
    none = torch.empty(0, 72, device="cuda")
    pb.pblock_rmsnorm_backward(pb.rmsnorm_config(0, 72, dtype="f32"), none, t["gamma"],
                               torch.empty(0, device="cuda"), none, none, dg, None)
    assert bool((dg == 0).all())


def test_rmsnorm_offsets_past_32_bits():
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say("[gpu] rmsnorm, 2.2e9 elements")
    rows, cols = 67000, 32768
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    t = make("bf16", 50, cols)
    x[-50:] = t["x"]
    cfg = pb.rmsnorm_config(rows, cols)
    rstd = torch.empty(rows, device="cuda")
    y = torch.empty_like(x)
    pb.pblock_rmsnorm_forward(cfg, x, t["gamma"], y, rstd=rstd)
    small = pb.rmsnorm_config(50, cols)
    y2, r2 = torch.empty_like(t["x"]), torch.empty(50, device="cuda")
    pb.pblock_rmsnorm_forward(small, t["x"], t["gamma"], y2, rstd=r2)
    assert torch.equal(y[-50:], y2) and torch.equal(rstd[-50:], r2) and not bool(y[:-50].any())
    dy = torch.zeros_like(x)
    dy[-50:] = t["dy"]
    ws = torch.empty(pb.pblock_rmsnorm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    dg, dx2, dg2 = torch.empty(cols, device="cuda"), torch.empty_like(y2), torch.empty(cols, device="cuda")
    pb.pblock_rmsnorm_backward(cfg, x, t["gamma"], rstd, dy, y, dg, ws)
    pb.pblock_rmsnorm_backward(small, t["x"], t["gamma"], r2, t["dy"], dx2, dg2, ws)
    assert torch.equal(y[-50:], dx2)
    # the same 50 terms a column in another order
    size = (t["dy"].double() * t["x"].double() * r2.double()[:, None]).abs().sum(0)
    assert bool(((dg.double() - dg2.double()).abs() <= 2 * 120 * 2.0 ** -24 * size).all())


def test_rmsnorm_streams_and_graph():
    """Two calls at once on two streams, each with its own workspace; a captured step
    replayed over new inputs."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say("[gpu] rmsnorm streams and graph")
    sets = []
    for seed in (1, 2):
        t = make("bf16", 300, 2048, seed=seed)
        cfg = pb.rmsnorm_config(300, 2048)
        t.update(cfg=cfg, y=torch.empty_like(t["x"]), total=torch.empty_like(t["x"]),
                 rstd=torch.empty(300, device="cuda"), dx=torch.empty_like(t["x"]),
                 dg=torch.empty(2048, device="cuda"),
                 ws=torch.empty(pb.pblock_rmsnorm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"))
        sets.append(t)

    def step(t, stream=None):
        pb.pblock_rmsnorm_forward(t["cfg"], t["x"], t["gamma"], t["y"], t["resid"], t["total"],
                                  rstd=t["rstd"], stream=stream)
        pb.pblock_rmsnorm_backward(t["cfg"], t["total"], t["gamma"], t["rstd"], t["dy"], t["dx"],
                                   t["dg"], t["ws"], dsum=t["dsum"], stream=stream)

    outs = lambda t: [t[k] for k in ("y", "total", "rstd", "dx", "dg")]  # noqa: E731
    want = []
    for t in sets:
        step(t)
        want.append([v.clone() for v in outs(t)])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for t, s in zip(sets, streams):
            step(t, s)
    torch.cuda.synchronize()
    for t, w in zip(sets, want):
        assert all(torch.equal(a, b) for a, b in zip(outs(t), w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(sets[0])
    for r in range(3):
        sets[0]["x"].normal_()
        step(sets[0])
        w = [v.clone() for v in outs(sets[0])]
        for v in outs(sets[0]):
            v.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs(sets[0]), w)), r


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rmsnorm_of_rows_whose_squares_pass_fp32(dtype):
    """Rows of 1e30 and 1e-30 beside ordinary ones, eps = 0: the squares do not fit into
    fp32, the results do."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    _say(f"[gpu] rmsnorm range {dtype}")
    for cols in (100, 1000, 5120):
        t = make(dtype, 6, cols, seed=cols, resid=False)
        scale = torch.tensor([1e30, 1.0, 1e-30, 1e19, 1e-19, 2e37], device="cuda")[:, None]
        x = (t["x"].float().clamp(-8, 8) * scale).to(t["act"])
        y, rstd = torch.empty_like(x), torch.empty(6, device="cuda")
        cfg = pb.rmsnorm_config(6, cols, eps=0.0, dtype=dtype)
        pb.pblock_rmsnorm_forward(cfg, x, t["gamma"], y, rstd=rstd)
        _, rr, ry = oo.rmsnorm(f64(x), f64(t["gamma"]), 0.0)
        assert np.all(np.abs(f64(y) - ry) <= (t["half"] + 2.0 ** -18) * np.abs(ry))
        assert np.all(np.abs(f64(rstd) - rr) <= 2.0 ** -18 * rr)

"""The root-mean-square norm within the roundings that its kernels make, and in place.

Forward, without the 8-bit output: s = x + resid is rounded to fp32 (2^-24; exact without
resid), its squares are summed in fp64, so 1 / rms is off by the roundings of s (2^-24 at
most) and its own: rstd 2^-23, without resid 2^-24.  y has s, r and two products: 5 and 3
times 2^-24, and its type's half step.  With the 8-bit output all of it is fp64 up to the
rounding of y to fp32 and its type: half a step and 2^-24.
"""
import numpy as np
import pytest

from oracle import operators_oracle as oo
from tests.test_gpu_rmsnorm import EPS, f64, make

pytestmark = pytest.mark.gpu
SLACK = 2.0 ** -34  # second-order terms and the fp64 sum


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(3, 7), (64, 100), (40, 1024), (30, 2049), (20, 5120), (7, 16384),
                                       (5, 32768)], ids=lambda v: str(v))
def test_rmsnorm_forward_within_its_roundings(dtype, rows, cols):
    import torch
    from paper_2402_15627_amd import pblock as pb
    print(f"[gpu] rmsnorm bounds {dtype} {rows} x {cols}", flush=True)
    for resid in (False, True):
        t = make(dtype, rows, cols, seed=cols, resid=resid)
        y, rstd = torch.empty_like(t["x"]), torch.empty(rows, device="cuda")
        cfg = pb.rmsnorm_config(rows, cols, dtype=dtype)
        _, rr, ry = oo.rmsnorm(f64(t["x"]), f64(t["gamma"]), EPS, f64(t["resid"]) if resid else None)
        pb.pblock_rmsnorm_forward(cfg, t["x"], t["gamma"], y, resid=t["resid"], rstd=rstd)
        assert np.all(np.abs(f64(rstd) - rr) <= ((2 if resid else 1) * 2.0 ** -24 + SLACK) * rr)
        assert np.all(np.abs(f64(y) - ry) <= (t["half"] + (5 if resid else 3) * 2.0 ** -24 + SLACK) * np.abs(ry))
        q = torch.empty(rows, cols, dtype=torch.uint8, device="cuda")
        sc = torch.empty(rows, 1, device="cuda")
        pb.pblock_rmsnorm_forward(cfg, t["x"], t["gamma"], y, resid=t["resid"], q8=q, scales=sc, rstd=rstd)
        assert np.all(np.abs(f64(rstd) - rr) <= (2.0 ** -24 + SLACK) * rr)
        assert np.all(np.abs(f64(y) - ry) <= (t["half"] + 2.0 ** -24 + SLACK) * np.abs(ry))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(37, 100), (5, 5120), (9, 1999), (700, 72), (3, 16384), (5, 16392),
                                       (300, 24577), (3, 32768)], ids=lambda v: str(v))
def test_rmsnorm_every_output_in_place(dtype, rows, cols):
    """The bits of separate buffers: sum and y over x or resid, dx over s, dy or dsum, also
    for the rows that the backward reads twice (over 16384 columns)."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    print(f"[gpu] rmsnorm in place {dtype} {rows} x {cols}", flush=True)
    t = make(dtype, rows, cols)
    cfg = pb.rmsnorm_config(rows, cols, dtype=dtype)
    new = lambda: torch.empty_like(t["x"])  # noqa: E731
    y, total, rstd = new(), new(), torch.empty(rows, device="cuda")
    pb.pblock_rmsnorm_forward(cfg, t["x"], t["gamma"], y, t["resid"], total, rstd=rstd)
    for sum_at, y_at in (("resid", "x"), ("x", "resid"), (None, "x"), (None, "resid"), ("x", None), ("resid", None)):
        u = {"x": t["x"].clone(), "resid": t["resid"].clone()}
        s2 = u[sum_at] if sum_at else new()
        y2 = u[y_at] if y_at else new()
        pb.pblock_rmsnorm_forward(cfg, u["x"], t["gamma"], y2, u["resid"], s2)
        assert torch.equal(s2, total) and torch.equal(y2, y), (sum_at, y_at)
    x2 = t["x"].clone()
    pb.pblock_rmsnorm_forward(cfg, x2, t["gamma"], x2)
    y3 = new()
    pb.pblock_rmsnorm_forward(cfg, t["x"], t["gamma"], y3)
    assert torch.equal(x2, y3)
    ws = torch.empty(pb.pblock_rmsnorm_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    dg, dg2, dx = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda"), new()
    for dsum in (True, False):
        pb.pblock_rmsnorm_backward(cfg, total, t["gamma"], rstd, t["dy"], dx, dg, ws,
                                   dsum=t["dsum"] if dsum else None)
        for which in ("s", "dy", "dsum") if dsum else ("s", "dy"):
            u = {"s": total.clone(), "dy": t["dy"].clone(), "dsum": t["dsum"].clone()}
            pb.pblock_rmsnorm_backward(cfg, u["s"], t["gamma"], rstd, u["dy"], u[which], dg2, ws,
                                       dsum=u["dsum"] if dsum else None)
            assert torch.equal(u[which], dx) and torch.equal(dg2, dg), (which, dsum)

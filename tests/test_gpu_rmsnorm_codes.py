"""The 8-bit output of the root-mean-square norm where its definition is easily missed:
quotients next to the middle of two codes, NaN and infinities.

A code is y / scale rounded to fp32 and that rounded to e4m3.  The kernel's fp64 product
with 1 / scale is off by a few 2^-53 from the oracle's quotient; the planted quotients
are checked to be farther than that from every border of the first rounding.
"""
import numpy as np
import pytest

from oracle import operators_oracle as oo
from tests.test_gpu_rmsnorm import EPS, codes_of, f64

pytestmark = pytest.mark.gpu
TINY = 2.0 ** -126


def e4m3_values():
    import torch
    v = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    return v  # 0 .. 448, ascending


def test_rmsnorm_codes_of_quotients_in_the_middle_of_two():
    import torch
    from paper_2402_15627_amd import pblock as pb
    print("[gpu] rmsnorm e4m3 middles", flush=True)
    cols = 4096
    rng = np.random.default_rng(4)
    x = rng.uniform(0.5, 2.0, cols).astype(np.float32) * rng.choice([-1, 1], cols).astype(np.float32)
    s = x.astype(np.float64)
    r = 1.0 / np.sqrt(np.mean(s * s) + EPS)
    v = e4m3_values()
    middle = rng.choice((v[8:-1] + v[9:]) / 2, cols)
    gamma = np.empty(cols, np.float32)
    gamma[0] = 448.0 / (s[0] * r)
    y0 = abs(s[0] * r * np.float64(gamma[0]))
    scale = np.float64(np.float32(y0 / 448.0))
    gamma[1:] = middle[1:] * scale / (s[1:] * r)  # rounded to fp32: within half a step of it
    y = (s * r * gamma.astype(np.float64))[None, :]
    q = y[0, 1:] / scale
    assert np.abs(q).max() <= 448.0 * (1 + 2.0 ** -23)
    # away from the borders of the rounding to fp32 (exact in fp64: eleven of its bits)
    step = 2.0 ** (np.floor(np.log2(np.abs(q))) - 23)
    to_border = np.abs(np.abs(q / step - np.floor(q / step)) - 0.5)
    keep = np.concatenate([[True], to_border > 2.0 ** -20])
    direct = v[np.argmin(np.abs(np.abs(q)[:, None] - v[None, :]), 1)]
    want = codes_of(y, np.array([[scale]]), 0)[0]
    other = direct != np.abs(want[1:].double().numpy())
    assert int((other & keep[1:]).sum()) > 300  # one rounding would give another code
    t = torch.from_numpy(x)[None].cuda()
    codes = torch.empty(1, cols, dtype=torch.float8_e4m3fn, device="cuda")
    sc = torch.empty(1, 1, device="cuda")
    pb.pblock_rmsnorm_forward(pb.rmsnorm_config(1, cols, dtype="f32"), t, torch.from_numpy(gamma).cuda(),
                              q8=codes, scales=sc)
    assert float(sc) == scale
    same = codes[0].cpu().view(torch.uint8) == want.view(torch.uint8)
    assert bool(same[torch.from_numpy(keep)].all()), int((~same).sum())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("cols", [70, 512, 5121])
def test_rmsnorm_codes_of_nan_and_infinity(dtype, group, cols):
    import torch
    from paper_2402_15627_amd import pblock as pb
    print(f"[gpu] rmsnorm e4m3 NaN and infinity {dtype} cols={cols} group={group}", flush=True)
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.empty(6, cols, device="cuda").normal_(generator=g).to(act)
    resid = torch.empty(6, cols, device="cuda").normal_(generator=g).to(act)
    gamma = torch.empty(cols, device="cuda").normal_(1.0, 0.2, generator=g).to(act)
    groups = -(-cols // group) if group else 1
    size = group or cols
    cfg = pb.rmsnorm_config(6, cols, dtype=dtype, group=group)

    def call(x, resid, gamma):
        q = torch.empty(6, cols, dtype=torch.float8_e4m3fn, device="cuda")
        sc, rstd = torch.empty(6, groups, device="cuda"), torch.empty(6, device="cuda")
        pb.pblock_rmsnorm_forward(cfg, x, gamma, resid=resid, q8=q, scales=sc, rstd=rstd)
        return q.float().cpu().numpy(), sc.cpu().numpy(), rstd.cpu().numpy()

    clean = call(x, resid, gamma)
    bad = x.clone()
    bad[1, 3], bad[4, 40] = float("nan"), -float("inf")
    other = resid.clone()
    other[2, 5] = float("inf")
    q, sc, rstd = call(bad, other, gamma)
    for row in (0, 3, 5):
        assert all(np.array_equal(a[row], b[row]) for a, b in zip((q, sc, rstd), clean)), row
    assert np.isnan(q[1]).all() and (sc[1] == TINY).all() and np.isnan(rstd[1])
    for row, c in ((4, 40), (2, 5)):  # r is 0
        rest = np.arange(cols) != c
        assert np.isnan(q[row, c]) and (q[row, rest] == 0).all() and (sc[row] == TINY).all() and rstd[row] == 0
    # a weight: its column alone is NaN; beside an infinite one its group is zeros
    for value in (float("nan"), float("inf")):
        weird = gamma.clone()
        weird[35] = value
        q, sc, rstd = call(x, resid, weird)
        k, cols_k = 35 // size, slice(35 // size * size, 35 // size * size + size)
        out = np.ones(cols, bool)
        out[cols_k] = False
        assert np.array_equal(q[:, out], clean[0][:, out]) and np.array_equal(rstd, clean[2])
        assert np.array_equal(np.delete(sc, k, 1), np.delete(clean[1], k, 1))
        assert np.isnan(q[:, 35]).all()
        beside = np.delete(q[:, cols_k], 35 - k * size, 1)
        if value == float("inf"):
            assert (sc[:, k] == np.inf).all() and (beside == 0).all()
        else:
            _, _, y = oo.rmsnorm(f64(x), f64(gamma), EPS, f64(resid))
            y[:, 35] = 0.0
            ref = oo.e4m3_scales(y, group)[:, k]
            assert np.all(np.abs(sc[:, k] - ref) <= 2.0 ** -23 * ref) and np.isfinite(beside).all()

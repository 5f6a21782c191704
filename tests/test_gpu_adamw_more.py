"""AdamW step on the GPU, beyond sizes: many tensors in a call, values that are not finite,
graphs, streams, seeds, many steps with 8-bit states.  Tolerances as in test_gpu_adamw."""
import numpy as np
import pytest

from oracle import score_oracle as so
from tests.test_gpu_adamw import HYPER, check, expected, make, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("e4m3", [False, True])
def test_many_tensors_are_one_after_another(e4m3):
    """130 tensors (three launches), some without elements or without a copy: each is the
    step of its own, and the bits are those of calls of one."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    sizes = [(n, n % 4) for n in (1, 7, 256, 300, 1024, 1500)] * 20 + [(4000, 0)] * 10
    all_, twice = ([make(n, i, e4m3, off, decay=0.1 * (i % 3)) for i, (n, off) in enumerate(sizes)]
                   for _ in range(2))
    for ts in (all_, twice):
        ts[5]["copy"] = ts[77]["copy"] = None
    want = [expected(t, **HYPER) for t in all_]
    none = torch.empty(0, device="cuda")
    empty = pb.adamw_tensor(none, none, none, none) if not e4m3 else pb.adamw_tensor(
        none, none, none.to(torch.uint8), none.to(torch.uint8), avg_scale=none, sq_scale=none)
    parts = [tensor(pb, t) for t in all_]
    parts.insert(3, empty)
    parts.append(empty)
    cfg = pb.adamw_config(**HYPER)
    pb.pblock_adamw_step(cfg, pb.AdamwTensors(parts))
    for t in twice:
        pb.pblock_adamw_step(cfg, [tensor(pb, t)])
    torch.cuda.synchronize()
    for t, s, e in zip(all_, twice, want):
        for k, x in t.items():
            if torch.is_tensor(x):
                assert torch.equal(x.view(torch.uint8), s[k].view(torch.uint8)), k
        if t["copy"] is None:
            t["copy"] = t["w"].to(torch.bfloat16)
        check(t, e)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_gradient_that_is_not_finite_shows(e4m3, value):
    """Its own weight is lost, and with 8-bit states its block's states; no other block's."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    t = make(1000, 3, e4m3)
    t["g"][300] = value
    u = make(1000, 3, e4m3)
    cfg = pb.adamw_config(**HYPER)
    pb.pblock_adamw_step(cfg, [tensor(pb, t)])
    pb.pblock_adamw_step(cfg, [tensor(pb, u)])
    torch.cuda.synchronize()
    assert not torch.isfinite(t["w"][300])
    others = torch.arange(1000, device="cuda") != 300
    assert torch.equal(t["w"][others], u["w"][others])
    if e4m3:
        assert not torch.isfinite(t["m_scale"][1]) and not torch.isfinite(t["r_scale"][1])
        same = torch.arange(4, device="cuda") != 1
        assert torch.equal(t["m_scale"][same], u["m_scale"][same])
        back = t["m"].view(torch.float8_e4m3fn).float() * t["m_scale"].repeat_interleave(256)[:1000]
        assert not torch.isfinite(back[256:512]).any() or not torch.isfinite(back[300])
        t["g"][300] = 0.0  # the next step does not make it whole again
        pb.pblock_adamw_step(cfg, [tensor(pb, t)])
        torch.cuda.synchronize()
        assert not torch.isfinite(t["w"][300])


@pytest.mark.parametrize("scale", [1e-22, 1e-12, 1e12, 1e18])
@pytest.mark.parametrize("e4m3", [False, True])
def test_values_far_from_one(scale, e4m3):
    """Squares near either end of fp32 and beyond take the general root and quotient."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    t = make(2000, 4, e4m3)
    t["g"].mul_(scale / 1e-3)
    t["g"][::7] = 0.0
    for k in ("m", "v") if not e4m3 else ("m_scale", "r_scale"):
        t[k].mul_(0.0)
    e = expected(t, **HYPER)
    pb.pblock_adamw_step(pb.adamw_config(**HYPER), [tensor(pb, t)])
    torch.cuda.synchronize()
    # (squares below the smallest normal number lose bits: an error of the update
    # where it is beside eps; at 1e-22 they are 0)
    tiny = scale < 1e-18
    w = t["w"].double().cpu().numpy()
    slack = 12 * 2.0 ** -24 * e["a_u"] + 2.0 ** -22 * abs(e["w0"])
    if not tiny:
        assert (abs(w - e["w"]) <= slack).all()
    assert np.isfinite(w).all()
    assert torch.equal(t["w"][::7] != t["w"][::7], torch.zeros_like(t["w"][::7], dtype=torch.bool))


def test_seeds_decide_codes_and_nothing_else():
    import torch
    from paper_2402_15627_amd import pblock as pb
    cfg = pb.adamw_config(**HYPER)
    runs = []
    for seed in (1, 1, 2, 1 << 40):
        t = make(5000, 9, True)
        t["seed"] = seed
        pb.pblock_adamw_step(cfg, [tensor(pb, t)])
        torch.cuda.synchronize()
        runs.append(t)
    a, b, c, d = runs
    for k in ("w", "m", "r", "m_scale", "r_scale"):
        assert torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)), k
    for x in (c, d):
        assert torch.equal(a["w"], x["w"]) and torch.equal(a["m_scale"], x["m_scale"])
        share = (a["m"] != x["m"]).float().mean()
        assert 0.1 < share < 0.7
    # a laid-out list takes the seeds of a new step
    parts = pb.AdamwTensors([tensor(pb, a), tensor(pb, c)])
    parts.seeds([5, 6])
    assert [r.seed for r in parts.array] == [5, 6]
    with pytest.raises(ValueError):
        parts.seeds([5])


def test_rounding_is_even_handed():
    """The mean over 64 seeds of 4096 elements' values is the value before it is rounded:
    a code's step is at most an eighth of the value, so the mean of 64 is off by at most
    an eighth / sqrt(4 64) of it in one standard deviation, and the relative error's mean
    over 4096 elements by a 64th of that: 1.3e-4."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    total, exact = 0, None
    for seed in range(64):
        t = make(4096, 11, True)
        t["seed"] = seed * 7919 + 3
        e = expected(t, **HYPER)
        pb.pblock_adamw_step(pb.adamw_config(**HYPER), [tensor(pb, t)])
        torch.cuda.synchronize()
        total = total + so.from_e4m3(t["m"].cpu().numpy(), t["m_scale"].cpu().numpy())
        exact = e["m"]
    big = abs(exact) > np.abs(exact).max() / 100  # (above the codes' smallest steps)
    rel = total[big] / 64 / exact[big] - 1
    assert abs(rel.mean()) <= 5 * 1.3e-4 and np.sqrt((rel ** 2).mean()) <= 0.125 / 16 * 1.1


def test_second_moments_follow_their_average():
    """A gradient of constant size that drops to a tenth: sqrt(v) in 8 bits comes down with
    the exact one (rounded to nearest it would stand still). Each step's rounding moves a
    code by a step of at most an eighth with a probability of its distance, 0.025 8 a step:
    over the average's 40 steps a standard deviation of 0.125 sqrt(40 0.2) / 2 or so for one
    element, a 64th of that for the mean of 4096."""
    import torch
    from paper_2402_15627_amd import pblock as pb
    n = 4096
    t = make(n, 12, True)
    t["r_scale"].mul_(0.0)
    t["m_scale"].mul_(0.0)
    v = np.zeros(n)
    for step in range(1, 121):
        t["g"].fill_(1e-3 if step <= 60 else 1e-4)
        cfg = pb.adamw_config(1e-4, 0.9, 0.95, step=step)
        part = tensor(pb, t)
        part.seed = step
        pb.pblock_adamw_step(cfg, [part])
        v = 0.95 * v + 0.05 * (1e-6 if step <= 60 else 1e-8)
    torch.cuda.synchronize()
    got = so.from_e4m3(t["r"].cpu().numpy(), t["r_scale"].cpu().numpy())
    assert abs(got.mean() / np.sqrt(v[0]) - 1) <= 0.05
    assert torch.isfinite(t["w"]).all()


@pytest.mark.parametrize("e4m3", [False, True])
def test_replays_and_streams(e4m3):
    import torch
    from paper_2402_15627_amd import pblock as pb
    cfg = pb.adamw_config(**HYPER)
    eager, captured, side = (make(3000, 21, e4m3) for _ in range(3))
    parts = pb.AdamwTensors([tensor(pb, captured)])
    g = torch.cuda.CUDAGraph()
    saved = {k: x.clone() for k, x in captured.items() if torch.is_tensor(x)}
    pb.pblock_adamw_step(cfg, parts)
    torch.cuda.synchronize()
    for k, x in saved.items():
        captured[k].copy_(x)
    with torch.cuda.graph(g):
        pb.pblock_adamw_step(cfg, parts)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        pb.pblock_adamw_step(cfg, [tensor(pb, eager)])
        pb.pblock_adamw_step(cfg, [tensor(pb, side)], stream=s)
        g.replay()
        torch.cuda.synchronize()
        for k, x in eager.items():
            if torch.is_tensor(x):
                assert torch.equal(x.view(torch.uint8), captured[k].view(torch.uint8)), k
                assert torch.equal(x.view(torch.uint8), side[k].view(torch.uint8)), k


def test_copies_of_another_type_are_refused():
    import torch
    from paper_2402_15627_amd import pblock as pb
    t, u = make(10, 1, False), make(10, 2, False, copy="f32")
    with pytest.raises(ValueError, match="copies of more than one type"):
        pb.AdamwTensors([tensor(pb, t), tensor(pb, u)])
    with pytest.raises(ValueError, match="param_copy is"):
        pb.pblock_adamw_step(pb.adamw_config(1e-3), [tensor(pb, t)], pb.PB_F32)
    with pytest.raises(ValueError, match="another type"):
        pb.AdamwTensors([tensor(pb, t), tensor(pb, make(10, 1, True))])
    torch.cuda.synchronize()

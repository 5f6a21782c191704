"""Refusals and sizes of the operators around the block, on a machine without a GPU:
every call below fails a host check (or has nothing to launch), so its pointers are
never read."""
import ctypes

import pytest
import torch

from paper_2402_15627_amd import pblock as pb

FAKE = 1 << 40
OK, BAD, UNSUPPORTED, SMALL = 0, 1, 2, 3


def align(v):
    return (v + 255) // 256 * 256


# ------------------------------------------------------- rotary positions
def rope(fn="pblock_rope_forward", n=None, tokens=4, seq=4, positions=None, tensors=None, **over):
    cfg = pb.rope_config(64, scaling=over.pop("scaling", "by_parts"), factor=2.0, orig_len=64.0)
    for k, v in over.items():
        setattr(cfg, k, v)
    x = tensors if tensors is not None else [pb.RopeTensor(FAKE, FAKE, 128, 128, 2)]
    arr = (pb.RopeTensor * max(len(x), 1))(*x)
    return getattr(pb.load_library(), fn)(ctypes.byref(cfg), len(x) if n is None else n, arr, tokens,
                                          seq, positions, None)


@pytest.mark.parametrize("fn", ["pblock_rope_forward", "pblock_rope_backward"])
@pytest.mark.parametrize("over,status", [
    (dict(head_dim=63), BAD), (dict(head_dim=0), BAD), (dict(head_dim=258), UNSUPPORTED),
    (dict(rot_dim=0), BAD), (dict(rot_dim=7), BAD), (dict(rot_dim=66), BAD),
    (dict(interleaved=2), BAD), (dict(base=0.0), BAD), (dict(base=float("inf")), BAD),
    (dict(magnitude=0.0), BAD), (dict(magnitude=float("nan")), BAD), (dict(magnitude=1e300), BAD),
    (dict(factor=0.0), BAD), (dict(orig_len=0.0), BAD), (dict(low_turns=-1.0), BAD),
    (dict(high_turns=1.0), BAD), (dict(dtype=5), BAD), (dict(tokens=-1), BAD),
    (dict(tokens=1 << 24), UNSUPPORTED), (dict(seq=0), BAD), (dict(positions=FAKE + 4), BAD),
    (dict(n=0), BAD), (dict(n=5), BAD),
    (dict(tensors=[pb.RopeTensor(None, FAKE, 128, 128, 2)]), BAD),
    (dict(tensors=[pb.RopeTensor(FAKE, FAKE + 1, 128, 128, 2)]), BAD),
    (dict(tensors=[pb.RopeTensor(FAKE, FAKE, 127, 128, 2)]), BAD),
    (dict(tensors=[pb.RopeTensor(FAKE, FAKE, 128, 256, 2)]), BAD),
    (dict(tensors=[pb.RopeTensor(FAKE, FAKE, 128, 128, 0)]), BAD),
    (dict(tensors=[pb.RopeTensor(FAKE, FAKE, 1 << 20, 1 << 20, 8193)]), UNSUPPORTED),
    (dict(tensors=[pb.RopeTensor(FAKE, FAKE, 1 << 32, 1 << 32, 2)]), UNSUPPORTED),
])
def test_rope_refusals(fn, over, status):
    assert rope(fn, **over) == status
    assert pb.pblock_last_error() != ""


def test_rope_scaling_values_are_read_only_by_their_kind():
    none = dict(tokens=0, factor=0.0, orig_len=-1.0, high_turns=0.0)
    assert rope(scaling="plain", **none) == OK
    assert rope(scaling="linear", **none) == BAD
    assert rope(scaling="linear", **dict(none, factor=2.0)) == OK
    cfg = pb.rope_config(64)
    cfg.scaling = 3
    arr = (pb.RopeTensor * 1)(pb.RopeTensor(FAKE, FAKE, 128, 128, 2))
    assert pb.load_library().pblock_rope_forward(ctypes.byref(cfg), 1, arr, 0, 1, None, None) == BAD
    assert pb.load_library().pblock_rope_forward(None, 1, arr, 0, 1, None, None) == BAD
    cfg.scaling = 0
    assert pb.load_library().pblock_rope_forward(ctypes.byref(cfg), 1, None, 0, 1, None, None) == BAD
    # no tokens: nothing is launched, no pointer is needed
    assert rope(tokens=0, tensors=[pb.RopeTensor(None, None, 128, 128, 2)]) == OK


# ------------------------------------------------- root-mean-square norm
def rms(**over):
    cfg = pb.rmsnorm_config(4, 64)
    a = dict(x=FAKE, resid=None, gamma=FAKE + (1 << 24), sum=None, y=FAKE, q8=None, scales=None, rstd=None)
    for k, v in over.items():
        if k in a:
            a[k] = v
        else:
            setattr(cfg, k, v)
    return pb.load_library().pblock_rmsnorm_forward(ctypes.byref(cfg), *a.values(), None)


def rms_back(nbytes=None, ws=FAKE + (1 << 26), **over):
    cfg = pb.rmsnorm_config(4, 64)
    a = dict(s=FAKE, gamma=FAKE + (1 << 24), rstd=FAKE + (1 << 25), dy=FAKE, dsum=None, dx=FAKE,
             dgamma=FAKE + (3 << 24))
    for k, v in over.items():
        if k in a:
            a[k] = v
        else:
            setattr(cfg, k, v)
    n = pb.pblock_rmsnorm_workspace_bytes(cfg) if nbytes is None else nbytes
    return pb.load_library().pblock_rmsnorm_backward(ctypes.byref(cfg), *a.values(), ws, n, None)


CONFIGS = [(dict(rows=-1), BAD), (dict(cols=0), BAD), (dict(cols=32769), UNSUPPORTED),
           (dict(rows=1 << 31), UNSUPPORTED), (dict(group=16), BAD), (dict(group=256), BAD),
           (dict(eps=-1e-5), BAD), (dict(eps=float("nan")), BAD), (dict(dtype=2), BAD),
           (dict(gamma=None), BAD), (dict(gamma=FAKE + 1), BAD)]


@pytest.mark.parametrize("over,status", CONFIGS + [
    (dict(x=None), BAD), (dict(x=FAKE + 1), BAD), (dict(y=None), BAD), (dict(resid=FAKE + 1), BAD),
    (dict(sum=FAKE + 256), BAD), (dict(resid=FAKE, sum=FAKE + 1), BAD),
    (dict(resid=FAKE, sum=FAKE), BAD),  # sum and y in one buffer
    (dict(y=FAKE + 2), BAD), (dict(y=FAKE + 4 * 64 * 2 - 2), BAD),  # y over a part of x
    (dict(resid=FAKE + 4096, sum=FAKE + 4096 - 2), BAD), (dict(resid=FAKE + 4096, sum=FAKE + 2), BAD),
    (dict(q8=FAKE), BAD), (dict(scales=FAKE), BAD), (dict(q8=FAKE, scales=FAKE + 2), BAD),
    (dict(rstd=FAKE + 2), BAD),
])
def test_rmsnorm_forward_refusals(over, status):
    assert rms(**over) == status
    assert pb.pblock_last_error() != ""


@pytest.mark.parametrize("over,status", CONFIGS + [
    (dict(s=None), BAD), (dict(rstd=None), BAD), (dict(rstd=FAKE + 2), BAD), (dict(dy=None), BAD),
    (dict(dsum=FAKE + 1), BAD), (dict(dx=None), BAD), (dict(dx=FAKE + 2), BAD),
    (dict(dsum=FAKE + 1024, dx=FAKE + 1022), BAD), (dict(dgamma=None), BAD),
    (dict(dgamma=FAKE + 2), BAD), (dict(ws=None), BAD), (dict(ws=FAKE + 16), BAD),
    (dict(nbytes=0), SMALL), (dict(nbytes=4 * 64 * 1 - 1), SMALL),
])
def test_rmsnorm_backward_refusals(over, status):
    assert rms_back(**over) == status
    assert pb.pblock_last_error() != ""


def test_rmsnorm_without_rows_and_its_workspace():
    assert rms(rows=0, x=None, y=None) == OK
    lib = pb.load_library()
    assert lib.pblock_rmsnorm_forward(None, *[FAKE] * 8, None, None) == BAD
    assert lib.pblock_rmsnorm_workspace_bytes(None) == 0
    # a row of fp32 per workgroup
    for rows in (1, 7, 100, 100000):
        for cols in (1, 5, 128, 129, 1024, 5120, 32768):
            n = pb.pblock_rmsnorm_workspace_bytes(pb.rmsnorm_config(rows, cols))
            assert n % 256 == 0 and n >= 4 * cols
    
    assert pb.pblock_rmsnorm_workspace_bytes(pb.rmsnorm_config(0, 64)) == 0
    assert pb.pblock_rmsnorm_workspace_bytes(pb.rmsnorm_config(4, 0)) == 0


# ------------------------------------------------------------- Muon step
def muon(ws=FAKE + (1 << 32), nbytes=1 << 30, copy=pb.PB_BF16, n=None, tensors=None, cfg_null=False, **over):
    cfg = pb.muon_config(1e-3)
    x = dict(param=FAKE, grad=FAKE + (1 << 20), momentum=FAKE + (2 << 20), param_copy=None, rows=8, cols=16, ld=16,
             weight_decay=0.1, scale=1.0)
    own = dict(mom_ptr="momentum")
    for k, v in over.items():
        if k in own:
            x[own[k]] = v
        elif k in x and k != "momentum":
            x[k] = v
        else:
            setattr(cfg, k, v)
    ts = tensors if tensors is not None else [pb.MuonTensor(*x.values())]
    arr = (pb.MuonTensor * max(len(ts), 1))(*ts)
    return pb.load_library().pblock_muon_step(None if cfg_null else ctypes.byref(cfg),
                                              len(ts) if n is None else n, arr, copy, ws, nbytes, None)


@pytest.mark.parametrize("over,status", [
    (dict(lr=float("nan")), BAD), (dict(momentum=1.0), BAD), (dict(momentum=-0.1), BAD),
    (dict(grad_scale=float("inf")), BAD), (dict(eps=0.0), BAD), (dict(nesterov=2), BAD),
    (dict(steps=0), BAD), (dict(steps=17), BAD), (dict(products=4), BAD), (dict(copy=3), BAD),
    (dict(n=0), BAD), (dict(n=17), BAD), (dict(param=None), BAD), (dict(grad=FAKE + 2), BAD),
    (dict(mom_ptr=None), BAD), (dict(param_copy=FAKE + 1), BAD), (dict(rows=-1), BAD),
    (dict(rows=65537, cols=65537, ld=65537), UNSUPPORTED),
    (dict(rows=4, cols=(1 << 20) + 1, ld=1 << 21), UNSUPPORTED),
    (dict(ld=15), BAD), (dict(ld=1 << 32), BAD), (dict(weight_decay=-1.0), BAD),
    (dict(scale=float("nan")), BAD), (dict(ws=None), BAD), (dict(ws=FAKE + 16), BAD),
    (dict(nbytes=1024), SMALL), (dict(cfg_null=True), BAD),
])
def test_muon_refusals(over, status):
    assert muon(**over) == status
    assert pb.pblock_last_error() != ""


@pytest.mark.parametrize("over,status", [
    (dict(dtype=7), BAD), (dict(steps=0), BAD), (dict(eps=-1.0), BAD), (dict(n=0), BAD),
    (dict(x=pb.OrthoTensor(None, FAKE, 8, 16, 16, 16)), BAD),
    (dict(x=pb.OrthoTensor(FAKE, FAKE + 1, 8, 16, 16, 16)), BAD),
    (dict(x=pb.OrthoTensor(FAKE, FAKE, 8, 16, 15, 16)), BAD),
    (dict(x=pb.OrthoTensor(FAKE, FAKE, 8, 16, 16, 24)), BAD),
    (dict(x=pb.OrthoTensor(FAKE, FAKE, 8, -1, 16, 16)), BAD),
    (dict(ws=None), BAD), (dict(nbytes=64), SMALL),
])
def test_orthogonalize_refusals(over, status):
    a = dict(n=1, x=pb.OrthoTensor(FAKE, FAKE, 8, 16, 16, 16), dtype=pb.PB_BF16, steps=5, eps=1e-7,
             ws=FAKE + (1 << 32), nbytes=1 << 30)
    a.update(over)
    assert pb.load_library().pblock_orthogonalize(a["n"], (pb.OrthoTensor * 1)(a["x"]), a["dtype"],
                                                  a["steps"], a["eps"], a["ws"], a["nbytes"],
                                                  None) == status
    assert pb.pblock_last_error() != ""


def test_rope_refuses_tensors_that_overlap():
    """Packed tensors interleave row by row: their columns decide.  The last calls pass
    every check and fail for want of a GPU (or launch nothing)."""
    R = pb.RopeTensor  # bf16, 2 heads of 64: 128 elements a row
    at = lambda n: FAKE + 2 * n  # noqa: E731
    assert rope(tensors=[R(FAKE, FAKE, 512, 512, 2), R(FAKE, FAKE, 512, 512, 2)]) == BAD
    assert "overlap" in pb.pblock_last_error()
    assert rope(tensors=[R(FAKE, FAKE, 512, 512, 2), R(at(127), at(127), 512, 512, 2)]) == BAD
    assert rope(tensors=[R(FAKE, FAKE, 512, 512, 2), R(at(3 * 512 + 500), at(3 * 512 + 500), 512, 512, 2)]) != BAD
    assert rope(tensors=[R(FAKE, FAKE, 512, 512, 2), R(at(2 * 512 + 500), at(2 * 512 + 500), 512, 512, 2)]) == BAD
    assert rope(tensors=[R(FAKE, at(64), 512, 512, 2)]) == BAD  # out over the next head of in
    assert rope(tensors=[R(FAKE, FAKE, 512, 512, 2), R(at(4096), at(128), 512, 512, 2)]) != BAD
    assert rope(tensors=[R(FAKE, FAKE, 512, 512, 2), R(at(128), at(128), 512, 512, 2)]) != BAD
    assert rope(tokens=0, tensors=[R(FAKE, FAKE, 512, 512, 2), R(FAKE, FAKE, 512, 512, 2)]) == OK


def test_muon_and_orthogonalize_refuse_matrices_that_overlap():
    M = lambda w, g, m: pb.MuonTensor(w, g, m, None, 8, 16, 64, 0.0, 1.0)  # noqa: E731
    f = lambda n: FAKE + 4 * n  # noqa: E731
    g, m = f(1 << 20), f(1 << 21)
    for bad in ([M(FAKE, g, m)] * 2, [M(FAKE, g, m), M(f(15), f(1 << 22), f(1 << 23))],
                [M(FAKE, FAKE, m)], [M(FAKE, g, f(64 + 8))], [M(FAKE, g, m), M(f(1 << 22), f(1 << 23), m)]):
        assert muon(tensors=bad) == BAD and "overlap" in pb.pblock_last_error()
    # columns of one weight side by side; a shared gradient is read alone
    assert muon(tensors=[M(FAKE, g, m), M(f(16), g + 64, m + 64), M(f(32), g, m + 128)], nbytes=1) == SMALL
    O = pb.OrthoTensor
    call = lambda *x: pb.load_library().pblock_orthogonalize(  # noqa: E731
        len(x), (O * len(x))(*x), pb.PB_F32, 5, 1e-7, FAKE, 1, None)
    assert call(O(FAKE, f(8), 8, 16, 64, 64)) == BAD
    assert call(O(FAKE, FAKE, 8, 16, 64, 64), O(f(32), f(4), 8, 16, 64, 64)) == BAD
    assert call(O(FAKE, FAKE, 8, 16, 64, 64), O(f(16), f(32), 8, 16, 64, 64)) == SMALL


def test_muon_refuses_copies_and_workspaces_over_tensors():
    f = lambda n: FAKE + 4 * n  # noqa: E731
    g, m, w2, g2, m2 = (f(k << 20) for k in range(1, 6))
    M = lambda copy, w=FAKE, gr=g, mo=m: pb.MuonTensor(w, gr, mo, copy, 8, 16, 64, 0.0, 1.0)  # noqa: E731
    for copy in (FAKE, FAKE + 64 * 4, g + 32, m + 3 * 256):  # bf16, rows of 128 bytes; of 256
        assert muon(tensors=[M(copy)]) == BAD and "copy" in pb.pblock_last_error()
    c = FAKE + (1 << 28)
    assert muon(tensors=[M(c), M(c + 30, w2, g2, m2)]) == BAD and "copy" in pb.pblock_last_error()
    assert muon(tensors=[M(c), M(c + 32, w2, g2, m2)], nbytes=1) == SMALL
    assert muon(tensors=[M(FAKE)], copy=pb.PB_F32) == BAD
    need = pb.pblock_muon_workspace_bytes(pb.muon_config(1e-3), [M(c)])
    for ws in (FAKE, FAKE - need + 256, m, c + 7 * 128, g - 256):
        assert muon(tensors=[M(c)], ws=ws // 256 * 256) == BAD and "ws" in pb.pblock_last_error()
    o = pb.OrthoTensor(FAKE, c, 8, 16, 64, 64)
    for ws in (FAKE, c):
        assert pb.load_library().pblock_orthogonalize(1, (pb.OrthoTensor * 1)(o), pb.PB_F32, 5, 1e-7, ws,
                                                      1 << 30, None) == BAD
        assert "ws" in pb.pblock_last_error()


def test_rmsnorm_refuses_outputs_over_other_tensors():
    """x is 512 bytes at FAKE, gamma 128 at FAKE + 2^24."""
    gamma, far = FAKE + (1 << 24), FAKE + (1 << 27)
    for over in (dict(q8=FAKE, scales=far), dict(q8=FAKE + 511, scales=far, y=far + 4096),
                 dict(q8=far, scales=FAKE + 508), dict(q8=far, scales=far + 252), dict(rstd=FAKE),
                 dict(rstd=gamma + 124), dict(y=gamma - 510), dict(resid=far, sum=gamma)):
        assert rms(**over) == BAD and "overlap" in pb.pblock_last_error(), over
    for over in (dict(dgamma=FAKE + 508), dict(dgamma=gamma), dict(dx=gamma), dict(ws=FAKE),
                 dict(dx=FAKE + (1 << 25)), dict(dgamma=FAKE + (1 << 26))):
        assert rms_back(**over) == BAD and "overlap" in pb.pblock_last_error(), over


def test_empty_matrices_and_workspaces():
    empty = [pb.MuonTensor(None, None, None, None, 0, 16, 16, 0.0, 1.0),
             pb.MuonTensor(None, None, None, None, 16, 0, 0, 0.0, 1.0)]
    cfg = pb.muon_config(1e-3)
    assert pb.pblock_muon_workspace_bytes(cfg, empty) == 0
    assert muon(tensors=empty, ws=None, nbytes=0) == OK
    # X twice, X X^T and its polynomial in planes of 2 bytes, padded to 64, at least
    ts = [pb.MuonTensor(FAKE, FAKE, FAKE, None, 100, 1000, 1000, 0.0, 1.0)]
    for products, planes in (("bf16", 1), ("f32", 2)):
        need = pb.pblock_muon_workspace_bytes(pb.muon_config(1e-3, products=products), ts)
        assert need >= planes * 2 * (2 * 128 * 1024 + 2 * 128 * 128)
    assert pb.pblock_muon_workspace_bytes(cfg, []) == 0
    assert pb.pblock_muon_workspace_bytes(cfg, ts * 17) == 0
    o = [pb.OrthoTensor(FAKE, FAKE, 1000, 100, 100, 100)]
    assert (pb.pblock_orthogonalize_workspace_bytes(o, "f32") >
            pb.pblock_orthogonalize_workspace_bytes(o, "bf16") > 0)


# ------------------------------------------------------------ the binding
def test_binding_refuses_what_tensors_say_of_themselves():
    bf, f32 = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64)
    g = torch.ones(64, dtype=torch.bfloat16)
    cfg = pb.rmsnorm_config(4, 64)
    with pytest.raises(ValueError, match="not on a GPU"):
        pb.pblock_rmsnorm_forward(cfg, bf, g, bf)
    with pytest.raises(ValueError, match="x is torch.float32"):
        pb.pblock_rmsnorm_forward(cfg, f32, g, bf)
    with pytest.raises(ValueError, match="x has 128"):
        pb.pblock_rmsnorm_forward(cfg, bf[:2], g, bf)
    with pytest.raises(ValueError, match="not contiguous"):
        pb.pblock_rmsnorm_forward(cfg, torch.zeros(64, 4, dtype=torch.bfloat16).t(), g, bf)
    with pytest.raises(ValueError, match="q8 is"):
        pb.pblock_rmsnorm_forward(cfg, bf, g, bf, q8=bf, scales=torch.zeros(4))
    with pytest.raises(ValueError, match="s is torch.float32"):
        pb.pblock_rmsnorm_backward(cfg, f32, g, torch.zeros(4), bf, bf, g, None)
    rc = pb.rope_config(32)
    with pytest.raises(ValueError, match="short of 4 tokens"):
        pb.pblock_rope_forward(rc, [pb.rope_tensor(bf[:, 8:], 64, 2)], 4)
    with pytest.raises(ValueError, match="positions is torch.float32"):
        pb.pblock_rope_forward(rc, [pb.rope_tensor(FAKE, 64, 2)], 4, positions=torch.zeros(4))
    with pytest.raises(ValueError, match="not on a GPU"):
        pb.pblock_rope_backward(rc, [pb.rope_tensor(bf, 64, 2)], 4)
    with pytest.raises(ValueError, match="scaling"):
        pb.rope_config(32, scaling="other")
    with pytest.raises(ValueError, match="dtype"):
        pb.rmsnorm_config(4, 64, dtype="fp8")
    with pytest.raises(ValueError, match="another stride"):
        pb.muon_tensor(f32, torch.zeros(4, 128)[:, :64], f32)
    with pytest.raises(ValueError, match="rows are not contiguous"):
        pb.muon_tensor(f32.t(), f32.t(), f32.t())
    with pytest.raises(ValueError, match="grad is"):
        pb.muon_tensor(f32, bf, f32)
    with pytest.raises(ValueError, match="param_copy is"):
        pb.pblock_muon_step(pb.muon_config(1e-3), [pb.muon_tensor(f32, f32, f32, f32)])
    with pytest.raises(ValueError, match="dimensions"):
        pb.ortho_tensor(torch.zeros(3), torch.zeros(3))
    with pytest.raises(ValueError, match="x is"):
        pb.pblock_orthogonalize([pb.ortho_tensor(f32, f32)], "bf16", None)


class _Tensor:
    def __init__(self, index):
        self.device = torch.device("cuda", index)

    def get_device(self):
        return self.device.index


def test_binding_refuses_two_devices_and_a_stream_of_another():
    call = pb._Call()
    call.on("a", _Tensor(1))
    call.on("b", _Tensor(1))
    with pytest.raises(ValueError, match="c is on another device"):
        call.on("c", _Tensor(0))
    assert call.ptr("d", None) is None and call.ptr("e", FAKE) == FAKE
    with pytest.raises(ValueError, match="stream is on device 0"):
        call.run(None, (), _Tensor(0))

"""The kind of products of attention with terms in its scores, on a machine without a GPU:
refusals and workspaces."""
import ctypes

import pytest

from paper_2402_15627_amd import pblock as pb


def config(products="f32", **over):
    return pb.score_attn_config(1, 40, 40, 4, 2, 64, products=products, **over)


def test_default_and_names():
    assert pb.score_attn_config(1, 4, 4, 1, 1, 64).products == pb.PB_F32
    assert config("bf16").products == pb.PB_BF16
    with pytest.raises((KeyError, ValueError)):
        config("f16")


@pytest.mark.parametrize("value", [-1, 2, 7])
def test_unknown_products_are_refused(value):
    cfg, lib = config(), pb.load_library()
    cfg.products = value
    at = 1 << 40
    ptrs = [at + (i << 32) for i in range(8)]
    assert lib.pblock_score_attn_forward(ctypes.byref(cfg), None, ptrs[0], 256, ptrs[1], ptrs[2], 128, ptrs[3],
                                         256, ptrs[4], None, 0, None) == 1
    assert "products" in pb.pblock_last_error()
    assert all(pb.pblock_score_attn_workspace_bytes(cfg, m) == 0 for m in range(3))


def test_workspaces_of_both_kinds():
    size = pb.pblock_score_attn_workspace_bytes
    for shape in ((1, 40, 40, 4, 2, 64), (1, 8192, 8192, 8, 8, 128), (1, 16, 60000, 2, 2, 64)):
        f32, bf16 = (pb.score_attn_config(*shape, products=p) for p in ("f32", "bf16"))
        assert size(f32, pb.ATTN_WS_FORWARD) == size(bf16, pb.ATTN_WS_FORWARD)
        assert size(f32, pb.ATTN_WS_BACKWARD_MIN) == size(bf16, pb.ATTN_WS_BACKWARD_MIN)
        assert size(f32, pb.ATTN_WS_BACKWARD) >= size(bf16, pb.ATTN_WS_BACKWARD)

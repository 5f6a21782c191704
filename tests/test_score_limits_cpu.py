"""Sizes of attention with terms in its scores whose launches would have 2^32 threads, on a
machine without a GPU."""
import pytest

from paper_2402_15627_amd import pblock as pb

MODES = (pb.ATTN_WS_FORWARD, pb.ATTN_WS_BACKWARD_MIN, pb.ATTN_WS_BACKWARD)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_table_of_2_to_the_26_entries_is_refused(dtype):
    """The sums of the table's gradient are a wave an entry."""
    cfg = lambda heads: pb.score_attn_config(1, 4, 4, heads, 1, 64, buckets=64, max_distance=99,  # noqa: E731
                                             dtype=dtype)
    assert all(pb.pblock_score_attn_workspace_bytes(cfg(1 << 20), m) == 0 for m in MODES)
    with pytest.raises(pb.PblockError, match="2.26 entries"):
        pb.pblock_score_attn_borders(cfg(1 << 20))
    assert len(pb.pblock_score_attn_borders(cfg((1 << 20) - 1))) == 64
    # the same heads without a table
    assert pb.pblock_score_attn_workspace_bytes(pb.score_attn_config(1, 4, 4, 1 << 20, 1, 64), MODES[1]) > 0

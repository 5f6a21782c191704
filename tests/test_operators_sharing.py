"""Memory that an output of the operators around the block shares with another tensor of
the call is refused on the host.  A call that passes every check fails for want of a GPU
(and is not made where there is one) or of workspace, so no pointer is read."""
import pytest
import torch

from paper_2402_15627_amd import pblock as pb
from tests.test_operators_cpu import BAD, FAKE, OK, SMALL, muon, rope

FAR = FAKE + (1 << 36)
NO_GPU = torch.cuda.device_count() == 0


def at(n):
    return FAKE + 2 * n


@pytest.mark.parametrize("fn", ["pblock_rope_forward", "pblock_rope_backward"])
def test_rope_refuses_an_output_over_the_positions(fn):
    """bf16, 4 tokens of 2 heads of 64, rows 512 elements apart: 128 elements are written
    in each.  Positions are 32 bytes."""
    x = [pb.RopeTensor(FAR, FAKE, 512, 512, 2)]
    for p in (FAKE, FAKE + 8, at(128) - 8, at(3 * 512), at(3 * 512 + 128) - 8, FAKE - 24, at(2 * 512) - 16):
        assert rope(fn, tensors=x, positions=p) == BAD, p
        assert "positions" in pb.pblock_last_error()
    # positions in the input, beside the output's columns or behind its rows are read only
    y = [pb.RopeTensor(FAR, FAKE, 512, 512, 2), pb.RopeTensor(FAR, at(256), 512, 512, 2)]
    assert rope(fn, tensors=y, positions=at(256 + 64)) == BAD
    for p in (FAR, at(128), at(512) - 32, FAKE - 32, at(3 * 512 + 128)) if NO_GPU else ():
        assert rope(fn, tensors=x, positions=p) != BAD, (p, pb.pblock_last_error())
    assert rope(fn, tensors=x, positions=FAKE, tokens=0) == OK

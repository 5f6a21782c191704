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


def test_rope_refuses_tensors_of_two_leading_dimensions_that_share_memory():
    """Rows that meet in one place alone, wherever the tensors begin."""
    R = pb.RopeTensor  # 2 heads of 64
    a = R(FAR, FAKE, 512, 512, 2)  # out: columns 0 .. 127 of rows of 512
    for b in (R(FAR, at(130), 512, 127 + 128, 2),  # rows at 130, 385, 640, 895: over row 1's tail
              R(FAR, at(200), 512, 313, 2),        # 200, 513, ...: over row 1
              R(FAR, at(384 + 1), 512, 640, 2),    # 385 .. 512: row 1's first element alone
              R(FAR, at(128), 512, 1280, 2), R(FAR, at(300), 512, 140, 2)):
        for pair in ([a, b], [b, a]):
            meet = any(p < q + 128 and q < p + 128 for p in range(0, 2048, 512)
                       for q in range((b.out - FAKE) // 2, (b.out - FAKE) // 2 + 4 * b.ld_out, b.ld_out))
            if meet:
                assert rope(tensors=pair) == BAD and "overlap" in pb.pblock_last_error(), (b.out, b.ld_out)
            elif NO_GPU:
                assert rope(tensors=pair) != BAD, pb.pblock_last_error()


@pytest.mark.parametrize("ld", [17, 24, 31, 40, 63, 64, 65, 96, 100, 128, 200])
def test_copies_of_another_type_are_told_apart_byte_by_byte(ld):
    """A bf16 copy between the fp32 weight's rows: its rows are half as far apart.  16
    columns, 5 rows; every place from two rows before the weight to two behind it."""
    w = FAKE
    g, m = FAKE + (1 << 30), FAKE + (2 << 30)
    for off in range(-10 * ld, 20 * ld, 2):
        t = [pb.MuonTensor(w, g, m, w + off, 5, 16, ld, 0.0, 1.0)]
        meet = any(4 * ld * i < off + 2 * ld * j + 32 and off + 2 * ld * j < 4 * ld * i + 64
                   for i in range(5) for j in range(5))
        got = muon(tensors=t, nbytes=1)
        assert got == (BAD if meet else SMALL), (off, pb.pblock_last_error())


def test_orthogonalize_with_two_leading_dimensions():
    f = lambda n: FAKE + 4 * n  # noqa: E731
    for ld_in in (16, 20, 37, 64):
        for ld_out in (16, 23, 64, 129):
            for off in range(-3 * ld_out - 20, 3 * ld_in + 20):
                x = pb.OrthoTensor(FAKE, f(off), 3, 16, ld_in, ld_out)
                meet = any(ld_in * i < off + ld_out * j + 16 and off + ld_out * j < ld_in * i + 16
                           for i in range(3) for j in range(3))
                if off == 0 and ld_in == ld_out:
                    meet = False  # in place
                got = pb.load_library().pblock_orthogonalize(1, (pb.OrthoTensor * 1)(x), pb.PB_F32, 5, 1e-7,
                                                             FAKE - (1 << 30), 1, None)
                assert got == (BAD if meet else SMALL), (ld_in, ld_out, off)

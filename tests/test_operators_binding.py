"""The binding of the operators around the block, without a GPU."""
import pytest
import torch

from paper_2402_15627_amd import pblock as pb

FAKE = 1 << 40


@pytest.mark.parametrize("fn", [pb.pblock_rope_forward, pb.pblock_rope_backward])
def test_rope_of_no_tokens_needs_no_sequence(fn):
    """Nothing is launched; positions, where given, are then an empty tensor."""
    cfg = pb.rope_config(64)
    part = [pb.rope_tensor(FAKE, 128, 2)]
    fn(cfg, part, 0, stream=0)
    fn(cfg, part, 0, seq=7, stream=0)
    fn(cfg, part, 0, positions=FAKE, stream=0)
    fn(cfg, [pb.RopeTensor(None, None, 128, 128, 2)], 0, stream=0)
    with pytest.raises(pb.PblockError, match="seq"):
        fn(cfg, part, 4, seq=0, stream=0)
    with pytest.raises(pb.PblockError, match="tokens"):
        fn(cfg, part, -1, stream=0)
    with pytest.raises(ValueError, match="positions has 3"):
        fn(cfg, part, 0, positions=torch.zeros(3, dtype=torch.int64), stream=0)

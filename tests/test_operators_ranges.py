"""Configurations whose derived values leave their type's range are refused."""
import pytest

from paper_2402_15627_amd import pblock as pb
from tests.test_operators_cpu import BAD, OK, rope


@pytest.mark.parametrize("over", [
    dict(magnitude=1e-50),                                    # 0 in fp32
    dict(scaling="linear", factor=1e-310),                    # frequencies past 1e308
    dict(scaling="by_parts", factor=1e-310, low_turns=1e6, high_turns=2e6),
    dict(base=5e-324, scaling="linear", factor=1e-30),
], ids=str)
def test_rope_refuses_what_leaves_its_range(over):
    over = dict(over)
    scaling = over.pop("scaling", "plain")
    assert rope(scaling=scaling, tokens=0, **over) == BAD
    assert pb.pblock_last_error() != ""


def test_rope_takes_what_stays_in_range():
    for over in (dict(magnitude=1.2e-38), dict(magnitude=3e38), dict(base=1e300), dict(base=1e-300)):
        assert rope(scaling="plain", tokens=0, **over) == OK
    assert rope(scaling="linear", tokens=0, factor=1e-300) == OK

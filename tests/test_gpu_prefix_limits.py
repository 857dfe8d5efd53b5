"""Shared prefixes on the GPU: the ends of what the arguments may be."""
import pytest

from paper_2510_24824_b200 import binding as B
from prefix_util import Problem

pytestmark = pytest.mark.gpu


# ---- the ends of 32 bits ------------------------------------------------------------------------------------------------
def test_the_lowest_lengths_are_clamped_as_any_below_zero():
    low = -2 ** 31
    for more in (dict(L=3, w=6), dict(q_len=4), dict(L=2, w=6, q_len=2)):
        p = Problem(41, [4] * 6, [300], [0, 5], lens=[304, low, low + 1, 302, -5, low + 2], **more)
        assert p.run() == B.PLT_DEV_SEQ_LEN_CLAMPED
        p.lens = [304, 0, 0, 302, 0, 0]
        p.hold()



def test_offsets_that_no_length_reaches():
    """The last loop never has a token: zero rows, although length - offset - newer tokens lies below the lowest whole number."""
    for q_len in (1, 3):
        p = Problem(43, [4] * 5, [300], [0, 4], lens=[304, 0, 1, 302, 4], L=2, w=6, q_len=q_len, offsets=[0, 2 ** 31 - 1])
        assert p.run() == 0
        assert (p.out[:, 1] == 0).all()
        p.hold()

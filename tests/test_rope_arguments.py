"""CPU checks of what the binding and the runner make of a rotation's arguments (no compute call is made)."""
import pytest

from paper_2510_24824_b200 import binding as B


def test_lists_that_are_too_short_are_refused_before_c_reads_them():
    args = ("bf16", 4, 2, 8, 4, 128, 512, 16)
    for more in (dict(inv_freq=[0.5] * 63), dict(inv_freq=[0.5] * 15, rotary_dim=32), dict(inv_freq=[]), dict(loop_offset=[0]), dict(loop_offset=[])):
        with pytest.raises(ValueError):
            B.make_rope_config(*args, **more)
    assert B.plt_rope_frequencies(B.make_rope_config(*args, inv_freq=[0.5] * 64, loop_offset=[0, 3]))[63] == 0.5
    assert B.plt_rope_frequencies(B.make_rope_config(*args, inv_freq=[0.25] * 16, rotary_dim=32))[15] == 0.25
    with pytest.raises(ValueError):
        B.make_prefix_config("bf16", 4, 2, 8, 4, 128, 512, 16, 100, loop_offset=[0])

"""CPU checks of the workspace that shared prefixes ask for (no compute call is made)."""
import pytest
import torch

from paper_2510_24824_b200 import binding as B

ONE = dict(dtype="bf16", max_batch=1, L=1, Hq=32, Hkv=8, d=128, max_seq_len=512, w=0, max_prefix_len=1000)


def _bytes(**kw):
    return B.plt_prefix_attn_workspace_bytes(B.make_prefix_config(**dict(ONE, **kw)))


def test_groups_that_cannot_have_a_sequence_take_no_partials():
    """One sequence fills one unit a head and begins one group: 8 * (1 + 1) units and a block's for 148 multiprocessors, of 256 rows of
    128 + 2 fp32 numbers each; further groups have five words in the plan and nothing else."""
    slot = 256 * (128 + 2) * 4
    few, many = _bytes(max_groups=1), _bytes(max_groups=1024)
    assert (8 * 2 + 148) * slot <= few < (8 * 2 + 148) * slot + (8 << 20)          # and the decode step's own
    assert many - few <= 5 * 4 * 1023 + 256
    assert _bytes(max_batch=4, max_groups=4) - _bytes(max_batch=4, max_groups=2) >= 8 * 2 * slot


def test_a_long_prefix_of_one_sequence_is_not_refused_for_its_groups():
    """2^24 tokens are 131072 tiles; 64 units of them fit the plan, however many groups may be named."""
    cfg = B.make_prefix_config(**dict(ONE, Hkv=32, max_groups=1024, max_prefix_len=1 << 24))
    assert B.plt_prefix_attn_workspace_bytes(cfg) > 0
    if not torch.cuda.is_available():
        with pytest.raises(B.PltError) as e:
            B.plt_prefix_attn_create(cfg)
        assert e.value.status == B.PLT_ERR_CUDA            # for want of a device, not of room in the plan


def test_what_create_refuses_has_no_size():
    for call in (B.plt_prefix_attn_workspace_bytes, B.plt_prefix_attn_create):
        with pytest.raises(B.PltError) as e:
            call(B.make_prefix_config(**dict(ONE, max_batch=4096, Hq=1024, Hkv=32, max_prefix_len=1 << 24)))
        assert e.value.status == B.PLT_ERR_UNSUPPORTED

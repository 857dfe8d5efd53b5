"""CPU checks of what cache eviction takes and refuses by size (no compute call is made)."""
import pytest

from paper_2510_24824_b200 import binding as B


def config(**kw):
    return B.make_evict_config(**dict(dict(dtype="bf16", max_batch=4096, L=1, Hq=8, Hkv=8, d=128, max_seq_len=64), **kw))


@pytest.mark.parametrize("kw", [dict(Hq=65536, Hkv=65536, d=64), dict(Hq=65536, Hkv=65536), dict(dtype="f32", Hq=32768, Hkv=32768),
                                dict(Hq=65536, Hkv=65536, d=64, heads_per_group=65536, max_seq_len=16)])
def test_more_blocks_than_a_launch_can_count_are_refused(kw):
    """Compaction takes a block for each sequence, head, cache and 64 bytes of a row."""
    for call in (B.plt_cache_evict_workspace_bytes, B.plt_cache_evict_create):
        with pytest.raises(B.PltError) as e:
            call(config(**kw))
        assert e.value.status == B.PLT_ERR_UNSUPPORTED and e.value.message


@pytest.mark.parametrize("kw", [dict(), dict(Hq=1024, Hkv=1024), dict(Hq=8192, Hkv=8192, max_batch=512), dict(dtype="f32", Hq=128, Hkv=128)])
def test_wide_layouts_below_that_are_taken(kw):
    assert B.plt_cache_evict_workspace_bytes(config(**kw)) > 0

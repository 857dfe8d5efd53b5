"""CPU checks of the cache-eviction boundary: exports, struct layout, refusals (no compute call is made), oracle pins."""
import ctypes
import re
import subprocess
from pathlib import Path

import numpy as np
import pytest

from oracle import plt_cache_evict as oracle_evict
from paper_2510_24824_b200 import binding as B

ROOT = Path(__file__).resolve().parents[1]


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "plt_cache_evict.h").read_text(), flags=re.S)
    names = sorted(set(re.findall(r"\b(plt_cache_evict_(?!t\b)\w+)\s*\(", text)))
    assert names == sorted(B.EVICT_EXPORTS)
    for n in names:
        assert hasattr(B.load_library(), n), f"{n} is declared in the header but not exported"


def test_struct_layout_matches_c(tmp_path):
    structs = [("plt_cache_evict_config", B.EvictConfig), ("plt_cache_evict_weights_args", B.EvictWeightsArgs),
               ("plt_cache_evict_select_args", B.EvictSelectArgs), ("plt_cache_evict_compact_args", B.EvictCompactArgs)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{ROOT}/include/plt_cache_evict.h"', 'int main(void){']
    for cname, st in structs:
        lines += [f'printf("%zu\\n", sizeof({cname}));']
        lines += [f'printf("%zu\\n", offsetof({cname}, {f}));' for f, _ in st._fields_]
    (tmp_path / "layout.c").write_text("\n".join(lines + ['return 0;}']))
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-o", str(tmp_path / "layout"), str(tmp_path / "layout.c")], check=True)
    vals = [int(x) for x in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for _, st in structs:
        want += [ctypes.sizeof(st)] + [getattr(st, f).offset for f, _ in st._fields_]
    assert vals == want


OK = dict(dtype="bf16", max_batch=4, L=2, Hq=8, Hkv=4, d=128, max_seq_len=512)


@pytest.mark.parametrize("change,code", [
    (dict(d=96), B.PLT_ERR_UNSUPPORTED), (dict(Hq=7), B.PLT_ERR_INVALID_ARG), (dict(L=9), B.PLT_ERR_UNSUPPORTED),
    (dict(Hq=256), B.PLT_ERR_UNSUPPORTED),
    (dict(Hq=128, maps=2), B.PLT_ERR_UNSUPPORTED), (dict(q_len=33), B.PLT_ERR_UNSUPPORTED), (dict(q_len=-1), B.PLT_ERR_INVALID_ARG),
    (dict(page_size=24), B.PLT_ERR_UNSUPPORTED), (dict(page_size=-16), B.PLT_ERR_INVALID_ARG), (dict(maps=3), B.PLT_ERR_INVALID_ARG),
    (dict(heads_per_group=3), B.PLT_ERR_INVALID_ARG), (dict(heads_per_group=-1), B.PLT_ERR_INVALID_ARG),
    (dict(kv_dtype="e4m3", d=64), B.PLT_ERR_UNSUPPORTED), (dict(kv_dtype="e4m3", dtype="f32"), B.PLT_ERR_UNSUPPORTED),
    (dict(kv_dtype=9), B.PLT_ERR_INVALID_ARG), (dict(dtype=9), B.PLT_ERR_INVALID_ARG), (dict(max_batch=0), B.PLT_ERR_INVALID_ARG),
    (dict(max_batch=4097), B.PLT_ERR_UNSUPPORTED), (dict(max_seq_len=(1 << 24) + 1), B.PLT_ERR_UNSUPPORTED),
    (dict(loop_offset=[0, -1]), B.PLT_ERR_INVALID_ARG),
])
def test_refusals(change, code):
    for call in (B.plt_cache_evict_workspace_bytes, B.plt_cache_evict_create):
        with pytest.raises(B.PltError) as e:
            call(B.make_evict_config(**dict(OK, **change)))
        assert e.value.status == code and e.value.message, (change, e.value)


def test_struct_sizes_and_nulls_are_checked():
    cfg = B.make_evict_config(**OK)
    assert B.plt_cache_evict_workspace_bytes(cfg) > 0
    cfg.struct_size = 8
    with pytest.raises(B.PltError) as e:
        B.plt_cache_evict_workspace_bytes(cfg)
    assert e.value.status == B.PLT_ERR_INVALID_ARG
    lib = B.load_library()
    assert lib.plt_cache_evict_create(None, ctypes.byref(ctypes.c_void_p())) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_cache_evict_create(ctypes.byref(B.make_evict_config(**OK)), None) == B.PLT_ERR_INVALID_ARG
    for name in ("weights", "select", "compact"):
        assert getattr(lib, f"plt_cache_evict_{name}")(None, None, None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_cache_evict_check(None, None, None) == B.PLT_ERR_INVALID_ARG
    B.plt_cache_evict_destroy(None)


def test_workspace_is_bounded():
    """The scores of a long batch do not grow the workspace beyond what one sequence or a quarter of a GB needs."""
    small = B.plt_cache_evict_workspace_bytes(B.make_evict_config(**OK))
    big = B.plt_cache_evict_workspace_bytes(B.make_evict_config(**dict(OK, max_batch=256, max_seq_len=32768)))
    assert small < 2 << 20 and 200 << 20 < big < 300 << 20


def test_create_without_a_device_fails_loudly():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    with pytest.raises(B.PltError) as e:
        B.plt_cache_evict_create(B.make_evict_config(**OK))
    assert e.value.status == B.PLT_ERR_CUDA


# ---- pins of the oracle -------------------------------------------------------------------------------------------
def test_weights_of_a_step_sum_to_its_rows():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 2, 3, 4, 8)), rng.standard_normal((2, 9, 2, 8))
    out, _ = oracle_evict.weights(q, k, [9, 2], np.full((2, 2, 9), 7.0), decay=0.0)
    # sequence 0: 2 loops x 3 tokens x 2 heads each; sequence 1 (2 tokens): loop 1 has rows that see 2, 1, 0 keys, loop 2 1, 0, 0
    assert np.allclose(out[0].sum(-1), 12.0) and np.allclose(out[1, :, :2].sum(-1), 6.0)
    assert (out[1, :, 2:] == 7.0).all()


def test_weights_written_out_for_one_key():
    q, k = np.zeros((1, 1, 1, 1, 2)), np.ones((1, 4, 1, 2))
    out, _ = oracle_evict.weights(q, k, [4], np.ones((1, 1, 4)), decay=0.5)
    assert np.allclose(out, 0.75)
    gate = np.zeros((1, 1, 1, 1))
    out, _ = oracle_evict.weights(np.zeros((1, 2, 1, 1, 2)), k, [4], np.zeros((1, 1, 4)), gate=gate)
    assert np.allclose(out[0, 0], [0.25 + 0.5 / 3] * 3 + [0.25])


def test_select_by_hand():
    w = np.array([[[5.0, 1.0, 1.0, np.nan, 9.0, 1.0, -0.0, 0.0]]])
    keep, new = oracle_evict.select(w, [8], 5, 1, 1)
    assert keep.tolist() == [[[0, 1, 2, 4, 7]]] and new.tolist() == [5]
    keep, _ = oracle_evict.select(w, [8], 7, 0, 0)
    assert keep.tolist() == [[[0, 1, 2, 4, 5, 6, 7]]]
    keep, new = oracle_evict.select(w, [3], 5, 1, 1)
    assert keep.tolist() == [[[0, 1, 2, -1, -1]]] and new.tolist() == [3]

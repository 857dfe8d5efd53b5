"""CPU checks of the differential-attention boundary: exports, struct layout, refusals (no compute call is made)."""
import ctypes
import re
import subprocess
from pathlib import Path

import pytest

from paper_2510_24824_b200 import binding as B

ROOT = Path(__file__).resolve().parents[1]


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "plt_diff_attn.h").read_text(), flags=re.S)
    names = sorted(set(re.findall(r"\b(plt_diff_(?:seq_)?attn_\w+)\s*\(", text)))
    assert names == sorted(B.DIFF_EXPORTS)
    for n in names:
        assert hasattr(B.load_library(), n), f"{n} is declared in the header but not exported"


def test_struct_layout_matches_c(tmp_path):
    structs = [("plt_diff_attn_config", B.DiffConfig), ("plt_diff_seq_attn_config", B.DiffSeqConfig), ("plt_diff_weights", B.DiffWeights)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{ROOT}/include/plt_diff_attn.h"', 'int main(void){']
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


OK = dict(dtype="bf16", max_batch=4, L=2, Hq=8, Hkv=2, d=128, max_seq_len=512, w=64)


@pytest.mark.parametrize("change,code", [
    (dict(d=96), B.PLT_ERR_UNSUPPORTED), (dict(Hq=7), B.PLT_ERR_INVALID_ARG), (dict(Hq=0), B.PLT_ERR_INVALID_ARG),
    (dict(L=9), B.PLT_ERR_UNSUPPORTED), (dict(Hq=64, Hkv=2), B.PLT_ERR_UNSUPPORTED), (dict(Hq=32, Hkv=2, q_len=2), B.PLT_ERR_UNSUPPORTED),
    (dict(w=0), B.PLT_ERR_INVALID_ARG), (dict(page_size=24), B.PLT_ERR_UNSUPPORTED), (dict(lambda_init=float("nan")), B.PLT_ERR_INVALID_ARG),
    (dict(norm_eps=0.0), B.PLT_ERR_INVALID_ARG), (dict(norm_eps=float("inf")), B.PLT_ERR_INVALID_ARG),
    (dict(kv_dtype="e4m3", d=64), B.PLT_ERR_UNSUPPORTED), (dict(dtype="f32", q_len=2), B.PLT_ERR_UNSUPPORTED),
    (dict(loop_offset=[0, -1]), B.PLT_ERR_INVALID_ARG), (dict(max_batch=0), B.PLT_ERR_INVALID_ARG), (dict(dtype=7), B.PLT_ERR_INVALID_ARG),
])
def test_step_refusals(change, code):
    for call in (B.plt_diff_attn_workspace_bytes, B.plt_diff_attn_create):
        with pytest.raises(B.PltError) as e:
            call(B.make_diff_config(**dict(OK, **change)))
        assert e.value.status == code and e.value.message, (change, e.value)


@pytest.mark.parametrize("change,code", [
    (dict(d=64), B.PLT_ERR_UNSUPPORTED), (dict(Hq=7), B.PLT_ERR_INVALID_ARG), (dict(L=9), B.PLT_ERR_UNSUPPORTED), (dict(w=0), B.PLT_ERR_INVALID_ARG),
    (dict(lambda_init=float("inf")), B.PLT_ERR_INVALID_ARG), (dict(norm_eps=-1.0), B.PLT_ERR_INVALID_ARG),
    (dict(max_batch=1 << 20, max_seq_len=1 << 20), B.PLT_ERR_UNSUPPORTED),
])
def test_prompt_refusals(change, code):
    with pytest.raises(B.PltError) as e:
        B.plt_diff_seq_attn_create(B.make_diff_seq_config(**dict({k: v for k, v in OK.items() if k != "dtype"}, **change)))
    assert e.value.status == code and e.value.message, (change, e.value)


def test_struct_sizes_and_nulls_are_checked():
    cfg = B.make_diff_config(**OK)
    assert B.plt_diff_attn_workspace_bytes(cfg) > 0
    cfg.struct_size = 8
    with pytest.raises(B.PltError) as e:
        B.plt_diff_attn_workspace_bytes(cfg)
    assert e.value.status == B.PLT_ERR_INVALID_ARG
    lib = B.load_library()
    assert lib.plt_diff_attn_create(None, ctypes.byref(ctypes.c_void_p())) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_diff_attn_create(ctypes.byref(B.make_diff_config(**OK)), None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_diff_attn_run(None, None, None, None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_diff_attn_step(None, None, None, None, None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_diff_attn_check(None, None, None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_diff_seq_attn_run(None, None, None, None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_diff_seq_attn_create(None, ctypes.byref(ctypes.c_void_p())) == B.PLT_ERR_INVALID_ARG
    B.plt_diff_attn_destroy(None)
    B.plt_diff_seq_attn_destroy(None)


def test_create_without_a_device_fails_loudly():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    for call in (lambda: B.plt_diff_attn_create(B.make_diff_config(**OK)),
                 lambda: B.plt_diff_seq_attn_create(B.make_diff_seq_config(**{k: v for k, v in OK.items() if k != "dtype"}))):
        with pytest.raises(B.PltError) as e:
            call()
        assert e.value.status == B.PLT_ERR_CUDA

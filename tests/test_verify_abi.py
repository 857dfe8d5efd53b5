"""CPU checks of draft verification's boundary: exports, struct layout, refusals (no compute call is made), oracle pins."""
import ctypes
import re
import subprocess
from pathlib import Path

import numpy as np
import pytest

from oracle import plt_draft_verify as oracle_verify
from paper_2510_24824_b200 import binding as B

ROOT = Path(__file__).resolve().parents[1]


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "plt_draft_verify.h").read_text(), flags=re.S)
    names = sorted(set(re.findall(r"\b(plt_draft_verify_(?!t\b)\w+)\s*\(", text)))
    assert names == sorted(B.VERIFY_EXPORTS)
    for n in names:
        assert hasattr(B.load_library(), n), f"{n} is declared in the header but not exported"


def test_struct_layout_matches_c(tmp_path):
    structs = [("plt_draft_verify_config", B.VerifyConfig), ("plt_draft_verify_args", B.VerifyArgs)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{ROOT}/include/plt_draft_verify.h"', 'int main(void){']
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


OK = dict(dtype="f32", max_batch=4, max_drafts=3, vocab=1000)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=7), B.PLT_ERR_INVALID_ARG), (dict(max_batch=0), B.PLT_ERR_INVALID_ARG), (dict(max_batch=4097), B.PLT_ERR_UNSUPPORTED),
    (dict(max_drafts=0), B.PLT_ERR_INVALID_ARG), (dict(max_drafts=65), B.PLT_ERR_UNSUPPORTED), (dict(vocab=0), B.PLT_ERR_INVALID_ARG),
    (dict(vocab=(1 << 24) + 1), B.PLT_ERR_UNSUPPORTED),
])
def test_refusals(change, code):
    for call in (B.plt_draft_verify_workspace_bytes, B.plt_draft_verify_create):
        with pytest.raises(B.PltError) as e:
            call(B.make_verify_config(**dict(OK, **change)))
        assert e.value.status == code and e.value.message, (change, e.value)


def test_struct_sizes_and_nulls_are_checked():
    cfg = B.make_verify_config(**OK)
    assert B.plt_draft_verify_workspace_bytes(cfg) > 0
    cfg.struct_size = 8
    with pytest.raises(B.PltError) as e:
        B.plt_draft_verify_workspace_bytes(cfg)
    assert e.value.status == B.PLT_ERR_INVALID_ARG
    lib = B.load_library()
    assert lib.plt_draft_verify_create(None, ctypes.byref(ctypes.c_void_p())) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_draft_verify_create(ctypes.byref(B.make_verify_config(**OK)), None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_draft_verify_run(None, None, None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_draft_verify_check(None, None, None) == B.PLT_ERR_INVALID_ARG
    B.plt_draft_verify_destroy(None)


def test_create_without_a_device_fails_loudly():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    with pytest.raises(B.PltError) as e:
        B.plt_draft_verify_create(B.make_verify_config(**OK))
    assert e.value.status == B.PLT_ERR_CUDA


# ---- pins of the oracle -------------------------------------------------------------------------------------------
def test_oracle_by_hand():
    p = np.array([[[0.5, 0.25, 0.25, 0.0], [0.0, 0.0, 0.5, 0.5], [0.25, 0.25, 0.25, 0.25]]])
    q = np.array([[[0.25, 0.5, 0.25, 0.0], [0.5, 0.0, 0.5, 0.0]]])
    # draft 0 (token 1): 0.6 * 0.5 >= 0.25: refused; what is left of p over q is token 0 alone
    t, n, _ = oracle_verify.verify(p, q, np.array([[1, 2]]), None, np.array([[0.6, 0.0]]), np.array([0.9]))
    assert t.tolist() == [[0, -1, -1]] and n.tolist() == [0]
    # 0.4 * 0.5 < 0.25 passes; draft 1 (token 0) has no probability: refused; left over: token 3
    t, n, _ = oracle_verify.verify(p, q, np.array([[1, 0]]), None, np.array([[0.4, 0.0]]), np.array([0.0]))
    assert t.tolist() == [[1, 3, -1]] and n.tolist() == [1]
    # both pass: the third row decides, its third quarter
    t, n, _ = oracle_verify.verify(p, q, np.array([[1, 2]]), None, np.array([[0.4, 0.9]]), np.array([0.5]))
    assert t.tolist() == [[1, 2, 2]] and n.tolist() == [2]
    # one draft only: the second row decides
    t, n, _ = oracle_verify.verify(p, q, np.array([[1, 2]]), [1], np.array([[0.4, 0.9]]), np.array([0.49]))
    assert t.tolist() == [[1, 2, -1]] and n.tolist() == [1]
    # a certain draft: refused with probability 1 - p, and what is left is p without it
    t, n, _ = oracle_verify.verify(p, None, np.array([[0, 2]]), None, np.array([[0.5, 0.0]]), np.array([0.6]))
    assert t.tolist() == [[2, -1, -1]] and n.tolist() == [0]


def test_oracle_keeps_the_targets_distribution():
    """Over a grid of numbers the first token comes out with the target's probabilities."""
    p, q = np.array([0.5, 0.3, 0.2]), np.array([0.2, 0.3, 0.5])
    m = 60
    grid = (np.arange(m) + 0.5) / m
    count = np.zeros(3)
    for x in range(3):
        for u in grid:
            r = grid
            t, _, _ = oracle_verify.verify(np.tile(p, (m, 2, 1)), np.tile(q, (m, 1, 1)), np.full((m, 1), x), None, np.full((m, 1), u), r)
            count += q[x] * np.bincount(t[:, 0], minlength=3)
    # a step of a grid is the most that a border can move
    assert np.abs(count / m ** 2 - p).max() <= 2.0 / m

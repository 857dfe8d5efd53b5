"""CPU checks of the rotation's boundary: exports, struct layout, refusals (no compute call is made), frequencies, oracle pins."""
import ctypes
import re
import subprocess
from pathlib import Path

import numpy as np
import pytest

from oracle import plt_rope as oracle_rope
from paper_2510_24824_b200 import binding as B

ROOT = Path(__file__).resolve().parents[1]


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "plt_rope.h").read_text(), flags=re.S)
    names = sorted(set(re.findall(r"\b(plt_rope_(?!t\b)\w+)\s*\(", text)))
    assert names == sorted(B.ROPE_EXPORTS)
    for n in names:
        assert hasattr(B.load_library(), n), f"{n} is declared in the header but not exported"


def test_struct_layout_matches_c(tmp_path):
    structs = [("plt_rope_config", B.RopeConfig), ("plt_rope_step_args", B.RopeStepArgs), ("plt_rope_seq_args", B.RopeSeqArgs)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{ROOT}/include/plt_rope.h"', 'int main(void){']
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


OK = dict(dtype="bf16", max_batch=4, L=2, Hq=8, Hkv=4, d=128, max_seq_len=512, w=64)


@pytest.mark.parametrize("change,code", [
    (dict(d=96), B.PLT_ERR_UNSUPPORTED), (dict(Hq=7), B.PLT_ERR_INVALID_ARG), (dict(L=9), B.PLT_ERR_UNSUPPORTED),
    (dict(w=0), B.PLT_ERR_INVALID_ARG), (dict(q_len=2), B.PLT_ERR_UNSUPPORTED), (dict(q_len=65, L=1), B.PLT_ERR_UNSUPPORTED),
    (dict(q_len=-1), B.PLT_ERR_INVALID_ARG), (dict(page_size=24), B.PLT_ERR_UNSUPPORTED), (dict(page_size=-16), B.PLT_ERR_INVALID_ARG),
    (dict(kv_dtype="e4m3", d=64), B.PLT_ERR_UNSUPPORTED), (dict(kv_dtype="e4m3", dtype="f32"), B.PLT_ERR_UNSUPPORTED),
    (dict(kv_dtype=9), B.PLT_ERR_INVALID_ARG), (dict(dtype=9), B.PLT_ERR_INVALID_ARG), (dict(max_batch=0), B.PLT_ERR_INVALID_ARG),
    (dict(max_batch=4097), B.PLT_ERR_UNSUPPORTED), (dict(loop_offset=[0, -1]), B.PLT_ERR_INVALID_ARG), (dict(Hq=2048), B.PLT_ERR_UNSUPPORTED),
    (dict(rotary_dim=24), B.PLT_ERR_UNSUPPORTED), (dict(rotary_dim=144), B.PLT_ERR_INVALID_ARG), (dict(rotary_dim=-16), B.PLT_ERR_INVALID_ARG),
    (dict(layout=2), B.PLT_ERR_INVALID_ARG), (dict(scaling=5), B.PLT_ERR_INVALID_ARG), (dict(scaling=-1), B.PLT_ERR_INVALID_ARG),
    (dict(norm_eps=0.0), B.PLT_ERR_INVALID_ARG), (dict(norm_eps=float("nan")), B.PLT_ERR_INVALID_ARG),
    (dict(attn_factor=float("inf")), B.PLT_ERR_INVALID_ARG), (dict(theta=1.0), B.PLT_ERR_INVALID_ARG),
    (dict(theta=float("nan")), B.PLT_ERR_INVALID_ARG), (dict(scaling="linear", factor=0.0), B.PLT_ERR_INVALID_ARG),
    (dict(scaling="wavelength", factor=2.0, low=4.0, high=4.0, original_len=100), B.PLT_ERR_INVALID_ARG),
    (dict(scaling="ramp", factor=2.0, low=0.0, high=4.0, original_len=100), B.PLT_ERR_INVALID_ARG),
    (dict(scaling="ramp", factor=2.0, low=1.0, high=4.0, original_len=0), B.PLT_ERR_INVALID_ARG),
    (dict(inv_freq=[float("inf")] * 64), B.PLT_ERR_INVALID_ARG),
])
def test_refusals(change, code):
    for call in (B.plt_rope_frequencies, B.plt_rope_create):
        with pytest.raises(B.PltError) as e:
            call(B.make_rope_config(**dict(OK, **change)))
        assert e.value.status == code and e.value.message, (change, e.value)


def test_struct_sizes_and_nulls_are_checked():
    cfg = B.make_rope_config(**OK)
    cfg.struct_size = 8
    with pytest.raises(B.PltError) as e:
        B.plt_rope_frequencies(cfg)
    assert e.value.status == B.PLT_ERR_INVALID_ARG
    lib = B.load_library()
    assert lib.plt_rope_create(None, ctypes.byref(ctypes.c_void_p())) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_rope_create(ctypes.byref(B.make_rope_config(**OK)), None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_rope_frequencies(ctypes.byref(B.make_rope_config(**OK)), None) == B.PLT_ERR_INVALID_ARG
    for name in ("step", "seq"):
        assert getattr(lib, f"plt_rope_{name}")(None, None, None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_rope_check(None, None, None) == B.PLT_ERR_INVALID_ARG
    B.plt_rope_destroy(None)


def test_create_without_a_device_fails_loudly():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    with pytest.raises(B.PltError) as e:
        B.plt_rope_create(B.make_rope_config(**OK))
    assert e.value.status == B.PLT_ERR_CUDA


@pytest.mark.parametrize("rd", [16, 48, 128])
@pytest.mark.parametrize("scaling,more", [
    ("none", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
    ("wavelength", dict(factor=8.0, low=1.0, high=4.0, original_len=8192)), ("wavelength", dict(factor=32.0, low=0.5, high=8.0, original_len=1)),
    ("ramp", dict(factor=16.0, low=1.0, high=32.0, original_len=4096)), ("ramp", dict(factor=40.0, low=1.0, high=1.5, original_len=3)),
])
def test_frequencies_are_the_definitions(rd, scaling, more):
    got = B.plt_rope_frequencies(B.make_rope_config(**dict(OK, rotary_dim=rd, theta=500000.0, scaling=scaling, **more)))
    # powers and products in 64 bits: a few roundings, and an exponent of up to ln(theta) * 1.0 that carries its own
    np.testing.assert_allclose(got, oracle_rope.frequencies(rd, 500000.0, scaling, **more), rtol=64 * 2.0 ** -53, atol=0)


def test_given_frequencies_pass_through():
    f = [0.5 ** i * (-1) ** i for i in range(8)]
    assert B.plt_rope_frequencies(B.make_rope_config(**dict(OK, rotary_dim=16, inv_freq=f, theta=0.0))) == f


# ---- pins of the oracle -------------------------------------------------------------------------------------------
def test_products_depend_on_distance_alone():
    rng = np.random.default_rng(0)
    q, k, f = rng.standard_normal(64), rng.standard_normal(64), oracle_rope.frequencies(32, 10000.0)
    for layout in ("half", "interleaved"):
        a = [oracle_rope.turn(q, p + 7, f, layout=layout) @ oracle_rope.turn(k, p, f, layout=layout) for p in (0, 3, 1000)]
        assert np.allclose(a, a[0], rtol=1e-12)


def test_turns_by_hand():
    f = np.array([np.pi / 2, np.pi])
    assert np.allclose(oracle_rope.turn([1.0, 2, 3, 4, 5], 1, f), [-3, -2, 1, -4, 5])
    assert np.allclose(oracle_rope.turn([1.0, 2, 3, 4, 5], 1, f, layout="interleaved"), [-2, 1, -3, -4, 5])
    assert np.allclose(oracle_rope.turn([3.0, 4, 0, 0], 0, f, gain=[1, 2, 1, 1], eps=0.0), [1.2, 3.2, 0, 0])
    assert np.allclose(oracle_rope.turn([1.0, 0, 0, 0, 5], 0, f, factor=2.0), [2, 0, 0, 0, 5])

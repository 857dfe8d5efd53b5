"""CPU checks of shared prefixes' boundary: exports, struct layout, refusals (no compute call is made), oracle pins."""
import ctypes
import re
import subprocess
from pathlib import Path

import pytest
import torch

from oracle import plt_prefix_attn as oracle_prefix
from paper_2510_24824_b200 import binding as B

ROOT = Path(__file__).resolve().parents[1]


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "plt_prefix_attn.h").read_text(), flags=re.S)
    names = sorted(set(re.findall(r"\b(plt_prefix_attn_(?!t\b)\w+)\s*\(", text)))
    assert names == sorted(B.PREFIX_EXPORTS)
    for n in names:
        assert hasattr(B.load_library(), n), f"{n} is declared in the header but not exported"


def test_struct_layout_matches_c(tmp_path):
    structs = [("plt_prefix_attn_config", B.PrefixConfig), ("plt_prefix_args", B.PrefixArgs)]
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{ROOT}/include/plt_prefix_attn.h"', 'int main(void){']
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


OK = dict(dtype="bf16", max_batch=4, L=2, Hq=8, Hkv=4, d=128, max_seq_len=512, w=64, max_prefix_len=1000, max_groups=2)


@pytest.mark.parametrize("change,code", [
    (dict(d=96), B.PLT_ERR_UNSUPPORTED), (dict(Hq=7), B.PLT_ERR_INVALID_ARG), (dict(L=9), B.PLT_ERR_UNSUPPORTED), (dict(Hq=256), B.PLT_ERR_UNSUPPORTED),
    (dict(w=0), B.PLT_ERR_INVALID_ARG), (dict(dtype="f32"), B.PLT_ERR_UNSUPPORTED), (dict(dtype=9), B.PLT_ERR_INVALID_ARG),
    (dict(kv_dtype="e4m3", d=64), B.PLT_ERR_UNSUPPORTED), (dict(kv_dtype=9), B.PLT_ERR_INVALID_ARG), (dict(max_batch=0), B.PLT_ERR_INVALID_ARG),
    (dict(max_batch=4097), B.PLT_ERR_UNSUPPORTED), (dict(page_size=24), B.PLT_ERR_UNSUPPORTED), (dict(q_len=17), B.PLT_ERR_UNSUPPORTED), (dict(loop_offset=[0, -1]), B.PLT_ERR_INVALID_ARG), (dict(max_prefix_len=0), B.PLT_ERR_INVALID_ARG),
    (dict(max_prefix_len=(1 << 24) + 1), B.PLT_ERR_UNSUPPORTED), (dict(max_groups=0), B.PLT_ERR_INVALID_ARG), (dict(max_groups=1025), B.PLT_ERR_UNSUPPORTED),
    (dict(max_seq_len=0x7fffffff), B.PLT_ERR_UNSUPPORTED),
])
def test_refusals(change, code):
    for call in (B.plt_prefix_attn_workspace_bytes, B.plt_prefix_attn_create):
        with pytest.raises(B.PltError) as e:
            call(B.make_prefix_config(**dict(OK, **change)))
        assert e.value.status == code and e.value.message, (change, e.value)


def test_struct_sizes_and_nulls_are_checked():
    cfg = B.make_prefix_config(**OK)
    assert B.plt_prefix_attn_workspace_bytes(cfg) > 0
    cfg.struct_size = 8
    with pytest.raises(B.PltError) as e:
        B.plt_prefix_attn_workspace_bytes(cfg)
    assert e.value.status == B.PLT_ERR_INVALID_ARG
    lib = B.load_library()
    assert lib.plt_prefix_attn_create(None, ctypes.byref(ctypes.c_void_p())) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_prefix_attn_create(ctypes.byref(B.make_prefix_config(**OK)), None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_prefix_attn_run(None, None, None, None) == B.PLT_ERR_INVALID_ARG
    assert lib.plt_prefix_attn_check(None, None, None) == B.PLT_ERR_INVALID_ARG
    B.plt_prefix_attn_destroy(None)


def test_plans_that_do_not_fit_are_refused():
    with pytest.raises(B.PltError) as e:
        B.plt_prefix_attn_create(B.make_prefix_config(**dict(OK, max_batch=4096, Hq=1024, Hkv=32, max_prefix_len=1 << 24)))
    assert e.value.status == B.PLT_ERR_UNSUPPORTED


def test_create_without_a_device_fails_loudly():
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    with pytest.raises(B.PltError) as e:
        B.plt_prefix_attn_create(B.make_prefix_config(**OK))
    assert e.value.status == B.PLT_ERR_CUDA


# ---- pins of the oracle -------------------------------------------------------------------------------------------
def test_oracle_is_the_plain_step_on_joined_caches():
    """With the prefix copied in front of every sequence's own keys it is the decode step's oracle."""
    import numpy as np

    import oracle
    from paper_2510_24824_b200.inputs import make_problem, shrunk_workload
    p = make_problem(shrunk_workload(0))
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x)).double()  # noqa: E731
    k, v, P = f(p.k_cache), f(p.v_cache), 5
    lens = [int(n) for n in p.seq_lens]
    k[:, :P], v[:, :P] = k[:1, :P], v[:1, :P]
    q = p.with_(k_cache=k.float().numpy(), v_cache=v.float().numpy())
    ref = oracle.decode_attn(q)
    gate = None if p.L == 1 else f(p.gate_logits).unsqueeze(2)
    win = (None, None) if p.L == 1 else (f(p.k_win), f(p.v_win))
    scale = p.sm_scale if p.sm_scale > 0 else p.d ** -0.5
    out, size, _ = oracle_prefix.attend(f(p.q).unsqueeze(2), [(k[0, :P], v[0, :P])], [0, p.B], k[:, P:], v[:, P:], lens, scale, [int(x) for x in p.offsets()],
                                        p.w, *win, None if p.win_lens is None else p.win_lens, gate)
    assert np.abs(out[:, :, 0].numpy() - ref).max() < 1e-12 and (size >= out.abs() - 1e-12).all()


def test_oracle_without_groups_and_inside_a_prefix():
    g = torch.Generator().manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    q, k, v, pk, pv = rand(2, 1, 1, 2, 8), rand(2, 4, 1, 8), rand(2, 4, 1, 8), rand(6, 1, 8), rand(6, 1, 8)
    out, _, _ = oracle_prefix.attend(q, [(pk, pv)], [0, 1], k, v, [3, 2], 0.3, [0])
    a = torch.softmax(q[0, 0, 0] @ pk[:3, 0].T * 0.3, -1) @ pv[:3, 0]
    b = torch.softmax(q[1, 0, 0] @ k[1, :2, 0].T * 0.3, -1) @ v[1, :2, 0]
    assert torch.allclose(out[0, 0, 0], a) and torch.allclose(out[1, 0, 0], b)

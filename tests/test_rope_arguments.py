"""CPU checks of what the binding and the runner make of a rotation's arguments (no compute call is made)."""
import subprocess
from pathlib import Path

import pytest
import torch

from paper_2510_24824_b200 import binding as B
from paper_2510_24824_b200.inputs import make_problem
from paper_2510_24824_b200.runner import DeviceProblem, Rope

ROOT = Path(__file__).resolve().parents[1]


def test_lists_that_are_too_short_are_refused_before_c_reads_them():
    args = ("bf16", 4, 2, 8, 4, 128, 512, 16)
    for more in (dict(inv_freq=[0.5] * 63), dict(inv_freq=[0.5] * 15, rotary_dim=32), dict(inv_freq=[]), dict(loop_offset=[0]), dict(loop_offset=[])):
        with pytest.raises(ValueError):
            B.make_rope_config(*args, **more)
    assert B.plt_rope_frequencies(B.make_rope_config(*args, inv_freq=[0.5] * 64, loop_offset=[0, 3]))[63] == 0.5
    assert B.plt_rope_frequencies(B.make_rope_config(*args, inv_freq=[0.25] * 16, rotary_dim=32))[15] == 0.25
    with pytest.raises(ValueError):
        B.make_prefix_config("bf16", 4, 2, 8, 4, 128, 512, 16, 100, loop_offset=[0])


def test_caches_that_a_handle_would_write_past_are_refused():
    spec = dict(name="args", dtype="bf16", B=2, L=2, Hq=8, Hkv=4, d=128, w=16, lens=("list", [40, 7]), max_seq_len=64, seed=1)
    p = make_problem(spec)
    o = Rope.__new__(Rope)
    o.handle, o.config = None, B.make_rope_config("bf16", 8, 2, 8, 4, 128, p.max_seq_len, 16)
    dp = DeviceProblem(p, "cpu")

    def prompt(n, dp):
        z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
        o.seq(z(n, 2, 5, 8, 128), z(n, 5, 4, 128), torch.ones(n, dtype=torch.int32), z(n, 2, 5, 8, 128), k_loc=z(n, 1, 5, 4, 128),
              k_loc_out=z(n, 1, 5, 4, 128), v_share=z(n, 5, 4, 128), dp=dp)

    with pytest.raises(ValueError, match="caches of 3 sequences"):
        prompt(3, dp)                              # the handle's batch holds 8, the caches 2
    for other in (dict(w=8), dict(Hkv=8), dict(L=3), dict(max_seq_len=48), dict(max_seq_len=96)):
        with pytest.raises(ValueError):
            o._caches(DeviceProblem(make_problem({**spec, **other}), "cpu"), 2)
    longer = DeviceProblem(make_problem({**spec, "max_seq_len": 96}), "cpu")
    o._caches(longer, 2, (96 * 4 * 128, 4 * 128, 128))
    o._caches(dp, 2)
    o._caches(dp, 1)


def test_the_header_names_every_bit_that_a_check_can_return(tmp_path):
    bits = ["PLT_DEV_SEQ_LEN_CLAMPED", "PLT_DEV_PAGE_ID_CLAMPED", "PLT_DEV_GROUP_CLAMPED"]
    (tmp_path / "bits.c").write_text(f'#include "{ROOT}/include/plt_rope.h"\n#include <stdio.h>\nint main(void) {{\n' +
                                     "".join(f'    printf("%u\\n", {b});\n' for b in bits) + "    return 0;\n}\n")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-o", str(tmp_path / "bits"), str(tmp_path / "bits.c")], check=True)
    out = subprocess.run([str(tmp_path / "bits")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(x) for x in out] == [getattr(B, b) for b in bits]

"""CPU checks of what the runner makes of the caller's tensors (no compute call is made)."""
import pytest
import torch

from paper_2510_24824_b200 import binding as B
from paper_2510_24824_b200 import runner
from paper_2510_24824_b200.inputs import make_problem, make_seq_problem
from paper_2510_24824_b200.runner import CacheEvict, DeviceProblem, _learned

P = make_problem(dict(name="args", dtype="bf16", B=3, L=2, Hq=8, Hkv=4, d=128, w=16, lens=("list", [40, 7, 2]), seed=1))
N = P.max_seq_len


def op(p=P, group=1, q_len=1):
    """A CacheEvict without its library handle."""
    o = CacheEvict.__new__(CacheEvict)
    o.handle = None
    o.config = B.make_evict_config(p.dtype, p.B, p.L, p.Hq, p.Hkv, p.d, p.max_seq_len, q_len=q_len, heads_per_group=group)
    return o


def tensors(p=P, group=1, budget=16, q_len=1):
    groups = p.Hkv // group
    return dict(dp=DeviceProblem(p, "cpu"), q=torch.zeros(p.B, p.L, q_len, p.Hq, p.d, dtype=torch.bfloat16),
                weights=torch.zeros(p.B, groups, p.max_seq_len), keep=torch.zeros(p.B, groups, budget, dtype=torch.int32),
                new_lens=torch.zeros(p.B, dtype=torch.int32))


def all_args(o, t, budget=16, gate=None):
    return (o.weights_args(t["dp"], t["q"], t["weights"], gate), o.select_args(t["dp"], t["weights"], t["keep"], t["new_lens"], budget, 1, 4),
            o.compact_args(t["dp"], t["keep"], t["new_lens"], t["weights"]))


@pytest.mark.parametrize("group", [1, 2, 4])
def test_totals_that_are_a_view_of_wider_rows(group):
    t = tensors(group=group)
    for wide in (torch.zeros(P.B, P.Hkv // group, N + 24)[..., :N], torch.zeros(P.B + 2, P.Hkv // group, N + 3)[1:-1, :, 2:N + 2]):
        t["weights"] = wide
        for a in all_args(op(group=group), t):
            assert a.weights_stride == wide.stride(0 if group == P.Hkv else 1)


def test_one_row_of_totals():
    p = make_problem(dict(name="args", dtype="bf16", B=1, L=1, Hq=4, Hkv=1, d=128, w=0, lens=("list", [40]), seed=1))
    t = tensors(p)
    t["weights"] = torch.zeros(64, 1, N).transpose(0, 1)[:, 3:4]            # strides that no row uses
    assert all(a.weights_stride >= N for a in all_args(op(p), t))


@pytest.mark.parametrize("name,bad", [
    ("weights", lambda t: t[:, :, : N - 1]),                                # rows shorter than the capacity
    ("weights", lambda t: t.double()), ("weights", lambda t: t[:2]), ("weights", lambda t: t[:, :3]), ("weights", lambda t: t[0]),
    ("weights", lambda t: torch.zeros(P.B, P.Hkv, 2 * N)[:, :, ::2]),       # elements apart
    ("weights", lambda t: torch.zeros(P.Hkv, P.B, N).transpose(0, 1)),      # rows in another order
    ("weights", lambda t: torch.zeros(P.B, 2 * P.Hkv, N)[:, : P.Hkv]),      # a gap between sequences
    ("keep", lambda t: t.long()), ("keep", lambda t: torch.zeros(P.B, P.Hkv, 32, dtype=torch.int32)[..., :16]),
    ("keep", lambda t: t[:2]), ("keep", lambda t: t[:, :3].contiguous()), ("keep", lambda t: t[0]),
    ("new_lens", lambda t: t.long()), ("new_lens", lambda t: t[:2]), ("new_lens", lambda t: torch.zeros(2 * P.B, dtype=torch.int32)[::2]),
    ("q", lambda t: t.float()), ("q", lambda t: t[:, :1]), ("q", lambda t: torch.zeros(P.L, P.B, 1, P.Hq, P.d, dtype=torch.bfloat16).transpose(0, 1)),
])
def test_tensors_that_a_kernel_would_misread(name, bad):
    t = tensors()
    all_args(op(), t)
    t[name] = bad(t[name])
    with pytest.raises(ValueError):
        all_args(op(), t)


def test_a_budget_that_is_not_the_width_of_keep_and_gates_of_another_shape():
    t = tensors()
    with pytest.raises(ValueError):
        all_args(op(), t, budget=15)
    good = torch.zeros(P.B, P.L - 1, 1, P.Hq)
    all_args(op(), t, gate=good)
    for bad in (good.double(), good[:2], torch.zeros(P.B, P.L - 1, 1, 2 * P.Hq)[..., ::2]):
        with pytest.raises(ValueError):
            all_args(op(), t, gate=bad)


def test_larger_buffers_and_several_tokens_are_taken():
    t = tensors(q_len=2)
    t["weights"], t["new_lens"] = torch.zeros(P.B + 1, P.Hkv, N), torch.zeros(P.B + 4, dtype=torch.int32)
    t["keep"] = torch.zeros(P.B + 1, P.Hkv, 16, dtype=torch.int32)
    all_args(op(q_len=2), t)


# ---- learned parameters of differential heads ------------------------------------------------------------------------
def learned(q1=(1, 64), k1=(1, 64), q2=(1, 64), k2=(1, 64), gain=(128,)):
    return _learned([torch.zeros(s) for s in (q1, k1, q2, k2)], None if gain is None else torch.ones(gain), "cpu", 8, 128)


def test_learned_parameters_of_every_allowed_shape():
    for rows in ((64,), (1, 64), (8, 64)):
        w = learned(rows, rows, rows, rows)
        assert w.lambda_heads == (8 if rows == (8, 64) else 1) and w.norm_gain
    assert not learned(gain=None).norm_gain


@pytest.mark.parametrize("bad", [dict(q1=(8, 64)), dict(k2=(8, 64)), dict(k1=(64, 8)), dict(q2=(1, 32)), dict(gain=(64,)), dict(gain=(2, 64)),
                                 dict(q1=(4, 64), k1=(4, 64), q2=(4, 64), k2=(4, 64)), dict(q1=(8, 8, 64))])
def test_learned_parameters_that_a_kernel_would_read_beyond(bad):
    with pytest.raises(ValueError):
        learned(**bad)


def test_learned_parameters_go_to_the_handles_device(monkeypatch):
    """Without a device of their own they follow device_index (nothing is created here)."""
    seen = []
    monkeypatch.setattr(runner, "_learned", lambda lambdas, gain, device, Hq, d: seen.append(str(device)))
    monkeypatch.setattr(runner, "to_torch", lambda a, dtype, device, pin=False: seen.append(str(device)))
    monkeypatch.setattr(runner.torch, "empty", lambda *a, device=None, **k: seen.append(str(device)))
    for name in ("plt_diff_attn_create", "plt_diff_seq_attn_create"):
        monkeypatch.setattr(B, name, lambda config: None)
    monkeypatch.setattr(B, "make_seq_args", lambda *a, **k: None)
    runner.DiffAttn(P, None, device_index=3)
    runner.DiffSeqAttn(make_seq_problem(B=1, L=1, T=2, Hq=1, Hkv=1, d=128, w=0), None, device_index=3)
    assert set(seen) == {"cuda:3"}

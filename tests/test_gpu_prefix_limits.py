"""Shared prefixes on the GPU: the framework's parity bound on sharply peaked rows, and the ends of what the arguments may be."""
import pytest
import torch

from paper_2510_24824_b200 import binding as B
from parity_bounds import assert_parity
from prefix_util import Problem

pytestmark = pytest.mark.gpu


# ---- sharp peaks on large values: the decode step's own bound -----------------------------------------------------------
def _peaked(seed, share, **kw):
    """A share of the prefixes' positions has its K and V rows tripled, as in the decode step's peaked workload."""
    p = Problem(seed, peak=1.0, **kw)
    g = torch.Generator("cuda").manual_seed(1000 + seed)
    k, v = p.shared_more["k_prefix"], p.shared_more["v_prefix"]
    for i, n in enumerate(p.plens):
        hot = torch.rand(n, generator=g, device="cuda") < share
        hot[int(torch.randint(n, (1,), generator=g, device="cuda"))] = True
        for x in (k, v):
            x[i, :n][hot] *= 3.0
        p.values["pre"][i] = (k[i, :n].double(), v[i, :n].double())
    return p


@pytest.mark.parametrize("seed", [2, 12, 22])
@pytest.mark.parametrize("share,kw", [
    (0.02, dict(own=[0] * 48, plens=[40], begin=[0, 48], Hq=32, Hkv=8)),
    (0.02, dict(own=[0] * 48, plens=[300], begin=[0, 48], Hq=32, Hkv=8)),
    (0.002, dict(own=[0] * 24, plens=[2000], begin=[0, 24], Hq=32, Hkv=8)),
    (0.02, dict(own=[0] * 24, plens=[2000], begin=[0, 24], Hq=32, Hkv=8, d=64)),
    (0.02, dict(own=[3] * 48, plens=[500], begin=[0, 48], Hq=16, Hkv=4, L=2, w=9)),
    (0.001, dict(own=[0, 5, 9], plens=[9000], begin=[0, 3], Hq=24, Hkv=8)),
], ids=["40", "300", "2000", "2000 of 64", "500 and windows", "9000"])
def test_peaked_rows_stay_within_the_decode_step_s_bound(seed, share, kw):
    p = _peaked(seed, share, **kw)
    assert p.run() == 0
    assert_parity(p.out.double().cpu().numpy(), p.expect()[0].cpu().numpy(), "bf16", f"peaks behind a prefix, seed {seed}")
    p.hold()


# ---- the ends of 32 bits ------------------------------------------------------------------------------------------------
def test_the_lowest_lengths_are_clamped_as_any_below_zero():
    low = -2 ** 31
    for more in (dict(L=3, w=6), dict(q_len=4), dict(L=2, w=6, q_len=2)):
        p = Problem(41, [4] * 6, [300], [0, 5], lens=[304, low, low + 1, 302, -5, low + 2], **more)
        assert p.run() == B.PLT_DEV_SEQ_LEN_CLAMPED
        p.lens = [304, 0, 0, 302, 0, 0]
        p.hold()



def test_offsets_that_no_length_reaches():
    """The last loop never has a token: zero rows, although length - offset - newer tokens lies below the lowest whole number."""
    for q_len in (1, 3):
        p = Problem(43, [4] * 5, [300], [0, 4], lens=[304, 0, 1, 302, 4], L=2, w=6, q_len=q_len, offsets=[0, 2 ** 31 - 1])
        assert p.run() == 0
        assert (p.out[:, 1] == 0).all()
        p.hold()


# ---- queries that are not numbers ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("kv", ["", "e4m3"])
@pytest.mark.parametrize("n", [30, 700])
def test_a_query_that_is_not_a_number_gives_none(kv, n):
    """Its own row alone: softmax of scores that are not numbers is none either, wherever the keys lie."""
    p = Problem(42, [0, 3, 0, 4], [n], [0, 4], kv=kv, Hq=8, Hkv=2)
    ref = p.expect()
    p.q[2, 0, 0, 5] = float("nan")
    p.q[1, 0, 0, 2, 7] = float("nan")
    assert p.run() == 0
    assert torch.isnan(p.out[2, 0, 0, 5]).all() and torch.isnan(p.out[1, 0, 0, 2]).all()
    bad = torch.zeros(p.out.shape, dtype=torch.bool, device="cuda")
    bad[2, 0, 0, 5] = bad[1, 0, 0, 2] = True
    assert torch.isfinite(p.out[~bad]).all()
    p.out = torch.where(bad, ref[0].to(p.out.dtype), p.out)
    p.hold(ref)

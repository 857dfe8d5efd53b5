"""CPU pins of the differential-attention oracle."""
import numpy as np
import pytest

import oracle
from paper_2510_24824_b200.inputs import make_problem, make_seq_problem

from diff_util import EPS, LAMBDA_INIT, learned, stored

TINY = dict(name="tiny", dtype="f32", B=3, L=3, Hq=4, Hkv=2, d=8, w=3, lens=("list", [7, 1, 2]), seed=3)


@pytest.mark.parametrize("heads", [1, 4])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("offset", [None, [0, 0, 0], [0, 2, 1]])
def test_oracle_equals_the_definition_written_out(heads, norm, offset):
    p = make_problem(dict(TINY, d=64, loop_offset=offset))
    lambdas, gain = learned(p.d, heads, norm=norm)
    want = oracle.brute_force_step(p, stored, lambdas, gain, LAMBDA_INIT, EPS)
    got = oracle.diff_attn(p, lambdas, gain, LAMBDA_INIT, EPS)
    assert np.abs(got - want).max() < 1e-12


def test_equal_halves_leave_one_map_times_one_minus_lambda():
    """Both halves alike: the maps agree, the difference is (1 - lambda) times the attention on the half rows."""
    p = make_problem(dict(TINY, d=64))
    q, k = p.q.copy(), p.k_cache.copy()
    q[..., 32:], k[..., 32:] = q[..., :32], k[..., :32]
    kw = p.k_win.copy()
    kw[..., 32:] = kw[..., :32]
    p = p.with_(q=q, k_cache=k, k_win=kw)
    lambdas, _ = learned(64, 1)
    lam = float(oracle.diff_lambda(lambdas, LAMBDA_INIT)[0])
    # the whole row's product is twice the half's, so half the scale gives the same softmax
    plain = oracle.decode_attn(p.with_(sm_scale=0.5 / np.sqrt(32.0)))
    assert np.abs(oracle.diff_attn(p, lambdas, None, LAMBDA_INIT) - (1.0 - lam) * plain).max() < 1e-12


def test_factor_of_zero_vectors_is_lambda_init():
    zero = [np.zeros((1, 32))] * 4
    assert oracle.diff_lambda(zero, 0.3)[0] == 0.3


def test_normed_heads_have_the_gain_as_root_mean_square():
    p = make_problem(dict(TINY, d=64))
    lambdas, _ = learned(64, 1)
    out = oracle.diff_attn(p, lambdas, np.ones(64), LAMBDA_INIT, 0.0 + 1e-30)
    rms = np.sqrt((out[0] ** 2).mean(-1))
    assert np.abs(rms - (1.0 - LAMBDA_INIT)).max() < 1e-12


def test_prompt_rows_are_decode_steps():
    """Row t of a prompt is the step at cache length t + 1 (one loop)."""
    s = make_seq_problem(B=1, L=1, T=6, Hq=2, Hkv=1, d=64, w=0, seed=4)
    lambdas, gain = learned(64, 2)
    rows = oracle.diff_seq_attn(s, lambdas, gain, LAMBDA_INIT, EPS)
    base = make_problem(dict(TINY, dtype="bf16", B=1, L=1, Hq=2, Hkv=1, d=64, lens=("list", [6])))
    for t in range(6):
        step = base.with_(q=s.q[:, :, t], k_cache=s.k_share, v_cache=s.v_share, seq_lens=np.array([t + 1], np.int32))
        assert np.abs(oracle.diff_attn(step, lambdas, gain, LAMBDA_INIT, EPS)[0, 0] - rows[0, 0, t]).max() < 1e-12

"""GPU parity of differential attention where no weight has to be rounded: integer scores in powers of two.

With sm_scale = ln 2 and queries and keys of -1, 0 and 1 every score is a whole power of two, so a weight relative to any
other score is 2^k, which bf16, f16 and E4M3 hold exactly. What is left of a map's error is the fp32 side, and the bound of the
comparison shrinks from 2^-8 of the largest value to a few 2^-16, far below the results themselves."""
import numpy as np
import pytest
import torch

import oracle
from paper_2510_24824_b200 import binding as B
from paper_2510_24824_b200.inputs import f32_to_bf16_bits, make_problem, make_seq_problem
from paper_2510_24824_b200.runner import DeviceProblem, DiffAttn, DiffSeqAttn

from diff_util import EPS, LAMBDA_INIT, assert_close, learned

pytestmark = pytest.mark.gpu

LN2 = float(np.log(2.0))
BASE = dict(name="exact", dtype="bf16", B=3, L=2, Hq=8, Hkv=2, d=128, w=48, lens=("list", [700, 77, 2]), seed=5)


def signs(rng, shape, share):
    return (rng.integers(0, 2, shape) * 2 - 1).astype(np.float32) * (rng.random(shape) < share)


def few(rng, shape, half, nonzero):
    """-1 or 1 in `nonzero` places of every half row, 0 elsewhere."""
    x = np.zeros(shape, np.float32).reshape(-1, half)
    at = np.argsort(rng.random(x.shape), axis=1)[:, :nonzero]
    np.put_along_axis(x, at, signs(rng, at.shape, 1.1), axis=1)
    return x.reshape(shape)


def e4m3(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()


def exact_fp32(keys, score):
    """Two sums of `keys` terms (weights, and weights times values of at most 1), each add off by 2^-23 of a partial sum that
    is no larger than the sum of magnitudes; a weight off by score 2^-23 from the scale's rounding, 2^-20 from exp2 and the
    merge of pieces. As in map_error, numerator and denominator one such share each."""
    return 2.0 * (keys * 2.0 ** -23 + score * 2.0 ** -23 + 2.0 ** -20)


def step_problem(nonzero=6, **kw):
    p = make_problem(dict(BASE, **kw))
    rng = np.random.default_rng(p.B + p.d + p.L)
    put = {"f32": lambda x: x, "bf16": f32_to_bf16_bits}[p.dtype]
    put_kv = e4m3 if p.kv_dtype == "e4m3" else put
    rows = {n: put_kv(signs(rng, getattr(p, n).shape, 0.7)) for n in ("k_cache", "k_win")}
    rows |= {n: put_kv(rng.uniform(-1.0, 1.0, getattr(p, n).shape).astype(np.float32)) for n in ("v_cache", "v_win")}
    if p.kv_dtype == "e4m3":
        rows |= dict(k_scale=np.ones(p.Hkv, np.float32), v_scale=np.ones(p.Hkv, np.float32))
    return p.with_(q=put(few(rng, p.q.shape, p.d // 2, nonzero)), sm_scale=LN2, **rows), nonzero


def check_step(p, nonzero, norm, **config):
    lambdas, gain = learned(p.d, p.Hq, norm=norm)
    dp = DeviceProblem(p, "cuda:0")
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS, **config) as op:
        got = op.run(dp).float().cpu().numpy().astype(np.float64)
        assert op.check() == 0
    e = exact_fp32(int(p.seq_lens.max()) + p.w, nonzero)
    assert_close(got, oracle.diff_maps(p), lambdas, gain, p.dtype, e, p.name)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("dtype,d,kv,page", [("bf16", 128, "", 0), ("bf16", 64, "", 16), ("bf16", 128, "", 64), ("bf16", 128, "e4m3", 0),
                                             ("bf16", 128, "e4m3", 64), ("f32", 128, "", 0), ("f32", 64, "", 32)])
@pytest.mark.parametrize("L", [1, 2, 3])
def test_step(dtype, d, kv, page, L, norm):
    check_step(*step_problem(dtype=dtype, d=d, kv_dtype=kv, page_size=page, L=L), norm)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("kv,Hq,Hkv", [("", 16, 2), ("", 64, 2), ("e4m3", 16, 2), ("e4m3", 16, 1)])
def test_step_on_tensor_memory(kv, Hq, Hkv, norm):
    """Three places a half: weights within 2^6 of one another, normal numbers of E4M3."""
    check_step(*step_problem(nonzero=3, kv_dtype=kv, Hq=Hq, Hkv=Hkv, L=1), norm, kernel_path=B.PLT_PATH_TCGEN05)


@pytest.mark.parametrize("norm", [False, True])
def test_step_split_over_the_grid(norm):
    check_step(*step_problem(B=1, Hq=4, Hkv=1, L=1, lens=("list", [5003])), norm)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv", [(129, 2, 1), (300, 6, 3), (1000, 4, 2)])
def test_prompt(T, Hq, Hkv, norm):
    p = make_seq_problem(B=2, L=1, T=T, Hq=Hq, Hkv=Hkv, d=128, w=0, lens=[T, T // 2 + 1], seed=T, sm_scale=LN2)
    rng = np.random.default_rng(T)
    p = p.with_(q=f32_to_bf16_bits(few(rng, p.q.shape, 64, 6)), k_share=f32_to_bf16_bits(signs(rng, p.k_share.shape, 0.7)),
                v_share=f32_to_bf16_bits(rng.uniform(-1.0, 1.0, p.v_share.shape).astype(np.float32)))
    lambdas, gain = learned(128, Hq, norm=norm)
    with DiffSeqAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        got = op.run().float().cpu().numpy().astype(np.float64)
        assert op.check() == 0
    assert_close(got, oracle.diff_seq_maps(p), lambdas, gain, "bf16", exact_fp32(T, 6), f"prompt of {T}")

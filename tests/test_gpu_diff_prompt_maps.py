"""GPU parity of the differential prompt kernel where its two maps take different times: one map's scores grow along the keys,
so that it moves its rows' reference (and rescales their accumulator) in every half tile, and the other map's never do."""
import numpy as np
import pytest
import torch

import oracle
from paper_2510_24824_b200.inputs import f32_to_bf16_bits, make_seq_problem
from paper_2510_24824_b200.runner import DiffSeqAttn

from diff_util import EPS, LAMBDA_INIT, assert_close, largest, learned, map_error

pytestmark = pytest.mark.gpu

HALF = 64
GROWTH = 0.85     # of q . k per key: 0.85 / 8 * log2(e) * 64 keys = 9.8 > 8 powers of two from half tile to half tile


def growing(grows, L, T, Hq, Hkv, seed):
    """Half `grows` of every query row is ones and of key row n is GROWTH n / 64 in each of its 64 elements; the other half is
    N(0, 1) clipped to 2. Values lie in [-1, 1]."""
    p = make_seq_problem(B=1, L=L, T=T, Hq=Hq, Hkv=Hkv, d=2 * HALF, w=64, seed=seed)
    rng = np.random.default_rng([seed, 3])
    q, k = (np.clip(rng.standard_normal(s, dtype=np.float32), -2.0, 2.0) for s in (p.q.shape, p.k_share.shape))
    half = slice(grows * HALF, (grows + 1) * HALF)
    q[..., half] = 1.0
    k[..., half] = (GROWTH / HALF * np.arange(T, dtype=np.float32))[None, :, None, None]
    v = [f32_to_bf16_bits(rng.uniform(-1.0, 1.0, s).astype(np.float32)) for s in (p.v_share.shape, p.v_loc.shape)]
    return p.with_(q=f32_to_bf16_bits(q), k_share=f32_to_bf16_bits(k), v_share=v[0], v_loc=v[1])


def bound(p):
    """map_error with the dot products of the kernel: each runs over the 64 elements of one half."""
    v = max(largest(p.v_share), largest(p.v_loc))
    return max(map_error("bf16", v, HALF, largest(p.q[..., h]), max(largest(p.k_share[..., h]), largest(p.k_loc[..., h])))
               for h in (slice(0, HALF), slice(HALF, 2 * HALF)))


@pytest.mark.parametrize("grows", [0, 1])
@pytest.mark.parametrize("L,T,Hq,Hkv", [(1, 129, 2, 1), (1, 256, 4, 2), (1, 300, 8, 4), (2, 300, 4, 2), (1, 1000, 8, 2), (2, 1100, 4, 1), (1, 2500, 4, 2)])
def test_one_map_rescales_in_every_half_tile(grows, L, T, Hq, Hkv):
    p = growing(grows, L, T, Hq, Hkv, seed=T + L)
    for norm in (False, True):
        lambdas, gain = learned(p.d, Hq, seed=2, norm=norm)
        with DiffSeqAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
            op.out.fill_(float("nan"))
            first = op.run().clone()
            assert op.check() == 0
            for _ in range(8):
                assert torch.equal(op.run(), first), "two runs on the same inputs differ"
            assert op.check() == 0
        if not norm:
            maps = oracle.diff_seq_maps(p)
        assert_close(first.float().cpu().numpy().astype(np.float64), maps, lambdas, gain, "bf16", bound(p), f"map {grows + 1} grows, norm {norm}")


def test_maps_that_take_turns():
    """The growing half changes with the sequence of the batch, next to sequences whose maps are alike."""
    parts = [growing(g, 1, 700, 4, 2, seed=90 + g) for g in (0, 1)]
    flat = make_seq_problem(B=1, L=1, T=700, Hq=4, Hkv=2, d=2 * HALF, w=64, seed=95)
    flat = flat.with_(v_share=parts[0].v_share, v_loc=parts[0].v_loc)
    all3 = [parts[0], flat, parts[1]]
    join = {n: np.concatenate([getattr(x, n) for x in all3]) for n in ("q", "k_share", "v_share", "k_loc", "v_loc", "gate_logits", "seq_lens")}
    p = flat.with_(B=3, **join)
    lambdas, gain = learned(p.d, 1, norm=False)
    with DiffSeqAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        got = op.run().float().cpu().numpy().astype(np.float64)
        assert op.check() == 0
    for b, x in enumerate(all3):
        assert_close(got[b:b + 1], oracle.diff_seq_maps(x), lambdas, gain, "bf16", bound(x), f"sequence {b}")

"""Shared by the tests of differential attention: parameters and the bound of one comparison (numpy only)."""
import numpy as np

import oracle
from paper_2510_24824_b200.inputs import bf16_bits_to_f32

LAMBDA_INIT, EPS = 0.8, 1e-5


def learned(d, heads, seed=0, norm=True):
    """The four vectors [heads, d / 2] and the gain [d] (or None), fp32."""
    rng = np.random.default_rng([seed, 11])
    lambdas = [(0.1 * rng.standard_normal((heads, d // 2))).astype(np.float32) for _ in range(4)]
    return lambdas, (1.0 + 0.1 * rng.standard_normal(d)).astype(np.float32) if norm else None


def stored(a):
    return bf16_bits_to_f32(a).astype(np.float64) if a.dtype == np.uint16 else a.astype(np.float64)


def largest(a, scale=None):
    """Largest finite magnitude of a stored tensor (E4M3 codes with their scales)."""
    if scale is not None:
        import torch
        x = torch.from_numpy(a).view(torch.float8_e4m3fn).float().numpy() * scale[:, None]
    else:
        x = stored(a)
    x = np.abs(x[np.isfinite(x)])
    return float(x.max()) if x.size else 0.0


def map_error(dtype, max_v, d, max_q=0.0, max_k=0.0, e4m3_terms=False):
    """How far one map's result can be from the exact one. Weights p' = p (1 + delta), |delta| <= u, move the weighted mean
    of values of magnitude max_v by at most 2 u max_v (numerator and denominator one u each).
    bf16: u = 2^-8 from rounding the weights, half a step; weights as two E4M3 terms: each leaves at most 2^-4 of what it holds,
    2^-8 together, to which the terms below the format's smallest steps add less than as much again. The fp32 side: a dot product of d terms is off by at most
    d 2^-24 sum|q k| <= d 2^-24 d max|q| max|k|, scaled by 1/sqrt(d/2); its exponential by that much relatively, and
    exp2, the sums and the merge by some 2^-20."""
    u = {"bf16": 2.0 ** -8, "f32": 0.0}[dtype] * (2.0 if e4m3_terms else 1.0)
    u += d * 2.0 ** -24 * d * max_q * max_k / np.sqrt(d / 2.0) + 2.0 ** -20
    return 2.0 * u * max_v


def assert_close(got, y, lambdas, gain, dtype, e_map, what=""):
    """got against the exact result. y [..., 2 H, d]: the two maps' exact results, each of which the kernel may have off by
    e_map. x = y_1 - lambda y_2 is then off by at most e = (1 + |lambda|) e_map in each element, its root mean square by no
    more (triangle inequality), hence x / rms by at most e / (rms - e) (1 + |x| / rms); the store adds half a step."""
    ref = oracle.diff_join(y, lambdas, gain, LAMBDA_INIT, EPS)
    assert got.shape == ref.shape and np.isfinite(got).all(), f"{what}: shape or non-finite output"
    lam = oracle.diff_lambda(lambdas, LAMBDA_INIT)[:, None]
    e = (1.0 + np.abs(lam)) * e_map
    if gain is not None:
        x = y[..., 0::2, :] - lam * y[..., 1::2, :]
        rms = np.sqrt((x * x).mean(-1, keepdims=True) + EPS)
        tight = rms > 2 * e
        scale = (1.0 - LAMBDA_INIT) * np.abs(gain)
        e = np.where(tight, scale * e / np.where(tight, rms - e, 1.0) * (1.0 + np.abs(x) / rms), 3.0 * scale * np.sqrt(x.shape[-1]))
    half_step = {"bf16": 2.0 ** -8, "f32": 2.0 ** -22}[dtype]     # bf16 2^-8; fp32 store and the norm's few operations
    bound = e + half_step * (np.abs(ref) + e) + 1e-30
    err = np.abs(got - ref)
    worst = float((err / bound).max()) if err.size else 0.0
    assert worst <= 1.0, f"{what}: error {err.max():.3e}, {worst:.2f} of its bound"
    zero = ~np.any(y, axis=-1)
    assert not got[zero[..., 0::2] & zero[..., 1::2]].any(), f"{what}: a row without a token is not zero"
    return worst

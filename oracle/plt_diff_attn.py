"""fp64 CPU oracle of differential attention (test infrastructure only; the product never imports it).

The two softmax maps of a head are attentions of their own on the same values: map m multiplies half m of the query and key
rows. A query row whose other half is zero has exactly map m's scores with the whole key row, so the maps' results y_1, y_2
come from the plain oracles on a problem with 2 Hq such rows; what is written out here is the factor, the difference and the
norm. `brute_force_step` forms everything from the definition in Python loops, without the plain oracles.
"""
from __future__ import annotations

from dataclasses import replace

import numpy as np

from .plt_oracle import decode_attn, decode_attn_multi
from .plt_seq_attn import seq_attn


def _halves(q: np.ndarray) -> np.ndarray:
    """[..., H, d] -> [..., 2 H, d]: row 2 h has the second half of head h zero, row 2 h + 1 the first (zero bits are 0.0)."""
    d = q.shape[-1]
    out = np.zeros(q.shape[:-2] + (2 * q.shape[-2], d), dtype=q.dtype)
    out[..., 0::2, : d // 2] = q[..., : d // 2]
    out[..., 1::2, d // 2:] = q[..., d // 2:]
    return out


def _two_rows(p):
    scale = p.sm_scale if p.sm_scale > 0 else 1.0 / float(np.sqrt(p.d / 2.0))
    return replace(p, Hq=2 * p.Hq, q=_halves(p.q), gate_logits=np.repeat(p.gate_logits, 2, axis=-1), sm_scale=scale)


def diff_lambda(lambdas, lambda_init: float) -> np.ndarray:
    """exp(q1 . k1) - exp(q2 . k2) + lambda_init per row of the four vectors [rows, d / 2]."""
    q1, k1, q2, k2 = (np.asarray(x, dtype=np.float64) for x in lambdas)
    return np.exp((q1 * k1).sum(-1)) - np.exp((q2 * k2).sum(-1)) + lambda_init


def diff_join(y: np.ndarray, lambdas, gain, lambda_init: float, eps: float) -> np.ndarray:
    """[..., 2 H, d] results of the maps -> [..., H, d]."""
    x = y[..., 0::2, :] - diff_lambda(lambdas, lambda_init)[:, None] * y[..., 1::2, :]
    if gain is None:
        return x
    rms = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return (1.0 - lambda_init) * np.asarray(gain, dtype=np.float64) * x / rms


def diff_maps(p, q=None, gate_logits=None, q_len: int = 1) -> np.ndarray:
    """The results of the maps of one decode step: [B, L, 2 Hq, d] ([B, L, q_len, 2 Hq, d] for a multi-token step, whose q
    and gate_logits are given apart)."""
    if q_len == 1:
        return decode_attn(_two_rows(p))
    return decode_attn_multi(_two_rows(p), _halves(q), np.repeat(gate_logits, 2, axis=-1), q_len)


def diff_attn(p, lambdas, gain=None, lambda_init: float = 0.8, eps: float = 1e-5) -> np.ndarray:
    """One decode step: [B, L, Hq, d] in float64."""
    return diff_join(diff_maps(p), lambdas, gain, lambda_init, eps)


def diff_seq_maps(p) -> np.ndarray:
    """The results of the maps of every row of a prompt: [B, L, T, 2 Hq, d]."""
    with np.errstate(over="ignore"):
        return seq_attn(_two_rows(p))


def diff_seq_attn(p, lambdas, gain=None, lambda_init: float = 0.8, eps: float = 1e-5) -> np.ndarray:
    """Every row of a prompt: [B, L, T, Hq, d] in float64."""
    return diff_join(diff_seq_maps(p), lambdas, gain, lambda_init, eps)


def brute_force_step(p, values, lambdas, gain=None, lambda_init: float = 0.8, eps: float = 1e-5) -> np.ndarray:
    """The same step from the definition, for tiny single-token problems on contiguous caches. `values`: maps a stored array
    to float64."""
    q, k, v, kw, vw = (values(a) for a in (p.q, p.k_cache, p.v_cache, p.k_win, p.v_win))
    half, G = p.d // 2, p.Hq // p.Hkv
    scale = p.sm_scale if p.sm_scale > 0 else 1.0 / np.sqrt(half)
    out = np.zeros((p.B, p.L, p.Hq, p.d))

    def attend(query, keys, vals):
        if len(keys) == 0:
            return np.zeros(p.d)
        e = [np.exp(scale * float(query @ key)) for key in keys]
        return sum(x * val for x, val in zip(e, vals)) / sum(e)

    for b in range(p.B):
        for l in range(p.L):
            cut = int(p.seq_lens[b]) - (l if p.loop_offset is None else int(p.loop_offset[l]))
            if cut <= 0:
                continue
            for h in range(p.Hq):
                g = h // G
                maps = []
                for m in (slice(0, half), slice(half, p.d)):
                    y = attend(q[b, l, h, m], k[b, :cut, g, m], v[b, :cut, g])
                    if l > 0:
                        wl = min(p.w, cut) if p.win_lens is None else int(p.win_lens[b, l - 1])
                        near = attend(q[b, l, h, m], kw[b, l - 1, :wl, g, m], vw[b, l - 1, :wl, g])
                        s = 1.0 / (1.0 + np.exp(-float(p.gate_logits[b, l - 1, h])))
                        y = s * near + (1.0 - s) * y
                    maps.append(y)
                row = h if len(np.asarray(lambdas[0])) > 1 else 0
                q1, k1, q2, k2 = (np.asarray(x[row], dtype=np.float64) for x in lambdas)
                lam = np.exp(q1 @ k1) - np.exp(q2 @ k2) + lambda_init
                x = maps[0] - lam * maps[1]
                out[b, l, h] = x if gain is None else (1.0 - lambda_init) * np.asarray(gain, dtype=np.float64) * x / np.sqrt(np.mean(x ** 2) + eps)
    return out

"""fp64 CPU oracle of cache eviction (test infrastructure only; the product never imports it): the three definitions written
out on plain arrays, one (sequence, head) at a time. Caches come as values [B, n, Hkv, d] (contiguous or gathered pages)."""
from __future__ import annotations

import numpy as np


def weights(q, k, lens, held, group=1, maps=1, decay=1.0, gate=None, scale=0.0, offsets=None):
    """q [B, L, Qn, Hq, d], k [B, N, Hkv, d], held [B, Hkv / group, N]; returns the totals and the largest sum |q||k| met."""
    B, L, Qn, Hq, d = q.shape
    Hkv = k.shape[2]
    G, part = Hq // Hkv, d // maps
    scale = scale if scale > 0 else 1.0 / np.sqrt(part)
    out, terms = held.astype(np.float64).copy(), 0.0
    for b in range(B):
        n = int(lens[b])
        new = np.zeros((Hkv // group, n))
        for l in range(L):
            for j in range(Qn):
                cut = max(0, n - (l if offsets is None else int(offsets[l])) - (Qn - 1 - j))
                if cut == 0:
                    continue
                for h in range(Hq):
                    kv = h // G
                    rho = 1.0
                    if gate is not None and l > 0:
                        with np.errstate(over="ignore"):
                            rho = 1.0 - 1.0 / (1.0 + np.exp(-float(gate[b, l - 1, j, h])))
                    for m in range(maps):
                        at = slice(m * part, (m + 1) * part)
                        x, y = q[b, l, j, h, at], k[b, :cut, kv, at]
                        s = scale * (y @ x)
                        e = np.exp(s - s.max())
                        new[kv // group, :cut] += rho * e / e.sum()
                        terms = max(terms, scale * float((np.abs(y) @ np.abs(x)).max()))
        out[b, :, :n] = new + (decay * out[b, :, :n] if decay != 0 else 0.0)
    return out, terms


def select(w, lens, budget, first, last):
    """w [B, groups, N] -> keep [B, groups, budget] int32 (-1 behind the kept ones), new lengths [B]."""
    B, groups, _ = w.shape
    keep, new = np.full((B, groups, budget), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        n = int(lens[b])
        new[b] = min(n, budget)
        for g in range(groups):
            if n <= budget:
                chosen = range(n)
            else:
                always = set(range(first)) | set(range(n - last, n))
                rest = [i for i in range(n) if i not in always]
                rest.sort(key=lambda i: (np.isnan(w[b, g, i]), 0.0 if np.isnan(w[b, g, i]) else -float(w[b, g, i]), i))
                chosen = sorted(always | set(rest[: budget - len(always)]))
            keep[b, g, : len(chosen)] = list(chosen)
    return keep, new


def compact(cache, keep, new, group=1):
    """cache [B, N, Hkv, ...] (any storage) -> the cache after the move."""
    out = cache.copy()
    for b in range(cache.shape[0]):
        for h in range(cache.shape[2]):
            at = keep[b, h // group, : new[b]]
            out[b, : new[b], h] = cache[b, at, h]
    return out

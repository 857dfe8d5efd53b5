"""fp64 CPU oracle of draft verification (test infrastructure only; the product never imports it): one sequence at a time, sums
exactly rounded (math.fsum) where they decide anything."""
from __future__ import annotations

import math

import numpy as np


def _weights(row):
    return [float(x) if x > 0 and np.isfinite(x) else 0.0 for x in row]


def verify(target, draft, drafts, lens, u, r):
    """target [B, K + 1, V], draft [B, K, V] or None -> tokens [B, K + 1], accepted [B], and the distance of r * total from the
    running sums on both sides of the chosen token, relative to the total (how near the choice is to another one)."""
    B, K = drafts.shape
    V = target.shape[2]
    tokens, accepted, near = np.full((B, K + 1), -1, np.int32), np.zeros(B, np.int32), np.full(B, np.inf)
    for b in range(B):
        held = K if lens is None else min(max(int(lens[b]), 0), K)
        n = 0
        while n < held:
            x = int(drafts[b, n])
            if not 0 <= x < V:
                break
            q = 1.0 if draft is None else float(draft[b, n, x])
            if not float(u[b, n]) * q < float(target[b, n, x]):
                break
            n += 1
        p = target[b, n].astype(np.float64)
        w = _weights(p)
        if n < held:
            if draft is not None:
                with np.errstate(invalid="ignore"):
                    rest = _weights(p - draft[b, n].astype(np.float64))
            else:
                rest = list(w)
                if 0 <= int(drafts[b, n]) < V:
                    rest[int(drafts[b, n])] = 0.0
            if any(rest):
                w = rest
        tokens[b, :n] = drafts[b, :n]
        accepted[b] = n
        total = math.fsum(w)
        if total > 0:
            limit = float(r[b]) * total
            sums = np.cumsum(w)
            past = np.nonzero(sums > limit)[0]
            token = int(past[0]) if len(past) else int(np.nonzero(w)[0][-1])
            tokens[b, n] = token
            below = sums[token] - w[token]
            near[b] = min(abs(sums[token] - limit), abs(limit - below) if below > 0 else np.inf) / total
    return tokens, accepted, near

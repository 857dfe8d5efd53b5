"""fp64 oracle of the decode step with shared prefixes (test infrastructure only; the product never imports it): one (sequence,
KV head) at a time, on the keys [prefix of the group ; own keys] laid one behind the other, softmax by its definition."""
from __future__ import annotations

import torch


def attend(q, prefixes, begin, own_k, own_v, lens, scale, offsets, w=0, k_win=None, v_win=None, win_lens=None, gate=None):
    """q [B, L, Qn, Hq, d]; prefixes: (k, v) [P_g, Hkv, d] of each group; begin: first sequence of each group and the end of the
    last; own_k, own_v [B, N, Hkv, d]; lens count the prefix.  Returns the result and, as the size that its error is measured
    by, the same with |v| in the place of v; and the largest sum of |q_i k_i| * scale met."""
    B, L, Qn, Hq, d = q.shape
    Hkv = own_k.shape[2]
    G = Hq // Hkv
    q = q.double()
    out, size, most = torch.zeros_like(q), torch.zeros_like(q), 0.0
    none = own_k[0, :0].double()

    def soft(x, k, v, seen):
        nonlocal most
        k, v = k[:seen], v[:seen]
        s = (x @ k.T) * scale
        most = max(most, float((x.abs() @ k.abs().T).max()) * scale)
        p = torch.exp(s - s.max(dim=-1, keepdim=True).values)
        p = p / p.sum(dim=-1, keepdim=True)
        return p @ v, p @ v.abs()

    for b in range(B):
        g = next((i for i in range(len(prefixes)) if begin[i] <= b < begin[i + 1]), None)
        pk, pv = prefixes[g] if g is not None else (none, none)
        n = int(lens[b])
        own = max(0, n - len(pk))
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            k = torch.cat([pk[:, h].double(), own_k[b, :own, h].double()])
            v = torch.cat([pv[:, h].double(), own_v[b, :own, h].double()])
            for l in range(L):
                for j in range(Qn):
                    newer = Qn - 1 - j
                    cut = n - offsets[l] - newer
                    if cut <= 0:
                        continue
                    x = q[b, l, j, heads]
                    y, z = soft(x, k, v, cut)
                    if l:
                        slots = min(w, n - offsets[l]) if win_lens is None else int(win_lens[b][l - 1])
                        near, far = torch.zeros_like(y), torch.zeros_like(y)
                        if slots - newer > 0:
                            near, far = soft(x, k_win[b, l - 1, :, h].double(), v_win[b, l - 1, :, h].double(), slots - newer)
                        m = torch.sigmoid(gate[b, l - 1, j, heads].double()).unsqueeze(-1)
                        y, z = m * near + (1 - m) * y, m * far + (1 - m) * z
                    out[b, l, j, heads], size[b, l, j, heads] = y, z
    return out, size, most

"""The measured calls of shared-prefix attention, of the rotation of queries and keys, and of draft verification: their
inputs, their plain forms and their cost.

  prefix      one decode step of a batch whose sequences share long prefixes, each prefix's cache read once for all of them
  rope_step   norm and rotation of a decode step's queries and keys, with the cache append, the window rings and the gates
  rope_seq    the same for every row of a prompt, with the rows' way into the decode cache
  verify      which of a step's drafted tokens the target's probabilities let pass, and the token after them

`run` computes them in elementary torch operations in fp32 (angles, and sums over a vocabulary, in fp64), or, where `own` is
true, through the framework's entry points.
"""
import math

import numpy as np
import torch

own = False


# ---- cases --------------------------------------------------------------------------------------------------------
def _prefix(name, **kw):
    case = dict(op="prefix", name=name, dtype="bf16", B=1, L=1, Hq=32, Hkv=8, d=128, w=64, P=4096, N=1024, groups=1, loose=0, page=0, q_len=1, ragged=True)
    case.update(kw)
    return case


def _rope(op, name, **kw):
    case = dict(op=op, name=name, dtype="bf16", B=1, L=1, Hq=32, Hkv=8, d=128, w=64, N=1024, page=0, q_len=1, ragged=True, rd=128, layout="half",
                scaling="none", norm=True, far=0)
    case.update(kw)
    return case


def listed():
    return [
        # two users of one short system prompt; latency is all there is
        _prefix("prefix_two", B=2, P=300, N=40),
        # the decode batch of the parallel loop configuration behind one system prompt: two loops, windows, gates
        _prefix("prefix_batch", B=64, L=2, P=4096, N=1024),
        # three prompts of different lengths and a few sequences without one, 8-bit caches in pages
        _prefix("prefix_groups_e4m3", B=96, Hkv=4, P=8192, N=2048, groups=3, loose=5, page=64, dtype="e4m3"),
        # four drafted tokens a step, heads of 64, odd lengths, pages of 48
        _prefix("prefix_drafts", B=21, Hq=16, Hkv=4, d=64, P=1777, N=301, page=48, q_len=5),
        # many samples of one long document
        _prefix("prefix_long", B=128, L=2, P=32768, N=512),
        # one user's step
        _rope("rope_step", "rope_step_one", N=700),
        # the decode batch of two loops with 8-bit caches in pages, positions scaled for long contexts
        _rope("rope_step", "rope_step_batch_e4m3", B=256, L=2, N=512, page=64, dtype="e4m3", scaling="ramp", far=100000),
        # ragged prompts of three loops in 32 bits, neighbouring pairs, a quarter of each head
        _rope("rope_seq", "rope_seq_ragged_f32", B=5, L=3, Hq=12, Hkv=4, d=64, N=701, dtype="f32", rd=16, layout="interleaved", norm=False),
        # long prompts of two loops into a cache in pages
        _rope("rope_seq", "rope_seq_long", B=2, L=2, N=8192, page=64, scaling="wavelength", ragged=False),
        # one user, three drafts
        dict(op="verify", name="verify_one", dtype="f32", B=1, K=3, V=32768, probs=True, ragged=False),
        # drafts without probabilities (copied from the prompt), an odd vocabulary in 16 bits
        dict(op="verify", name="verify_copied_bf16", dtype="bf16", B=48, K=7, V=50257, probs=False, ragged=True),
        # a large batch
        dict(op="verify", name="verify_batch", dtype="f32", B=256, K=4, V=131072, probs=True, ragged=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the same ranges: one token to long prefixes and prompts, small and odd batches, every type and layout."""
    op = rng.choice(["prefix", "prefix", "prefix", "rope_step", "rope_seq", "verify"])
    if op == "verify":
        V, K = _log(rng, 50, 131072), rng.choice([1, 2, 3, 4, 7, 8])
        return dict(op=op, name="drawn", dtype=rng.choice(["f32", "f32", "bf16"]), B=_log(rng, 1, max(1, min(256, 256 * 131072 * 5 // (V * (K + 1))))), K=K, V=V,
                    probs=rng.random() < 0.7, ragged=rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "e4m3"] if op == "prefix" else ["bf16", "bf16", "f32", "e4m3"])
    d = 128 if dtype == "e4m3" else rng.choice([64, 128, 128])
    L, Hkv, G = rng.choice([1, 1, 2, 3]), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 8])
    page, ragged = rng.choice([0, 0, 32, 64]), rng.random() < 0.6
    q_len = rng.choice([1, 1, 2, 4]) if (op == "prefix" or L == 1) and op != "rope_seq" else 1
    while L * q_len * G > 64:
        G -= 1
    w = rng.choice([16, 64, 200])
    if op == "prefix":
        P, N = _log(rng, 1, 32768), _log(rng, 1, 2048)
        rows = L * q_len * Hkv * G
        B = _log(rng, 1, max(1, min(200, 128 * 64 * 32768 // (max(P, 128) * rows), (1 << 28) // (N * Hkv * d))))
        groups = rng.choice([1, 1, 2, 4])
        return _prefix("drawn", dtype=dtype, B=B, L=L, Hq=Hkv * G, Hkv=Hkv, d=d, w=w, P=P, N=N, groups=min(groups, B), loose=rng.choice([0, 0, 1]) if B > groups else 0,
                       page=page, q_len=q_len, ragged=ragged)
    more = dict(dtype=dtype, L=L, Hq=Hkv * G, Hkv=Hkv, d=d, w=w, page=page, q_len=q_len, ragged=ragged, rd=rng.choice([16, 32, d // 2, d, d]),
                layout=rng.choice(["half", "half", "interleaved"]), scaling=rng.choice(["none", "linear", "base", "wavelength", "ramp"]), norm=rng.random() < 0.6,
                far=rng.choice([0, 0, 1000, 1000000]))
    if op == "rope_step":
        N = _log(rng, 1, 4096)
        return _rope(op, "drawn", B=_log(rng, 1, max(1, min(256, (1 << 28) // (N * Hkv * d)))), N=max(N, q_len), **more)
    N = _log(rng, 1, 8192)
    return _rope(op, "drawn", B=_log(rng, 1, max(1, min(64, 2 * 2 * 8192 * 40 // (N * L * Hkv * (G + 1))))), N=N, **more)


# ---- inputs -------------------------------------------------------------------------------------------------------
THETA, NORM_EPS = 500000.0, 1e-6
#: positions trained on, the stretch beyond them, and the two limits of each scaling
SCALING = {"none": dict(), "linear": dict(factor=4.0), "base": dict(factor=4.0), "wavelength": dict(factor=8.0, low=1.0, high=4.0, original_len=8192),
           "ramp": dict(factor=16.0, low=1.0, high=32.0, original_len=4096, attn_factor=0.1 * math.log(16.0) + 1.0)}


def _lengths(case, seed):
    """Own tokens of each sequence: all N, or spread log-uniformly over a factor of 64, the longest and a single token among
    them; another seed gives the same lengths to other sequences. A step has at least its own tokens."""
    B, N, least = case["B"], case["N"], min(case["N"], case["q_len"])
    if not case["ragged"]:
        return np.full(B, N, dtype=np.int32)
    lens = np.rint(np.exp(np.random.default_rng([B, N]).uniform(math.log(max(1.0, N / 64)), math.log(N), size=B))).astype(np.int32)
    lens[0] = N
    if B > 2:
        lens[1] = 1
    return np.random.default_rng([seed, 1]).permutation(np.clip(lens, least, N)).astype(np.int32)


def _groups(case):
    """(first sequence of each group and the end of the last, tokens of each prefix): groups of unequal sizes, prefixes from P
    down to a third of it; the last `loose` sequences have none."""
    n, G = case["B"] - case["loose"], case["groups"]
    shares = np.cumsum([0.0] + [1.0 / (g + 1) for g in range(G)])
    begin = np.rint(shares / shares[-1] * n).astype(np.int32)
    return begin, np.array([max(1, round(case["P"] * (1.0 - 2.0 * g / (3.0 * G)))) for g in range(G)], dtype=np.int32)


def _random(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _act(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _codes(x, scale):
    return torch.clamp(x / scale.view(-1, 1), -448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _rows(gen, shape, case, scale):
    x = _random(gen, *shape)
    return _codes(x, scale) if scale is not None else x.to(_act(case))


def _cap(case):
    page = case["page"]
    return -(-case["N"] // page) * page if page else case["N"]


def _pages(case, tokens):
    return -(-tokens // case["page"])


def _cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _verify_inputs(case, gen):
    B, K, V = case["B"], case["K"], case["V"]
    kind = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    s = {"case": case}
    logits = _random(gen, B, K + 1, V) * 2.5
    target = torch.softmax(logits, dim=-1)
    # a small model's view of the same context: near the target's, not equal to it
    logits = logits[:, :K] + 0.7 * _random(gen, B, K, V)
    draft = torch.softmax(logits, dim=-1)
    noise = torch.rand(B, K, V, generator=gen, device="cuda").clamp_(min=1e-20)
    s["draft_tokens"] = torch.argmax(logits - torch.log(-torch.log(noise)), dim=-1).to(torch.int32)
    s["target"] = target.to(kind)
    s["draft"] = draft.to(kind) if case["probs"] else None
    s["accept_u"] = torch.rand(B, K, generator=gen, device="cuda")
    s["sample_u"] = torch.rand(B, generator=gen, device="cuda")
    s["draft_lens"] = torch.randint(0, K + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if case["ragged"] else None
    s["seq_lens"] = torch.randint(K + 1, 5000, (B,), generator=gen, device="cuda", dtype=torch.int32)
    s["tokens"] = torch.empty(B, K + 1, dtype=torch.int32, device="cuda")
    s["accepted"] = torch.empty(B, dtype=torch.int32, device="cuda")
    s["new_lens"] = torch.empty(B, dtype=torch.int32, device="cuda")
    return s


def _inputs(case, seed):
    """Every tensor of a call, from the seed alone."""
    gen = torch.Generator("cuda").manual_seed(seed)
    op, B = case["op"], case["B"]
    if op == "verify":
        return _verify_inputs(case, gen)
    L, Hq, Hkv, d, Qn, page = case["L"], case["Hq"], case["Hkv"], case["d"], case["q_len"], case["page"]
    s = {"case": case}
    s["k_scale"], s["v_scale"] = ((torch.rand(Hkv, generator=gen, device="cuda") * 0.01 + 0.005) for _ in range(2)) if case["dtype"] == "e4m3" else (None, None)
    lens = _lengths(case, seed)
    own_pages = 0
    if page:
        per = _cap(case) // page
        own_pages = B * per
        extra = case["groups"] * _pages(case, case["P"]) if op == "prefix" else 0
        s["pool_pages"] = own_pages + extra + 3
        table = torch.randperm(s["pool_pages"], generator=gen, device="cuda").to(torch.int32)
        s["page_table"] = table[:own_pages].view(B, per).contiguous()
    shape = (s["pool_pages"], page, Hkv, d) if page else (B, case["N"], Hkv, d)
    s["k_cache"], s["v_cache"] = _rows(gen, shape, case, s["k_scale"]), _rows(gen, shape, case, s["v_scale"])
    if L > 1 and op != "rope_seq":
        s["k_win"], s["v_win"] = (_rows(gen, (B, L - 1, case["w"], Hkv, d), case, x) for x in (s["k_scale"], s["v_scale"]))
    if op == "prefix":
        s["q"] = (_random(gen, B, L, Qn, Hq, d) * 1.5).to(_act(case))
        begin, plens = _groups(case)
        s["group_begin"], s["prefix_lens"] = _cuda(begin), _cuda(plens)
        tokens = lens.astype(np.int64)
        for g, n in enumerate(plens):
            tokens[begin[g]:begin[g + 1]] += n
        s["seq_lens"] = _cuda(tokens.astype(np.int32))
        if page:
            per = _pages(case, case["P"])
            s["prefix_table"] = table[own_pages:own_pages + case["groups"] * per].view(case["groups"], per).contiguous()
            s["k_prefix"] = s["v_prefix"] = None
        else:
            s["k_prefix"], s["v_prefix"] = (_rows(gen, (case["groups"], case["P"], Hkv, d), case, x) for x in (s["k_scale"], s["v_scale"]))
        if L > 1:
            s["gate_logits"] = _random(gen, B, L - 1, Qn, Hq)
        s["out"] = torch.empty_like(s["q"])
        return s
    rows = case["N"] if op == "rope_seq" else Qn
    act = _act(case)
    s["q"] = (_random(gen, B, L, rows, Hq, d) * 1.5).to(act)
    s["q_gain"], s["k_gain"] = ((1.0 + 0.1 * _random(gen, d)) for _ in range(2)) if case["norm"] else (None, None)
    s["q_out"] = torch.empty_like(s["q"])
    # tokens in front of the ones of this cache: a shared prefix, or an earlier part of a document
    s["before"] = torch.full((B,), case["far"], dtype=torch.int32, device="cuda")
    if op == "rope_step":
        s["k_new"], s["v_new"] = (_random(gen, B, L, Qn, Hkv, d).to(act) for _ in range(2))
        s["seq_lens"] = _cuda((lens.astype(np.int64) + case["far"]).astype(np.int32))
        if L > 1:
            s["w_gate"], s["b_gate"] = 0.1 * _random(gen, Hq, d), 0.1 * _random(gen, Hq)
            s["gate_logits"] = torch.empty(B, L - 1, Hq, device="cuda")
        return s
    s["seq_lens"] = _cuda(lens)
    s["k_share"], s["v_share"] = (_random(gen, B, rows, Hkv, d).to(act) for _ in range(2))
    s["q_out"].zero_()
    if L > 1:
        s["k_loc"] = _random(gen, B, L - 1, rows, Hkv, d).to(act)
        s["k_loc_out"] = torch.zeros_like(s["k_loc"])
    return s


_handles = {}


def _bind(s):
    """The handle (one for each configuration, as a program keeps it) and the argument structs of the call."""
    from paper_2510_24824_b200 import binding as P
    case = s["case"]
    op, B = case["op"], case["B"]
    key = (op,) + tuple(case[k] for k in sorted(case) if k not in ("name", "ragged", "loose", "far", "probs"))
    fresh = key not in _handles
    if op == "verify":
        if fresh:
            _handles[key] = P.plt_draft_verify_create(P.make_verify_config(case["dtype"], B, case["K"], case["V"]))
        args = P.make_verify_args(B, s["target"], s["draft_tokens"], s["accept_u"], s["sample_u"], s["tokens"], s["accepted"], draft_probs=s["draft"],
                                  draft_lens=s["draft_lens"], seq_lens=s["seq_lens"], new_lens=s["new_lens"])
        s["call"] = (P.plt_draft_verify_run, _handles[key], args)
        return s
    dt, kv = ("bf16", "e4m3") if case["dtype"] == "e4m3" else (case["dtype"], "")
    w = case["w"] if case["L"] > 1 else 0
    sizes = (dt, B, case["L"], case["Hq"], case["Hkv"], case["d"], _cap(case), w)
    pages = dict(page_table=s["page_table"], max_pages=s["page_table"].shape[1], num_pool_pages=s["pool_pages"]) if case["page"] else {}
    if op == "prefix":
        if fresh:
            _handles[key] = P.plt_prefix_attn_create(P.make_prefix_config(*sizes, max_prefix_len=case["P"], max_groups=case["groups"], page_size=case["page"],
                                                                          kv_dtype=kv, q_len=case["q_len"]))
        args = P.make_args(B, s["q"], s["k_cache"], s["v_cache"], s["seq_lens"], s["out"], k_win=s.get("k_win"), v_win=s.get("v_win"),
                           gate_logits=s.get("gate_logits"), k_scale=s["k_scale"], v_scale=s["v_scale"], **pages)
        table = dict(page_table=s["prefix_table"], max_pages=s["prefix_table"].shape[1]) if case["page"] else {}
        shared = P.make_prefix_args(case["groups"], s["group_begin"], s["prefix_lens"], k_prefix=s["k_prefix"], v_prefix=s["v_prefix"], **table)
        s["call"] = (P.plt_prefix_attn_run, _handles[key], args, shared)
        return s
    if fresh:
        _handles[key] = P.plt_rope_create(P.make_rope_config(*sizes, page_size=case["page"], kv_dtype=kv, q_len=case["q_len"], rotary_dim=case["rd"],
                                                             layout=case["layout"], theta=THETA, scaling=case["scaling"], norm_eps=NORM_EPS, **SCALING[case["scaling"]]))
    both = dict(q_gain=s["q_gain"], k_gain=s["k_gain"], prefix_lens=s["before"], k_scale=s["k_scale"], v_scale=s["v_scale"], **pages)
    if op == "rope_step":
        args = P.make_rope_step_args(B, s["q"], s["k_new"], s["v_new"], s["q_out"], s["k_cache"], s["v_cache"], s["seq_lens"], k_win=s.get("k_win"), v_win=s.get("v_win"),
                                     w_gate=s.get("w_gate"), b_gate=s.get("b_gate"), gate_logits=s.get("gate_logits"), **both)
        s["call"] = (P.plt_rope_step, _handles[key], args)
    else:
        args = P.make_rope_seq_args(B, case["N"], s["q"], s["k_share"], s["seq_lens"], s["q_out"], k_loc=s.get("k_loc"), k_loc_out=s.get("k_loc_out"), start=s["before"],
                                    v_share=s["v_share"], k_cache=s["k_cache"], v_cache=s["v_cache"], **both)
        s["call"] = (P.plt_rope_seq, _handles[key], args)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    return _bind(s) if own else s


# ---- plain forms --------------------------------------------------------------------------------------------------
def _values(x, scale, table=None, dtype=torch.float32):
    """Cache rows as values, through a page table where there is one: [sequences, tokens, Hkv, d]."""
    if table is not None:
        x = x[table.long()].flatten(1, 2)
    x = x.view(torch.float8_e4m3fn).to(dtype) if x.dtype == torch.uint8 else x.to(dtype)
    return x if scale is None else x * scale.to(dtype).view(-1, 1)


def _partial(x, seen, v, eq):
    """Of scores x where `seen`: their maximum, sum of exp(x - maximum), and that sum's weighted values."""
    x = torch.where(seen, x, -math.inf)
    top = x.amax(dim=-1)
    e = torch.exp(x - torch.where(top > -math.inf, top, 0.0).unsqueeze(-1))
    return top, e.sum(dim=-1), torch.einsum(eq, e, v)


def _plain_prefix(s):
    case = s["case"]
    B, L, Qn, Hkv, d = case["B"], case["L"], case["q_len"], case["Hkv"], case["d"]
    q = s["q"].float().unflatten(3, (Hkv, -1)) / math.sqrt(d)                      # [B, L, Qn, Hkv, G, d]
    # tokens that each row sees, and how many of them the prefix holds
    n = s["seq_lens"].long().view(-1, 1, 1)
    loop = torch.arange(L, device="cuda").view(1, -1, 1)
    newer = torch.arange(Qn - 1, -1, -1, device="cuda").view(1, 1, -1)
    cut = (n - loop - newer).clamp(min=0)
    at = torch.arange(B, device="cuda")
    group = (at.view(-1, 1) >= s["group_begin"][1:].view(1, -1)).sum(dim=1)         # the number of groups: none
    inside = group < case["groups"]
    group = group.clamp(max=case["groups"] - 1)
    plen = torch.where(inside, s["prefix_lens"].long()[group], 0).view(-1, 1, 1)
    # the prefixes, each against the queries of all its sequences
    most = int(_groups(case)[0][1:].max() if case["groups"] == 1 else np.diff(_groups(case)[0]).max())
    member = s["group_begin"].long()[:-1].view(-1, 1) + torch.arange(most, device="cuda")
    member = member.clamp(max=B - 1)                                                # [groups, most]
    pages = case["page"] > 0
    kp = _values(s["k_cache"] if pages else s["k_prefix"], s["k_scale"], s.get("prefix_table"))
    vp = _values(s["v_cache"] if pages else s["v_prefix"], s["v_scale"], s.get("prefix_table"))
    key = torch.arange(kp.shape[1], device="cuda")
    vp = torch.where((key.view(1, -1) < s["prefix_lens"].view(-1, 1))[:, :, None, None], vp, 0.0)
    seen = key < torch.minimum(cut, plen)[member].unsqueeze(-1)                     # [groups, most, L, Qn, P]
    x = torch.einsum("gblrhxd,gnhd->gblrhxn", q[member], kp)
    place = (at - s["group_begin"].long()[group]).clamp(0, most - 1)
    top1, sum1, y1 = (t[group, place] for t in _partial(x, seen[:, :, :, :, None, None], vp, "gblrhxn,gnhd->gblrhxd"))
    del x
    has = inside.view(-1, 1, 1, 1, 1)
    top1, sum1, y1 = torch.where(has, top1, -math.inf), torch.where(has, sum1, 0.0), torch.where(has.unsqueeze(-1), y1, 0.0)
    # what each sequence holds itself
    k, v = _values(s["k_cache"], s["k_scale"], s.get("page_table")), _values(s["v_cache"], s["v_scale"], s.get("page_table"))
    key = torch.arange(k.shape[1], device="cuda")
    v = torch.where((key.view(1, -1) < (n - plen).view(-1, 1))[:, :, None, None], v, 0.0)
    seen = key < (cut - plen).unsqueeze(-1)
    top2, sum2, y2 = _partial(torch.einsum("blrhxd,bnhd->blrhxn", q, k), seen[:, :, :, None, None], v, "blrhxn,bnhd->blrhxd")
    top = torch.maximum(top1, top2)
    top = torch.where(top > -math.inf, top, 0.0)
    a, b = torch.exp(top1 - top), torch.exp(top2 - top)
    total = a * sum1 + b * sum2
    y = (a.unsqueeze(-1) * y1 + b.unsqueeze(-1) * y2) / torch.where(total > 0, total, 1.0).unsqueeze(-1)
    if L > 1:
        kw, vw = _values(s["k_win"], s["k_scale"]), _values(s["v_win"], s["v_scale"])
        wl = ((n - loop).clamp(0, case["w"]) - newer)[:, 1:]
        seen = torch.arange(case["w"], device="cuda") < wl.unsqueeze(-1)
        _, total, near = _partial(torch.einsum("blrhxd,blnhd->blrhxn", q[:, 1:], kw), seen[:, :, :, None, None], vw, "blrhxn,blnhd->blrhxd")
        near = near / torch.where(total > 0, total, 1.0).unsqueeze(-1)
        g = torch.sigmoid(s["gate_logits"]).unflatten(-1, (Hkv, -1)).unsqueeze(-1)
        y = torch.cat([y[:, :1], g * near + (1.0 - g) * y[:, 1:]], dim=1)
    y = torch.where((cut > 0).view(B, L, Qn, 1, 1, 1), y, 0.0)
    return y.flatten(3, 4).to(s["q"].dtype)


def _frequencies(case):
    """Radians a position for each rotated pair, [rd / 2] in 64 bits."""
    rd, more = case["rd"], SCALING[case["scaling"]]
    at = torch.arange(0, rd, 2, dtype=torch.float64, device="cuda") / rd
    f = THETA ** -at
    if case["scaling"] == "linear":
        return f / more["factor"]
    if case["scaling"] == "base":
        return (THETA * more["factor"] ** (rd / (rd - 2))) ** -at
    if case["scaling"] == "wavelength":
        turns = more["original_len"] * f / (2 * math.pi)
        keep = ((turns - more["low"]) / (more["high"] - more["low"])).clamp(0.0, 1.0)
        return f * keep + f / more["factor"] * (1 - keep)
    if case["scaling"] == "ramp":
        pair = [rd * math.log(more["original_len"] / (t * 2 * math.pi)) / (2 * math.log(THETA)) for t in (more["high"], more["low"])]
        first, last = max(math.floor(pair[0]), 0), min(math.ceil(pair[1]), rd - 1)
        far = ((torch.arange(rd // 2, dtype=torch.float64, device="cuda") - first) / max(last - first, 0.001)).clamp(0.0, 1.0)
        return f / more["factor"] * far + f * (1 - far)
    return f


def _rotated(x, at, gain, case, dtype=torch.float32):
    """Rows x [..., heads, d] normed and turned to the positions `at` [...]."""
    x = x.to(dtype)
    if gain is not None:
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + NORM_EPS) * gain.to(dtype)
    rd = case["rd"]
    angle = at.double().unsqueeze(-1) * _frequencies(case)
    factor = SCALING[case["scaling"]].get("attn_factor", 1.0)
    c, sn = ((t * factor).to(dtype).unsqueeze(-2) for t in (torch.cos(angle), torch.sin(angle)))
    a, b = (x[..., : rd // 2], x[..., rd // 2: rd]) if case["layout"] == "half" else (x[..., 0:rd:2], x[..., 1:rd:2])
    a, b = a * c - b * sn, b * c + a * sn
    turned = torch.cat([a, b], dim=-1) if case["layout"] == "half" else torch.stack([a, b], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., rd:]], dim=-1)


def _stored(x, cache, scale):
    """Values as the cache holds them."""
    return _codes(x, scale) if cache.dtype == torch.uint8 else x.to(cache.dtype)


def _cell(s, b, at):
    """Row of the flattened cache that position `at` of sequence b has."""
    page = s["case"]["page"]
    return s["page_table"].long()[b, at // page] * page + at % page if page else b * s["case"]["N"] + at


def _seen(x):
    return x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x


def _step_outputs(s):
    out = [s["q_out"], _seen(s["k_cache"]), _seen(s["v_cache"])]
    return out + ([_seen(s["k_win"]), _seen(s["v_win"]), s["gate_logits"]] if s["case"]["L"] > 1 else [])


def _plain_rope_step(s):
    case = s["case"]
    B, L, Qn, Hkv, d = case["B"], case["L"], case["q_len"], case["Hkv"], case["d"]
    loop = torch.arange(L, device="cuda").view(1, -1, 1)
    newer = torch.arange(Qn - 1, -1, -1, device="cuda").view(1, 1, -1)
    at = s["seq_lens"].long().view(-1, 1, 1) - loop - newer - 1                    # [B, L, Qn] positions
    q = torch.where((at >= 0)[..., None, None], _rotated(s["q"], at, s["q_gain"], case), 0.0)
    s["q_out"].copy_(q)
    k = _stored(_rotated(s["k_new"], at, s["k_gain"], case), s["k_cache"], s["k_scale"])
    v = _stored(s["v_new"].float(), s["v_cache"], s["v_scale"])
    place = at[:, 0] - s["before"].long().view(-1, 1)
    b, j = (place >= 0).nonzero(as_tuple=True)
    cell = _cell(s, b, place[b, j])
    s["k_cache"].view(-1, Hkv, d)[cell] = k[b, 0, j]
    s["v_cache"].view(-1, Hkv, d)[cell] = v[b, 0, j]
    if L > 1:
        b, l = (at[:, 1:, 0] >= 0).nonzero(as_tuple=True)
        slot = at[b, l + 1, 0] % case["w"]
        s["k_win"][b, l, slot] = k[b, l + 1, 0]
        s["v_win"][b, l, slot] = v[b, l + 1, 0]
        s["gate_logits"].copy_((q[:, 1:, 0] * s["w_gate"]).sum(dim=-1) + s["b_gate"])
    return _step_outputs(s)


def _seq_outputs(s):
    return [s["q_out"], _seen(s["k_cache"]), _seen(s["v_cache"])] + ([s["k_loc_out"]] if s["case"]["L"] > 1 else [])


def _plain_rope_seq(s):
    case = s["case"]
    L, T, Hkv, d = case["L"], case["N"], case["Hkv"], case["d"]
    t = torch.arange(T, device="cuda")
    at = s["before"].long().view(-1, 1, 1) + t - torch.arange(L, device="cuda").view(1, -1, 1)      # [B, L, T]
    live = (at >= 0) & (t < s["seq_lens"].view(-1, 1, 1))
    s["q_out"].copy_(torch.where(live[..., None, None], _rotated(s["q"], at, s["q_gain"], case).to(s["q"].dtype), s["q_out"]))
    if L > 1:
        s["k_loc_out"].copy_(torch.where(live[:, 1:, :, None, None], _rotated(s["k_loc"], at[:, 1:], s["k_gain"], case).to(s["q"].dtype), s["k_loc_out"]))
    b, i = (t < s["seq_lens"].view(-1, 1)).nonzero(as_tuple=True)
    cell = _cell(s, b, i)
    s["k_cache"].view(-1, Hkv, d)[cell] = _stored(_rotated(s["k_share"], at[:, 0], s["k_gain"], case), s["k_cache"], s["k_scale"])[b, i]
    s["v_cache"].view(-1, Hkv, d)[cell] = _stored(s["v_share"].float(), s["v_cache"], s["v_scale"])[b, i]
    return _seq_outputs(s)


def _plain_verify(s):
    case = s["case"]
    B, K = case["B"], case["K"]
    at = torch.arange(K, device="cuda")
    drafts = s["draft_tokens"].long()
    p = s["target"][:, :K].gather(2, drafts.unsqueeze(-1)).squeeze(-1).double()
    q = s["draft"].gather(2, drafts.unsqueeze(-1)).squeeze(-1).double() if case["probs"] else torch.ones_like(p)
    held = s["draft_lens"].long() if case["ragged"] else torch.full((B,), K, device="cuda")
    passed = (s["accept_u"].double() * q < p) & (at < held.view(-1, 1))
    n = torch.cumprod(passed.long(), dim=1).sum(dim=1)
    row = torch.arange(B, device="cuda")
    p = s["target"][row, n].double()
    cut = (n < held).view(-1, 1)                                                    # a draft was refused
    last = n.clamp(max=K - 1)
    if case["probs"]:
        rest = (p - s["draft"][row, last].double()).clamp(min=0.0)
    else:
        rest = p.scatter(1, drafts[row, last].view(-1, 1), 0.0)
    rest = torch.where(cut & (rest.sum(dim=1, keepdim=True) > 0), rest, p)
    total = torch.cumsum(rest, dim=1)
    past = total > s["sample_u"].double().view(-1, 1) * total[:, -1:]
    vocab = torch.arange(case["V"], device="cuda")
    token = torch.where(past.any(dim=1), torch.argmax(past.to(torch.int8), dim=1), torch.where(rest > 0, vocab, -1).amax(dim=1))
    out = torch.where(at < n.view(-1, 1), drafts, -1)
    s["tokens"].copy_(torch.cat([out, torch.full_like(out[:, :1], -1)], dim=1).scatter(1, n.view(-1, 1), token.view(-1, 1)))
    s["accepted"].copy_(n)
    s["new_lens"].copy_((s["seq_lens"] - (K - n)).clamp(min=0))
    return s["tokens"], s["accepted"], s["new_lens"]


def run(s):
    op = s["case"]["op"]
    if own:
        call = s["call"]
        call[0](*call[1:], torch.cuda.current_stream().cuda_stream)
        if op == "prefix":
            return s["out"]
        if op == "verify":
            return s["tokens"], s["accepted"], s["new_lens"]
        return _step_outputs(s) if op == "rope_step" else _seq_outputs(s)
    return {"prefix": _plain_prefix, "rope_step": _plain_rope_step, "rope_seq": _plain_rope_seq, "verify": _plain_verify}[op](s)


# ---- cost ---------------------------------------------------------------------------------------------------------
def work(case):
    """Bytes: every input that the result needs read once and every output written once. Flops: the products over the keys
    that are seen."""
    op, B = case["op"], case["B"]
    if op == "verify":
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": float(B) * case["V"] * size * (2 if case["probs"] else 1) + 4.0 * B * (5 * case["K"] + 8), "flops": 0}
    es = {"bf16": 2, "f32": 4, "e4m3": 1}[case["dtype"]]
    qb = 4 if case["dtype"] == "f32" else 2
    L, Hq, Hkv, d, Qn = case["L"], case["Hq"], case["Hkv"], case["d"], case["q_len"]
    lens = _lengths(case, 1).astype(np.float64)
    if op == "prefix":
        begin, plens = _groups(case)
        prefix, shared = float(plens.sum()), float((np.diff(begin) * plens).sum())
        tokens = float(lens.sum())
        slots = float(B) * case["w"] * (L - 1)
        bytes_ = (prefix + tokens + slots) * Hkv * d * 2 * es + 2.0 * B * L * Qn * Hq * d * qb + 4.0 * B * (L - 1) * Qn * Hq
        return {"bytes": bytes_, "flops": 4.0 * ((shared + tokens) * L + slots) * Qn * Hq * d}
    if op == "rope_step":
        rows = float(B) * L * Qn
        return {"bytes": rows * d * (2.0 * Hq * qb + 2.0 * Hkv * (qb + es)) + 4.0 * B * (L - 1) * Hq + (4.0 * Hq * d if L > 1 else 0.0), "flops": 0}
    rows = float(lens.sum())
    return {"bytes": rows * d * (2.0 * L * Hq * qb + 2.0 * (L - 1) * Hkv * qb + 2.0 * Hkv * (qb + es)), "flops": 0}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def _real(x, scale, h):
    x = x.view(torch.float8_e4m3fn).double() if x.dtype == torch.uint8 else x.double()
    return x if scale is None else x * float(scale[h])


def _exact_prefix(s):
    case, out = s["case"], torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    B, L, Qn, Hq, d = out.shape
    G, page, scale = Hq // case["Hkv"], case["page"], case["d"] ** -0.5
    begin, plens = _groups(case)
    group = [next((g for g in range(case["groups"]) if begin[g] <= b < begin[g + 1]), -1) for b in range(B)]
    every = s["seq_lens"].tolist()
    for h in range(case["Hkv"]):
        heads = slice(h * G, (h + 1) * G)
        held = {}
        for g, n in enumerate(plens):
            if page:
                at = torch.arange(n, device="cuda")
                cells = s["prefix_table"][g].long()[at // page], at % page
                k, v = s["k_cache"][cells[0], cells[1], h], s["v_cache"][cells[0], cells[1], h]
            else:
                k, v = s["k_prefix"][g, :n, h], s["v_prefix"][g, :n, h]
            k, v = _real(k, s["k_scale"], h), _real(v, s["v_scale"], h)
            if begin[g + 1] > begin[g]:
                held[g] = (k, v, s["q"][begin[g]:begin[g + 1], :, :, heads].double() @ k.T * scale)
        for b in range(B):
            g, n = group[b], every[b]
            own_n = n - (int(plens[g]) if g >= 0 else 0)
            at = torch.arange(own_n, device="cuda")
            k, v = ((x[s["page_table"][b].long()[at // page], at % page, h] if page else x[b, :own_n, h]) for x in (s["k_cache"], s["v_cache"]))
            k, v = _real(k, s["k_scale"], h), _real(v, s["v_scale"], h)
            q = s["q"][b, :, :, heads].double()                                     # [L, Qn, G, d]
            x = q @ k.T * scale
            if g >= 0:
                x, v = torch.cat([held[g][2][b - int(begin[g])], x], dim=-1), torch.cat([held[g][1], v])
            cut = n - torch.arange(L, device="cuda").view(-1, 1) - torch.arange(Qn - 1, -1, -1, device="cuda").view(1, -1)
            hidden = torch.arange(n, device="cuda") >= cut[:, :, None, None]
            y = torch.nan_to_num(torch.softmax(x.masked_fill(hidden, -math.inf), dim=-1)) @ v
            if L > 1:
                kw, vw = _real(s["k_win"][b, :, :, h], s["k_scale"], h), _real(s["v_win"][b, :, :, h], s["v_scale"], h)
                slots = (n - torch.arange(1, L, device="cuda")).clamp(0, case["w"]).view(-1, 1) - torch.arange(Qn - 1, -1, -1, device="cuda").view(1, -1)
                x = torch.einsum("lrxd,lnd->lrxn", q[1:], kw) * scale
                x = x.masked_fill(torch.arange(case["w"], device="cuda") >= slots[:, :, None, None], -math.inf)
                near = torch.einsum("lrxn,lnd->lrxd", torch.nan_to_num(torch.softmax(x, dim=-1)), vw)
                gate = torch.sigmoid(s["gate_logits"][b, :, :, heads].double()).unsqueeze(-1)
                y[1:] = gate * near + (1 - gate) * y[1:]
            out[b, :, :, heads] = torch.where((cut > 0)[:, :, None, None], y, 0.0)
    return out


def _turn64(x, at, gain, case):
    """_rotated's result from its definition, a pair as a complex number."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x ** 2).mean(dim=-1, keepdim=True) + NORM_EPS) * gain.double()
    rd, half = case["rd"], case["rd"] // 2
    first, second = (slice(0, half), slice(half, rd)) if case["layout"] == "half" else (slice(0, rd, 2), slice(1, rd, 2))
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous())
    angle = at.double()[..., None, None] * _frequencies(case)
    z = z * torch.polar(torch.full_like(angle, SCALING[case["scaling"]].get("attn_factor", 1.0)), angle)
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _held64(x, cache, scale):
    """What the cache holds of a value, in 64 bits: a code's value, or the value."""
    return torch.clamp(x / scale.double().view(-1, 1), -448.0, 448.0).to(torch.float8_e4m3fn).double() if cache.dtype == torch.uint8 else x


def _exact_rope(s):
    case = s["case"]
    B, L, rows = s["q"].shape[:3]
    seq, page = case["op"] == "rope_seq", case["page"]
    q, caches = s["q_out"].double() if seq else torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), [_seen(s[n]).double() for n in ("k_cache", "v_cache")]
    wins = [_seen(s[n]).double() for n in ("k_win", "v_win")] if L > 1 and not seq else []
    local = s["k_loc_out"].double() if L > 1 and seq else None
    for b in range(B):
        n, far = int(s["seq_lens"][b]), case["far"]
        for l in range(L):
            if seq:
                r = torch.arange(min(max(0, l - far), n), n, device="cuda")
                at = far + r - l
            else:
                at = n - l - torch.arange(rows, 0, -1, device="cuda")
                r = torch.arange(rows, device="cuda")[at >= 0]
                at = at[at >= 0]
            if not len(r):
                continue
            q[b, l, r] = _turn64(s["q"][b, l, r], at, s["q_gain"], case)
            if l == 0:
                k, v = ((s["k_share"], s["v_share"]) if seq else (s["k_new"][:, 0], s["v_new"][:, 0]))
                place = at - far
                r, at, place = r[place >= 0], at[place >= 0], place[place >= 0]
                cell = (s["page_table"][b].long()[place // page], place % page) if page else (b, place)
                caches[0][cell] = _held64(_turn64(k[b, r], at, s["k_gain"], case), s["k_cache"], s["k_scale"])
                caches[1][cell] = _held64(v[b, r].double(), s["v_cache"], s["v_scale"])
            elif seq:
                local[b, l - 1, r] = _turn64(s["k_loc"][b, l - 1, r], at, s["k_gain"], case)
            else:
                wins[0][b, l - 1, at % case["w"]] = _held64(_turn64(s["k_new"][b, l, r], at, s["k_gain"], case), s["k_win"], s["k_scale"])
                wins[1][b, l - 1, at % case["w"]] = _held64(s["v_new"][b, l, r].double(), s["v_win"], s["v_scale"])
    out = [q] + caches + wins
    if local is not None:
        out.append(local)
    if wins:
        out.append((q[:, 1:, 0] * s["w_gate"].double()).sum(dim=-1) + s["b_gate"].double())
    return out


def exact(case, seed):
    if case["op"] == "verify":
        return None                                   # tokens and counts: whole numbers
    s = _inputs(case, seed)
    return _exact_prefix(s) if case["op"] == "prefix" else _exact_rope(s)

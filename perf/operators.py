"""The measured calls of differential attention and of cache eviction: their inputs, their plain forms and their cost.

Five operators, all on the caches of the decode-step attention (K and V rows of d elements per KV head, contiguous or in
pages, bf16, fp32 or E4M3 codes):

  diff_step    one decode step of differential attention: the difference of two softmax maps, one on each half of the
               query and key rows, with a learned factor and a norm for each head
  diff_prompt  the same for every row of a prompt at once
  weights      adds to a running total the attention weight that a step's queries give each cached key
  select       the positions of a cache to keep under a budget, by that total
  compact      moves the kept rows (and their totals) to the front of the cache

`run` computes them in elementary torch operations in fp32, or, where `own` is true, through the framework's entry points.
"""
import math

import numpy as np
import torch

own = False

GIB = 1 << 30


# ---- cases --------------------------------------------------------------------------------------------------------
def _attn(op, name, **kw):
    case = dict(op=op, name=name, dtype="bf16", B=1, L=1, Hq=32, Hkv=8, d=128, w=64, N=4096, page=0, q_len=1, ragged=False)
    case.update(kw)
    return case


def listed():
    return [
        # a chat turn of one user: one sequence, a short cache; latency is all there is
        _attn("diff_step", "diff_step_one", N=300, norm=True, lambda_heads=1),
        # the decode batch of the parallel loop configuration: two loops, windows, gate
        _attn("diff_step", "diff_step_batch", B=64, L=2, N=4096, norm=True, lambda_heads=1),
        # a serving mix in pages of 64 tokens with 8-bit caches, lengths from 1 token up
        _attn("diff_step", "diff_step_paged_e4m3", B=96, N=16384, Hkv=4, dtype="e4m3", page=64, ragged=True, norm=True, lambda_heads=32),
        # ragged short prompts of two loops
        _attn("diff_prompt", "diff_prompt_ragged", B=4, L=2, Hq=16, Hkv=4, N=701, ragged=True, norm=True, lambda_heads=1),
        # one prompt of the paper's prefill length
        _attn("diff_prompt", "diff_prompt_5000", N=5000, norm=True, lambda_heads=1),
        # one user's step
        _attn("weights", "weights_one", N=700, group=1, maps=1, gate=False, decay=1.0),
        # the decode batch with two loops, ragged
        _attn("weights", "weights_batch", B=64, L=2, N=8192, ragged=True, group=1, maps=1, gate=True, decay=1.0),
        # long caches of 8-bit codes in pages, the last four tokens' queries together, heads kept in pairs
        _attn("weights", "weights_long_e4m3", B=8, N=32768, q_len=4, dtype="e4m3", page=64, group=2, maps=1, gate=False, decay=0.5),
        # one sequence grown to 5000 tokens is cut to 1024
        dict(op="select", name="select_one", B=1, groups=8, N=5000, budget=1024, first=4, last=64, ragged=False),
        # a batch at long context
        dict(op="select", name="select_batch", B=48, groups=8, N=32768, budget=4096, first=4, last=128, ragged=True),
        # one sequence, contiguous cache
        dict(op="compact", name="compact_one", dtype="bf16", B=1, Hkv=8, d=128, N=5000, page=0, group=1, budget=1024, first=4, last=64, ragged=False),
        # the batch in pages
        dict(op="compact", name="compact_batch_paged", dtype="bf16", B=64, Hkv=8, d=128, N=8192, page=64, group=1, budget=4096, first=4, last=128, ragged=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the same ranges: one token to long caches, small and odd batches, every type and layout."""
    op = rng.choice(["diff_step", "diff_step", "diff_prompt", "weights", "weights", "select", "compact"])
    if op == "select":
        N, groups = _log(rng, 128, 65536), rng.choice([1, 2, 4, 8])
        B = _log(rng, 1, max(1, min(48, 8 * 32768 * 48 // (N * groups))))
        budget = _log(rng, N // 16, 3 * N // 4)
        first, last = rng.choice([0, 4]), rng.choice([1, 16, 64])
        return dict(op=op, B=B, groups=groups, N=N, budget=max(budget, first + last), first=first, last=last, ragged=rng.random() < 0.5)
    page = rng.choice([0, 0, 16, 64])
    if op == "compact":
        dtype, Hkv = rng.choice(["bf16", "bf16", "f32", "e4m3"]), rng.choice([1, 2, 4, 8])
        d = 128 if dtype == "e4m3" else rng.choice([64, 128])
        N = _log(rng, 100, 16384)
        es = {"bf16": 2, "f32": 4, "e4m3": 1}[dtype]
        B = _log(rng, 1, max(1, min(64, GIB // (N * Hkv * d * es))))
        first, last = rng.choice([0, 4]), rng.choice([1, 16, 64])
        budget = max(first + last, _log(rng, max(1, N // 16), N // 2))
        return dict(op=op, dtype=dtype, B=B, Hkv=Hkv, d=d, N=N, page=page, group=rng.choice([1, 1, Hkv]), budget=budget, first=first, last=last, ragged=rng.random() < 0.5)
    Hkv, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8])
    if op == "diff_prompt":
        N = _log(rng, 1, 3000)
        L = rng.choice([1, 1, 2, 3])
        B = _log(rng, 1, max(1, min(8, (5000 * 5000 * 32) // (N * N * L * Hkv * G * 2))))
        return _attn(op, "", B=B, L=L, Hq=Hkv * G, Hkv=Hkv, N=N, w=rng.choice([16, 64, 200]), ragged=rng.random() < 0.5, norm=rng.random() < 0.7,
                     lambda_heads=rng.choice([1, Hkv * G])) | {"name": "drawn"}
    dtype = rng.choice(["bf16", "bf16", "bf16", "e4m3", "f32"])
    d = 128 if dtype == "e4m3" else rng.choice([64, 128, 128])
    page = 32 if dtype == "e4m3" and page == 16 else page       # the attention on 8-bit caches takes pages of 32 tokens up
    L = rng.choice([1, 1, 2, 3])
    maps = 2 if op == "diff_step" else rng.choice([1, 1, 2])
    q_len = rng.choice([1, 1, 1, 2, 3]) if dtype != "f32" else 1
    while maps * L * q_len * G > 64:
        G //= 2
    N = _log(rng, 1, 32768)
    es = {"bf16": 2, "f32": 4, "e4m3": 1}[dtype]
    rows = maps * L * q_len * G
    # the caches and the plain form's scores stay below the largest listed case's
    most = min(GIB // 2 // (N * Hkv * d * es), 64 * 8192 * 8 * 8 // (N * Hkv * rows))
    B = _log(rng, 1, max(1, min(96, most)))
    case = _attn(op, "drawn", B=B, L=L, Hq=Hkv * G, Hkv=Hkv, d=d, w=rng.choice([16, 64, 200]), N=N, page=page, q_len=q_len, dtype=dtype, ragged=rng.random() < 0.5)
    if op == "diff_step":
        return case | dict(norm=rng.random() < 0.7, lambda_heads=rng.choice([1, Hkv * G]))
    return case | dict(group=rng.choice([1, 1, 2 if Hkv > 1 else 1, Hkv]), maps=maps, gate=rng.random() < 0.5, decay=rng.choice([0.0, 0.5, 1.0]) if N > 8 else 1.0)


# ---- inputs -------------------------------------------------------------------------------------------------------
LAMBDA_INIT, NORM_EPS = 0.8, 1e-5


def _lengths(case, seed):
    """Full caches, or lengths spread log-uniformly over a factor of 64, the longest and one of a single token among
    them; another seed gives the same lengths to other sequences."""
    B, N = case["B"], case["N"]
    if not case["ragged"]:
        return np.full(B, N, dtype=np.int32)
    lens = np.rint(np.exp(np.random.default_rng([B, N]).uniform(math.log(max(1.0, N / 64)), math.log(N), size=B))).astype(np.int32)
    lens[0] = N
    if B > 2:
        lens[1] = 1
    return np.random.default_rng([seed, 1]).permutation(np.clip(lens, 1, N)).astype(np.int32)


def _random(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _rows(gen, shape, dtype, heads_dim):
    """Cache rows: N(0, 1); as codes with a scale for each head where they are E4M3."""
    if dtype != "e4m3":
        return _random(gen, *shape).to(torch.bfloat16 if dtype == "bf16" else torch.float32), None
    scale = torch.rand(shape[heads_dim], generator=gen, device="cuda") * 0.01 + 0.005
    codes = torch.clamp(_random(gen, *shape) / scale.view(-1, 1), -448.0, 448.0).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), scale


def _cap(case):
    page = case.get("page", 0)
    return -(-case["N"] // page) * page if page else case["N"]


def _cache_shape(case):
    page = case.get("page", 0)
    return (case["B"] * (_cap(case) // page) + 3, page, case["Hkv"], case["d"]) if page else (case["B"], case["N"], case["Hkv"], case["d"])


def _inputs(case, seed):
    """Every tensor of a call, from the seed alone."""
    gen = torch.Generator("cuda").manual_seed(seed)
    op, B = case["op"], case["B"]
    lens = _lengths(case, seed)
    s = {"case": case, "seq_lens": torch.from_numpy(lens).cuda()}
    if op == "select":
        # totals as attention leaves them: heavy-tailed, and not a few positions that nothing attended yet
        w = torch.exp(1.5 * _random(gen, B, case["groups"], case["N"]) - 2.0)
        s["weights"] = torch.where(torch.rand(w.shape, generator=gen, device="cuda") < 0.05, torch.zeros_like(w), w)
        s["keep"] = torch.empty(B, case["groups"], case["budget"], dtype=torch.int32, device="cuda")
        s["new_lens"] = torch.empty(B, dtype=torch.int32, device="cuda")
        return s
    if case.get("page"):
        pages = s["pool_pages"] = _cache_shape(case)[0]
        per = _cap(case) // case["page"]
        s["page_table"] = torch.randperm(pages, generator=gen, device="cuda")[: B * per].to(torch.int32).view(B, per).contiguous()
    if op == "compact":
        for name in ("k_cache", "v_cache"):
            s[name], _ = _rows(gen, _cache_shape(case), case["dtype"], 2)
        groups = case["Hkv"] // case["group"]
        s["weights"] = torch.rand(B, groups, _cap(case), generator=gen, device="cuda")
        # a kept set as `select` makes it: the first and last positions and a random choice between, ascending
        n, k = s["seq_lens"].view(B, 1, 1), case["budget"]
        at = torch.arange(_cap(case), device="cuda").view(1, 1, -1)
        order = torch.rand(B, groups, _cap(case), generator=gen, device="cuda")
        order = torch.where((at < case["first"]) | (at >= n - case["last"]), 2.0, order)
        order = torch.where(at < n, order, -1.0)
        top = torch.argsort(order, dim=2, descending=True)[:, :, :k]
        top = torch.where(top < n, top, 1 << 30).sort(dim=2).values
        s["keep"] = torch.where(top < n, top, -1).to(torch.int32).contiguous()
        s["new_lens"] = torch.clamp(s["seq_lens"], max=k)
        return s
    L, Hq, Hkv, d, Qn, dt = case["L"], case["Hq"], case["Hkv"], case["d"], case["q_len"], case["dtype"]
    act = torch.float32 if dt == "f32" else torch.bfloat16
    rows = case["N"] if op == "diff_prompt" else Qn
    s["q"] = (_random(gen, B, L, rows, Hq, d) * 1.5).to(act)
    s["k_cache"], s["k_scale"] = _rows(gen, _cache_shape(case), dt, 2)
    if L > 1:
        s["gate_logits"] = _random(gen, B, L - 1, rows, Hq)
    if op == "weights":
        # a total of the size that a few steps leave
        few = 4.0 * L * Qn * (Hq // Hkv) * case["maps"] * case["group"] / case["N"]
        s["weights"] = torch.rand(B, Hkv // case["group"], _cap(case), generator=gen, device="cuda") * few
        return s
    s["v_cache"], s["v_scale"] = _rows(gen, _cache_shape(case), dt, 2)
    if L > 1:
        slots = case["N"] if op == "diff_prompt" else case["w"]
        for name, scale in (("k_win", s["k_scale"]), ("v_win", s["v_scale"])):
            x = _random(gen, B, L - 1, slots, Hkv, d)
            s[name] = x.to(act) if dt != "e4m3" else torch.clamp(x / scale.view(-1, 1), -448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    # the learned factor's four vectors (as they are initialised: N(0, 0.1)) and the norm's gain
    s["lambdas"] = [(_random(gen, case["lambda_heads"], d // 2) * 0.1).contiguous() for _ in range(4)]
    s["gain"] = (1.0 + 0.1 * _random(gen, d)).contiguous() if case["norm"] else None
    s["out"] = torch.empty_like(s["q"])
    return s


_handles = {}


def _bind(s):
    """The handle (one for each configuration, as a program keeps it) and the argument structs of the call."""
    from paper_2510_24824_b200 import binding as P
    case = s["case"]
    op, B = case["op"], case["B"]
    pages = dict(page_table=s.get("page_table"), max_pages=s["page_table"].shape[1], num_pool_pages=s["pool_pages"]) if case.get("page") else {}
    dt, kv = ("bf16", "e4m3") if case.get("dtype") == "e4m3" else (case.get("dtype", "bf16"), "")
    key = (op,) + tuple(case[k] for k in sorted(case) if k not in ("name", "ragged", "gate", "decay", "budget", "first", "last"))
    fresh = key not in _handles
    if op == "diff_step":
        if fresh:
            _handles[key] = P.plt_diff_attn_create(P.make_diff_config(
                dt, B, case["L"], case["Hq"], case["Hkv"], case["d"], _cap(case), case["w"] if case["L"] > 1 else 0, page_size=case["page"],
                kv_dtype=kv, q_len=case["q_len"], lambda_init=LAMBDA_INIT, norm_eps=NORM_EPS))
        args = P.make_args(B, s["q"], s["k_cache"], s["v_cache"], s["seq_lens"], s["out"], k_win=s.get("k_win"), v_win=s.get("v_win"),
                           gate_logits=s.get("gate_logits"), k_scale=s["k_scale"], v_scale=s["v_scale"], **pages)
        calls = (P.plt_diff_attn_run, _handles[key], args, P.make_diff_weights(*s["lambdas"], norm_gain=s["gain"]))
    elif op == "diff_prompt":
        if fresh:
            _handles[key] = P.plt_diff_seq_attn_create(P.make_diff_seq_config(
                B, case["L"], case["Hq"], case["Hkv"], case["d"], case["N"], case["w"] if case["L"] > 1 else 0, lambda_init=LAMBDA_INIT, norm_eps=NORM_EPS))
        args = P.make_seq_args(B, s["q"], s["k_cache"], s["v_cache"], s["seq_lens"], s["out"], k_loc=s.get("k_win"), v_loc=s.get("v_win"), gate_logits=s.get("gate_logits"))
        calls = (P.plt_diff_seq_attn_run, _handles[key], args, P.make_diff_weights(*s["lambdas"], norm_gain=s["gain"]))
    else:
        if fresh:
            select = op == "select"
            _handles[key] = P.plt_cache_evict_create(P.make_evict_config(
                "bf16" if select else dt, B, 1 if op != "weights" else case["L"], case.get("Hq", case.get("Hkv", case.get("groups"))),
                case.get("Hkv", case.get("groups")), case.get("d", 128), case["N"] if select else _cap(case), page_size=case.get("page", 0),
                kv_dtype=kv, q_len=case.get("q_len", 1), maps=case.get("maps", 1), heads_per_group=case.get("group", 1)))
        if op == "weights":
            args = P.make_evict_weights_args(B, s["q"], s["k_cache"], s["seq_lens"], s["weights"], gate_logits=s.get("gate_logits") if case["gate"] else None,
                                             decay=case["decay"], k_scale=s["k_scale"], **pages)
            calls = (P.plt_cache_evict_weights, _handles[key], args)
        elif op == "select":
            args = P.make_evict_select_args(B, s["weights"], s["seq_lens"], s["keep"], s["new_lens"], case["budget"], keep_first=case["first"], keep_last=case["last"])
            calls = (P.plt_cache_evict_select, _handles[key], args)
        else:
            args = P.make_evict_compact_args(B, s["k_cache"], s["v_cache"], s["seq_lens"], s["keep"], s["new_lens"], case["budget"], weights=s["weights"], **pages)
            calls = (P.plt_cache_evict_compact, _handles[key], args)
    s["call"] = calls
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    return _bind(s) if own else s


# ---- plain forms --------------------------------------------------------------------------------------------------
def _values(s, name, scale=None, dtype=torch.float32):
    """A cache as [B, capacity, Hkv, d] values."""
    x = s[name]
    if x.dtype == torch.uint8:
        x = x.view(torch.float8_e4m3fn)
    if s["case"].get("page") and name in ("k_cache", "v_cache"):
        x = x[s["page_table"].long()].flatten(1, 2) if x.dtype != torch.float8_e4m3fn else x.view(torch.uint8)[s["page_table"].long()].flatten(1, 2).view(torch.float8_e4m3fn)
    x = x.to(dtype)
    return x if scale is None else x * scale.to(dtype).view(-1, 1)


def _softmax(x, seen):
    """exp(x - max) / sum over the last axis where `seen`; rows that see nothing are zero."""
    x = torch.where(seen, x, -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    e = torch.exp(x - torch.where(top > -math.inf, top, 0.0))
    total = e.sum(dim=-1, keepdim=True)
    return e / torch.where(total > 0, total, 1.0)


def _split(q, Hkv, maps):
    """[B, L, rows, Hq, d] -> [B, L, rows, Hkv, G, maps, d / maps]."""
    B, L, R, Hq, d = q.shape
    return q.view(B, L, R, Hkv, Hq // Hkv, maps, d // maps)


def _scores(q, k, maps, eq):
    """Scaled products of the query halves with the key halves."""
    k = k.unflatten(-1, (maps, -1))
    return torch.einsum(eq, q, k) / math.sqrt(q.shape[-1])


def _step_limits(s):
    """[B, L, q_len] keys each row of a step sees; of the loops' windows likewise."""
    case = s["case"]
    n = s["seq_lens"].long().view(-1, 1, 1)
    loop = torch.arange(case["L"], device="cuda").view(1, -1, 1)
    newer = torch.arange(case["q_len"] - 1, -1, -1, device="cuda").view(1, 1, -1)
    cut = (n - loop).clamp(min=0)
    return (cut - newer).clamp(min=0), (cut.clamp(max=case["w"]) - newer).clamp(min=0)


def _finish(y1, y2, s, dtype=torch.float32):
    """The difference of the two maps' results and the norm of each head. y: [B, L, rows, Hkv, G, d]."""
    l1, m1, l2, m2 = (t.to(dtype) for t in s["lambdas"])
    lam = torch.exp((l1 * m1).sum(dim=-1)) - torch.exp((l2 * m2).sum(dim=-1)) + LAMBDA_INIT
    x = y1.flatten(3, 4) - lam.view(-1, 1) * y2.flatten(3, 4)
    if s["gain"] is not None:
        x = (1.0 - LAMBDA_INIT) * s["gain"].to(dtype) * x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + NORM_EPS)
    return x


def _gated(y, local, s):
    """Loops 2..L mix the result on their own window in by their gate."""
    g = torch.sigmoid(s["gate_logits"]).view(*y[:, 1:].shape[:5], 1, 1)
    return torch.cat([y[:, :1], g * local + (1.0 - g) * y[:, 1:]], dim=1)


def _plain_step(s):
    case = s["case"]
    k, v = _values(s, "k_cache", s["k_scale"]), _values(s, "v_cache", s["v_scale"])
    q = _split(s["q"].float(), case["Hkv"], 2)
    cut, wl = _step_limits(s)
    at = torch.arange(k.shape[1], device="cuda")
    v = torch.where((at.view(1, -1) < s["seq_lens"].view(-1, 1))[:, :, None, None], v, 0.0)
    p = _softmax(_scores(q, k, 2, "blrhgmd,bnhmd->blrhgmn"), at < cut.view(*cut.shape, 1, 1, 1, 1))
    y = torch.einsum("blrhgmn,bnhd->blrhgmd", p, v)
    if case["L"] > 1:
        kw, vw = _values(s, "k_win", s["k_scale"]), _values(s, "v_win", s["v_scale"])
        slot, wl = torch.arange(case["w"], device="cuda"), wl[:, 1:]
        p = _softmax(_scores(q[:, 1:], kw, 2, "blrhgmd,blnhmd->blrhgmn"), slot < wl.reshape(*wl.shape, 1, 1, 1, 1))
        y = _gated(y, torch.einsum("blrhgmn,blnhd->blrhgmd", p, vw), s)
    return _finish(y[..., 0, :], y[..., 1, :], s).to(s["q"].dtype)


def _plain_prompt(s):
    case = s["case"]
    T, L = case["N"], case["L"]
    k, v = s["k_cache"].float(), s["v_cache"].float()
    q = _split(s["q"].float(), case["Hkv"], 2).permute(0, 1, 3, 4, 5, 2, 6)          # [B, L, Hkv, G, 2, T, d / 2]
    t, loop = torch.arange(T, device="cuda"), torch.arange(L, device="cuda")
    live = (t.view(1, 1, -1) < s["seq_lens"].view(-1, 1, 1)) & (t.view(1, 1, -1) >= loop.view(1, -1, 1))      # [B, L, T]
    seen = live.unsqueeze(-1) & (t.view(1, 1, 1, -1) < t.view(1, 1, -1, 1) + 1 - loop.view(1, -1, 1, 1))      # [B, L, T, T]
    p = _softmax(_scores(q, k, 2, "blhgmtd,bnhmd->blhgmtn"), seen[:, :, None, None, None])
    y = torch.einsum("blhgmtn,bnhd->blhgmtd", p, v)
    del p
    if L > 1:
        kw, vw = s["k_win"].float(), s["v_win"].float()
        first = torch.maximum(loop[1:].view(-1, 1), t.view(1, -1) + 1 - case["w"])                             # [L - 1, T]
        band = (t.view(1, 1, -1) >= first.unsqueeze(-1)) & (t.view(1, 1, -1) <= t.view(1, -1, 1))
        p = _softmax(_scores(q[:, 1:], kw, 2, "blhgmtd,blnhmd->blhgmtn"), (live[:, 1:].unsqueeze(-1) & band)[:, :, None, None, None])
        g = torch.sigmoid(s["gate_logits"]).unflatten(-1, (case["Hkv"], -1)).permute(0, 1, 3, 4, 2)[:, :, :, :, None, :, None]
        y = torch.cat([y[:, :1], g * torch.einsum("blhgmtn,blnhd->blhgmtd", p, vw) + (1.0 - g) * y[:, 1:]], dim=1)
    y = torch.where(live[:, :, None, None, None, :, None], y, 0.0).permute(0, 1, 5, 2, 3, 4, 6)
    return _finish(y[..., 0, :], y[..., 1, :], s).to(s["q"].dtype)


def _plain_weights(s):
    case = s["case"]
    k = _values(s, "k_cache", s["k_scale"])
    q = _split(s["q"].float(), case["Hkv"], case["maps"])
    cut, _ = _step_limits(s)
    at = torch.arange(k.shape[1], device="cuda")
    p = _softmax(_scores(q, k, case["maps"], "blrhgmd,bnhmd->blrhgmn"), at < cut.view(*cut.shape, 1, 1, 1, 1))
    if case["gate"] and case["L"] > 1:
        share = 1.0 - torch.sigmoid(s["gate_logits"])
        p = p * torch.cat([torch.ones_like(share[:, :1]), share], dim=1).view(*p.shape[:5], 1, 1)
    new = p.sum(dim=(1, 2, 4, 5)).unflatten(1, (-1, case["group"])).sum(dim=2)
    held = s["weights"]
    total = held * case["decay"] + new if case["decay"] else new
    held.copy_(torch.where(at < s["seq_lens"].view(-1, 1, 1), total, held))
    return held


def _plain_select(s):
    case = s["case"]
    k, n = case["budget"], s["seq_lens"].view(-1, 1, 1)
    at = torch.arange(case["N"], device="cuda")
    key = torch.where((at < case["first"]) | (at >= n - case["last"]), math.inf, s["weights"])
    key = torch.where(at < n, key, -math.inf)
    top = torch.sort(key, dim=2, descending=True, stable=True).indices[:, :, :k]     # ties: the lowest position first
    top = torch.where(torch.arange(k, device="cuda") < n, top, 1 << 30).sort(dim=2).values
    s["keep"].copy_(torch.where(torch.arange(k, device="cuda") < n, top, -1))
    s["new_lens"].copy_(s["seq_lens"].clamp(max=k))
    return s["keep"], s["new_lens"]


def _plain_compact(s):
    case = s["case"]
    new, old = s["new_lens"].long().view(-1, 1, 1), s["seq_lens"].long().view(-1, 1, 1)
    slot = torch.arange(case["budget"], device="cuda").view(1, 1, -1)
    kept = (slot < new).expand(s["keep"].shape)
    b, g, i = kept.nonzero(as_tuple=True)
    source = s["keep"].long()[b, g, i]
    cell = lambda at: (b * case["N"] + at if not case["page"] else s["page_table"].long()[b, at // case["page"]] * case["page"] + at % case["page"])  # noqa: E731
    for name in ("k_cache", "v_cache"):
        flat = s[name].view(-1, case["Hkv"] // case["group"], case["group"], case["d"])
        flat[cell(i), g] = flat[cell(source), g]
    w = s["weights"]
    w[b, g, i] = w[b, g, source]
    at = torch.arange(w.shape[2], device="cuda")
    w.copy_(torch.where((at >= new) & (at < old), 0.0, w))
    return _compact_outputs(s)


def _compact_outputs(s):
    seen = (lambda x: x.view(torch.float8_e4m3fn)) if s["case"]["dtype"] == "e4m3" else (lambda x: x)
    return [seen(s["k_cache"]), seen(s["v_cache"]), s["weights"]]


def run(s):
    op = s["case"]["op"]
    if own:
        call = s["call"]
        call[0](*call[1:], torch.cuda.current_stream().cuda_stream)
        if op in ("diff_step", "diff_prompt"):
            return s["out"]
        if op == "weights":
            return s["weights"]
        return (s["keep"], s["new_lens"]) if op == "select" else _compact_outputs(s)
    return {"diff_step": _plain_step, "diff_prompt": _plain_prompt, "weights": _plain_weights, "select": _plain_select, "compact": _plain_compact}[op](s)


# ---- cost ---------------------------------------------------------------------------------------------------------
def work(case):
    """Bytes: every input read once and every output written once. Flops: the products over the keys that are seen."""
    lens = _lengths(case, 1).astype(np.float64)
    op, B, tokens = case["op"], case["B"], float(lens.sum())
    if op == "select":
        return {"bytes": 4.0 * case["groups"] * (tokens + B * case["budget"]) + 8 * B, "flops": 0}
    es = {"bf16": 2, "f32": 4, "e4m3": 1}[case["dtype"]]
    Hkv, d = case["Hkv"], case["d"]
    if op == "compact":
        moved = float(np.where(lens > case["budget"], case["budget"] - case["first"], 0).sum())
        groups = Hkv // case["group"]
        return {"bytes": moved * (4.0 * Hkv * d * es + 12.0 * groups) + 4.0 * groups * float(np.maximum(lens - case["budget"], 0).sum()), "flops": 0}
    L, Hq, Qn = case["L"], case["Hq"], case["q_len"]
    qb = 4 if case["dtype"] == "f32" else 2
    if op == "weights":
        per = 8.0 if case["decay"] else 4.0
        gates = 4.0 * B * (L - 1) * Qn * Hq if case["gate"] else 0.0
        return {"bytes": tokens * (Hkv * d * es + per * Hkv / case["group"]) + B * L * Qn * Hq * d * qb + gates, "flops": 2.0 * tokens * L * Qn * Hq * d}
    if op == "diff_step":
        slots = float(np.minimum(lens, case["w"]).sum()) * (L - 1)
        qo = 2.0 * B * L * Qn * Hq * d * qb + 4.0 * B * (L - 1) * Qn * Hq
        return {"bytes": (tokens + slots) * Hkv * d * 2 * es + qo, "flops": (tokens * L + slots) * Qn * Hq * d * 6.0}
    pairs = sum((L * n * (n + 1) / 2) + (L - 1) * sum(min(t + 1, case["w"]) for t in range(int(n))) for n in lens)
    return {"bytes": 2.0 * tokens * d * (L * Hq + Hkv * (2 * L)) + 2.0 * B * case["N"] * L * Hq * d, "flops": pairs * Hq * d * 6.0}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def _row64(q, k, v, scale):
    """softmax(scale * q k^T) and its product with v, for queries [r, c] on keys [n, c]."""
    x = (q @ k.T) * scale
    x = torch.exp(x - x.max(dim=1, keepdim=True).values)
    x = x / x.sum(dim=1, keepdim=True)
    return x if v is None else x @ v


def _cache64(s, name, scale, b, n):
    case, x = s["case"], s[name]
    if case.get("page"):
        at = torch.arange(n, device="cuda")
        x = x[s["page_table"][b].long()[at // case["page"]], at % case["page"]]
    else:
        x = x[b, :n]
    x = x.view(torch.float8_e4m3fn).double() if x.dtype == torch.uint8 else x.double()
    return x * scale.double()[:, None] if scale is not None else x


def _join64(a1, a2, s, h):
    l1, m1, l2, m2 = (t.double()[h if t.shape[0] > 1 else 0] for t in s["lambdas"])
    x = a1 - (math.exp(float(l1 @ m1)) - math.exp(float(l2 @ m2)) + LAMBDA_INIT) * a2
    if s["gain"] is not None:
        x = x / torch.sqrt((x ** 2).mean(dim=1, keepdim=True) + NORM_EPS) * s["gain"].double() * (1 - LAMBDA_INIT)
    return x


def _exact_step(s):
    case, out = s["case"], torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    B, L, Qn, Hq, d = out.shape
    G, half = Hq // case["Hkv"], d // 2
    for b in range(B):
        n = int(s["seq_lens"][b])
        k, v = _cache64(s, "k_cache", s["k_scale"], b, n), _cache64(s, "v_cache", s["v_scale"], b, n)
        for l in range(L):
            for j in range(Qn):
                cut = n - l - (Qn - 1 - j)
                slots = min(case["w"], n - l) - (Qn - 1 - j) if l else 0
                for kv in range(case["Hkv"]) if cut > 0 else ():
                    qs = s["q"][b, l, j, kv * G:(kv + 1) * G].double()
                    ys = [_row64(qs[:, m * half:(m + 1) * half], k[:cut, kv, m * half:(m + 1) * half], v[:cut, kv], half ** -0.5) for m in (0, 1)]
                    if l:
                        g = torch.sigmoid(s["gate_logits"][b, l - 1, j, kv * G:(kv + 1) * G].double())[:, None]
                        near = [torch.zeros_like(y) for y in ys]
                        if slots > 0:
                            kw, vw = ((t.view(torch.float8_e4m3fn).double() * sc.double()[kv] if t.dtype == torch.uint8 else t.double()) for t, sc in
                                      ((s["k_win"][b, l - 1, :slots, kv], s["k_scale"]), (s["v_win"][b, l - 1, :slots, kv], s["v_scale"])))
                            near = [_row64(qs[:, m * half:(m + 1) * half], kw[:, m * half:(m + 1) * half], vw, half ** -0.5) for m in (0, 1)]
                        ys = [g * a + (1 - g) * y for a, y in zip(near, ys)]
                    for i in range(G):
                        out[b, l, j, kv * G + i] = _join64(ys[0][i:i + 1], ys[1][i:i + 1], s, kv * G + i)[0]
    return out


def _exact_prompt(s):
    case, out = s["case"], torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    B, L, T, Hq, d = out.shape
    half = d // 2
    for b in range(B):
        n = int(s["seq_lens"][b])
        row, col = torch.arange(n, device="cuda")[:, None], torch.arange(n, device="cuda")[None, :]
        for l in range(L):
            if n <= l:
                continue
            for h in range(Hq):
                kv = h // (Hq // case["Hkv"])
                ys = []
                for m in (0, 1):
                    part = slice(m * half, (m + 1) * half)
                    q = s["q"][b, l, l:n, h, part].double()
                    x = (q @ s["k_cache"][b, :n, kv, part].double().T) * half ** -0.5
                    x = x.masked_fill(col > row[l:] - l, -math.inf)
                    y = torch.softmax(x, dim=1) @ s["v_cache"][b, :n, kv].double()
                    if l:
                        g = torch.sigmoid(s["gate_logits"][b, l - 1, l:n, h].double())[:, None]
                        x = (q @ s["k_win"][b, l - 1, :n, kv, part].double().T) * half ** -0.5
                        x = x.masked_fill((col > row[l:]) | (col < l) | (col <= row[l:] - case["w"]), -math.inf)
                        y = g * (torch.softmax(x, dim=1) @ s["v_win"][b, l - 1, :n, kv].double()) + (1 - g) * y
                    ys.append(y)
                out[b, l, l:n, h] = _join64(ys[0], ys[1], s, h)
    return out


def _exact_weights(s):
    case, held = s["case"], s["weights"].double()
    B, L, Qn, Hq, d = s["q"].shape
    G, part = Hq // case["Hkv"], d // case["maps"]
    for b in range(B):
        n = int(s["seq_lens"][b])
        k = _cache64(s, "k_cache", s["k_scale"], b, n)
        new = torch.zeros(held.shape[1], n, dtype=torch.float64, device="cuda")
        for l in range(L):
            for j in range(Qn):
                cut = n - l - (Qn - 1 - j)
                for kv in range(case["Hkv"]) if cut > 0 else ():
                    share = torch.ones(G, 1, dtype=torch.float64, device="cuda")
                    if l and case["gate"]:
                        share = 1 - torch.sigmoid(s["gate_logits"][b, l - 1, j, kv * G:(kv + 1) * G].double())[:, None]
                    for m in range(case["maps"]):
                        at = slice(m * part, (m + 1) * part)
                        p = _row64(s["q"][b, l, j, kv * G:(kv + 1) * G, at].double(), k[:cut, kv, at], None, part ** -0.5)
                        new[kv // case["group"], :cut] += (share * p).sum(dim=0)
        held[b, :, :n] = new + (held[b, :, :n] * case["decay"] if case["decay"] else 0.0)
    return held


def _exact_compact(s):
    case = s["case"]
    caches = [(x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x).double() for x in (s["k_cache"], s["v_cache"])]
    held = s["weights"].double()
    for b in range(case["B"]):
        n, m = int(s["seq_lens"][b]), int(s["new_lens"][b])
        slot = torch.arange(m, device="cuda")
        for g in range(held.shape[1]):
            source, heads = s["keep"][b, g, :m].long(), slice(g * case["group"], (g + 1) * case["group"])
            for x in caches:
                if case["page"]:
                    table = s["page_table"][b].long()
                    x[table[slot // case["page"]], slot % case["page"], heads] = x[table[source // case["page"]], source % case["page"], heads]
                else:
                    x[b, :m, heads] = x[b, source, heads]
            held[b, g, :m] = held[b, g, source]
            held[b, g, m:n] = 0.0
    return caches + [held]


def exact(case, seed):
    if case["op"] == "select":
        return None                                   # positions: whole numbers
    s = _inputs(case, seed)
    return {"diff_step": _exact_step, "diff_prompt": _exact_prompt, "weights": _exact_weights, "compact": _exact_compact}[case["op"]](s)

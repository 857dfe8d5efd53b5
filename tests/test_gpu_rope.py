"""Norm and rotation of queries and keys on the GPU against the fp64 oracle.

Error of a row in fp32, in units u = 2^-24 (relative): the norm's sum of squares 19 additions and products, the mean and eps 2,
square root, quotient, gain and product 3, together 14 after the root halves the sum's share. Cosine and sine: 2 each, the angle
below 1 (absolute), attn_factor 1, the two products and the sum 3. So |error| <= 24 u factor (|a| + |b|) on a pair, 14 u |x| where
nothing turns; then one rounding to the stored type. Positions up to 2^31 add pos * f * 2^-51 of angle from 64-bit frequencies."""
import numpy as np
import pytest
import torch

from oracle import plt_rope as oracle_rope
from paper_2510_24824_b200 import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SCALINGS = {"none": {}, "linear": dict(factor=4.0), "base": dict(factor=8.0), "wavelength": dict(factor=8.0, low=1.0, high=4.0, original_len=8192),
            "ramp": dict(factor=16.0, low=1.0, high=32.0, original_len=4096, attn_factor=1.2772588722239781)}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def values(x, scale=None):
    """A stored tensor's values in 64 bits; scale: per head, the last axis but one."""
    x = x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x
    x = x.double().cpu().numpy()
    return x if scale is None else x * scale.double().cpu().numpy()[:, None]


class Case:
    def __init__(self, seed=0, dtype="bf16", kv="", B_=3, L=1, Hq=4, Hkv=2, d=128, cap=64, w=16, page=0, q_len=1, rd=0, layout="half",
                 scaling="none", norm=True, far=0, theta=10000.0):
        self.__dict__.update({k: v for k, v in locals().items() if k != "self"})
        g = torch.Generator("cuda").manual_seed(seed)
        self.gen, self.rd = g, rd or d
        self.act = torch.float32 if dtype == "f32" else torch.bfloat16
        self.freq = oracle_rope.frequencies(self.rd, theta, scaling, **{k: v for k, v in SCALINGS[scaling].items() if k != "attn_factor"})
        self.factor = SCALINGS[scaling].get("attn_factor", 1.0)
        self.rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.q_gain, self.k_gain = (1 + 0.2 * self.rand(d), 1 + 0.2 * self.rand(d)) if norm else (None, None)
        e4m3 = kv == "e4m3"
        self.k_scale, self.v_scale = (torch.rand(Hkv, generator=g, device="cuda") * 0.01 + 0.01 for _ in range(2)) if e4m3 else (None, None)
        self.pool = (B_ * -(-cap // page) + 2) if page else 0
        shape = (self.pool, page, Hkv, d) if page else (B_, cap, Hkv, d)
        self.table = torch.randperm(self.pool, generator=g, device="cuda")[:-2].to(torch.int32).view(B_, -1).contiguous() if page else None
        fill = lambda *s: torch.randint(0, 120, s, generator=g, device="cuda").to(torch.uint8) if e4m3 else self.rand(*s).to(self.act)  # noqa: E731
        self.k_cache, self.v_cache = fill(*shape), fill(*shape)
        self.k_win, self.v_win = (fill(B_, L - 1, w, Hkv, d), fill(B_, L - 1, w, Hkv, d)) if L > 1 else (None, None)
        self.op = B.plt_rope_create(B.make_rope_config(dtype, B_, L, Hq, Hkv, d, cap, w if L > 1 else 0, page_size=page, kv_dtype=kv, q_len=q_len,
                                                       rotary_dim=rd, layout=layout, theta=theta, scaling=scaling, **SCALINGS[scaling]))
        self.pages = dict(page_table=self.table, max_pages=self.table.shape[1], num_pool_pages=self.pool) if page else {}
        self.scales = dict(k_scale=self.k_scale, v_scale=self.v_scale)

    def row(self, x, pos, gain):
        """Row(s) [heads, d] at a position in 64 bits, and the bound of the fp32 error."""
        x = x.double().cpu().numpy()
        y = oracle_rope.turn(x, pos, self.freq, None if gain is None else gain.double().cpu().numpy(), 1e-6, self.layout, self.factor)
        z = oracle_rope.turn(x, 0, self.freq * 0, None if gain is None else gain.double().cpu().numpy(), 1e-6, self.layout, 1.0)
        a, b = (slice(0, self.rd // 2), slice(self.rd // 2, self.rd)) if self.layout == "half" else (slice(0, self.rd, 2), slice(1, self.rd, 2))
        size = np.abs(z).copy() * 14 * U
        pair = (np.abs(z[..., a]) + np.abs(z[..., b])) * self.factor * (24 * U + abs(float(pos)) * np.abs(self.freq) * 2.0 ** -51)
        size[..., a], size[..., b] = pair, pair
        return y, size

    def stored(self, got, want, err, kind, scale=None):
        """got (as stored, [heads, d]) against want with the fp32 bound err."""
        got = values(got, scale)
        if scale is not None:
            s = scale.double().cpu().numpy()[:, None]
            want = np.clip(want, -448 * s, 448 * s)
            bound = 2.0 ** -4 * np.abs(want) + 2.0 ** -10 * s + 2 * err + 2 * U * np.abs(want)     # half a step, or of a subnormal
        else:
            bound = HALF_STEP[kind] * (np.abs(want) + err) + err
        assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())

    def cell(self, b, at):
        return (int(self.table[b, at // self.page]), at % self.page) if self.page else (b, at)


STEPS = [
    dict(), dict(dtype="f32"), dict(kv="e4m3"), dict(d=64), dict(dtype="f32", d=64, layout="interleaved"), dict(layout="interleaved"),
    dict(rd=16), dict(rd=48, layout="interleaved"), dict(rd=64), dict(rd=112, norm=False), dict(d=64, rd=32, dtype="f32"),
    dict(L=3, w=5), dict(L=2, kv="e4m3", page=32), dict(L=2, dtype="f32", page=16, Hkv=4), dict(page=48, q_len=3, cap=100), dict(q_len=5, d=64),
    dict(Hq=1, Hkv=1), dict(Hq=40, Hkv=8, L=2), dict(Hq=9, Hkv=3, d=64, L=8, w=3), dict(Hq=33, Hkv=11),
    dict(far=2 ** 30), dict(far=1000000, scaling="ramp"), dict(far=123457, scaling="wavelength", dtype="f32"), dict(scaling="linear", L=2),
    dict(scaling="base", layout="interleaved", q_len=2), dict(far=2 ** 31 - 200, dtype="f32", theta=500000.0),
]


@pytest.mark.parametrize("kw", STEPS, ids=str)
@pytest.mark.parametrize("fused", [False, True])
def test_step(kw, fused):
    c = Case(seed=len(str(kw)), **kw)
    n, Qn = c.B_, c.q_len
    own = [c.cap, min(Qn, c.cap), max(1, c.cap // 2)]          # a full cache, the first step, something between
    lens = torch.tensor([x + c.far for x in own], dtype=torch.int32, device="cuda")
    before = torch.full((n,), c.far, dtype=torch.int32, device="cuda") if c.far else None
    if fused:      # one projection's rows hold q, k and v
        wide = (c.rand(n, c.L, Qn, (c.Hq + 2 * c.Hkv) * c.d + 64) * 1.5).to(c.act)
        flat = wide.view(-1, wide.shape[-1])
        offs = (0, c.Hq * c.d, (c.Hq + c.Hkv) * c.d)
        q, k, v = (flat[:, o:o + h * c.d].unflatten(1, (h, c.d)).unflatten(0, (n, c.L, Qn)) for o, h in zip(offs, (c.Hq, c.Hkv, c.Hkv)))
        strides = (wide.shape[-1],) * 3
    else:
        q, k, v = ((c.rand(n, c.L, Qn, h, c.d) * 1.5).to(c.act) for h in (c.Hq, c.Hkv, c.Hkv))
        strides = (0, 0, 0)
    q_out = torch.full((n, c.L, Qn, c.Hq, c.d), float("nan"), device="cuda").to(c.act)
    gates = dict(w_gate=0.2 * c.rand(c.Hq, c.d), b_gate=c.rand(c.Hq), gate_logits=torch.full((n, max(1, c.L - 1), c.Hq), float("nan"), device="cuda"))
    old = {name: getattr(c, name).clone() for name in ("k_cache", "v_cache", "k_win", "v_win") if getattr(c, name) is not None}
    B.plt_rope_step(c.op, B.make_rope_step_args(n, q, k, v, q_out, c.k_cache, c.v_cache, lens, prefix_lens=before, q_gain=c.q_gain, k_gain=c.k_gain,
                                                k_win=c.k_win, v_win=c.v_win, row_strides=strides, **c.pages, **c.scales, **gates))
    torch.cuda.synchronize()
    assert B.plt_rope_check(c.op) == 0
    for b in range(n):
        for l in range(c.L):
            for j in range(Qn):
                pos = own[b] + c.far - l - 1 - (Qn - 1 - j)
                if pos < 0:
                    assert (q_out[b, l, j] == 0).all()
                    if l:
                        assert torch.equal(gates["gate_logits"][b, l - 1], gates["b_gate"])
                    continue
                y, err = c.row(q[b, l, j], pos, c.q_gain)
                c.stored(q_out[b, l, j], y, err, c.act)
                if l:
                    w, bias = gates["w_gate"].double().cpu().numpy(), gates["b_gate"].double().cpu().numpy()
                    want = (w * y).sum(-1) + bias
                    bound = (np.abs(w) * err).sum(-1) + 21 * U * (np.abs(w) * np.abs(y)).sum(-1) + U * np.abs(want)
                    assert (np.abs(gates["gate_logits"][b, l - 1].double().cpu().numpy() - want) <= bound).all()
                y, err = c.row(k[b, l, j], pos, c.k_gain)
                plain, zero = v[b, l, j].double().cpu().numpy(), np.zeros((c.Hkv, c.d))
                if l == 0:
                    if pos < c.far:
                        continue
                    at = c.cell(b, pos - c.far)
                    c.stored(c.k_cache[at], y, err, c.act, c.k_scale)
                    c.stored(c.v_cache[at], plain, zero, c.act, c.v_scale)
                    old["k_cache"][at], old["v_cache"][at] = c.k_cache[at], c.v_cache[at]
                else:
                    at = (b, l - 1, pos % c.w)
                    c.stored(c.k_win[at], y, err, c.act, c.k_scale)
                    c.stored(c.v_win[at], plain, zero, c.act, c.v_scale)
                    old["k_win"][at], old["v_win"][at] = c.k_win[at], c.v_win[at]
    for name, was in old.items():          # nothing else was touched
        assert torch.equal(getattr(c, name).view(torch.uint8), was.view(torch.uint8)), name


SEQS = [
    dict(), dict(dtype="f32"), dict(kv="e4m3"), dict(d=64, L=2), dict(dtype="f32", d=64, layout="interleaved", L=3), dict(rd=32, layout="interleaved"),
    dict(rd=80, norm=False), dict(page=16, L=2), dict(kv="e4m3", page=48, L=2), dict(Hq=1, Hkv=1), dict(Hq=24, Hkv=8, L=2, scaling="ramp"),
    dict(Hq=7, Hkv=7, d=64, dtype="f32"), dict(Hq=6, Hkv=3, scaling="wavelength"),
]


@pytest.mark.parametrize("kw", SEQS, ids=str)
@pytest.mark.parametrize("start", [0, 3, 100000])
@pytest.mark.parametrize("in_place", [False, True])
def test_prompt(kw, start, in_place):
    c = Case(seed=len(str(kw)) + start, B_=4, cap=64, **kw)
    n, T = 4, 29
    lens, begins = [T, 0, 1, 17], [start, start, start + 2, start]
    before = [start, start, start, max(0, start - 5)]
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, ks, vs = (c.rand(n, c.L, T, c.Hq, c.d) * 1.5).to(c.act), (c.rand(n, T, c.Hkv, c.d) * 1.5).to(c.act), c.rand(n, T, c.Hkv, c.d).to(c.act)
    kl = (c.rand(n, c.L - 1, T, c.Hkv, c.d) * 1.5).to(c.act) if c.L > 1 else None
    for b in range(n):         # rows behind a sequence's end are not read
        q[b, :, lens[b]:] = float("nan")
    src = [x.clone() if x is not None else None for x in (q, ks, kl)]
    outs = [q, ks, kl] if in_place else [torch.full_like(x, 7.0) if x is not None else None for x in (q, ks, kl)]
    was = [x.clone() if x is not None else None for x in outs]
    old_k, old_v = c.k_cache.clone(), c.v_cache.clone()
    B.plt_rope_seq(c.op, B.make_rope_seq_args(n, T, q, ks, dev(lens), outs[0], k_share_out=outs[1], k_loc=kl, k_loc_out=outs[2], q_gain=c.q_gain,
                                              k_gain=c.k_gain, start=dev(begins), prefix_lens=dev(before), v_share=vs, k_cache=c.k_cache,
                                              v_cache=c.v_cache, **c.pages, **c.scales))
    torch.cuda.synchronize()
    assert B.plt_rope_check(c.op) == 0
    for b in range(n):
        for t in range(T):
            for l in range(c.L):
                pos = begins[b] + t - l
                if t >= lens[b] or pos < 0:
                    for o, w, at in ((outs[0], was[0], (b, l, t)), (outs[2], was[2], (b, l - 1, t)) if l else (outs[1], was[1], (b, t))):
                        assert torch.equal(o[at].view(torch.uint8), w[at].view(torch.uint8))
                    continue
                y, err = c.row(src[0][b, l, t], pos, c.q_gain)
                c.stored(outs[0][b, l, t], y, err, c.act)
                k_in, k_out = (src[2][b, l - 1, t], outs[2][b, l - 1, t]) if l else (src[1][b, t], outs[1][b, t])
                y, err = c.row(k_in, pos, c.k_gain)
                c.stored(k_out, y, err, c.act)
                if l == 0:
                    at = c.cell(b, pos - before[b])
                    c.stored(c.k_cache[at], y, err, c.act, c.k_scale)
                    c.stored(c.v_cache[at], vs[b, t].double().cpu().numpy(), np.zeros((c.Hkv, c.d)), c.act, c.v_scale)
                    old_k[at], old_v[at] = c.k_cache[at], c.v_cache[at]
    assert torch.equal(c.k_cache.view(torch.uint8), old_k.view(torch.uint8)) and torch.equal(c.v_cache.view(torch.uint8), old_v.view(torch.uint8))


def test_prompt_in_parts_and_step_by_step_give_the_same_bits():
    """A prompt at once, in two parts, and one step a token: the same queries and the same cache."""
    c = Case(seed=3, B_=2, cap=40, norm=True)
    T = 37
    q, k, v = ((c.rand(2, 1, T, h, c.d)).to(c.act) for h in (c.Hq, c.Hkv, c.Hkv))
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    whole = torch.empty_like(q)
    caches = [(torch.zeros_like(c.k_cache), torch.zeros_like(c.v_cache)) for _ in range(3)]
    args = dict(q_gain=c.q_gain, k_gain=c.k_gain)
    B.plt_rope_seq(c.op, B.make_rope_seq_args(2, T, q, k, dev(T, T), whole, v_share=v, k_cache=caches[0][0], v_cache=caches[0][1], **args))
    outs = []
    for lo, hi in ((0, 20), (20, T)):
        part = [x[:, :, lo:hi].contiguous() for x in (q, k, v)]
        out = torch.empty_like(part[0])
        B.plt_rope_seq(c.op, B.make_rope_seq_args(2, hi - lo, part[0], part[1], dev(hi - lo, hi - lo), out, start=dev(lo, lo), v_share=part[2],
                                                  k_cache=caches[1][0], v_cache=caches[1][1], **args))
        outs.append(out)
    steps = []
    for t in range(T):
        part = [x[:, :, t:t + 1].contiguous() for x in (q, k, v)]
        out = torch.empty_like(part[0])
        B.plt_rope_step(c.op, B.make_rope_step_args(2, part[0], part[1], part[2], out, caches[2][0], caches[2][1], dev(t + 1, t + 1), **args))
        steps.append(out)
    torch.cuda.synchronize()
    assert torch.equal(torch.cat(outs, 2), whole) and torch.equal(torch.cat(steps, 2), whole)
    for a, b in caches[1:]:
        assert torch.equal(a, caches[0][0]) and torch.equal(b, caches[0][1])


@pytest.mark.parametrize("kw", [dict(Hq=1, Hkv=1), dict(Hq=3, Hkv=1, d=64, L=2, w=9, layout="interleaved"), dict(Hq=4, Hkv=2, dtype="f32", d=64, page=32),
                                dict(Hq=2, Hkv=2, kv="e4m3", page=48)], ids=str)
@pytest.mark.parametrize("T", [260, 700])
def test_blocks_of_many_tokens_give_the_same_bits(kw, T):
    """A large call goes in larger blocks than a small one: every sequence of it gives what a call of its own gives, and nothing else
    is written."""
    n = 60
    c = Case(seed=9, B_=n, cap=720, **kw)
    lens = [(37 * b) % (T + 1) for b in range(n)]
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    q, ks, vs = (c.rand(n, c.L, T, c.Hq, c.d) * 1.5).to(c.act), (c.rand(n, T, c.Hkv, c.d) * 1.5).to(c.act), c.rand(n, T, c.Hkv, c.d).to(c.act)
    kl = (c.rand(n, c.L - 1, T, c.Hkv, c.d) * 1.5).to(c.act) if c.L > 1 else None

    def call(rows, caches):
        outs = [torch.full_like(x[rows], 7.0) if x is not None else None for x in (q, ks, kl)]
        pages = dict(c.pages, page_table=c.table[rows].contiguous()) if c.page else {}
        B.plt_rope_seq(c.op, B.make_rope_seq_args(len(lens[rows]), T, q[rows], ks[rows], dev(lens[rows]), outs[0], k_share_out=outs[1],
                                                  k_loc=None if kl is None else kl[rows], k_loc_out=outs[2], q_gain=c.q_gain, k_gain=c.k_gain, start=dev([5] * len(lens[rows])),
                                                  v_share=vs[rows], k_cache=caches[0] if c.page else caches[0][rows], v_cache=caches[1] if c.page else caches[1][rows],
                                                  **pages, **c.scales))
        return outs
    caches = [[x.clone() for x in (c.k_cache, c.v_cache)] for _ in range(2)]
    whole = call(slice(0, n), caches[0])
    parts = [call(slice(b, b + 1), caches[1]) for b in range(n)]
    torch.cuda.synchronize()
    assert B.plt_rope_check(c.op) == 0
    for i, x in enumerate(whole):
        if x is not None:
            assert torch.equal(x.view(torch.uint8), torch.cat([o[i] for o in parts]).view(torch.uint8))
    for a, b in zip(*caches):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    y, err = c.row(q[1, 0, 36], 41, c.q_gain)
    c.stored(whole[0][1, 0, 36], y, err, c.act)


def test_no_turn_and_no_norm_is_the_plain_pre_step():
    """With frequencies of 0 and no gains, rope_step and run do what plt_decode_attn_step does."""
    from paper_2510_24824_b200.inputs import make_problem, shrunk_workload
    from paper_2510_24824_b200.runner import DecodeAttn, DeviceProblem, Rope
    for kw in (dict(), dict(kv_dtype="e4m3")):
        p = make_problem(shrunk_workload(2, **kw))
        a, b = DeviceProblem(p), DeviceProblem(p)
        g = torch.Generator("cuda").manual_seed(1)
        k, v = (torch.randn(p.B, p.L, p.Hkv, p.d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        w, bias = torch.randn(p.Hq, p.d, generator=g, device="cuda") * 0.1, torch.randn(p.Hq, generator=g, device="cuda")
        a.win_lens = b.win_lens = None
        q = b.q.clone()
        b.q.zero_()
        with DecodeAttn(p) as op, Rope(p, inv_freq=[0.0] * 64) as rope:
            op.step(a, k, v, w, bias)
            rope.step(b, q, k, v, w_gate=w, b_gate=bias)
            op.run(b)
            torch.cuda.synchronize()
            assert rope.check() == 0 and op.check() == 0
        assert torch.equal(b.q, q)
        for name in ("k_cache", "v_cache", "k_win", "v_win"):
            assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8)), name
        # the gates' sums run in another order: two fp32 sums of d terms
        size = (w.abs() * q[:, 1:].float().abs()).sum(-1) + bias.abs()
        assert ((a.gate_logits.view_as(size) - b.gate_logits.view_as(size)).abs() <= 2 * 21 * U * size + 128 * U * size).all()


def test_lengths_and_pages_out_of_range():
    """Clamped lengths are flagged; a row with a bad page id is not stored; a prompt's rows beyond the cache are left out."""
    c = Case(seed=5, B_=3, cap=32, page=16)
    q, k, v = ((c.rand(3, 1, 1, h, c.d)).to(c.act) for h in (c.Hq, c.Hkv, c.Hkv))
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    out = torch.empty_like(q)
    step = lambda lens, table, before=None: B.plt_rope_step(c.op, B.make_rope_step_args(  # noqa: E731
        3, q, k, v, out, c.k_cache, c.v_cache, lens, prefix_lens=before, page_table=table, max_pages=2, num_pool_pages=c.pool))
    step(dev(33, -2, 5), c.table)
    assert B.plt_rope_check(c.op) == B.PLT_DEV_SEQ_LEN_CLAMPED
    assert torch.equal(c.v_cache[int(c.table[0, 1]), 15], v[0, 0, 0]) and (out[1] == 0).all()
    bad = c.table.clone()
    bad[0, 0], bad[1, 0] = c.pool, -1
    before = [c.k_cache.clone(), c.v_cache.clone()]
    step(dev(3, 4, 0), bad)
    assert B.plt_rope_check(c.op) == B.PLT_DEV_PAGE_ID_CLAMPED
    assert torch.equal(c.k_cache, before[0]) and torch.equal(c.v_cache, before[1])
    step(dev(3, 4, 5), c.table, dev(-1, 0, 0))
    assert B.plt_rope_check(c.op) == B.PLT_DEV_GROUP_CLAMPED
    # a prompt that runs past the cache
    T = 40
    q, k, v = ((c.rand(3, 1, T, h, c.d)).to(c.act) for h in (c.Hq, c.Hkv, c.Hkv))
    out = torch.empty_like(q)
    c.v_cache.zero_()
    B.plt_rope_seq(c.op, B.make_rope_seq_args(3, T, q, k, dev(T, 41, -1), out, v_share=v, k_cache=c.k_cache, v_cache=c.v_cache, **c.pages))
    assert B.plt_rope_check(c.op) == B.PLT_DEV_SEQ_LEN_CLAMPED
    assert torch.equal(c.v_cache[c.table[0].long()].flatten(0, 1), v[0, 0, :32]) and (c.v_cache[c.table[2].long()] == 0).all()


def test_replayed_steps_on_other_streams_and_two_handles():
    """A captured step replayed with other lengths and rows in the same buffers gives what a call does; two handles whose calls
    run on two streams do not meet."""
    dev = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cases = [Case(seed=8 + i, L=2, w=6, layout=layout) for i, layout in enumerate(("half", "interleaved"))]
    new = [[(c.rand(3, 2, 1, h, c.d)).to(c.act) for h in (c.Hq, c.Hkv, c.Hkv)] for c in cases for _ in range(4)]
    lens = [dev(1, 9, 30), dev(2, 10, 31), dev(64, 1, 2), dev(0, 33, 17)]

    def state(c):
        return [x.clone() for x in (c.k_cache, c.v_cache, c.k_win, c.v_win)]

    def call(c, rows, n, to, out, stream=0):
        B.plt_rope_step(c.op, B.make_rope_step_args(3, *rows, out, to[0], to[1], n, q_gain=c.q_gain, k_gain=c.k_gain, k_win=to[2], v_win=to[3]), stream)
    want = []
    for i, c in enumerate(cases):
        to, outs = state(c), []
        for s in range(4):
            outs.append(torch.empty_like(new[0][0]))
            call(c, new[4 * i + s], lens[s], to, outs[-1])
        want.append((to, outs))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for i, c in enumerate(cases):       # one captured, one called
        c.to, c.out, c.rows, c.n = state(c), torch.empty_like(new[0][0]), [x.clone() for x in new[4 * i]], lens[0].clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(cases[0], cases[0].rows, cases[0].n, cases[0].to, cases[0].out, torch.cuda.current_stream().cuda_stream)
    got = [[], []]
    for s in range(4):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                for x, y in zip(c.rows, new[4 * i + s]):
                    x.copy_(y)
                c.n.copy_(lens[s])
                if i == 0:
                    graph.replay()
                else:
                    call(c, c.rows, c.n, c.to, c.out, streams[i].cuda_stream)
                got[i].append(c.out.clone())
    torch.cuda.synchronize()
    for i, c in enumerate(cases):
        assert B.plt_rope_check(c.op) == 0
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i][1])) and all(torch.equal(a, b) for a, b in zip(c.to, want[i][0]))


def test_refusals_of_a_call():
    c = Case(seed=6, L=2)
    q, k, v = ((c.rand(3, 2, 1, h, c.d)).to(c.act) for h in (c.Hq, c.Hkv, c.Hkv))
    out, lens = torch.full_like(q, 7.0), torch.tensor([3, 4, 5], dtype=torch.int32, device="cuda")
    base = dict(batch=3, q=q, k_new=k, v_new=v, q_out=out, k_cache=c.k_cache, v_cache=c.v_cache, seq_lens=lens, k_win=c.k_win, v_win=c.v_win)
    for kw, code in ((dict(batch=4), B.PLT_ERR_CAPACITY), (dict(batch=-1), B.PLT_ERR_INVALID_ARG), (dict(q=None), B.PLT_ERR_INVALID_ARG),
                     (dict(k_win=None), B.PLT_ERR_INVALID_ARG), (dict(w_gate=out), B.PLT_ERR_INVALID_ARG), (dict(q=q.data_ptr() + 8), B.PLT_ERR_INVALID_ARG),
                     (dict(row_strides=(516, 0, 0)), B.PLT_ERR_INVALID_ARG), (dict(row_strides=(0, 128, 0)), B.PLT_ERR_INVALID_ARG),
                     (dict(q_out=q, row_strides=(1024, 0, 0)), B.PLT_ERR_INVALID_ARG), (dict(kv_strides=(1024, 256, 64)), B.PLT_ERR_INVALID_ARG),
                     (dict(kv_strides=(1024, 257, 128)), B.PLT_ERR_INVALID_ARG), (dict(seq_lens=lens.data_ptr() + 2), B.PLT_ERR_INVALID_ARG)):
        with pytest.raises(B.PltError) as e:
            B.plt_rope_step(c.op, B.make_rope_step_args(**{**base, **kw}))
        assert e.value.status == code and e.value.message, kw
    s = dict(batch=3, rows=1, q=q, k_share=k, seq_lens=lens, q_out=out, k_share_out=k, k_loc=v, k_loc_out=v)
    for kw, code in ((dict(batch=4), B.PLT_ERR_CAPACITY), (dict(rows=0), B.PLT_ERR_INVALID_ARG), (dict(k_share_out=None), B.PLT_ERR_INVALID_ARG),
                     (dict(k_loc=None), B.PLT_ERR_INVALID_ARG), (dict(k_cache=c.k_cache), B.PLT_ERR_INVALID_ARG),
                     (dict(k_cache=c.k_cache, v_cache=c.v_cache), B.PLT_ERR_INVALID_ARG), (dict(q_out=out.data_ptr() + 2), B.PLT_ERR_INVALID_ARG)):
        with pytest.raises(B.PltError) as e:
            B.plt_rope_seq(c.op, B.make_rope_seq_args(**{**s, **kw}))
        assert e.value.status == code and e.value.message, kw
    B.plt_rope_step(c.op, B.make_rope_step_args(**{**base, "batch": 0}))
    torch.cuda.synchronize()
    assert (out == 7.0).all() and B.plt_rope_check(c.op) == 0
    shifted = B.plt_rope_create(B.make_rope_config("bf16", 3, 2, 4, 2, 128, 64, 16, loop_offset=[1, 2]))
    with pytest.raises(B.PltError) as e:
        B.plt_rope_seq(shifted, B.make_rope_seq_args(**s))
    assert e.value.status == B.PLT_ERR_UNSUPPORTED
    B.plt_rope_destroy(shifted)


def test_caches_beyond_4_gb_offsets():
    """Strides that spread a small cache over more than 2^32 elements' bytes."""
    c = Case(seed=7, B_=2, cap=3, Hq=2, Hkv=1)
    far = 1 << 31                                            # elements between the two sequences: 4 GB of bf16
    big = torch.empty(far + 3 * 128 + 128, dtype=torch.bfloat16, device="cuda")
    big2 = torch.empty_like(big)
    q, k, v = ((c.rand(2, 1, 1, h, c.d)).to(c.act) for h in (2, 1, 1))
    out = torch.empty_like(q)
    B.plt_rope_step(c.op, B.make_rope_step_args(2, q, k, v, out, big, big2, torch.tensor([3, 2], dtype=torch.int32, device="cuda"), kv_strides=(far, 128, 128)))
    torch.cuda.synchronize()
    assert torch.equal(big2[2 * 128:3 * 128], v[0, 0, 0, 0]) and torch.equal(big2[far + 128:far + 256], v[1, 0, 0, 0])
    y, err = c.row(k[1, 0, 0], 1, None)
    c.stored(big[far + 128:far + 256].view(1, -1), y, err, c.act)

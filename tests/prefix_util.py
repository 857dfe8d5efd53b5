"""Problems of shared-prefix attention for the GPU tests, and the bound that a result is held to."""
import torch

from oracle import plt_prefix_attn as oracle_prefix
from paper_2510_24824_b200 import binding as B


class Problem:
    """Sequences with own lengths `own` behind prefixes `plens`, whose groups start at `begin` (and end at its last entry).
    lens: total lengths where they are not prefix + own."""

    def __init__(self, seed, own, plens, begin, L=1, Hq=4, Hkv=2, d=128, cap=None, pcap=None, w=16, page=0, q_len=1, kv="", lens=None, offsets=None,
                 peak=1.5, max_groups=None, max_batch=None, junk=float("nan"), kernel_path=0, strided=False, win_lens=None, scale=0.0, own_strided=False):
        g = torch.Generator("cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.own, self.plens, self.begin, self.L, self.q_len, self.kv = own, plens, begin, L, q_len, kv
        n, groups = len(own), len(plens)
        cap, pcap = cap or max(max(own), 1), pcap or max(plens + [1])
        self.group = [next((i for i in range(groups) if begin[i] <= b < begin[i + 1]), None) for b in range(n)]
        self.lens = lens or [o + (plens[i] if i is not None else 0) for o, i in zip(own, self.group)]
        self.offsets = offsets or list(range(L))
        self.q = (rand(n, L, q_len, Hq, d) * peak).bfloat16()
        e4m3 = kv == "e4m3"
        self.k_scale, self.v_scale = ((torch.rand(Hkv, generator=g, device="cuda") * 0.01 + 0.005 for _ in range(2)) if e4m3 else (None, None))

        def rows(scale, *s):
            x = rand(*s)
            return (x / scale.view(-1, 1)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if e4m3 else x.bfloat16()

        def soil(x, held):      # what lies behind the held rows may be anything
            if e4m3:
                x[held:] = 0x7f
            else:
                x[held:] = junk

        def value(x, scale):
            return x.view(torch.float8_e4m3fn).double() * scale.double().view(-1, 1) if e4m3 else x.double()

        # plain arrays first
        self.k_own, self.v_own = rows(self.k_scale, n, cap, Hkv, d), rows(self.v_scale, n, cap, Hkv, d)
        self.k_pre, self.v_pre = ([rows(s, pcap, Hkv, d) for _ in range(groups)] for s in (self.k_scale, self.v_scale))
        for i, p in enumerate(plens):
            soil(self.k_pre[i], p)
            soil(self.v_pre[i], p)
        for b in range(n):
            held = max(0, self.lens[b] - (plens[self.group[b]] if self.group[b] is not None else 0))
            soil(self.k_own[b], held)
            soil(self.v_own[b], held)
        self.k_win = self.v_win = self.gate = None
        if L > 1:
            self.k_win, self.v_win = rows(self.k_scale, n, L - 1, w, Hkv, d), rows(self.v_scale, n, L - 1, w, Hkv, d)
            self.gate = rand(n, L - 1, q_len, Hq) * 2
        self.values = dict(k_own=value(self.k_own, self.k_scale), v_own=value(self.v_own, self.v_scale),
                           pre=[(value(a, self.k_scale)[:p], value(c, self.v_scale)[:p]) for a, c, p in zip(self.k_pre, self.v_pre, plens)],
                           k_win=None if L == 1 else value(self.k_win, self.k_scale), v_win=None if L == 1 else value(self.v_win, self.v_scale))
        self.w, self.d, self.win_lens, self.scale = w, d, win_lens, scale
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.seq_lens, self.group_begin, self.prefix_lens = dev(self.lens), dev(begin if groups else [0]), dev(plens if groups else [0])
        self.out = torch.full_like(self.q, float("nan"))
        more, shared = {}, {}
        if page:
            per, pper = -(-cap // page), -(-pcap // page)
            pool = n * per + groups * pper + 2
            order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
            self.table, self.ptable = order[: n * per].view(n, per).contiguous(), order[n * per: n * per + groups * pper].view(groups, pper).contiguous()
            self.pool = pool

            def paged(own, pre):
                x = torch.empty(pool, page, Hkv, d, dtype=own.dtype, device="cuda")
                soil(x, 0)
                for table, rows_ in [(self.table[b], own[b]) for b in range(n)] + [(self.ptable[i], pre[i]) for i in range(groups)]:
                    full = torch.empty(len(table) * page, Hkv, d, dtype=own.dtype, device="cuda")
                    soil(full, 0)
                    full[: len(rows_)] = rows_
                    x[table.long()] = full.view(-1, page, Hkv, d)
                return x
            self.k_cache, self.v_cache = paged(self.k_own, self.k_pre), paged(self.v_own, self.v_pre)
            more = dict(page_table=self.table, max_pages=per, num_pool_pages=pool)
            shared = dict(page_table=self.ptable, max_pages=pper)
        else:
            self.k_cache, self.v_cache = self.k_own, self.v_own
            if own_strided:          # [sequences, Hkv, tokens, d + a pad]
                wide = [torch.zeros(n, Hkv, cap, d + 16, dtype=self.k_own.dtype, device="cuda") for _ in range(2)]
                for x, y in zip(wide, (self.k_own, self.v_own)):
                    x[..., :d] = y.transpose(1, 2)
                self.k_cache, self.v_cache = wide
                more["kv_strides"] = (wide[0].stride(0), wide[0].stride(2), wide[0].stride(1))
            if groups:
                kp, vp = torch.stack(self.k_pre), torch.stack(self.v_pre)
                if strided:      # [groups, Hkv, tokens, d + a pad]
                    wide = [torch.zeros(groups, Hkv, pcap, d + 16, dtype=kp.dtype, device="cuda") for _ in range(2)]
                    for x, y in zip(wide, (kp, vp)):
                        x[..., :d] = y.transpose(1, 2)
                    kp, vp = wide
                    shared["strides"] = (kp.stride(0), kp.stride(2), kp.stride(1))
                shared.update(k_prefix=kp, v_prefix=vp)
        self.config = B.make_prefix_config("bf16", max_batch or n, L, Hq, Hkv, d, cap, w if L > 1 else 0, max_prefix_len=pcap,
                                           max_groups=max_groups or max(groups, 1), page_size=page, kv_dtype=kv, q_len=q_len, loop_offset=offsets,
                                           kernel_path=kernel_path, sm_scale=scale)
        self.args = B.make_args(n, self.q, self.k_cache, self.v_cache, self.seq_lens, self.out, k_win=self.k_win, v_win=self.v_win,
                                gate_logits=self.gate, k_scale=self.k_scale, v_scale=self.v_scale, **more)
        self.shared = B.make_prefix_args(groups, self.group_begin, self.prefix_lens, **shared)
        if win_lens is not None:
            self.kept_win = dev(win_lens)
            self.args.win_lens = self.kept_win.data_ptr()
        self.more, self.shared_more = more, shared

    def expect(self, lens=None, plens=None, begin=None):
        v = self.values
        pre = v["pre"] if plens is None else [(a[:p], c[:p]) for (a, c), p in zip(v["pre"], plens)]
        return oracle_prefix.attend(self.q, pre, begin or self.begin, v["k_own"], v["v_own"], lens or self.lens, self.scale or self.d ** -0.5, self.offsets, self.w,
                                    v["k_win"], v["v_win"], self.win_lens, self.gate)

    def run(self, handle=None, stream=0):
        own = handle is None
        handle = handle or B.plt_prefix_attn_create(self.config)
        B.plt_prefix_attn_run(handle, self.args, self.shared, stream)
        bits = B.plt_prefix_attn_check(handle, stream)
        if own:
            B.plt_prefix_attn_destroy(handle)
        return bits

    def hold(self, ref=None):
        """The result against the oracle.  Half a step of bf16 (2^-8) for the stored result; half a step for the probabilities in
        front of |v|; a score of d products in fp32 is off by (d + 2) 2^-24 of the sum of their sizes, which moves a probability by
        that much and the denominator likewise; sums of fp32 weights and the merge: 2^-16 covers up to 2^7 joined parts."""
        out, size, most = ref or self.expect()
        got = self.out.double()
        bound = 2.0 ** -8 * out.abs() + (2.0 ** -8 + 2 * (self.d + 2) * 2.0 ** -24 * most + 2.0 ** -16) * size + 1e-30
        assert torch.isfinite(got).all()
        worst = float(((got - out).abs() / bound).max())
        assert worst <= 1.0, worst
        assert (got[out.abs().amax(-1) == 0] == 0).all()
        return worst

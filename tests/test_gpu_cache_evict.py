"""GPU parity of cache eviction (plt_cache_evict_* through the C ABI) against the fp64 oracle, and a run of its three calls
with the attention that reads the cache."""
import numpy as np
import pytest
import torch

import oracle
from oracle import plt_cache_evict as oracle_evict
from paper_2510_24824_b200 import binding as B
from paper_2510_24824_b200.inputs import f32_to_bf16_bits, make_problem
from paper_2510_24824_b200.runner import CacheEvict, DecodeAttn, DeviceProblem, DiffAttn, to_torch

from diff_util import EPS, LAMBDA_INIT, assert_close, largest, learned, map_error, stored
from gpu_util import assert_parity

pytestmark = pytest.mark.gpu

BASE = dict(name="evict", dtype="bf16", B=3, L=2, Hq=8, Hkv=4, d=128, w=16, lens=("list", [300, 77, 2]), seed=21)


def problem(**kw):
    tail = kw.pop("tail_fill", None)
    return make_problem(dict(BASE, **kw), tail_fill=tail)


def values(p, name):
    """A shared cache as float64 [B, capacity, Hkv, d] (pages gathered, codes with their scales)."""
    a = getattr(p, name)
    if p.page_size:
        a = a[p.page_table].reshape(p.B, -1, p.Hkv, p.d)
    if p.kv_dtype == "e4m3":
        x = torch.from_numpy(np.ascontiguousarray(a)).view(torch.float8_e4m3fn).to(torch.float64).numpy()
        return x * getattr(p, name[0] + "_scale").astype(np.float64)[:, None]
    return stored(a)


def check_weights(p, q_len=1, maps=1, group=1, decay=1.0, gated=True, stride=0, seed=3, held=None):
    rng = np.random.default_rng(seed)
    q = rng.standard_normal((p.B, p.L, q_len, p.Hq, p.d)).astype(np.float32) * 1.5
    q = f32_to_bf16_bits(q) if p.dtype == "bf16" else q
    gate = rng.standard_normal((p.B, p.L - 1, q_len, p.Hq)).astype(np.float32) if gated and p.L > 1 else None
    pitch = stride or p.max_seq_len
    if held is None:
        held = rng.random((p.B, p.Hkv // group, pitch)).astype(np.float32)
    dp = DeviceProblem(p, "cuda:0")
    dq, dg, dw = to_torch(q, p.dtype, "cuda:0"), to_torch(gate, "", "cuda:0"), to_torch(held, "", "cuda:0")
    with CacheEvict(p, q_len=q_len, maps=maps, heads_per_group=group) as op:
        op.weights(dp, dq, dw, gate_logits=dg, decay=decay)
        assert op.check() == 0
        first = dw.clone()
        dw.copy_(torch.from_numpy(held))
        op.weights(dp, dq, dw, gate_logits=dg, decay=decay)
        assert op.check() == 0
        assert torch.equal(first.view(torch.int32), dw.view(torch.int32)), "two calls on the same inputs differ"
    got = first.cpu().numpy()
    k = np.nan_to_num(values(p, "k_cache"))
    n = k.shape[1]
    want, terms = oracle_evict.weights(stored(q), k, p.seq_lens, held[:, :, :n], group, maps, decay, gate, p.sm_scale, p.loop_offset)
    # a score is a sum of d products, each add off by at most 2^-23 of the running sum <= sum |q k|; a weight's exponent and
    # its denominator's by twice that; exp2, the sums over rows and pieces and the store add some 2^-19
    new = want - np.where(np.arange(n) < p.seq_lens[:, None, None], decay * held[:, :, :n].astype(np.float64), held[:, :, :n]) if decay else want
    bound = (2.0 * p.d * 2.0 ** -23 * terms + 2.0 ** -19) * np.abs(new) + 2.0 ** -21 * np.abs(want) + 1e-30
    err = np.abs(got[:, :, :n] - want)
    live = np.arange(n) < p.seq_lens[:, None, None]
    live = np.broadcast_to(live, err.shape)
    assert (err[live] <= bound[live]).all(), f"worst {np.max(err[live] / bound[live]):.2f} of its bound"
    same = got.view(np.int32) == held.view(np.int32)
    assert same[:, :, :n][~live].all() and same[:, :, n:].all(), "totals behind a sequence's length were written"


@pytest.mark.parametrize("dtype,d,kv", [("bf16", 128, ""), ("bf16", 64, ""), ("f32", 128, ""), ("f32", 64, ""), ("bf16", 128, "e4m3")])
@pytest.mark.parametrize("L", [1, 3])
def test_weights_types_and_loops(dtype, d, kv, L):
    check_weights(problem(dtype=dtype, d=d, kv_dtype=kv, L=L, tail_fill=None if kv else float("nan")))


@pytest.mark.parametrize("lens", [[0, 1, 2], [1, 1, 1], [31, 32, 33], [127, 128, 129], [255, 256, 257], [1500, 3, 700]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_lengths(lens, dtype):
    check_weights(problem(lens=("list", lens), L=3, dtype=dtype))


@pytest.mark.parametrize("Hq,Hkv,L,q_len,maps", [(1, 1, 1, 1, 1), (3, 1, 1, 1, 1), (5, 1, 1, 1, 2), (12, 2, 2, 1, 1), (8, 2, 2, 1, 2),
                                                (16, 4, 2, 3, 1), (16, 4, 1, 5, 2), (12, 4, 3, 2, 2), (6, 3, 2, 1, 1), (64, 1, 1, 1, 1)])
@pytest.mark.parametrize("kv", ["", "e4m3"])
def test_weights_rows_and_heads(Hq, Hkv, L, q_len, maps, kv):
    check_weights(problem(Hq=Hq, Hkv=Hkv, L=L, kv_dtype=kv, lens=("list", [200, 40, 3])), q_len=q_len, maps=maps)


@pytest.mark.parametrize("Hq,L,q_len,maps", [(5, 1, 1, 1), (4, 2, 2, 2), (32, 2, 1, 1)])
def test_weights_rows_fp32(Hq, L, q_len, maps):
    check_weights(problem(Hq=Hq, Hkv=1, L=L, dtype="f32", lens=("list", [200, 40, 3])), q_len=q_len, maps=maps)


@pytest.mark.parametrize("group", [1, 2, 4])
@pytest.mark.parametrize("decay", [0.0, 0.5, 1.0])
def test_weights_groups_and_decay(group, decay):
    p = problem()
    held = None
    if decay == 0.0:
        held = np.full((p.B, p.Hkv // group, p.max_seq_len), np.nan, np.float32)      # not read
    check_weights(p, group=group, decay=decay, held=held)


@pytest.mark.parametrize("page", [16, 32, 48, 64, 256])
@pytest.mark.parametrize("dtype,kv,Hkv", [("bf16", "", 4), ("bf16", "e4m3", 1), ("bf16", "", 1), ("f32", "", 2)])
def test_weights_pages(page, dtype, kv, Hkv):
    check_weights(problem(page_size=page, dtype=dtype, kv_dtype=kv, Hkv=Hkv, Hq=2 * Hkv, lens=("list", [300, 77, 1])))


def test_weights_without_gate_with_offsets_and_wide_rows():
    check_weights(problem(loop_offset=[1, 5]), gated=False, stride=333)
    check_weights(problem(loop_offset=[0, 0]), stride=301)


def test_weights_gates_at_their_ends():
    p = problem(lens=("list", [100, 50, 2]))
    q = f32_to_bf16_bits(np.random.default_rng(0).standard_normal((p.B, p.L, 1, p.Hq, p.d)).astype(np.float32))
    dp, dq = DeviceProblem(p, "cuda:0"), to_torch(q, "bf16", "cuda:0")
    with CacheEvict(p) as op:
        for end, rows in ((float("inf"), 1.0), (float("-inf"), 2.0)):
            w = torch.zeros(p.B, p.Hkv, p.max_seq_len, device="cuda")
            op.weights(dp, dq, w, gate_logits=torch.full((p.B, p.L - 1, 1, p.Hq), end, device="cuda"))
            assert op.check() == 0
            assert torch.allclose(w.sum(-1), torch.full((p.B, p.Hkv), 2.0 * rows, device="cuda"), atol=1e-4)


def test_weights_split_over_the_whole_grid_and_in_parts_of_the_batch():
    """One long sequence; and a batch whose scores do not fit the scratch, which runs in several pairs of launches."""
    check_weights(problem(B=1, lens=("list", [20011]), Hq=4, Hkv=1, L=1))
    lens = [300, 77, 0, 5, 300, 1, 222]
    for kw in (dict(Hq=128, Hkv=4, max_seq_len=40000), dict(Hq=16, Hkv=4, max_seq_len=524288, page_size=64)):
        p = problem(B=7, L=2, lens=("list", lens), **kw)
        rows = p.L * p.Hq // p.Hkv
        whole = p.B * p.max_seq_len * p.Hkv * rows * 4
        assert B.plt_cache_evict_workspace_bytes(B.make_evict_config("bf16", p.B, p.L, p.Hq, p.Hkv, p.d, p.max_seq_len, p.page_size)) < whole
        check_weights(p)


def test_weights_strided_cache():
    p = problem()
    rng = np.random.default_rng(2)
    q = f32_to_bf16_bits(rng.standard_normal((p.B, p.L, 1, p.Hq, p.d)).astype(np.float32))
    dp, dq = DeviceProblem(p, "cuda:0"), to_torch(q, "bf16", "cuda:0")
    with CacheEvict(p) as op:
        dense, strided = (torch.zeros(p.B, p.Hkv, p.max_seq_len, device="cuda") for _ in range(2))
        op.weights(dp, dq, dense)
        heads_first = dp.k_cache.permute(0, 2, 1, 3).contiguous()
        dp.k_cache = heads_first
        op.weights(dp, dq, strided, kv_strides=(p.Hkv * p.max_seq_len * p.d, p.d, p.max_seq_len * p.d))
        assert op.check() == 0
    assert torch.equal(dense, strided)


def test_weights_of_many_rows_in_parts_of_the_batch():
    """64 rows a head: a handle whose capacity makes it take the batch in parts, against one that takes it whole."""
    p = problem(B=7, Hq=128, Hkv=4, page_size=64, lens=("list", [300, 77, 0, 5, 300, 1, 222]))
    cap = 1 << 21
    config = B.make_evict_config("bf16", p.B, p.L, p.Hq, p.Hkv, p.d, cap, p.page_size)
    assert B.plt_cache_evict_workspace_bytes(config) < p.B * cap * p.Hkv * 4 * 4
    q = f32_to_bf16_bits(np.random.default_rng(6).standard_normal((p.B, p.L, 1, p.Hq, p.d)).astype(np.float32))
    dp, dq = DeviceProblem(p, "cuda:0"), to_torch(q, "bf16", "cuda:0")
    gate = dp.gate_logits.view(p.B, p.L - 1, 1, p.Hq)
    whole, parts = torch.zeros(p.B, p.Hkv, p.max_seq_len, device="cuda"), torch.zeros(p.B, p.Hkv, cap, device="cuda")
    with CacheEvict(p) as op:
        op.weights(dp, dq, whole, gate_logits=gate)
        assert op.check() == 0
    table = torch.zeros(p.B, cap // p.page_size, dtype=torch.int32, device="cuda")
    table[:, : p.max_pages] = dp.page_table
    h = B.plt_cache_evict_create(config)
    try:
        a = B.make_evict_weights_args(p.B, dq, dp.k_cache, dp.seq_lens, parts, gate_logits=gate, page_table=table, max_pages=table.shape[1],
                                      num_pool_pages=p.num_pool_pages, weights_stride=cap)
        stream = torch.cuda.current_stream().cuda_stream
        B.plt_cache_evict_weights(h, a, stream)
        assert B.plt_cache_evict_check(h, stream) == 0
    finally:
        B.plt_cache_evict_destroy(h)
    n = p.max_seq_len
    assert not parts[:, :, n:].any() and torch.allclose(parts[:, :, :n], whole, rtol=2e-5, atol=1e-8)
    # a row's weights add up to its share of the gate
    live = (dp.seq_lens > 1).float()
    rho = (1 - torch.sigmoid(gate.double())).view(p.B, p.Hkv, -1).sum(-1) + p.Hq // p.Hkv
    assert torch.allclose(whole.double().sum(-1)[live > 0], rho[live > 0], rtol=1e-5)


@pytest.mark.parametrize("Hq,L,q_len,maps", [(17, 1, 1, 1), (12, 2, 1, 1), (8, 2, 2, 1), (33, 1, 1, 1), (24, 2, 1, 1), (8, 2, 2, 2), (64, 1, 1, 1)])
@pytest.mark.parametrize("kv,d", [("", 64), ("", 128), ("e4m3", 128)])
@pytest.mark.parametrize("heads,group,page", [(1, 1, 0), (2, 2, 64), (8, 1, 32), (8, 8, 0)])
def test_weights_above_sixteen_rows(Hq, L, q_len, maps, kv, d, heads, group, page):
    """Every share of the rows full, begun and empty, and heads of a group in one block and in several."""
    check_weights(problem(Hq=Hq * heads, Hkv=heads, L=L, d=d, kv_dtype=kv, page_size=page, lens=("list", [700, 33, 2])), q_len=q_len, maps=maps,
                  group=group, decay=0.5)


@pytest.mark.parametrize("Hq,dtype", [(16, "bf16"), (80, "bf16"), (16, "f32")])
def test_weights_replayed_with_other_lengths_queries_and_keys(Hq, dtype):
    p = problem(Hq=Hq, dtype=dtype, lens=("list", [2100, 900, 40]))
    dp, other = DeviceProblem(p, "cuda:0"), DeviceProblem(problem(Hq=Hq, dtype=dtype, lens=("list", [17, 2100, 0]), max_seq_len=2100, seed=77), "cuda:0")
    q, w = dp.q.view(p.B, p.L, 1, p.Hq, p.d), torch.zeros(p.B, p.Hkv, p.max_seq_len, device="cuda")
    side = torch.cuda.Stream()
    with CacheEvict(p) as op:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            op.weights(dp, q, w, decay=0.25)          # the first call of the handle
        for t in ("q", "k_cache", "seq_lens"):
            getattr(dp, t).copy_(getattr(other, t))
        w.fill_(0.5)
        want = w.clone()
        torch.cuda.synchronize()
        for _ in range(3):
            graph.replay()
            op.weights(other, other.q.view(p.B, p.L, 1, p.Hq, p.d), want, decay=0.25)
        torch.cuda.synchronize()
        assert op.check() == 0
    assert torch.equal(w, want)
    assert bool((w[2] == 0.5).all()) and bool((w[0, :, 17:] == 0.5).all())


# ---- select -------------------------------------------------------------------------------------------------------
def check_select(w, lens, budget, first=0, last=1, stride=0):
    Bn, groups, N = w.shape
    store = np.zeros((Bn, groups, stride or N), np.float32)
    store[:, :, :N] = w
    keep = torch.full((Bn, groups, budget), 77, dtype=torch.int32, device="cuda")
    new = torch.full((Bn,), -5, dtype=torch.int32, device="cuda")
    h = B.plt_cache_evict_create(B.make_evict_config("bf16", Bn, 1, groups, groups, 128, N))
    try:
        dw, dl = to_torch(store, "", "cuda:0"), to_torch(np.asarray(lens, np.int32), "", "cuda:0")
        a = B.make_evict_select_args(Bn, dw, dl, keep, new, budget, first, last, weights_stride=stride)
        B.plt_cache_evict_select(h, a, torch.cuda.current_stream().cuda_stream)
        assert B.plt_cache_evict_check(h, torch.cuda.current_stream().cuda_stream) == 0
    finally:
        B.plt_cache_evict_destroy(h)
    want, lengths = oracle_evict.select(store[:, :, :N], lens, budget, first, last)
    assert np.array_equal(new.cpu().numpy(), lengths)
    got = keep.cpu().numpy()
    assert np.array_equal(got, want), f"{(got != want).sum()} positions differ"


@pytest.mark.parametrize("N,budget", [(1, 1), (2, 1), (33, 32), (1024, 100), (4096, 1), (4097, 4096), (5000, 1024), (9001, 700)])
def test_select_sizes(N, budget):
    rng = np.random.default_rng(N)
    check_select(np.exp(1.5 * rng.standard_normal((2, 3, N))).astype(np.float32), [N, max(1, N // 2)], budget, 0, min(1, budget))


@pytest.mark.parametrize("first,last", [(0, 0), (4, 64), (0, 300), (300, 0), (100, 200)])
def test_select_protected_positions(first, last):
    rng = np.random.default_rng(7)
    check_select(rng.random((2, 2, 2000)).astype(np.float32), [2000, 1999], 300, first, last)


def test_select_ties_and_special_values():
    rng = np.random.default_rng(8)
    w = rng.integers(0, 4, (4, 3, 6000)).astype(np.float32)      # long runs of equal totals
    w[1] = 0.0                                                    # all equal
    w[2] = -w[2]
    w[2, :, ::7] = -0.0
    w[3, :, ::3] = np.nan
    w[3, :, 1::50] = np.inf
    w[3, :, 2::50] = -np.inf
    check_select(w, [6000, 6000, 5999, 6000], 1500, 3, 17)
    check_select(w, [0, 1, 1500, 1501], 1500, 3, 17)
    check_select(w[3:], [6000], 5000, 3, 17)                      # some of the NaN are kept


def test_select_long_rows_on_several_blocks_each():
    rng = np.random.default_rng(9)
    w = np.exp(2.0 * rng.standard_normal((2, 2, 70001))).astype(np.float32)
    w[0, 1] = np.round(w[0, 1])
    check_select(w, [70001, 4099], 3001, 4, 64, stride=70003)
    check_select(w[:1, :1], [65536], 60000, 0, 1, stride=70001)


# ---- compact ------------------------------------------------------------------------------------------------------
def check_compact(p, group=1, budget=64, first=2, last=5, with_totals=True, stride=0, seed=4):
    rng = np.random.default_rng(seed)
    groups, pitch = p.Hkv // group, stride or p.max_seq_len
    keep, new = oracle_evict.select(rng.random((p.B, groups, p.max_seq_len)).astype(np.float32), p.seq_lens, budget, first, last)
    totals = rng.random((p.B, groups, pitch)).astype(np.float32)
    dp = DeviceProblem(p, "cuda:0")
    dk, dn, dw = (to_torch(x, "", "cuda:0") for x in (keep, new, totals))
    with CacheEvict(p, heads_per_group=group) as op:
        op.compact(dp, dk, dn, weights=dw if with_totals else None)
        assert op.check() == 0
    for name in ("k_cache", "v_cache"):
        before = getattr(p, name)
        want = before.copy()
        if p.page_size:
            moved = oracle_evict.compact(before[p.page_table].reshape(p.B, -1, p.Hkv, p.d), keep, new, group)
            for b in range(p.B):
                for i in range(int(new[b])):
                    want[p.page_table[b, i // p.page_size], i % p.page_size] = moved[b, i]
        else:
            want = oracle_evict.compact(before, keep, new, group)
        got = getattr(dp, name).cpu()
        got = got.view(torch.uint8).numpy() if got.dtype != torch.float32 else got.numpy().view(np.uint8)
        assert np.array_equal(got, np.ascontiguousarray(want).view(np.uint8)), f"{name} differs"
    if with_totals:
        want = totals.copy()
        for b in range(p.B):
            for g in range(groups):
                want[b, g, : new[b]] = totals[b, g, keep[b, g, : new[b]]]
                want[b, g, new[b]: p.seq_lens[b]] = 0.0
        assert np.array_equal(dw.cpu().numpy(), want)


@pytest.mark.parametrize("dtype,d,kv", [("bf16", 128, ""), ("bf16", 64, ""), ("f32", 128, ""), ("f32", 64, ""), ("bf16", 128, "e4m3")])
@pytest.mark.parametrize("page", [0, 16])
def test_compact_types(dtype, d, kv, page):
    check_compact(problem(dtype=dtype, d=d, kv_dtype=kv, page_size=page, tail_fill=None if kv else float("nan")))


@pytest.mark.parametrize("lens", [[0, 1, 2], [64, 65, 66], [2000, 1, 700], [5000, 4999, 3]])
@pytest.mark.parametrize("budget", [7, 64, 1900])
def test_compact_lengths(lens, budget):
    check_compact(problem(lens=("list", lens)), budget=min(budget, max(7, max(lens))) if max(lens) >= 7 else 2, first=0 if max(lens) < 7 else 2,
                  last=1 if max(lens) < 7 else 5)


@pytest.mark.parametrize("group", [1, 2, 4])
@pytest.mark.parametrize("page", [0, 64])
def test_compact_groups_and_pages(group, page):
    check_compact(problem(lens=("list", [900, 300, 65]), page_size=page), group=group, budget=256)


def test_compact_without_totals_wide_rows_and_a_large_batch():
    check_compact(problem(), with_totals=False)
    check_compact(problem(lens=("list", [3000, 200, 2900])), stride=3333, budget=1000)
    check_compact(problem(B=40, Hkv=8, lens=("uniform", 1, 400)), budget=100)


def test_compact_clamps_and_flags_what_is_out_of_range():
    p = problem(lens=("list", [100, 50, 20]))
    keep, new = oracle_evict.select(np.random.default_rng(0).random((3, 4, 100)).astype(np.float32), p.seq_lens, 40, 1, 1)
    wild = keep.copy()
    wild[0, 0, 3], wild[0, 1, 4] = -9, 10 ** 8
    dp = DeviceProblem(p, "cuda:0")
    with CacheEvict(p) as op:
        op.compact(dp, to_torch(wild, "", "cuda:0"), to_torch(new, "", "cuda:0"))
        assert op.check() == B.PLT_DEV_KEEP_CLAMPED
        fixed = keep.copy()
        fixed[0, 0, 3], fixed[0, 1, 4] = 3, 99
        want = oracle_evict.compact(p.k_cache, fixed, new)
        assert np.array_equal(dp.k_cache.cpu().view(torch.uint8).numpy(), want.view(np.uint8))
        dp = DeviceProblem(p, "cuda:0")
        op.compact(dp, to_torch(keep, "", "cuda:0"), to_torch(np.array([-3, 1000, 20], np.int32), "", "cuda:0"))
        assert op.check() == B.PLT_DEV_KEEP_CLAMPED
        assert np.array_equal(dp.k_cache[0].cpu().view(torch.uint8).numpy(), p.k_cache[0].view(np.uint8))


def test_refusals_of_calls():
    p = problem(page_size=16, lens=("list", [60, 50, 20]))
    dp = DeviceProblem(p, "cuda:0")
    w = torch.zeros(p.B, p.Hkv, p.max_seq_len, device="cuda")
    keep, new = torch.zeros(p.B, p.Hkv, 32, dtype=torch.int32, device="cuda"), torch.zeros(p.B, dtype=torch.int32, device="cuda")
    q = torch.zeros(p.B, p.L, 1, p.Hq, p.d, dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    with CacheEvict(p) as op:
        make = {"weights": lambda: op.weights_args(dp, q, w), "select": lambda: op.select_args(dp, w, keep, new, 32, 1, 4),
                "compact": lambda: op.compact_args(dp, keep, new, w)}
        bad = [("weights", "q", None), ("weights", "q", q.data_ptr() + 2), ("weights", "weights", None), ("weights", "weights", w.data_ptr() + 2),
               ("weights", "decay", -1.0), ("weights", "decay", float("nan")), ("weights", "weights_stride", 5), ("weights", "kv_stride_n", 3),
               ("weights", "page_table", None), ("weights", "num_pool_pages", 0), ("weights", "struct_size", 3), ("weights", "seq_lens", None),
               ("select", "budget", 0), ("select", "budget", p.max_seq_len + 1), ("select", "keep_first", -1), ("select", "keep_first", 29),
               ("select", "keep_last", 0), ("select", "new_lens", dp.seq_lens.data_ptr()), ("select", "keep", None), ("select", "struct_size", 1),
               ("compact", "keep", None), ("compact", "keep_stride", 0), ("compact", "keep_stride", p.max_seq_len + 1),
               ("compact", "v_cache", dp.k_cache.data_ptr()), ("compact", "new_lens", dp.seq_lens.data_ptr()), ("compact", "k_cache", dp.k_cache.data_ptr() + 2),
               ("compact", "page_table", None), ("compact", "struct_size", 1), ("compact", "batch", -1)]
        for name, field, value in bad:
            a = make[name]()
            setattr(a, field, value)
            with pytest.raises(B.PltError) as e:
                getattr(B, f"plt_cache_evict_{name}")(op.handle, a, stream)
            assert e.value.status == B.PLT_ERR_INVALID_ARG and e.value.message, (name, field)
        for name, field, value in (("weights", "batch", 4), ("compact", "max_pages", 1)):
            a = make[name]()
            setattr(a, field, value)
            with pytest.raises(B.PltError) as e:
                getattr(B, f"plt_cache_evict_{name}")(op.handle, a, stream)
            assert e.value.status == B.PLT_ERR_CAPACITY, (name, field)
        assert op.check() == 0


def test_a_handle_for_a_larger_batch_and_other_buffers_between_calls():
    """max_batch above the batch; the same handle on other addresses, another length and another stream in turn."""
    big = problem(lens=("list", [300, 77, 2]))
    small = problem(B=2, lens=("list", [200, 300]), max_seq_len=300, seed=8)
    side = torch.cuda.Stream()
    with CacheEvict(big, max_batch=9) as op:
        for p in (big, small, big):
            q = f32_to_bf16_bits(np.random.default_rng(p.B).standard_normal((p.B, p.L, 1, p.Hq, p.d)).astype(np.float32))
            dp, dq = DeviceProblem(p, "cuda:0"), to_torch(q, "bf16", "cuda:0")
            w = torch.zeros(p.B + 1, p.Hkv, p.max_seq_len, device="cuda")
            w[p.B] = 3.0
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                op.weights(dp, dq, w)
                assert op.check() == 0
            want, _ = oracle_evict.weights(stored(q), values(p, "k_cache"), p.seq_lens, np.zeros((p.B, p.Hkv, p.max_seq_len)))
            assert np.allclose(w[: p.B].cpu().numpy(), want, rtol=1e-3, atol=1e-7)
            assert bool((w[p.B] == 3.0).all()), "rows behind the batch were written"


def test_compact_caches_that_share_one_buffer_and_repeated_positions():
    """K and V as the two halves of one tensor (strides), and a position that is kept twice."""
    p = problem(lens=("list", [300, 120, 40]))
    dp = DeviceProblem(p, "cuda:0")
    both = torch.stack([dp.k_cache, dp.v_cache], dim=3).contiguous()          # [B, N, Hkv, 2, d]
    dp.k_cache, dp.v_cache = both[:, :, :, 0], both[:, :, :, 1]
    n, h, d = p.max_seq_len, p.Hkv, p.d
    keep, new = oracle_evict.select(np.random.default_rng(3).random((p.B, h, n)).astype(np.float32), p.seq_lens, 50, 2, 5)
    keep[:, :, 10] = keep[:, :, 11]
    with CacheEvict(p) as op:
        op.compact(dp, to_torch(keep, "", "cuda:0"), to_torch(new, "", "cuda:0"), kv_strides=(n * h * 2 * d, h * 2 * d, 2 * d))
        assert op.check() == 0
    for i, name in enumerate(("k_cache", "v_cache")):
        want = oracle_evict.compact(getattr(p, name), keep, new)
        assert np.array_equal(both[:, :, :, i].contiguous().cpu().view(torch.int16).numpy().view(np.uint16), want)


def test_infinite_and_huge_scores():
    """Keys that drive scores far apart, and a cache row of the largest values: weights stay finite and sum to their rows."""
    p = problem(L=1, Hq=4, Hkv=4, lens=("list", [300, 77, 2]))
    k = stored(p.k_cache) * 40.0
    k[:, 1] *= 8.0
    p = p.with_(k_cache=f32_to_bf16_bits(k.astype(np.float32)))
    check_weights(p, decay=0.0)


def test_compact_flags_clamped_lengths_where_nothing_moves():
    """Every kept position is its own slot and there are no totals: the lengths out of range still show."""
    p = problem(lens=("list", [100, 50, 20]))
    keep = np.tile(np.arange(100, dtype=np.int32), (3, 4, 1))
    for lens, new, bits in (([100, 50, 20], [100, 50, 20], 0), ([10 ** 6, 50, 20], [100, 50, 20], B.PLT_DEV_SEQ_LEN_CLAMPED),
                            ([100, -4, 20], [100, 0, 20], B.PLT_DEV_SEQ_LEN_CLAMPED), ([100, 50, 20], [100, 50, 21], B.PLT_DEV_KEEP_CLAMPED)):
        dp = DeviceProblem(p, "cuda:0")
        dp.seq_lens = to_torch(np.array(lens, np.int32), "", "cuda:0")
        with CacheEvict(p) as op:
            op.compact(dp, to_torch(keep, "", "cuda:0"), to_torch(np.array(new, np.int32), "", "cuda:0"))
            assert op.check() == bits, (lens, new)
        assert np.array_equal(dp.k_cache.cpu().view(torch.int16).numpy().view(np.uint16), p.k_cache)


@pytest.mark.parametrize("page", [0, 64])
def test_offsets_beyond_32_bits(page):
    """The same cache in a few MB and spread over more than 2^32 bytes: totals, attention and compaction agree bit for bit."""
    p = problem(B=1, lens=("list", [2300]), page_size=page)
    lambdas, gain = learned(p.d, 1)
    row, budget = p.Hkv * p.d, 700
    near, far = DeviceProblem(p, "cuda:0"), DeviceProblem(p, "cuda:0")
    if page:
        pages = (1 << 33) // (page * row * 2) // 2 + 200                 # 2^32 bytes and some
        pools = []
        for name in ("k_cache", "v_cache"):
            pool = torch.empty(pages, page, p.Hkv, p.d, dtype=torch.bfloat16, device="cuda")
            pool[pages - p.num_pool_pages:] = getattr(near, name).flip(0)
            pools.append(pool)
        far.k_cache, far.v_cache = pools
        far.page_table = (pages - 1 - near.page_table).to(torch.int32)
        strides, count = (0, 0, 0), pages
        rows = [lambda t, which: getattr(near, which)[near.page_table[0].long()].view(-1, row)[:t],
                lambda t, which: getattr(far, which)[far.page_table[0].long()].view(-1, row)[:t]]
    else:
        wide = 1 << 20                                                   # elements between rows: 4.8 GB
        both = torch.empty(p.max_seq_len, wide, dtype=torch.bfloat16, device="cuda")
        far.k_cache, far.v_cache = both, both[:, wide // 2:]
        both[:, :row], both[:, wide // 2:wide // 2 + row] = near.k_cache.view(-1, row), near.v_cache.view(-1, row)
        strides, count = (p.max_seq_len * wide, wide, p.d), 0
        rows = [lambda t, which: getattr(near, which).view(-1, row)[:t],
                lambda t, which: getattr(far, which)[:t, :row]]
    q = near.q.view(p.B, p.L, 1, p.Hq, p.d)
    results = []
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as attn, CacheEvict(p, maps=2) as op:
        for dp, (sb, sn, sh), n in ((near, (0, 0, 0), p.num_pool_pages), (far, strides, count)):
            stream = torch.cuda.current_stream().cuda_stream
            a = dp.args()
            a.kv_stride_b, a.kv_stride_n, a.kv_stride_h, a.num_pool_pages = sb, sn, sh, n
            B.plt_diff_attn_run(attn.handle, a, attn.weights, stream)
            w = torch.zeros(p.B, p.Hkv, p.max_seq_len, device="cuda")
            a = op.weights_args(dp, q, w, kv_strides=(sb, sn, sh))
            a.num_pool_pages = n
            B.plt_cache_evict_weights(op.handle, a, stream)
            keep, new = torch.empty(p.B, p.Hkv, budget, dtype=torch.int32, device="cuda"), torch.empty(p.B, dtype=torch.int32, device="cuda")
            op.select(dp, w, keep, new, budget, 4, 16)
            a = op.compact_args(dp, keep, new, w, kv_strides=(sb, sn, sh))
            a.num_pool_pages = n
            B.plt_cache_evict_compact(op.handle, a, stream)
            assert attn.check() == 0 and op.check() == 0
            results.append((dp.out.clone(), w, keep))
    for one, other in zip(*results):
        assert torch.equal(one, other)
    for which in ("k_cache", "v_cache"):
        assert torch.equal(rows[0](p.max_seq_len, which), rows[1](p.max_seq_len, which)), which
    moved = oracle_evict.compact(values(p, "k_cache"), results[0][2].cpu().numpy(), np.array([budget]))
    assert np.array_equal(rows[0](budget, "k_cache").float().cpu().numpy(), moved.reshape(-1, row)[:budget].astype(np.float32))


def test_two_handles_at_once_on_two_streams():
    """Handles own their workspaces: calls of two of them that overlap on the device give what each gives alone."""
    problems = [problem(B=24, Hq=16, Hkv=4, lens=("uniform", 1, 1500), seed=31), problem(B=20, Hq=40, Hkv=4, lens=("uniform", 1, 1700), seed=32)]
    lambdas, gain = learned(128, 1)
    alone, budget = [], 200
    jobs = []
    for p in problems:                        # 8 and 20 packed rows (16 and 40 with both maps): K once, K twice
        dp = DeviceProblem(p, "cuda:0")
        q = dp.q.view(p.B, p.L, 1, p.Hq, p.d)
        w = torch.zeros(p.B, p.Hkv, p.max_seq_len, device="cuda")
        keep, new = torch.empty(p.B, p.Hkv, budget, dtype=torch.int32, device="cuda"), torch.empty(p.B, dtype=torch.int32, device="cuda")
        jobs.append((p, dp, q, w, keep, new, DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS), CacheEvict(p), torch.cuda.Stream()))

    def work(job):
        p, dp, q, w, keep, new, attn, op, _ = job
        attn.run(dp)
        op.weights(dp, q, w, decay=0.0)
        op.select(dp, w, keep, new, budget, 2, 8)
        return dp.out, w, keep, new
    for job in jobs:
        alone.append([t.clone() for t in work(job)])
    torch.cuda.synchronize()
    for _ in range(20):
        for job in jobs:
            with torch.cuda.stream(job[-1]):
                work(job)
    torch.cuda.synchronize()
    for job, want in zip(jobs, alone):
        assert job[6].check() == 0 and job[7].check() == 0
        for got, t in zip((job[1].out, job[3], job[4], job[5]), want):
            live = t == t if t.is_floating_point() else slice(None)
            assert torch.equal(got[live], t[live])
        job[6].close()
        job[7].close()


def test_a_batch_of_none_does_nothing():
    p = problem()
    dp = DeviceProblem(p, "cuda:0")
    w = torch.full((p.B, p.Hkv, p.max_seq_len), 7.0, device="cuda")
    keep, new = torch.full((p.B, p.Hkv, 32), 5, dtype=torch.int32, device="cuda"), torch.full((p.B,), 5, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    with CacheEvict(p) as op:
        for name, a in (("weights", op.weights_args(dp, dp.q.view(p.B, p.L, 1, p.Hq, p.d), w)), ("select", op.select_args(dp, w, keep, new, 32, 1, 4)),
                        ("compact", op.compact_args(dp, keep, new, w))):
            a.batch = 0
            getattr(B, f"plt_cache_evict_{name}")(op.handle, a, stream)
        assert op.check() == 0
    assert bool((w == 7.0).all()) and bool((keep == 5).all()) and bool((new == 5).all())


# ---- together -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("page,kv", [(0, ""), (32, ""), (32, "e4m3")])
@pytest.mark.parametrize("diff", [False, True])
def test_a_cache_held_to_its_budget_between_steps(page, kv, diff):
    """Attention, totals, selection and compaction in one captured graph, then attention on the smaller cache: every stage
    against its oracle on what the stage before left."""
    p = problem(page_size=page, kv_dtype=kv, lens=("list", [400, 150, 30]), max_seq_len=448)
    budget, first, last = 100, 4, 16
    lambdas, gain = learned(p.d, 1)
    dp = DeviceProblem(p, "cuda:0")
    w = torch.rand(p.B, p.Hkv, p.max_seq_len, device="cuda") * 0.01
    held = w.cpu().numpy()
    keep, new = torch.empty(p.B, p.Hkv, budget, dtype=torch.int32, device="cuda"), torch.empty(p.B, dtype=torch.int32, device="cuda")
    q = dp.q.view(p.B, p.L, 1, p.Hq, p.d)
    attn = DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS) if diff else DecodeAttn(p)
    out2 = torch.full_like(dp.out, float("nan"))
    side = torch.cuda.Stream()
    with attn, CacheEvict(p, maps=2 if diff else 1) as op:
        def step():
            attn.run(dp)
            op.weights(dp, q, w, gate_logits=dp.gate_logits.view(p.B, p.L - 1, 1, p.Hq), decay=0.5)
            op.select(dp, w, keep, new, budget, first, last)
            op.compact(dp, keep, new, weights=w)
            lens, dp.seq_lens = dp.seq_lens, new
            attn.run(dp, out=out2)
            dp.seq_lens = lens
        saved = [t.clone() for t in (dp.k_cache, dp.v_cache, w)]
        with torch.cuda.stream(side):
            step()                                    # outside a capture first: tensor maps are encoded
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        for t, s in zip((dp.k_cache, dp.v_cache, w), saved):
            t.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert attn.check() == 0 and op.check() == 0
    want_w, _ = oracle_evict.weights(stored(p.q)[:, :, None], values(p, "k_cache"), p.seq_lens, held[:, :, : values(p, "k_cache").shape[1]], 1,
                                     2 if diff else 1, 0.5, p.gate_logits[:, :, None])
    got_keep, got_new = keep.cpu().numpy(), new.cpu().numpy()
    assert np.array_equal(got_new, np.minimum(p.seq_lens, budget))
    # the kept totals are those of the exact ranking up to the totals' own error
    for b in range(p.B):
        n, m = int(p.seq_lens[b]), int(got_new[b])
        for g in range(p.Hkv):
            at = got_keep[b, g, :m]
            assert (np.diff(at) > 0).all() and at[0] >= 0 and at[-1] == n - 1 and (at[: min(first, m)] == np.arange(min(first, m))).all()
            dropped = np.setdiff1d(np.arange(n), at)
            inner = at[(at >= first) & (at < n - last)]
            if len(dropped) and len(inner):
                assert want_w[b, g, inner].min() >= want_w[b, g, dropped].max() - 1e-4 * want_w[b, g].max()
            assert np.allclose(w[b, g, :m].cpu().numpy(), want_w[b, g, at], rtol=1e-3, atol=1e-7)
            assert not w[b, g, m:n].any()
    # the attention on the smaller cache: the problem with the moved rows
    after = p.with_(seq_lens=got_new, k_cache=_numpy(dp.k_cache, p), v_cache=_numpy(dp.v_cache, p))
    moved = oracle_evict.compact(values(p, "k_cache"), got_keep, got_new)
    for b in range(p.B):
        assert np.array_equal(values(after, "k_cache")[b, : got_new[b]], moved[b, : got_new[b]])
    got = out2.float().cpu().numpy().astype(np.float64)
    if diff:
        fp8 = p.kv_dtype == "e4m3"
        e = map_error("bf16", max(largest(a, p.v_scale if fp8 else None) for a in (p.v_cache, p.v_win)), p.d, largest(p.q),
                      max(largest(a, p.k_scale if fp8 else None) for a in (p.k_cache, p.k_win)))
        assert_close(got, oracle.diff_maps(after), lambdas, gain, "bf16", e, "after")
    else:
        assert_parity(got, oracle.decode_attn(after), "bf16", "after")


def _numpy(t, p):
    t = t.cpu()
    return t.view(torch.int16).numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.numpy()

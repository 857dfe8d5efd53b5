"""GPU parity of differential attention (plt_diff_attn_* and plt_diff_seq_attn_* through the C ABI) against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2510_24824_b200 import binding as B
from paper_2510_24824_b200.inputs import f32_to_bf16_bits, make_problem, make_seq_problem
from paper_2510_24824_b200.runner import DeviceProblem, DiffAttn, DiffSeqAttn, to_torch

from diff_util import EPS, LAMBDA_INIT, assert_close, largest, learned, map_error

pytestmark = pytest.mark.gpu

BASE = dict(name="diff", dtype="bf16", B=3, L=2, Hq=8, Hkv=2, d=128, w=48, lens=("list", [300, 77, 2]), seed=5)


def spec(**kw):
    return dict(BASE, **kw)


def e_map(p, e4m3_terms=False):
    fp8 = p.kv_dtype == "e4m3"
    v = max(largest(a, p.v_scale if fp8 else None) for a in (p.v_cache, p.v_win))
    k = max(largest(a, p.k_scale if fp8 else None) for a in (p.k_cache, p.k_win))
    return map_error(p.dtype, v, p.d, largest(p.q), k, e4m3_terms)


def run(p, heads=1, norm=True, seed=0, **config):
    lambdas, gain = learned(p.d, heads, seed, norm)
    dp = DeviceProblem(p, "cuda:0")
    dp.out.fill_(float("nan"))
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS, **config) as op:
        op.run(dp)
        assert op.check() == 0
        first = dp.out.clone()
        op.run(dp)
        assert op.check() == 0
        assert torch.equal(first, dp.out), "two runs on the same inputs differ"
    got = first.float().cpu().numpy().astype(np.float64)
    return assert_close(got, oracle.diff_maps(p), lambdas, gain, p.dtype, e_map(p, config.get("kernel_path") == B.PLT_PATH_TCGEN05), p.name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("L", [1, 2, 3])
def test_types_head_sizes_and_loops(dtype, d, L):
    run(make_problem(spec(dtype=dtype, d=d, L=L), tail_fill=float("nan")))


@pytest.mark.parametrize("lens", [[0, 1, 2], [1, 1, 1], [63, 64, 65], [127, 128, 129], [1023, 1, 500]])
def test_lengths_from_nothing_up(lens):
    run(make_problem(spec(lens=("list", lens), L=3), tail_fill=float("nan")))


@pytest.mark.parametrize("heads", [(8, 8), (8, 1), (16, 2), (4, 4), (12, 4), (32, 1)])
def test_head_layouts(heads):
    Hq, Hkv = heads
    run(make_problem(spec(Hq=Hq, Hkv=Hkv, L=1)), heads=Hq)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("per_head", [False, True])
def test_parameters(norm, per_head):
    run(make_problem(spec()), heads=8 if per_head else 1, norm=norm, seed=9)


@pytest.mark.parametrize("page,kv", [(16, ""), (64, ""), (128, ""), (32, "e4m3"), (64, "e4m3"), (128, "e4m3")])
def test_pages(page, kv):
    run(make_problem(spec(page_size=page, kv_dtype=kv, lens=("list", [500, 64, 1])), tail_fill=float("nan") if not kv else None))


def test_e4m3_and_fp32_pages():
    run(make_problem(spec(kv_dtype="e4m3", L=3)))
    run(make_problem(spec(dtype="f32", page_size=32, lens=("list", [200, 33, 1]))))


@pytest.mark.parametrize("kv,Hq,Hkv", [("", 16, 2), ("", 64, 2), ("e4m3", 16, 2), ("e4m3", 16, 1)])
def test_tensor_memory_kernels(kv, Hq, Hkv):
    """The tcgen05 kernels with 16, 32 or 64 packed rows."""
    run(make_problem(spec(kv_dtype=kv, Hq=Hq, Hkv=Hkv, L=1, lens=("list", [700, 128, 1]))), kernel_path=B.PLT_PATH_TCGEN05)


def test_gates_at_their_ends_and_window_lengths():
    p = make_problem(spec())
    gate = p.gate_logits.copy()
    gate[0], gate[1] = np.inf, -np.inf
    run(p.with_(gate_logits=gate, win_lens=np.array([[0], [5], [1]], np.int32)))


def test_long_sequence_spread_over_the_whole_grid():
    run(make_problem(spec(B=1, lens=("list", [20011]), Hq=4, Hkv=1, L=1)))


@pytest.mark.parametrize("q_len", [2, 4])
def test_several_tokens_in_one_step(q_len):
    p = make_problem(spec(L=2, Hq=4, Hkv=1, lens=("list", [300, 77, 2]), w=40))
    rng = np.random.default_rng(8)
    q = f32_to_bf16_bits(rng.standard_normal((p.B, p.L, q_len, p.Hq, p.d)).astype(np.float32))
    gate = rng.standard_normal((p.B, p.L - 1, q_len, p.Hq)).astype(np.float32)
    lambdas, gain = learned(p.d, p.Hq)
    dp = DeviceProblem(p, "cuda:0")
    dq, dg = to_torch(q, "bf16", "cuda:0"), to_torch(gate, "", "cuda:0")
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda:0")
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS, q_len=q_len) as op:
        a = dp.args(out)
        a.q, a.gate_logits = dq.data_ptr(), dg.data_ptr()
        B.plt_diff_attn_run(op.handle, a, op.weights, torch.cuda.current_stream().cuda_stream)
        assert op.check() == 0
    y = oracle.diff_maps(p, q, gate, q_len)
    e = map_error("bf16", max(largest(p.v_cache), largest(p.v_win)), p.d, largest(q), max(largest(p.k_cache), largest(p.k_win)))
    assert_close(out.float().cpu().numpy().astype(np.float64), y, lambdas, gain, "bf16", e, f"q_len {q_len}")


@pytest.mark.parametrize("kv", ["", "e4m3"])
def test_step_appends_and_attends(kv):
    """The pre-step's cache rows, window slots and gate logits, then the attention on them."""
    p = make_problem(spec(kv_dtype=kv, page_size=32, lens=("list", [50, 32, 1])))
    rng = np.random.default_rng(3)
    k_new, v_new = (f32_to_bf16_bits(rng.standard_normal((p.B, p.L, p.Hkv, p.d)).astype(np.float32)) for _ in range(2))
    w_gate = (rng.standard_normal((p.Hq, p.d)) / np.sqrt(p.d)).astype(np.float32)
    b_gate = rng.standard_normal(p.Hq).astype(np.float32)
    lambdas, gain = learned(p.d, 1)
    dp = DeviceProblem(p, "cuda:0")
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        out = op.step(dp, to_torch(k_new, "bf16", "cuda:0"), to_torch(v_new, "bf16", "cuda:0"), to_torch(w_gate, "", "cuda:0"),
                      to_torch(b_gate, "", "cuda:0"))
        assert op.check() == 0
    after, logits = oracle.prestep(p, k_new, v_new, w_gate.astype(np.float64), b_gate.astype(np.float64))
    assert np.array_equal(dp.k_cache.cpu().view(torch.uint8).numpy(), np.ascontiguousarray(after.k_cache).view(np.uint8))
    assert np.array_equal(dp.v_win.cpu().view(torch.uint8).numpy(), np.ascontiguousarray(after.v_win).view(np.uint8))
    # the logits are fp32 dot products of d terms; the attention is compared on the very logits it used
    used = dp.gate_logits.cpu().numpy()
    assert np.abs(used - after.gate_logits).max() < 1e-4
    y = oracle.diff_maps(after.with_(gate_logits=used))
    assert_close(out.float().cpu().numpy().astype(np.float64), y, lambdas, gain, "bf16", e_map(after), "step")


def test_graph_replay_on_another_stream_and_new_lengths():
    p = make_problem(spec(lens=("list", [300, 200, 100])))
    lambdas, gain = learned(p.d, 1)
    dp = DeviceProblem(p, "cuda:0")
    side = torch.cuda.Stream()
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        with torch.cuda.stream(side):
            op.run(dp)
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                op.run(dp)
        for lens in ([300, 200, 100], [1, 299, 0]):
            dp.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            dp.out.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            q = p.with_(seq_lens=np.array(lens, np.int32))
            assert_close(dp.out.float().cpu().numpy().astype(np.float64), oracle.diff_maps(q), lambdas, gain, "bf16", e_map(q), f"{lens}")
        assert op.check() == 0


def test_bad_lengths_and_pages_are_clamped_and_flagged():
    p = make_problem(spec(page_size=16, lens=("list", [50, 40, 30])))
    lambdas, gain = learned(p.d, 1)
    bad = DeviceProblem(p.with_(seq_lens=np.array([-4, p.max_seq_len + 9, 30], np.int32)), "cuda:0")
    with DiffAttn(p, lambdas, gain) as op:
        op.run(bad)
        assert op.check() == B.PLT_DEV_SEQ_LEN_CLAMPED
        assert not bad.out[0].any()
        table = p.page_table.copy()
        table[1, 0] = 10 ** 6
        op.run(DeviceProblem(p.with_(page_table=table), "cuda:0"))
        assert op.check() == B.PLT_DEV_PAGE_ID_CLAMPED


def test_a_handle_for_a_larger_batch():
    p = make_problem(spec(lens=("list", [300, 77, 2])))
    lambdas, gain = learned(p.d, 1)
    dp = DeviceProblem(p, "cuda:0")
    out = torch.full((p.B + 1, p.L, p.Hq, p.d), 5.0, dtype=torch.bfloat16, device="cuda")
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS, max_batch=70) as op:
        op.run(dp, out=out)
        assert op.check() == 0
    assert_close(out[: p.B].float().cpu().numpy().astype(np.float64), oracle.diff_maps(p), lambdas, gain, "bf16", e_map(p), "max_batch 70")
    assert bool((out[p.B] == 5.0).all()), "rows behind the batch were written"


def test_strided_head_major_cache():
    p = make_problem(spec(lens=("list", [320, 100, 7])))
    lambdas, gain = learned(p.d, p.Hq)
    dp = DeviceProblem(p, "cuda:0")
    dp.k_cache, dp.v_cache = (t.permute(0, 2, 1, 3).contiguous() for t in (dp.k_cache, dp.v_cache))
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        a = dp.args()
        a.kv_stride_b, a.kv_stride_h, a.kv_stride_n = p.Hkv * 320 * p.d, 320 * p.d, p.d
        B.plt_diff_attn_run(op.handle, a, op.weights, torch.cuda.current_stream().cuda_stream)
        assert op.check() == 0
    assert_close(dp.out.float().cpu().numpy().astype(np.float64), oracle.diff_maps(p), lambdas, gain, "bf16", e_map(p), "HND strides")


def test_refusals_of_a_call():
    p = make_problem(spec())
    lambdas, gain = learned(p.d, 1)
    dp = DeviceProblem(p, "cuda:0")
    with DiffAttn(p, lambdas, gain) as op:
        good = [torch.zeros(1, p.d // 2, device="cuda") for _ in range(4)]
        stream = torch.cuda.current_stream().cuda_stream

        def refused(args, weights, status=B.PLT_ERR_INVALID_ARG):
            dp.out.fill_(7.0)
            with pytest.raises(B.PltError) as e:
                B.plt_diff_attn_run(op.handle, args, weights, stream)
            assert e.value.status == status and e.value.message
            torch.cuda.synchronize()
            assert bool((dp.out == 7.0).all()), "a refused call wrote its output"

        for bad in (B.make_diff_weights(*good, lambda_heads=3), B.make_diff_weights(None, *good[1:], lambda_heads=1),
                    B.make_diff_weights(good[0].data_ptr() + 2, *good[1:], lambda_heads=1),
                    B.make_diff_weights(*good, norm_gain=good[0].data_ptr() + 1)):
            refused(dp.args(), bad)
        short = B.make_diff_weights(*good)
        short.struct_size = 4
        refused(dp.args(), short)
        for field, value, status in (("batch", -1, B.PLT_ERR_INVALID_ARG), ("batch", 4, B.PLT_ERR_CAPACITY), ("q", None, B.PLT_ERR_INVALID_ARG),
                                     ("gate_logits", None, B.PLT_ERR_INVALID_ARG), ("k_cache", dp.k_cache.data_ptr() + 2, B.PLT_ERR_INVALID_ARG),
                                     ("kv_stride_n", 3, B.PLT_ERR_INVALID_ARG), ("struct_size", 3, B.PLT_ERR_INVALID_ARG)):
            a = dp.args()
            setattr(a, field, value)
            refused(a, op.weights, status)
        a = dp.args()
        a.batch = 0
        B.plt_diff_attn_run(op.handle, a, op.weights, stream)     # nothing to do is not an error
        assert op.check() == 0


# ---- prompts ------------------------------------------------------------------------------------------------------
def run_seq(p, heads=1, norm=True, seed=0):
    lambdas, gain = learned(p.d, heads, seed, norm)
    with DiffSeqAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        op.out.fill_(float("nan"))
        op.run()
        assert op.check() == 0
        first = op.out.clone()
        op.run()
        assert op.check() == 0
        assert torch.equal(first, op.out), "two runs on the same inputs differ"
    v, k = (max(largest(a), largest(b)) for a, b in ((p.v_share, p.v_loc), (p.k_share, p.k_loc)))
    e = map_error("bf16", v, p.d, largest(p.q), k)
    return assert_close(first.float().cpu().numpy().astype(np.float64), oracle.diff_seq_maps(p), lambdas, gain, "bf16", e, p.name)


@pytest.mark.parametrize("L", [1, 2, 3])
@pytest.mark.parametrize("n", [1, 2, 127, 128, 129, 257, 700])
def test_prompt_lengths_around_the_tiles(n, L):
    run_seq(make_seq_problem(B=2, L=L, T=n, Hq=4, Hkv=2, d=128, w=64, lens=[n, max(1, n // 2)], seed=n + L))


@pytest.mark.parametrize("heads", [(1, 1), (3, 3), (6, 2), (3, 1)])
def test_prompt_head_layouts_and_parameters(heads):
    Hq, Hkv = heads
    run_seq(make_seq_problem(B=2, L=2, T=200, Hq=Hq, Hkv=Hkv, d=128, w=33, lens=[200, 0], seed=4), heads=Hq, norm=Hq != 3)


def test_prompt_offsets_windows_and_garbage_behind_the_lengths():
    p = make_seq_problem(B=2, L=3, T=300, Hq=2, Hkv=1, d=128, w=1, lens=[300, 131], seed=6, loop_offset=[0, 0, 5])
    for name in ("k_share", "v_share"):
        a = getattr(p, name).copy()
        a[1, 131:] = 0x7FC0           # NaN
        p = p.with_(**{name: a})
    for name in ("k_loc", "v_loc"):
        a = getattr(p, name).copy()
        a[1, :, 131:] = 0x7FC0
        p = p.with_(**{name: a})
    lambdas, gain = learned(128, 1)
    clean = p.with_(**{n: np.where(getattr(p, n) == 0x7FC0, 0, getattr(p, n)).astype(np.uint16) for n in ("k_share", "v_share", "k_loc", "v_loc")})
    with DiffSeqAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        got = op.run().float().cpu().numpy().astype(np.float64)
        assert op.check() == 0
    e = map_error("bf16", max(largest(clean.v_share), largest(clean.v_loc)), 128, largest(p.q), max(largest(clean.k_share), largest(clean.k_loc)))
    assert_close(got, oracle.diff_seq_maps(clean), lambdas, gain, "bf16", e, "garbage")


def test_prompt_with_sharp_rows():
    """Scores far apart (rescaled accumulators) and large values."""
    p = make_seq_problem(B=1, L=2, T=400, Hq=2, Hkv=2, d=128, w=50, seed=7)
    big = f32_to_bf16_bits((np.random.default_rng(1).standard_normal(p.q.shape) * 6.0).astype(np.float32))
    run_seq(p.with_(q=big))


def test_prompt_graph_replay_with_new_lengths():
    p = make_seq_problem(B=2, L=2, T=300, Hq=2, Hkv=1, d=128, w=64, seed=12)
    lambdas, gain = learned(128, 1)
    side = torch.cuda.Stream()
    with DiffSeqAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        with torch.cuda.stream(side):
            op.run()
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                op.run()
        for lens in ([300, 129], [0, 1]):
            op.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            op.out.fill_(float("nan"))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            q = p.with_(seq_lens=np.array(lens, np.int32))
            e = map_error("bf16", max(largest(p.v_share), largest(p.v_loc)), 128, largest(p.q), max(largest(p.k_share), largest(p.k_loc)))
            assert_close(op.out.float().cpu().numpy().astype(np.float64), oracle.diff_seq_maps(q), lambdas, gain, "bf16", e, f"{lens}")
        assert op.check() == 0
        bad = torch.tensor([-1, 10 ** 6], dtype=torch.int32)
        op.seq_lens.copy_(bad)
        op.run()
        assert op.check() == B.PLT_DEV_SEQ_LEN_CLAMPED


def test_prompt_rows_are_decode_steps():
    """The last row of a prompt and the decode step at its length give the same head outputs."""
    s = make_seq_problem(B=1, L=1, T=150, Hq=4, Hkv=2, d=128, w=0, seed=8)
    lambdas, gain = learned(128, 4)
    with DiffSeqAttn(s, lambdas, gain, LAMBDA_INIT, EPS) as op:
        row = op.run()[0, 0, -1].float()
        assert op.check() == 0
    p = make_problem(spec(B=1, L=1, Hq=4, lens=("list", [150]))).with_(q=np.ascontiguousarray(s.q[:, :, -1]), k_cache=s.k_share, v_cache=s.v_share)
    dp = DeviceProblem(p, "cuda:0")
    with DiffAttn(p, lambdas, gain, LAMBDA_INIT, EPS) as op:
        step = op.run(dp)[0, 0].float()
        assert op.check() == 0
    y = oracle.diff_maps(p)
    e = map_error("bf16", largest(p.v_cache), 128, largest(p.q), largest(p.k_cache))
    for got in (row, step):
        assert_close(got.cpu().numpy().astype(np.float64)[None, None], y, lambdas, gain, "bf16", e, "last row")

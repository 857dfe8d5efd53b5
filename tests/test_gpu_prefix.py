"""Decode steps behind shared prefixes on the GPU against the fp64 oracle."""
import pytest
import torch

from paper_2510_24824_b200 import binding as B
from prefix_util import Problem

pytestmark = pytest.mark.gpu

CASES = [
    dict(own=[5, 1, 17], plens=[300], begin=[0, 3]),
    dict(own=[1], plens=[1], begin=[0, 1]),
    dict(own=[1], plens=[128], begin=[0, 1], Hq=1, Hkv=1),
    dict(own=[3], plens=[129], begin=[0, 1], Hq=8, Hkv=8),
    dict(own=[2, 2], plens=[127], begin=[0, 2], d=64),
    dict(own=[40] * 40, plens=[1000], begin=[0, 40], Hq=8, Hkv=2),                   # 160 rows: both tiles
    dict(own=[9] * 70, plens=[513], begin=[0, 70], Hq=8, Hkv=2, d=64),              # 280 rows: two units a head
    dict(own=[7, 8, 9, 10, 11], plens=[256, 40, 700], begin=[0, 2, 3, 5]),           # three groups
    dict(own=[7, 8, 9, 10, 11, 12], plens=[256, 40, 700], begin=[1, 2, 2, 4]),       # sequences in front, an empty group, sequences behind
    dict(own=[20, 3, 5], plens=[260], begin=[0, 3], L=3, w=5),
    dict(own=[20, 3, 5], plens=[260], begin=[0, 3], L=2, Hq=12, Hkv=4, d=64, w=40),
    dict(own=[9, 30, 4], plens=[130], begin=[0, 3], q_len=4),
    dict(own=[9, 30, 4], plens=[130], begin=[0, 3], q_len=3, L=2, w=7),
    dict(own=[9, 30, 64], plens=[333], begin=[0, 3], page=16),
    dict(own=[9, 30, 64], plens=[333, 50], begin=[0, 2, 3], page=48),
    dict(own=[9, 300, 64], plens=[333, 1000], begin=[0, 1, 3], page=64, L=2),
    dict(own=[9, 300, 64], plens=[1000], begin=[0, 2], page=256),
    dict(own=[5, 1, 17], plens=[300], begin=[0, 3], kv="e4m3"),
    dict(own=[50] * 40, plens=[700], begin=[0, 40], Hq=8, Hkv=2, kv="e4m3", L=2),
    dict(own=[9, 300, 64], plens=[333, 1000], begin=[0, 1, 3], page=32, kv="e4m3"),
    dict(own=[9, 300, 64], plens=[129, 1], begin=[0, 1, 3], page=64, kv="e4m3", q_len=2),
    dict(own=[6, 7, 8], plens=[500], begin=[0, 3], Hq=10, Hkv=2, L=2),               # an odd group of heads
    dict(own=[33] * 9, plens=[2000], begin=[0, 9], Hq=64, Hkv=1),                    # 64 packed rows a sequence
    dict(own=[6, 7, 8], plens=[400], begin=[0, 3], strided=True),
    dict(own=[6, 7, 8], plens=[400, 90], begin=[0, 1, 3], strided=True, d=64, pcap=500),
    dict(own=[12, 25], plens=[5000], begin=[0, 2], Hq=32, Hkv=8),                    # many blocks share a unit
    dict(own=[4] * 130, plens=[64] * 65, begin=list(range(0, 131, 2))),              # many short groups: pieces of one key tile
    dict(own=[2] * 12, plens=[130] * 12, begin=list(range(13)), Hq=32, Hkv=8),
    dict(own=[8, 9], plens=[200], begin=[0, 2], offsets=[2, 5], L=2),
    dict(own=[8, 9, 10], plens=[200], begin=[0, 3], L=3, w=9, win_lens=[[0, 9], [3, 1], [9, 0]]),
    dict(own=[8, 9, 10], plens=[200], begin=[0, 3], scale=0.01),
    dict(own=[8, 9, 40], plens=[200], begin=[0, 3], own_strided=True, L=2),
    dict(own=[1000, 3, 700, 900] * 8, plens=[1000, 300], begin=[0, 20, 30], L=2, Hq=32, Hkv=8),      # multiprocessors divided between the passes
    dict(own=[1000, 3, 700, 900] * 8, plens=[1000, 300], begin=[0, 20, 30], L=2, Hq=32, Hkv=8, kv="e4m3", page=64),
    dict(own=[300] * 8, plens=[6000], begin=[0, 8], Hq=48, Hkv=8, d=64),                             # 6 heads: query rows without TMA
    dict(own=[300] * 8, plens=[6000], begin=[0, 8], Hq=24, Hkv=8, kv="e4m3", L=2),
    dict(own=[2] * 40, plens=[9000] * 40, begin=list(range(41)), Hq=2, Hkv=1),                       # a plan of many groups, several pieces a block
    dict(own=[2] * 20, plens=[2500] * 20, begin=list(range(21)), Hq=32, Hkv=8),                      # more units than blocks
    dict(own=[900], plens=[12615], begin=[0, 1], Hq=3, Hkv=1, kv="e4m3", q_len=2, page=32),          # pieces of a tile each, many to a row
    dict(own=[6, 0, 3], plens=[20000, 3000], begin=[0, 1, 3], Hq=4, Hkv=2, d=64, L=2, w=9),          # several tiles each, many to a row
    dict(own=[5], plens=[128 * 9], begin=[0, 1], Hq=8, Hkv=1),                                       # at the borders of the merge's forms
    dict(own=[5], plens=[128 * 8], begin=[0, 1], Hq=8, Hkv=1),
]


@pytest.mark.parametrize("kw", CASES, ids=str)
def test_against_the_oracle(kw):
    p = Problem(len(str(kw)), **kw)
    assert p.run() == 0
    p.hold()


@pytest.mark.parametrize("kv", ["", "e4m3"])
def test_lengths_that_end_inside_the_prefix(kv):
    """Slots without a sequence, rows that see part of the prefix or nothing at all, and windows of rows without own keys."""
    lens = [0, 1, 2, 100, 128, 129, 255, 299, 300, 301, 305]
    own = [max(0, n - 300) for n in lens]
    p = Problem(3, own, [300], [0, len(lens)], L=3, w=6, kv=kv, lens=lens, cap=8)
    assert p.run() == 0
    p.hold()
    p = Problem(4, own, [300], [0, len(lens)], q_len=4, kv=kv, lens=lens, cap=8)
    assert p.run() == 0
    p.hold()


@pytest.mark.parametrize("plens,begin", [([], []), ([0, 0], [0, 1, 3]), ([77, 0], [0, 1, 3]), ([77], [0, 0]), ([50, 60], [2, 2, 2])])
def test_without_prefixes(plens, begin):
    """No groups, prefixes of length 0 and groups without a sequence: what plt_decode_attn_run gives, within both's bounds."""
    p = Problem(5, [40, 30, 3], plens, begin, L=2, w=8, pcap=100)
    assert p.run() == 0
    p.hold(p.expect(begin=begin or [0]))


def test_peaked_rows_move_the_reference():
    """Scores that grow along the prefix outrun the reference in many tiles."""
    for kv in ("", "e4m3"):
        p = Problem(6, [5] * 40, [1500], [0, 40], Hq=8, Hkv=2, kv=kv, peak=6.0)
        assert p.run() == 0
        p.hold()


def test_a_ramp_of_scores_rescales_every_tile():
    p = Problem(7, [3, 4], [900], [0, 2], Hq=2, Hkv=1)
    ramp = torch.linspace(-12, 12, 900, device="cuda").view(-1, 1, 1) * torch.ones(1, 1, 128, device="cuda")
    p.q.fill_(1.0)
    k = p.shared_more["k_prefix"]
    k[0, :900] = (ramp / 4).bfloat16()
    p.values["pre"][0] = (k[0, :900].double(), p.values["pre"][0][1])
    assert p.run() == 0
    p.hold()


@pytest.mark.parametrize("seqs,P", [(2, 40000), (100, 20000)])
def test_long_prefixes(seqs, P):
    for kv in ("", "e4m3"):
        p = Problem(8, [3] * seqs, [P], [0, seqs], Hq=8, Hkv=2, kv=kv)
        assert p.run() == 0
        p.hold()


def test_other_paths_of_the_own_pass():
    """The tensor-memory kernels of the decode step behind a prefix."""
    p = Problem(9, [700, 300], [300], [0, 2], Hq=64, Hkv=1, kernel_path=B.PLT_PATH_TCGEN05)
    assert p.run() == 0
    p.hold()
    p = Problem(9, [700, 300, 0], [300], [0, 3], Hq=16, Hkv=2, L=2, lens=[1000, 600, 200], kernel_path=B.PLT_PATH_TCGEN05)
    assert p.run() == 0
    p.hold()


def test_tcgen05_pass_over_own_codes():
    """Queries and probabilities there are sums of two E4M3 terms, each off by at most 2^-4 of what it is rounded from: together 2^-8,
    twice (a score moves by that share of its terms' sizes), so this path has a bound of its own."""
    p = Problem(10, [700, 300, 0], [300], [0, 3], Hq=16, Hkv=2, L=2, kv="e4m3", lens=[1000, 600, 200], kernel_path=B.PLT_PATH_TCGEN05, peak=0.5)
    assert p.run() == 0
    out, size, most = p.expect()
    got = p.out.double()
    assert ((got - out).abs() <= 2.0 ** -8 * out.abs() + (2.0 ** -7 + 2.0 ** -8 * most) * size + 1e-30).all()


def test_clamped_groups_lengths_and_pages():
    p = Problem(11, [5, 6, 7], [200], [0, 3], page=16)
    h = B.plt_prefix_attn_create(p.config)
    call = lambda begin, plens, lens, table=None: (  # noqa: E731
        p.out.fill_(float("nan")),
        B.plt_prefix_attn_run(h, _args(p, lens),
                              B.make_prefix_args(1, _dev(begin), _dev(plens), page_table=p.ptable if table is None else table, max_pages=p.ptable.shape[1])),
        B.plt_prefix_attn_check(h))[-1]
    good = [205, 206, 207]
    assert call([0, 3], [200], good) == 0
    p.hold()
    # a group that runs past the batch is cut; one that ends before it begins is empty
    assert call([0, 9], [200], good) == B.PLT_DEV_GROUP_CLAMPED
    p.hold()
    assert call([-4, 3], [200], good) == B.PLT_DEV_GROUP_CLAMPED
    p.hold()
    assert call([2, 1], [200], [5, 6, 7]) == B.PLT_DEV_GROUP_CLAMPED
    p.hold(p.expect(lens=[5, 6, 7], begin=[2, 2]))
    assert call([0, 3], [201], good) == B.PLT_DEV_GROUP_CLAMPED          # above max_prefix_len: as 200
    p.hold()
    assert call([0, 3], [-1], [5, 6, 7]) == B.PLT_DEV_GROUP_CLAMPED       # below 0: as 0
    p.hold(p.expect(lens=[5, 6, 7], plens=[0]))
    assert call([0, 3], [200], [205, 2000, -7]) == B.PLT_DEV_SEQ_LEN_CLAMPED
    assert torch.equal(p.out[2], torch.zeros_like(p.out[2]))
    for bad in (-1, p.pool):
        table = p.ptable.clone()
        table[0, 1] = bad
        assert call([0, 3], [200], good, table) == B.PLT_DEV_PAGE_ID_CLAMPED
    assert call([0, 3], [200], good) == 0
    p.hold()
    B.plt_prefix_attn_destroy(h)


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _args(p, lens):
    p.kept = _dev(lens)      # the argument struct holds an address alone
    return B.make_args(len(p.own), p.q, p.k_cache, p.v_cache, p.kept, p.out, k_win=p.k_win, v_win=p.v_win, gate_logits=p.gate,
                       k_scale=p.k_scale, v_scale=p.v_scale, **p.more)


def test_the_same_bits_again_on_another_stream_and_from_a_graph():
    p = Problem(12, [5, 60, 17, 30], [700, 90], [0, 2, 4], L=2, w=9)
    h = B.plt_prefix_attn_create(p.config)
    assert p.run(h) == 0
    p.hold()
    first = p.out.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            p.out.fill_(0)
            B.plt_prefix_attn_run(h, p.args, p.shared, side.cuda_stream)
    side.synchronize()
    assert torch.equal(p.out, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.plt_prefix_attn_run(h, p.args, p.shared, torch.cuda.current_stream().cuda_stream)
    p.out.fill_(0)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p.out, first)
    # other lengths, prefixes and groups in the same buffers
    p.seq_lens.copy_(_dev([604, 640, 605, 50]))
    p.prefix_lens.copy_(_dev([600, 50]))
    p.group_begin.copy_(_dev([0, 3, 4]))
    graph.replay()
    assert B.plt_prefix_attn_check(h) == 0
    p.hold(p.expect(lens=[604, 640, 605, 50], plens=[600, 50], begin=[0, 3, 4]))
    B.plt_prefix_attn_destroy(h)


def test_two_handles_at_once_and_batches_below_the_largest():
    a, b = Problem(13, [5, 60, 17], [700], [0, 3], max_batch=64, max_groups=5), Problem(14, [9] * 30, [400, 33], [0, 20, 30], L=2)
    ha, hb = B.plt_prefix_attn_create(a.config), B.plt_prefix_attn_create(b.config)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        B.plt_prefix_attn_run(ha, a.args, a.shared, sa.cuda_stream)
        B.plt_prefix_attn_run(hb, b.args, b.shared, sb.cuda_stream)
    torch.cuda.synchronize()
    a.hold()
    b.hold()
    assert B.plt_prefix_attn_check(ha) == 0 and B.plt_prefix_attn_check(hb) == 0
    # an empty batch touches nothing
    a.out.fill_(7)
    empty = B.make_args(0, a.q, a.k_cache, a.v_cache, a.seq_lens, a.out)
    B.plt_prefix_attn_run(ha, empty, a.shared)
    torch.cuda.synchronize()
    assert (a.out == 7).all()
    B.plt_prefix_attn_destroy(ha)
    B.plt_prefix_attn_destroy(hb)


def test_a_batch_of_none_writes_nothing():
    p = Problem(20, [5, 6], [200], [0, 2])
    h = B.plt_prefix_attn_create(p.config)
    B.plt_prefix_attn_run(h, B.make_args(0, p.q, p.k_cache, p.v_cache, p.seq_lens, p.out), p.shared)
    torch.cuda.synchronize()
    assert torch.isnan(p.out.float()).all() and B.plt_prefix_attn_check(h) == 0
    assert p.run(handle=h) == 0
    p.hold()
    B.plt_prefix_attn_destroy(h)


def test_window_lengths_out_of_range_are_clamped_and_flagged():
    p = Problem(17, [8, 9, 10], [200], [0, 3], L=2, w=9, win_lens=[[-3], [10], [5]])
    assert p.run() == B.PLT_DEV_WIN_LEN_CLAMPED
    p.win_lens = [[0], [9], [5]]
    p.hold()


def test_large_values_behind_a_row_s_last_key_weigh_nothing():
    """Finite values of 2^126 in the part of the prefix that no row sees: not a trace of them in the output."""
    p = Problem(18, [0, 0], [300], [0, 2], lens=[200, 131])
    p.shared_more["v_prefix"][:, 200:300] = 2.0 ** 126
    assert p.run() == 0
    p.hold()


def test_a_head_whose_codes_have_scale_zero():
    """Keys of scale 0 are all alike to every query: the mean of the values that a row sees."""
    p = Problem(19, [0, 0, 0], [200], [0, 3], kv="e4m3", lens=[150, 199, 200])
    p.k_scale[0] = 0.0
    for k, _ in p.values["pre"]:
        k[:, 0] = 0
    assert p.run() == 0
    p.hold()


def test_runner_class():
    from paper_2510_24824_b200.inputs import make_problem, shrunk_workload
    from paper_2510_24824_b200.runner import DecodeAttn, DeviceProblem, PrefixAttn
    # a prefix copied in front of every sequence's own keys is the plain step, within both's bounds
    p = make_problem(shrunk_workload(2))
    dp, P = DeviceProblem(p), 40
    dp.k_cache[:, :P], dp.v_cache[:, :P] = dp.k_cache[:1, :P].clone(), dp.v_cache[:1, :P].clone()
    with DecodeAttn(p) as op:
        whole = op.run(dp).clone()
    kp, vp = (x[:1, :P].contiguous() for x in (dp.k_cache, dp.v_cache))
    dp.k_cache, dp.v_cache = (torch.cat([x[:, P:], x[:, :P]], dim=1).contiguous() for x in (dp.k_cache, dp.v_cache))
    with PrefixAttn(p, P) as op:
        out = op.run(dp, op.prefix_args(_dev([0, p.B]), _dev([P]), kp, vp))
        assert op.check() == 0
        with pytest.raises(ValueError):
            op.prefix_args(_dev([0, p.B]), _dev([P]), kp.float(), vp)
        with pytest.raises(ValueError):
            op.prefix_args(_dev([0]), _dev([P]), kp, vp)
    # each is within 2^-8 |ref| + 2^-8 sum p |v| of the true result; |v| stays below 6
    assert float((out.float() - whole.float()).abs().max()) <= 2 * (2.0 ** -8 + 2.0 ** -8) * 6


def test_refusals_of_a_call():
    p = Problem(15, [5, 6], [200], [0, 2])
    h = B.plt_prefix_attn_create(p.config)
    kp, vp = p.shared_more["k_prefix"], p.shared_more["v_prefix"]
    base = dict(num_groups=1, group_begin=p.group_begin, prefix_lens=p.prefix_lens, k_prefix=kp, v_prefix=vp)
    for kw, code in ((dict(num_groups=2), B.PLT_ERR_CAPACITY), (dict(num_groups=-1), B.PLT_ERR_INVALID_ARG), (dict(group_begin=None), B.PLT_ERR_INVALID_ARG),
                     (dict(prefix_lens=None), B.PLT_ERR_INVALID_ARG), (dict(k_prefix=None), B.PLT_ERR_INVALID_ARG), (dict(v_prefix=None), B.PLT_ERR_INVALID_ARG),
                     (dict(k_prefix=kp.data_ptr() + 8), B.PLT_ERR_INVALID_ARG), (dict(strides=(51200, 256, 64)), B.PLT_ERR_INVALID_ARG),
                     (dict(strides=(51200, 257, 128)), B.PLT_ERR_INVALID_ARG), (dict(strides=(51200, 256, 0)), B.PLT_ERR_INVALID_ARG),
                     (dict(strides=(1 << 41, 256, 128)), B.PLT_ERR_UNSUPPORTED), (dict(group_begin=p.group_begin.data_ptr() + 1), B.PLT_ERR_INVALID_ARG)):
        with pytest.raises(B.PltError) as e:
            B.plt_prefix_attn_run(h, p.args, B.make_prefix_args(**{**base, **kw}))
        assert e.value.status == code and e.value.message, kw
    for kw, code in ((dict(batch=3), B.PLT_ERR_CAPACITY), (dict(q=None), B.PLT_ERR_INVALID_ARG), (dict(out=p.out.data_ptr() + 2), B.PLT_ERR_INVALID_ARG)):
        a = dict(batch=2, q=p.q, k_cache=p.k_cache, v_cache=p.v_cache, seq_lens=p.seq_lens, out=p.out)
        with pytest.raises(B.PltError) as e:
            B.plt_prefix_attn_run(h, B.make_args(**{**a, **kw}), p.shared)
        assert e.value.status == code and e.value.message, kw
    torch.cuda.synchronize()
    assert torch.isnan(p.out.float()).all() and B.plt_prefix_attn_check(h) == 0
    B.plt_prefix_attn_destroy(h)
    paged = Problem(16, [5, 6], [200], [0, 2], page=16)
    h = B.plt_prefix_attn_create(paged.config)
    for kw, code in ((dict(page_table=None), B.PLT_ERR_INVALID_ARG), (dict(max_pages=12), B.PLT_ERR_CAPACITY)):
        with pytest.raises(B.PltError) as e:
            B.plt_prefix_attn_run(h, paged.args, B.make_prefix_args(1, paged.group_begin, paged.prefix_lens, **{**paged.shared_more, **kw}))
        assert e.value.status == code
    B.plt_prefix_attn_destroy(h)

"""Shared prefixes on the GPU: the plan's way from the kernel that makes it to the ones that walk it, and the borders between its forms."""
import pytest
import torch

from paper_2510_24824_b200 import binding as B
from prefix_util import Problem

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _plans():
    """(total lengths, prefix lengths, first sequences) on the same twelve sequences: few groups, none, and more than the prefix kernel
    plans for by itself."""
    few = [([700 + 3 * b for b in range(12)], [690, 300], [0, 7, 12]), ([b for b in range(12)], [0, 5], [2, 4, 9]),
           ([310 + b for b in range(12)], [300, 640], [0, 11, 12]), ([900] * 12, [600, 650], [3, 3, 12])]
    many = ([620 + b for b in range(12)], [600 - 9 * g for g in range(33)], [min(g // 2, 12) for g in range(34)])
    return few[:2] + [([5 + b for b in range(12)], [], [0])] + few[2:] + [many, ([650 - 50 * b for b in range(12)], [700, 1], [1, 10, 12])]


@pytest.mark.parametrize("L", [1, 2])
@pytest.mark.parametrize("captured", [False, True])
def test_every_call_walks_its_own_plan(L, captured):
    """Calls behind one another on one handle, no host between them: each one's lengths and groups, and none of the call's before."""
    p = Problem(31, [12] * 12, [700] * 33, [0, 6] + [12] * 32, L=L, w=9, cap=900)
    p.k_own.nan_to_num_(0.25)
    p.v_own.nan_to_num_(0.25)
    p.values.update(k_own=p.k_own.double(), v_own=p.v_own.double())
    plans = _plans()
    lens = [_dev(n) for n, _, _ in plans]
    shared = [B.make_prefix_args(len(pre), _dev(first), _dev(pre or [0]), **p.shared_more) for _, pre, first in plans]
    outs = [torch.full_like(p.out, float("nan")) for _ in plans]
    h = B.plt_prefix_attn_create(p.config)

    def steps():
        stream = torch.cuda.current_stream().cuda_stream
        for n, args, out in zip(lens, shared, outs):
            p.seq_lens.copy_(n)
            B.plt_prefix_attn_run(h, p.args, args, stream)
            out.copy_(p.out)

    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            steps()
        for _ in range(3):
            graph.replay()
    else:
        for _ in range(3):
            steps()
    assert B.plt_prefix_attn_check(h) == 0
    for (n, pre, first), got in zip(plans, outs):
        p.out = got
        p.hold(p.expect(lens=n, plens=pre, begin=first))
    B.plt_prefix_attn_destroy(h)


BORDERS = {
    # up to 31 groups are planned by the prefix kernel itself, the last one's end by its 32nd lane
    "31 groups": dict(own=[4, 2] * 31, plens=[130 + 40 * g for g in range(31)], begin=list(range(0, 63, 2))),
    "31 groups, some sequences without": dict(own=[4] * 35, plens=[90] * 31, begin=list(range(2, 34)), L=2, w=9),
    "31 groups of codes": dict(own=[4, 2] * 31, plens=[300] * 31, begin=list(range(0, 63, 2)), kv="e4m3", Hq=8),
    "32 groups": dict(own=[4, 2] * 32, plens=[130 + 40 * g for g in range(32)], begin=list(range(0, 65, 2))),
    "32 groups of codes": dict(own=[4] * 40, plens=[300] * 32, begin=list(range(3, 36)), kv="e4m3", L=2, w=5),
    # 3, 5 and 6 heads of a KV head: query rows by the softmax's threads, in units of both tiles
    "wide": dict(own=[9] * 70, plens=[520], begin=[0, 70], Hq=12, Hkv=4),
    "wide codes": dict(own=[9] * 70, plens=[520], begin=[0, 70], Hq=12, Hkv=4, kv="e4m3"),
    "two units": dict(own=[9] * 100, plens=[400, 70], begin=[0, 99, 100], Hq=12, Hkv=4, d=64),
    "two units of codes": dict(own=[9] * 100, plens=[400, 70], begin=[0, 99, 100], Hq=12, Hkv=4, kv="e4m3"),
    "loops and tokens": dict(own=[9] * 30, plens=[300], begin=[0, 30], Hq=10, Hkv=2, L=2, q_len=2, w=11),
    "several pieces a block": dict(own=[2] * 60, plens=[2000 - 20 * g for g in range(20)], begin=list(range(0, 61, 3)), Hq=24, Hkv=8, L=5, w=4),
    "several pieces of codes": dict(own=[2] * 60, plens=[2000 - 20 * g for g in range(20)], begin=list(range(0, 61, 3)), Hq=24, Hkv=8, L=5, w=4, kv="e4m3"),
    # more sequences than the plan's threads
    "600 sequences": dict(own=[b % 7 for b in range(600)], plens=[200, 33, 1], begin=[5, 300, 560, 598], Hq=2, Hkv=1, L=2, w=6),
    "600 sequences, 40 groups": dict(own=[b % 7 for b in range(600)], plens=[60 + g for g in range(40)], begin=list(range(0, 601, 15)), Hq=2, Hkv=1, L=2, w=6),
    # the tensor-memory kernels over the own caches behind each way of planning
    "tcgen05, no group": dict(own=[700, 300, 0], plens=[], begin=[], Hq=16, Hkv=2, L=2, kernel_path=B.PLT_PATH_TCGEN05),
    "tcgen05, 33 groups": dict(own=[70 + b for b in range(33)], plens=[130] * 33, begin=list(range(34)), Hq=16, Hkv=2, L=2, kernel_path=B.PLT_PATH_TCGEN05),
}


@pytest.mark.parametrize("name", BORDERS)
def test_at_the_borders_of_the_plans(name):
    p = Problem(51, **BORDERS[name])
    assert p.run() == 0
    p.hold()

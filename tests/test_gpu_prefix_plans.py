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

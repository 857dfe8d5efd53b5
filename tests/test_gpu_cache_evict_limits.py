"""GPU tests of cache eviction at the ends of its ranges."""
import numpy as np
import pytest
import torch

from oracle import plt_cache_evict as oracle_evict
from paper_2510_24824_b200 import binding as B
from paper_2510_24824_b200.runner import CacheEvict, DeviceProblem, to_torch

from test_gpu_cache_evict import check_select, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [8 * 48 * 1024, 8 * 48 * 1024 + 1, 400003])
def test_select_rows_that_fill_and_exceed_a_clusters_shared_memory(N):
    """Up to 8 x 48 K keys stay in shared memory; longer rows are read again by every pass."""
    rng = np.random.default_rng(N)
    w = np.exp(2.0 * rng.standard_normal((2, 2, N))).astype(np.float32)
    w[0, 1] = np.minimum(np.round(w[0, 1]), 3.0)          # long runs of equal totals
    w[1, 0, ::3] = np.nan
    check_select(w, [N, 4099], 3001, 4, 64)
    check_select(w, [N - 7, N], 300000, 0, 1, stride=N + 2)


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
@pytest.mark.parametrize("which", [0, 2])
def test_compact_writes_no_page_for_an_id_outside_the_pool(bad, which):
    """Page `which` of sequence 1 is outside the pool: its rows stay, every other row of every sequence moves as it should, and
    the pages that a clamped id would name (the pool's first and last) are those of their owners."""
    p = problem(page_size=16, B=3, lens=("list", [100, 90, 70]))
    budget = 40
    keep, new = oracle_evict.select(np.random.default_rng(0).random((3, 4, p.max_seq_len)).astype(np.float32), p.seq_lens, budget, 2, 5)
    table = p.page_table.copy()
    lost = int(table[1, which])
    table[1, which] = bad
    dp = DeviceProblem(p.with_(page_table=table), "cuda:0")
    with CacheEvict(p) as op:
        op.compact(dp, to_torch(keep, "", "cuda:0"), to_torch(new, "", "cuda:0"))
        assert op.check() == B.PLT_DEV_PAGE_ID_CLAMPED
    for name in ("k_cache", "v_cache"):
        before = getattr(p, name)
        want = before.copy()
        for b in range(p.B):
            for h in range(p.Hkv):
                for i, k in enumerate(keep[b, h, : new[b]]):
                    (to, at), (source, row) = divmod(i, 16), divmod(int(k), 16)
                    if b != 1 or which not in (to, source):
                        want[p.page_table[b, to], at, h] = before[p.page_table[b, source], row, h]
        got = getattr(dp, name).cpu().view(torch.int16).numpy().view(np.uint16)
        assert np.array_equal(got, want), name
        assert np.array_equal(got[lost], before[lost])

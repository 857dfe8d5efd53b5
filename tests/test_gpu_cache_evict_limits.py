"""GPU tests of cache eviction at the ends of its ranges."""
import numpy as np
import pytest

from test_gpu_cache_evict import check_select

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

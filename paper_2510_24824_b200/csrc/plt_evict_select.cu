// plt_cache_evict_select: the positions of a cache to keep, by their attention-weight totals.
//
// Per (sequence, head group) the `budget` largest of N totals, ties to the lowest position, in ascending order. A total maps
// to a 32-bit key that orders like it (protected positions above everything, NaN below); three radix passes (11, 11, 10
// bits, from the top) find the key T of the budget-th largest, each a histogram of the next digit of the keys that share the
// digits found so far; a last pass walks the positions in order and writes those above T and as many equal to T as are left.
// After the first pass few keys take part in the histograms, so the passes are reads (the later ones from L1 / L2) and a few
// block-wide scans: bound by latency for one sequence and by the SM's load path for long rows.
//
// One block of 1024 threads per row, or a cluster of up to 8 on long rows when the batch leaves SMs idle: each block then
// holds a run of the row, histograms are summed over the cluster through distributed shared memory, and every block takes
// the same decisions on the same sums.
#include <cooperative_groups.h>

#include "plt_common.cuh"
#include "plt_evict.h"
#include "plt_ptx.cuh"

namespace plt {

namespace {

namespace cg = cooperative_groups;

constexpr int kSelThreads = 1024;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelBins = 2048;
constexpr int kSelRun = 4;                              // 32-element pieces a warp takes per step of the last pass
constexpr int kSelTile = kSelThreads * kSelRun;

// Orders like the value: NaN 0, then from -inf up; -0 and 0 alike. All ones is left for protected positions.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.f);        // -0 + 0 = 0
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

struct Row {
    const float* w;
    int n, first, last0;                                // [0, first) and [last0, n) are protected
    __device__ __forceinline__ uint32_t key(int i) const { return i < first || i >= last0 ? 0xffffffffu : order_key(w[i]); }
};

// Inclusive sum over the block; total: the block's. `warp_sums`: 32 words of shared memory.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* warp_sums, uint32_t& total) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    __syncthreads();                                    // an earlier scan's sums have been read
    if (lane == 31) warp_sums[wid] = v;
    __syncthreads();
    uint32_t s = warp_sums[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += t;
    }
    total = __shfl_sync(0xffffffffu, s, 31);
    const uint32_t before = __shfl_sync(0xffffffffu, s, (wid + 31) & 31);
    return v + (wid > 0 ? before : 0u);
}

template <bool CLUSTER>
__global__ void __launch_bounds__(kSelThreads) plt_evict_select_kernel(const __grid_constant__ SelectParams p, const int csize) {
    __shared__ uint32_t hist[kSelBins];                 // this block's counts (read by the whole cluster)
    __shared__ uint32_t warp_sums[32];
    __shared__ uint32_t s_pick[3];                      // digit picked, keys above it (cluster), keys above it (this block)
    __shared__ uint32_t s_mine[2];                      // keys above T and equal to T in this block (read by the cluster)
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int row = CLUSTER ? (int)(blockIdx.x / csize) : (int)blockIdx.x, rank = CLUSTER ? (int)(blockIdx.x % csize) : 0;
    const int b = row / p.groups, g = row - b * p.groups;
    int n = p.seq_lens[b];
    if (n < 0 || n > p.max_seq_len) {
        if (tid == 0) atomicOr(p.status, kDevSeqLenClamped);
        n = n < 0 ? 0 : p.max_seq_len;
    }
    const int kept = n < p.budget ? n : p.budget;
    int32_t* out = p.keep + (int64_t)row * p.budget;
    if (g == 0 && rank == 0 && tid == 0) p.new_lens[b] = kept;
    if (n <= p.budget) {                                // every block of the row takes this way
        for (int i = rank * kSelThreads + tid; i < p.budget; i += csize * kSelThreads) out[i] = i < n ? i : -1;
        return;
    }
    const Row r{p.weights + (int64_t)row * p.weights_stride, n, p.keep_first, n - p.keep_last};
    // this block's run of the row: whole tiles
    const int tiles = (n + kSelTile - 1) / kSelTile;
    const int i0 = min(n, (int)((int64_t)tiles * rank / csize) * kSelTile);
    const int i1 = min(n, (int)((int64_t)tiles * (rank + 1) / csize) * kSelTile);

    uint32_t prefix = 0, left = (uint32_t)kept;         // digits found so far; how many of the keys that share them are kept
    uint32_t above_mine = 0, equal_mine = 0;            // in this block: keys above T, keys equal to T
    int shift = 32;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10;
        const int bins = 1 << bits, prev = shift;
        shift -= bits;
        for (int i = tid; i < kSelBins; i += kSelThreads) hist[i] = 0;
        __syncthreads();
        for (int base = i0; base < i1; base += kSelThreads * 4) {
            uint32_t k[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = base + u * kSelThreads + tid;
                k[u] = i < i1 ? r.key(i) : 0u;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = base + u * kSelThreads + tid;
                const bool in = i < i1 && (pass == 0 || (k[u] >> prev) == prefix);
                const uint32_t mask = __ballot_sync(0xffffffffu, in);
                if (mask == 0) continue;
                const uint32_t digit = (k[u] >> shift) & (uint32_t)(bins - 1);
                // lanes that agree on the digit (long runs of equal totals) add once
                const uint32_t lead = __shfl_sync(0xffffffffu, digit, __ffs(mask) - 1);
                if (__all_sync(0xffffffffu, !in || digit == lead)) {
                    if (lane == 0) atomicAdd(&hist[lead], (uint32_t)__popc(mask));
                } else if (in) {
                    atomicAdd(&hist[digit], 1u);
                }
            }
        }
        if constexpr (CLUSTER) cg::this_cluster().sync(); else __syncthreads();
        // thread t has bins 2 t and 2 t + 1 counted from the top; the picked one is where the running count reaches `left`
        uint32_t c[2], mine[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int bin = kSelBins - 1 - (2 * tid + u);
            mine[u] = c[u] = hist[bin];
            if constexpr (CLUSTER)
                for (int q = 1; q < csize; ++q) c[u] += *cg::this_cluster().map_shared_rank(&hist[bin], (rank + q) % csize);
        }
        uint32_t total, total_mine;
        const uint32_t upto = block_scan(c[0] + c[1], warp_sums, total);
        const uint32_t upto_mine = block_scan(mine[0] + mine[1], warp_sums, total_mine);
        uint32_t before = upto - c[0] - c[1], before_mine = upto_mine - mine[0] - mine[1];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (before < left && before + c[u] >= left) {
                s_pick[0] = (uint32_t)(kSelBins - 1 - (2 * tid + u));
                s_pick[1] = before;
                s_pick[2] = before_mine;
                s_mine[1] = mine[u];
            }
            before += c[u];
            before_mine += mine[u];
        }
        __syncthreads();
        prefix = (prefix << bits) | s_pick[0];
        left -= s_pick[1];
        above_mine += s_pick[2];
        equal_mine = s_mine[1];
        if constexpr (CLUSTER) cg::this_cluster().sync(); else __syncthreads();   // counts and picks have been read
    }
    // T = prefix; `left` of the keys equal to it are kept, the lowest positions first
    uint32_t above = 0, equal = 0;                      // before this block's run
    if constexpr (CLUSTER) {
        if (tid == 0) {
            s_mine[0] = above_mine;
            s_mine[1] = equal_mine;
        }
        cg::this_cluster().sync();
        for (int q = 0; q < rank; ++q) {
            const uint32_t* other = cg::this_cluster().map_shared_rank(&s_mine[0], q);
            above += other[0];
            equal += other[1];
        }
        cg::this_cluster().sync();                      // no block ends while another reads its counts
    }
    for (int base = i0; base < i1; base += kSelTile) {
        uint32_t mg[kSelRun], me[kSelRun], ng = 0, ne = 0;
#pragma unroll
        for (int u = 0; u < kSelRun; ++u) {
            const int i = base + (wid * kSelRun + u) * 32 + lane;
            const uint32_t k = i < i1 ? r.key(i) : 0u;
            mg[u] = __ballot_sync(0xffffffffu, i < i1 && k > prefix);
            me[u] = __ballot_sync(0xffffffffu, i < i1 && k == prefix);
            ng += __popc(mg[u]);
            ne += __popc(me[u]);
        }
        // both counts of a tile fit 16 bits: one scan over the warps' sums (kept by lane 31 of each)
        uint32_t total;
        const uint32_t mine = ng | (ne << 16);
        const uint32_t incl = block_scan(lane == 31 ? mine : 0u, warp_sums, total);
        const uint32_t mine_before = __shfl_sync(0xffffffffu, incl, 31) - mine;
        uint32_t ag = above + (mine_before & 0xffffu), ae = equal + (mine_before >> 16);
        const uint32_t below = (1u << lane) - 1u;
#pragma unroll
        for (int u = 0; u < kSelRun; ++u) {
            const int i = base + (wid * kSelRun + u) * 32 + lane;
            const uint32_t g0 = ag + __popc(mg[u] & below), e0 = ae + __popc(me[u] & below);
            if ((mg[u] >> lane) & 1u) out[g0 + min(e0, left)] = i;
            else if (((me[u] >> lane) & 1u) && e0 < left) out[g0 + e0] = i;
            ag += __popc(mg[u]);
            ae += __popc(me[u]);
        }
        above += total & 0xffffu;
        equal += total >> 16;
    }
}

// Blocks per row: as many as leave each 4096 positions of a full row and the grid within what two blocks per SM take. A row
// of 65536 among 8 took ... us with one block and ... us with eight; batches that fill the SMs gain nothing from it.
int select_cluster(const SelectParams& p, int batch) {
    int c = 1;
    while (c < 8 && (int64_t)batch * p.groups * c * 2 <= 296 && p.max_seq_len / (2 * c) >= kSelTile) c *= 2;
    return c;
}

}  // namespace

cudaError_t launch_select(const SelectParams& p, int batch, cudaStream_t stream) {
    const int c = select_cluster(p, batch);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(batch * p.groups * c));
    cfg.blockDim = dim3(kSelThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)c;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = c > 1 ? 1 : 0;
    return c > 1 ? cudaLaunchKernelEx(&cfg, plt_evict_select_kernel<true>, p, c) : cudaLaunchKernelEx(&cfg, plt_evict_select_kernel<false>, p, 1);
}

}  // namespace plt

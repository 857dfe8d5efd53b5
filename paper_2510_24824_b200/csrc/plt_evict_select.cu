// plt_cache_evict_select: the positions of a cache to keep, by their attention-weight totals.
//
// Per (sequence, head group) the `budget` largest of N totals, ties to the lowest position, in ascending order. A total maps
// to a 32-bit key that orders like it (protected positions above everything, NaN below); three radix passes (11, 11, 10
// bits, from the top) find the key T of the budget-th largest, each a histogram of the next digit of the keys that share the
// digits found so far. Every warp then knows the keys of its run that are above T and equal to T (the third pass counts those
// that the first two digits tell apart, and only a warp with others counts once more), one scan over the warps gives each its
// place in the output, and the runs are written without further synchronisation.
//
// A block of 1024 threads takes a row, or a cluster of up to 8 blocks where rows are long and few: each block then holds a
// part of the row, histograms are summed over the cluster through distributed shared memory, and every block takes the same
// decisions on the same sums. A block's keys are read from memory once and stay with it, in registers (up to 8 per thread)
// or shared memory (up to 48 K keys), by the capacity, which bounds the length; longer parts are read again by every pass.
// The floor is one read of the totals; what bounds it is the chain of passes (histogram, scan, pick) and, on long rows, the
// histogram's shared-memory atomics. A row of 32768, alone on its SM, 18 us: load 2.4, passes 3.2 / 2.1 / 1.9, picks 0.65 each,
// scan, positions out and the end 6. 384 rows of up to 32768: 25.6 us (18 MB at 700 GB/s), all of 32768: 60, and with all totals equal,
// where one bin of each histogram takes every addition: 65; 8 rows of 5000: 9.2, of 65536: 16.6.
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

// Orders like the value: NaN 1, then from -inf up; -0 and 0 alike. All ones is left for protected positions, 0 for places
// behind the row's end, which are below everything that can be picked and so need no test of their own.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);        // -0 + 0 = 0
    const uint32_t k = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return x == x ? k : 1u;
}

struct Row {
    const float* w;
    uint32_t first, inner;                              // [0, first) and [first + inner, n) are protected
    __device__ __forceinline__ uint32_t key(int i, float x) const { return (uint32_t)i - first >= inner ? 0xffffffffu : order_key(x); }
    __device__ __forceinline__ uint32_t key(int i) const { return key(i, w[i]); }
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

// Where a block's keys stay between the passes.
enum Home { kMemory, kRegisters, kShared };
constexpr int kRegKeys = 8;                             // per thread
constexpr int kSharedKeys = 48 * 1024;                  // per block

template <int HOME, bool CLUSTER>
__global__ void __launch_bounds__(kSelThreads) plt_evict_select_kernel(const __grid_constant__ SelectParams p, const int csize) {
    __shared__ uint32_t hist[kSelBins];                 // this block's counts
    __shared__ uint32_t sums[CLUSTER ? 2 : 1][CLUSTER ? kSelBins : 1];   // the cluster's, for this pass and the next
    __shared__ uint32_t warp_sums[32];
    __shared__ uint32_t s_pick[4];                      // digit picked; keys above it: in the cluster, in this block; equal: in this block
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
    const Row r{p.weights + (int64_t)row * p.weights_stride, (uint32_t)p.keep_first, (uint32_t)(n - p.keep_last - p.keep_first)};
    // Warp w of the csize * 32 warps of the row has the run [w0, w1): `steps` pieces of 32 positions.
    const int steps = (n + csize * kSelThreads - 1) / (csize * kSelThreads);
    const int w0 = min(n, (rank * kSelWarps + wid) * steps * 32), w1 = min(n, w0 + steps * 32);
    constexpr int IPT = HOME == kRegisters ? kRegKeys : 1;
    uint32_t held[IPT];
    extern __shared__ uint32_t s_keys[];
    uint32_t* run = s_keys + wid * steps * 32;          // kShared: this warp's keys; no other warp reads them
    if constexpr (HOME == kRegisters) {
#pragma unroll
        for (int j = 0; j < IPT; ++j) {
            const int i = w0 + j * 32 + lane;
            held[j] = j < steps && i < w1 ? r.key(i) : 0u;
        }
    } else if constexpr (HOME == kShared) {
        // the totals as they are, all on their way at once; the first pass turns them into keys. Rows that start on a 16-byte
        // boundary move four to an instruction, up to the last whole four.
        int i0 = w0;
        if (((uintptr_t)r.w & 15u) == 0) {
            i0 = w0 + ((w1 - w0) & ~3);
            for (int i = w0 + 4 * lane; i < i0; i += 128)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(run + (i - w0))), "l"(r.w + i) : "memory");
        }
        for (int i = i0 + lane; i < w1; i += 32)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(run + (i - w0))), "l"(r.w + i) : "memory");
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();                                   // the copies of the other lanes
    }
    const int whole = (w1 - w0) / 32;                   // pieces that have all their positions
    // Calls f(piece, key) for every piece of the warp's run, with key 0 behind the end; `fresh`: the first call.
    auto walk = [&](bool fresh, auto&& f) {
        if constexpr (HOME == kRegisters) {
#pragma unroll
            for (int j = 0; j < IPT; ++j)
                if (j < steps) f(j, held[j]);
        } else {
            auto key_of = [&](int j) {
                const int i = w0 + j * 32 + lane;
                if constexpr (HOME == kShared) {
                    uint32_t k = run[j * 32 + lane];
                    if (fresh) run[j * 32 + lane] = k = r.key(i, __uint_as_float(k));
                    return k;
                } else {
                    return r.key(i);
                }
            };
#pragma unroll 4
            for (int j = 0; j < whole; ++j) f(j, key_of(j));
            if (whole < steps && w0 + whole * 32 < w1) f(whole, w0 + whole * 32 + lane < w1 ? key_of(whole) : 0u);
        }
    };

    uint32_t prefix = 0, left = (uint32_t)kept;         // digits found so far; how many of the keys that share them are kept
    uint32_t above_mine = 0, equal_mine = 0;            // in this block: keys above T, keys equal to T
    uint32_t ng = 0, ne = 0;                            // in this warp's run: keys above T, keys equal to T
    bool near = false;                                  // a key of the run shares T's first two digits
    int shift = 32;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10;
        const uint32_t digits = (1u << bits) - 1u;
        const int prev = shift;
        shift -= bits;
        for (int i = tid; i < kSelBins; i += kSelThreads) hist[i] = 0;
        if (CLUSTER && pass == 0) {
            for (int i = tid; i < kSelBins; i += kSelThreads) sums[0][i] = 0;
            cg::this_cluster().sync();                  // no block adds before all have cleared
        }
        __syncthreads();
        if (pass == 0) walk(true, [&](int, uint32_t k) { atomicAdd(&hist[k >> shift], 1u); });
        else if (pass == 1) walk(false, [&](int, uint32_t k) {
            if ((k >> prev) == prefix) atomicAdd(&hist[(k >> shift) & digits], 1u);
        });
        else walk(false, [&](int, uint32_t k) {
            ng += (k >> prev) > prefix;
            if ((k >> prev) == prefix) {
                atomicAdd(&hist[k & digits], 1u);
                near = true;
            }
        });
        __syncthreads();
        const uint32_t* counts = hist;
        if constexpr (CLUSTER) {
            // Bins that hold something are few: each block adds its own to every block's sums. The sums of the next pass are
            // cleared before the barrier behind which anyone adds to them.
            cg::cluster_group cluster = cg::this_cluster();
#pragma unroll
            for (int u = 0; u < kSelBins / kSelThreads; ++u) {
                const int bin = tid + u * kSelThreads;
                const uint32_t v = hist[bin];
                sums[(pass + 1) & 1][bin] = 0;
                if (v != 0)
                    for (int q = 0; q < csize; ++q) atomicAdd(cluster.map_shared_rank(&sums[pass & 1][bin], q), v);
            }
            cluster.sync();
            counts = sums[pass & 1];
        }
        // thread t has bins 2 t and 2 t + 1 counted from the top; the picked one is where the running count reaches `left`
        uint32_t c[2], mine[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int bin = kSelBins - 1 - (2 * tid + u);
            mine[u] = hist[bin];
            c[u] = counts[bin];
        }
        uint32_t total, before = block_scan(c[0] + c[1], warp_sums, total) - c[0] - c[1], before_mine = before;
        if constexpr (CLUSTER) before_mine = block_scan(mine[0] + mine[1], warp_sums, total) - mine[0] - mine[1];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (before < left && before + c[u] >= left) {
                s_pick[0] = (uint32_t)(kSelBins - 1 - (2 * tid + u));
                s_pick[1] = before;
                s_pick[2] = before_mine;
                s_pick[3] = mine[u];
            }
            before += c[u];
            before_mine += mine[u];
        }
        __syncthreads();
        prefix = (prefix << bits) | s_pick[0];
        left -= s_pick[1];
        above_mine += s_pick[2];
        equal_mine = s_pick[3];
    }
    // T = prefix; `left` of the keys equal to it are kept, the lowest positions first
    uint32_t above = 0, equal = 0;                      // before this block's part
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
    if (__any_sync(0xffffffffu, near)) {                // the last pass counted what the first two digits tell
        ng = 0;
        walk(false, [&](int, uint32_t k) {
            ng += k > prefix;
            ne += k == prefix;
        });
    }
    ng = __reduce_add_sync(0xffffffffu, ng);
    ne = __reduce_add_sync(0xffffffffu, ne);
    uint32_t total;
    const uint32_t ig = block_scan(lane == 31 ? ng : 0u, warp_sums, total), ie = block_scan(lane == 31 ? ne : 0u, warp_sums, total);
    above += __shfl_sync(0xffffffffu, ig, 31) - ng;
    equal += __shfl_sync(0xffffffffu, ie, 31) - ne;
    const uint32_t below = (1u << lane) - 1u;
    uint32_t to = above + min(equal, left);             // the warp's next place
    const bool ties = ne > 0 && equal < left;           // of the warp's run, some equal to T are kept
    if (!ties) {
        int32_t* dst = out + to;
        int at = w0 + lane;
        walk(false, [&](int j, uint32_t k) {
            const bool take = k > prefix;
            const uint32_t mask = __ballot_sync(0xffffffffu, take);
            if (take) dst[__popc(mask & below)] = at + j * 32;
            dst += __popc(mask);
        });
        return;
    }
    walk(false, [&](int j, uint32_t k) {
        const bool tie = k == prefix;
        const uint32_t me = __ballot_sync(0xffffffffu, tie);
        const bool take = k > prefix || (tie && equal + __popc(me & below) < left);
        equal += __popc(me);
        const uint32_t mask = __ballot_sync(0xffffffffu, take);
        if (take) out[to + __popc(mask & below)] = w0 + j * 32 + lane;
        to += __popc(mask);
    });
}

// Blocks per row: as few as can hold a full row, and more while the grid leaves SMs idle and every block keeps 4096
// positions (blocks per row, 8 rows of 65536: two 26.1 us, four 20.7, eight 16.6; 8 rows of 32768: one 20.7, two 19.4, four 16.6,
// eight 14.6; 384 rows of up to 32768, which fill the device: one 25.6, two 40.0; 8 rows of 5000: one 9.2, two 12.5). The rule
// knows the capacity, not the lengths: a row that is short in a long capacity is spread over as many blocks.
int select_cluster(const SelectParams& p, int batch) {
    int c = 1;
    while (c < 8 && p.max_seq_len / c >= 2 * 4096 && ((int64_t)batch * p.groups * c * 2 <= p.sm_count || p.max_seq_len > c * kSharedKeys)) c *= 2;
    return c;
}

template <int HOME, bool CLUSTER>
cudaError_t launch_home(const SelectParams& p, int batch, int c, cudaStream_t stream) {
    auto fn = plt_evict_select_kernel<HOME, CLUSTER>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(batch * p.groups * c));
    cfg.blockDim = dim3(kSelThreads);
    cfg.stream = stream;
    if (HOME == kShared) {
        const int steps = (p.max_seq_len + c * kSelThreads - 1) / (c * kSelThreads);   // of the longest row
        cfg.dynamicSmemBytes = (size_t)steps * kSelThreads * 4;
        const cudaError_t e = allow_max_dynamic_smem((const void*)fn);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)c;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CLUSTER ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, fn, p, c);
}

template <int HOME>
cudaError_t launch_cluster(const SelectParams& p, int batch, int c, cudaStream_t stream) {
    return c > 1 ? launch_home<HOME, true>(p, batch, c, stream) : launch_home<HOME, false>(p, batch, c, stream);
}

}  // namespace

cudaError_t launch_select(const SelectParams& p, int batch, cudaStream_t stream) {
    const int c = select_cluster(p, batch);
    if (p.max_seq_len <= c * kRegKeys * kSelThreads) return launch_cluster<kRegisters>(p, batch, c, stream);
    if (p.max_seq_len <= c * kSharedKeys) return launch_cluster<kShared>(p, batch, c, stream);
    return launch_home<kMemory, true>(p, batch, c, stream);      // select_cluster gives rows this long eight blocks
}

}  // namespace plt

// plt_cache_evict_compact: moves the kept rows of the caches to the front, in place.
//
// Slot i of a head takes row keep[i] >= i. Reading is safe as long as the slot has not been overwritten, i.e. before slot
// keep[i] itself is written, and since keep[i] >= i that is never before slot i is: a block that walks the slots in order,
// reading a chunk of rows, waiting for all its threads' reads, then writing the chunk, always reads old values, and may read
// ahead as far as it likes. So no scratch copy of the cache is needed and every row moves once: 2 x its bytes, the floor.
// The order binds the slots of one head only; heads, K and V, and the 16-byte columns of a row are independent, which is
// where the blocks come from: one per (sequence, head, K or V, piece of the row). Rows are cut into pieces of down to 64
// bytes only while that is needed to give every SM a block. Two chunks of loads are in flight per block, the next chunk's
// page ids and positions included. Bound: HBM on batches, the chain position -> page id -> row for one sequence.
#include "plt_common.cuh"
#include "plt_evict.h"
#include "plt_ptx.cuh"

namespace plt {

namespace {

constexpr int kCmpThreads = 256;
constexpr int kCmpUnroll = 8;         // rows in flight per thread and chunk

struct Slots {                        // the slots of one (sequence, group)
    const int32_t* keep;
    int n, m;                         // lengths before and after
};

__device__ __forceinline__ Slots read_slots(const CompactParams& p, int b, int g, uint32_t& flags) {
    Slots s;
    s.n = p.seq_lens[b];
    if (s.n < 0 || s.n > p.max_seq_len) {
        flags |= kDevSeqLenClamped;
        s.n = s.n < 0 ? 0 : p.max_seq_len;
    }
    const int most = min(p.keep_stride, s.n);
    s.m = p.new_lens[b];
    if (s.m < 0 || s.m > most) {
        flags |= kDevKeepClamped;
        s.m = s.m < 0 ? 0 : most;
    }
    s.keep = p.keep + ((int64_t)b * (p.Hkv / p.hpg) + g) * p.keep_stride;
    return s;
}

__device__ __forceinline__ int source_of(const Slots& s, int i, uint32_t& flags) {
    int k = s.keep[i];
    if (k < i || k >= s.n) {
        flags |= kDevKeepClamped;
        k = k < i ? i : s.n - 1;
    }
    return k;
}

// Byte offset of a position's row of KV head 0.
__device__ __forceinline__ int64_t cell(const CompactParams& p, const int32_t* pages, int b, int pos, uint32_t& flags) {
    if (p.page_size == 0) return (int64_t)b * p.stride_b + (int64_t)pos * p.stride_n;
    int page = pages[pos / p.page_size];
    if (page < 0 || page >= p.num_pool_pages) {
        flags |= kDevPageIdClamped;
        page = page < 0 ? 0 : p.num_pool_pages - 1;
    }
    return (int64_t)page * p.stride_b + (int64_t)(pos % p.page_size) * p.stride_n;
}

// `lanes`: 16-byte columns of a block's piece of a row (a power of two, at most 32); `pieces`: pieces of a row.
__global__ void __launch_bounds__(kCmpThreads) plt_evict_compact_kernel(const __grid_constant__ CompactParams p, const int lanes,
                                                                        const int pieces, const int row_blocks) {
    uint32_t flags = 0;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < row_blocks) {
        int id = blockIdx.x;
        const int piece = id % pieces; id /= pieces;
        const int which = id & 1; id >>= 1;
        const int h = id % p.Hkv, b = id / p.Hkv;
        const Slots s = read_slots(p, b, h / p.hpg, flags);
        const int32_t* pages = p.page_table + (int64_t)b * p.max_pages;
        char* base = (which ? p.v : p.k) + (int64_t)h * p.stride_h + (piece * lanes + tid % lanes) * 16;
        const int per = kCmpThreads / lanes;             // rows per step
        const int chunk = per * kCmpUnroll, row0 = tid / lanes;
        uint4 x[kCmpUnroll];
        int64_t to[kCmpUnroll];                          // where the row goes; -1: it stays (or there is none)
        auto load = [&](int c0, uint4 (&v)[kCmpUnroll], int64_t (&dst)[kCmpUnroll]) {
            int64_t from[kCmpUnroll];
#pragma unroll
            for (int u = 0; u < kCmpUnroll; ++u) {
                const int i = c0 + u * per + row0;
                dst[u] = -1;
                from[u] = 0;
                if (i < s.m) {
                    const int k = source_of(s, i, flags);
                    if (k != i) {
                        from[u] = cell(p, pages, b, k, flags);
                        dst[u] = cell(p, pages, b, i, flags);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kCmpUnroll; ++u)
                if (dst[u] >= 0) v[u] = *(const uint4*)(base + from[u]);
        };
        load(0, x, to);
        for (int c0 = 0; c0 < s.m; c0 += chunk) {
            uint4 y[kCmpUnroll];
            int64_t to2[kCmpUnroll];
            load(c0 + chunk, y, to2);
            __syncthreads();                             // every row of this chunk (and of the next) has been read
#pragma unroll
            for (int u = 0; u < kCmpUnroll; ++u)
                if (to[u] >= 0) *(uint4*)(base + to[u]) = x[u];
#pragma unroll
            for (int u = 0; u < kCmpUnroll; ++u) {
                x[u] = y[u];
                to[u] = to2[u];
            }
        }
    } else {
        // the totals of one (sequence, group): the same walk on single elements, then zeros up to the old length
        const int groups = p.Hkv / p.hpg, id = blockIdx.x - row_blocks, b = id / groups, g = id - b * groups;
        const Slots s = read_slots(p, b, g, flags);
        float* w = p.weights + (int64_t)id * p.weights_stride;
        for (int c0 = 0; c0 < s.m; c0 += kCmpThreads * kCmpUnroll) {
            float x[kCmpUnroll];
#pragma unroll
            for (int u = 0; u < kCmpUnroll; ++u) {
                const int i = c0 + u * kCmpThreads + tid;
                x[u] = i < s.m ? w[source_of(s, i, flags)] : 0.f;
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kCmpUnroll; ++u) {
                const int i = c0 + u * kCmpThreads + tid;
                if (i < s.m) w[i] = x[u];
            }
        }
        __syncthreads();
        for (int i = s.m + tid; i < s.n; i += kCmpThreads) w[i] = 0.f;
    }
    if (flags) atomicOr(p.status, flags);
}

}  // namespace

cudaError_t launch_compact(const CompactParams& p, int batch, int sm_count, cudaStream_t stream) {
    int pieces = 1, lanes = p.row_bytes / 16;
    while (lanes > 4 && (int64_t)batch * p.Hkv * 2 * pieces < sm_count) {
        lanes /= 2;
        pieces *= 2;
    }
    const int row_blocks = batch * p.Hkv * 2 * pieces;
    const int blocks = row_blocks + (p.weights ? batch * (p.Hkv / p.hpg) : 0);
    plt_evict_compact_kernel<<<(unsigned)blocks, kCmpThreads, 0, stream>>>(p, lanes, pieces, row_blocks);
    return cudaGetLastError();
}

}  // namespace plt

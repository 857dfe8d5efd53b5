// plt_cache_evict_compact: moves the kept rows of the caches to the front, in place.
//
// Slot i of a head takes row keep[i] >= i. Reading is safe as long as the slot has not been overwritten, i.e. before slot
// keep[i] itself is written, and since keep[i] >= i that is never before slot i is: a block that walks the slots in order,
// reading a chunk of rows, waiting for all its threads' reads, then writing the chunk, always reads old values. So no scratch
// copy of the cache is needed and every row moves once: 2 x its bytes, the floor. The order binds the slots of one head only,
// and only within the same bytes of the rows: heads, K and V, and the 16-byte columns of a row are independent. A block owns
// a 64-byte piece of the rows of one (sequence, head, K or V). The chain position -> page id -> row is taken apart: one thread
// per row works out the next chunk's addresses into shared memory while the rows of the current one are under way, from
// positions it fetched a chunk earlier. (Every thread working out the addresses of the rows it moves, 4 lanes to a row, took
// 2.1x the time on pages of 64 tokens: integer divisions.) A chunk is 512 rows.
//
// Bound: HBM, reads and writes mixed: 64 sequences of 8192, 4096 kept, 8 heads of 128 bf16: 370 us, 0.91 of the copy rate, in pages
// of 64 tokens 392, 0.86; ragged lengths, half of which keep everything: 85 us, 0.68. One sequence of 5000, 1024 kept: 8.3 to 8.6
// us, the chain lengths -> positions -> pages -> rows. What moves is what lies behind the first dropped position: a cache one
// position over its budget moves half of its rows on average (64 sequences of 4097, 4096 kept: 249 us). (Blocks of 1024 threads with 1024 rows a chunk: 8.6 there, 468 us on the full batch.)
#include "plt_common.cuh"
#include "plt_evict.h"
#include "plt_ptx.cuh"

namespace plt {

namespace {

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

// Clamped position that slot i < m takes.
__device__ __forceinline__ int clamp_source(const Slots& s, int i, int k, uint32_t& flags) {
    if (k >= i && k < s.n) return k;
    flags |= kDevKeepClamped;
    return k < i ? i : s.n - 1;
}

__device__ __forceinline__ int clamp_page(const CompactParams& p, int page, uint32_t& flags) {
    if (page >= 0 && page < p.num_pool_pages) return page;
    flags |= kDevPageIdClamped;
    return page < 0 ? 0 : p.num_pool_pages - 1;
}

constexpr int kColumns = 4;           // 16-byte columns of a block's piece of a row

// Byte offsets of a row's source and destination, from the head's first row; to = -1: the row stays.
struct Move {
    int64_t from, to;
};

__device__ __forceinline__ int64_t row_offset(const CompactParams& p, const int32_t* pages, int b, int pos, uint32_t& flags) {
    if (p.page_size == 0) return (int64_t)b * p.stride_b + (int64_t)pos * p.stride_n;
    const int page = p.page_shift >= 0 ? pos >> p.page_shift : pos / p.page_size;
    return (int64_t)clamp_page(p, pages[page], flags) * p.stride_b + (int64_t)(pos - page * p.page_size) * p.stride_n;
}

constexpr int kMoveThreads = 256;

__global__ void __launch_bounds__(kMoveThreads) plt_evict_compact_kernel(const __grid_constant__ CompactParams p, const int pieces,
                                                                         const int row_blocks) {
    constexpr int THREADS = kMoveThreads, U = 8;                                         // U: rows of a thread in flight
    constexpr int STEP = THREADS / kColumns, CHUNK = STEP * U, MINE = CHUNK / THREADS;   // rows: per step, per chunk, planned per thread
    __shared__ Move moves[3][CHUNK];     // a buffer is rewritten two barriers after its last use
    uint32_t flags = 0;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < row_blocks) {
        int id = blockIdx.x;
        const int piece = id % pieces; id /= pieces;
        const int which = id & 1; id >>= 1;
        const int h = id % p.Hkv, b = id / p.Hkv;
        const Slots s = read_slots(p, b, h / p.hpg, flags);
        const int32_t* pages = p.page_table + (int64_t)b * p.max_pages;
        // A sequence that keeps all it has moves nothing: seen in one sweep with 16 loads a thread in flight. In a batch of ragged
        // lengths these are many, and their blocks take the places of those with work (64 sequences of up to 8192, budget 4096:
        // chunk by chunk 97 us, a sweep of 4 loads at a time 92, of 16 82).
        if (s.m == s.n) {
            bool moved = false;
            for (int i0 = tid; i0 < s.m; i0 += 16 * THREADS) {
                int k[16];
#pragma unroll
                for (int u = 0; u < 16; ++u) k[u] = i0 + u * THREADS < s.m ? s.keep[i0 + u * THREADS] : i0 + u * THREADS;
#pragma unroll
                for (int u = 0; u < 16; ++u) moved |= k[u] != i0 + u * THREADS;
            }
            if (!__syncthreads_or(moved)) {
                if (flags) atomicOr(p.status, flags);     // a length may have been clamped
                return;
            }
        }
        char* base = (which ? p.v : p.k) + (int64_t)h * p.stride_h + (piece * kColumns + tid % kColumns) * 16;
        int k[MINE];                     // positions of the chunk that is planned next
        auto fetch = [&](int c0) {
#pragma unroll
            for (int j = 0; j < MINE; ++j) k[j] = c0 + j * THREADS + tid < s.m ? s.keep[c0 + j * THREADS + tid] : 0;
        };
        auto plan = [&](int c0, Move* to) {
#pragma unroll
            for (int j = 0; j < MINE; ++j) {
                const int i = c0 + j * THREADS + tid;
                Move m{0, -1};
                if (i < s.m) {
                    const int from = clamp_source(s, i, k[j], flags);
                    if (from != i) {
                        uint32_t bad = 0;          // a page outside the pool: the row stays, no other sequence's page is written
                        const int64_t src = row_offset(p, pages, b, from, bad), dst = row_offset(p, pages, b, i, bad);
                        if (bad == 0) m = Move{src, dst};
                        flags |= bad;
                    }
                }
                to[j * THREADS + tid] = m;
            }
        };
        fetch(0);
        plan(0, moves[0]);
        fetch(CHUNK);
        __syncthreads();
        int buf = 0;
        for (int c0 = 0; c0 < s.m; c0 += CHUNK) {
            const Move* now = moves[buf] + tid / kColumns;
            uint4 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Move m = now[u * STEP];
                if (m.to >= 0) x[u] = *(const uint4*)(base + m.from);
            }
            buf = buf == 2 ? 0 : buf + 1;
            plan(c0 + CHUNK, moves[buf]);
            fetch(c0 + 2 * CHUNK);
            __syncthreads();             // every row of the chunk has been read, the next one's addresses are in place
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t to = now[u * STEP].to;
                if (to >= 0) *(uint4*)(base + to) = x[u];
            }
        }
    } else {
        // the totals of one (sequence, group): the same walk on single elements, then zeros up to the old length
        constexpr int V = 8;
        const int groups = p.Hkv / p.hpg, id = blockIdx.x - row_blocks, b = id / groups, g = id - b * groups;
        const Slots s = read_slots(p, b, g, flags);
        float* w = p.weights + (int64_t)id * p.weights_stride;
        for (int c0 = 0; c0 < s.m; c0 += THREADS * V) {
            int k[V];
            float x[V];
#pragma unroll
            for (int u = 0; u < V; ++u) {
                const int i = c0 + u * THREADS + tid;
                k[u] = i < s.m ? s.keep[i] : 0;
            }
#pragma unroll
            for (int u = 0; u < V; ++u) {
                const int i = c0 + u * THREADS + tid;
                x[u] = i < s.m ? w[clamp_source(s, i, k[u], flags)] : 0.f;
            }
            __syncthreads();
#pragma unroll
            for (int u = 0; u < V; ++u) {
                const int i = c0 + u * THREADS + tid;
                if (i < s.m) w[i] = x[u];
            }
        }
        __syncthreads();
        for (int i = s.m + tid; i < s.n; i += THREADS) w[i] = 0.f;
    }
    if (flags) atomicOr(p.status, flags);
}

}  // namespace

cudaError_t launch_compact(const CompactParams& p, int batch, cudaStream_t stream) {
    const int pieces = p.row_bytes / (16 * kColumns);
    const int row_blocks = batch * p.Hkv * 2 * pieces;
    const unsigned grid = (unsigned)(row_blocks + (p.weights ? batch * (p.Hkv / p.hpg) : 0));
    plt_evict_compact_kernel<<<grid, kMoveThreads, 0, stream>>>(p, pieces, row_blocks);
    return cudaGetLastError();
}

}  // namespace plt

// The rest of plt_cache_evict_weights: choice of the scores kernel's variant, the scores kernel for fp32 caches, and the
// kernels that join the pieces' statistics, turn scores into weights and add them up.
#include "plt_common.cuh"
#include "plt_evict.h"
#include "plt_evict_scores.cuh"
#include "plt_ptx.cuh"

namespace plt {

cudaError_t scores_bf16_d128(int op, int mode, const ScoreVariant&, const CUtensorMap*, const EvictWeights*, int, cudaStream_t, int*);
cudaError_t scores_bf16_d64(int op, int mode, const ScoreVariant&, const CUtensorMap*, const EvictWeights*, int, cudaStream_t, int*);
cudaError_t scores_e4m3(int op, int mode, const ScoreVariant&, const CUtensorMap*, const EvictWeights*, int, cudaStream_t, int*);

namespace {

cudaError_t score_dispatch(int op, int mode, const ScoreVariant& v, const CUtensorMap* map, const EvictWeights* e, int grid,
                           cudaStream_t stream, int* out) {
    if (v.fp8) return scores_e4m3(op, mode, v, map, e, grid, stream, out);
    return v.D == 128 ? scores_bf16_d128(op, mode, v, map, e, grid, stream, out) : scores_bf16_d64(op, mode, v, map, e, grid, stream, out);
}

// ---- fp32 caches --------------------------------------------------------------------------------------------------
// Plain fp32 FMA (tensor-core formats would round the products). A tile of 32 keys in shared memory; warp = packed rows
// wid, wid + 8, ..; lane = key, so a row's statistics stay with the lane until the end of the piece. Not tuned: a tile is loaded,
// then multiplied, with nothing in flight meanwhile. 8 rows, 64 ragged sequences of up to 8192 keys, 8 KV heads of 128: the call
// takes 387 us, 4.4 times its floor; one sequence of 700: 15.8.
constexpr int kFThreads = 256;
constexpr int kFRows = kMaxRows / (kFThreads / 32);   // rows per warp at most

template <int D>
struct FCfg {
    static constexpr int KROW = D + 4;   // padded row: conflict-free float4 reads, lane = key
    __host__ __device__ static size_t smem_bytes(int R, int max_batch) {
        return (size_t)(kEvictF32Keys * KROW + R * D) * 4 + (size_t)(2 * max_batch + 4) * 4;
    }
};

template <int D>
__global__ void __launch_bounds__(kFThreads) plt_evict_scores_f32(const __grid_constant__ EvictWeights e) {
    using C = FCfg<D>;
    constexpr int TK = kEvictF32Keys;
    const Params& p = e.p;
    extern __shared__ float4 smem_f4[];
    float* sK = (float*)smem_f4;                 // [TK][KROW]
    float* sQ = sK + TK * C::KROW;               // [R][D]
    int32_t* s_prefix = (int32_t*)(sQ + p.R * D);
    int32_t* s_lens = s_prefix + p.B + 1;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const int R = p.R;
    uint32_t flags = 0;
    build_prefix(p, s_prefix, flags, s_lens);
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t T = s_prefix[p.B];
    const int cta = blockIdx.x, nctas = evict_ctas(T, (int)gridDim.x, kEvictScoreTiles);
    const bool in_plan = cta < nctas;
    const int64_t lo = in_plan ? cta_begin(T, cta, nctas) : 0, hi = in_plan ? cta_begin(T, cta + 1, nctas) : 0;
    const float* kc = (const float*)p.k_cache;

    PieceWalk walk(p, s_prefix, lo, hi, s_lens);
    Piece pc;
    while (walk.next(pc, flags)) {
        const int kvh = pc.hg;   // one KV head per item
        __syncthreads();
        for (int i = tid; i < R * D; i += kFThreads) {
            const int r = i / D, c = i - r * D;
            const int lq = r / p.G;
            const int64_t head_row = ((int64_t)pc.b * p.L * p.Qn + lq) * p.Hq + kvh * p.G + (r - lq * p.G);
            const bool other_half = p.qsplit && c / (D / 2) != (int)(head_row & 1);
            sQ[i] = other_half ? 0.f : ((const float*)p.q)[(head_row >> p.qsplit) * D + c];
        }
        int cutr[kFRows];
        float m[kFRows], l[kFRows];
#pragma unroll
        for (int k = 0; k < kFRows; ++k) {
            const int r = wid + k * (kFThreads / 32), lq = r < R ? r / p.G : 0;
            cutr[k] = 0;
#pragma unroll
            for (int q = 0; q < kMaxLoops; ++q)
                if (r < R && q == lq / p.Qn) cutr[k] = max(pc.sp.cut[q] - (p.Qn - 1 - lq % p.Qn), 0);
            m[k] = -1e30f;
            l[k] = 0.f;
        }
        const int64_t tile0 = (int64_t)s_prefix[pc.b] + (int64_t)pc.hg * line_len(p, pc.sp.gt) + p.piece_cost;
        for (int t = pc.t0; t < pc.t1; ++t) {
            const int key0 = t * TK;
            __syncthreads();   // the tile before has been read (and the query rows are in place)
            for (int i = tid; i < TK * (D / 4); i += kFThreads) {
                const int j = i / (D / 4), c4 = (i - j * (D / 4)) * 4, key = key0 + j;
                float4 k4 = make_float4(0.f, 0.f, 0.f, 0.f);
                if (key < pc.sp.cmax) {
                    int64_t off;
                    if (p.page_size > 0) {
                        int page = p.page_table[(int64_t)pc.b * p.max_pages + key / p.page_size];
                        if (page < 0 || page >= p.num_pool_pages) {
                            flags |= kDevPageIdClamped;
                            page = page < 0 ? 0 : p.num_pool_pages - 1;
                        }
                        off = (int64_t)page * p.kv_stride_b + (int64_t)(key % p.page_size) * p.kv_stride_n;
                    } else {
                        off = (int64_t)(e.b0 + pc.b) * p.kv_stride_b + (int64_t)key * p.kv_stride_n;
                    }
                    k4 = *(const float4*)(kc + off + (int64_t)kvh * p.kv_stride_h + c4);
                }
                *(float4*)(sK + j * C::KROW + c4) = k4;
            }
            __syncthreads();
            float* dst = e.scores + ((tile0 + t) * TK + lane) * (int64_t)e.row_pitch;
            if (R + wid < e.row_pitch) dst[R + wid] = -INFINITY;   // no row: weight 0
#pragma unroll
            for (int k = 0; k < kFRows; ++k) {
                const int r = wid + k * (kFThreads / 32);
                if (r < R) {
                    float s = 0.f;
                    const float4* kr = (const float4*)(sK + lane * C::KROW);
                    const float4* qr = (const float4*)(sQ + r * D);
#pragma unroll 8
                    for (int c = 0; c < D / 4; ++c) {
                        const float4 a = qr[c], b4 = kr[c];
                        s = fmaf(a.x, b4.x, s);
                        s = fmaf(a.y, b4.y, s);
                        s = fmaf(a.z, b4.z, s);
                        s = fmaf(a.w, b4.w, s);
                    }
                    s = key0 + lane < cutr[k] ? s * p.scale_log2 : -INFINITY;
                    if (s - m[k] > 8.f) {
                        l[k] *= fast_exp2(m[k] - s);
                        m[k] = s;
                    }
                    l[k] += fast_exp2(s - m[k]);
                    dst[r] = s;
                }
            }
        }
        const int64_t slot = slot_of(item_index(p, pc.b, pc.hg, 0), cta);
        if (tid == 0) note_piece(p, pc, cta);
#pragma unroll
        for (int k = 0; k < kFRows; ++k) {
            const int r = wid + k * (kFThreads / 32);
            float mm = m[k], ll = l[k];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float m2 = __shfl_xor_sync(0xffffffffu, mm, o), l2 = __shfl_xor_sync(0xffffffffu, ll, o);
                const float mx = fmaxf(mm, m2);
                ll = ll * fast_exp2(mm - mx) + l2 * fast_exp2(m2 - mx);
                mm = mx;
            }
            if (lane == 0 && r < R) *(float2*)(e.ml + (slot * R + r) * 2) = make_float2(mm, ll);
        }
    }
    if (flags) atomicOr(p.status, flags);
}

// ---- scores to weights --------------------------------------------------------------------------------------------
// weight of a key = sum over rows of 2^(score - m) * (rho / l), m and l joined over the pieces of the row's item.
//
// Two kernels: `join` leaves (m, rho / l) of every row, a warp per 8 rows of a (sequence, KV head) with its lanes over the
// pieces; `add` then has no chain of dependent loads and no barrier left. A warp of it takes 128 keys of one (sequence, head
// group). The rows of a key lie side by side in the scratch, so LPK lanes share a key, four rows each in one 16-byte load: a
// warp's load is 512 consecutive bytes, and a lane's statistics stay in its registers over the keys. (With a key per lane the
// same loads touch a line each.) The sum's order is fixed by the rows alone. Bound: L2 / HBM on the scores.
__device__ __forceinline__ int scored_tiles(const EvictWeights& e, int n) {
    return (max(n - e.min_delta, 0) + (1 << e.tile_shift) - 1) >> e.tile_shift;
}

constexpr int kJoinThreads = 128;
constexpr int kJoinRows = 8;                              // rows of a warp

// Folds the statistics (m2, l2) into (m, l).
__device__ __forceinline__ void fold(float& m, float& l, float m2, float l2) {
    const float mm = fmaxf(m, m2);
    l = l * fast_exp2(m - mm) + l2 * fast_exp2(m2 - mm);
    m = mm;
}

__global__ void __launch_bounds__(kJoinThreads) plt_evict_join(const __grid_constant__ EvictWeights e) {
    const Params& p = e.p;
    const int lane = threadIdx.x & 31;
    const int chunks = (p.R + kJoinRows - 1) / kJoinRows;
    const int task = blockIdx.x * (kJoinThreads / 32) + (threadIdx.x >> 5);
    const int id = task / chunks, r0 = (task - id * chunks) * kJoinRows;    // sequence * Hkv + head, first row
    grid_launch_dependents();
    if (id >= p.B * p.Hkv) return;
    const int b = id / p.Hkv, h = id - b * p.Hkv, hg = h / p.hpc, hl = h - hg * p.hpc;
    uint32_t flags = 0;                                   // reported by the other kernels
    const int n = seq_len_clamped(p, b, flags);
    const int item = item_index(p, b, hg, 0);
    // lane j (of 8) ends up with row r0 + j: its factor rho
    const int row = r0 + (lane & (kJoinRows - 1));
    float rho = 1.f;
    const int lq = row / p.G, loop = lq / p.Qn;
    const bool gated = e.gate != nullptr && row < p.R && loop > 0;
    grid_dependency_wait();
    int2 c = make_int2(0, -1);
    if (scored_tiles(e, n) > 0) c = *(const int2*)(p.item_blocks + 2 * item);
    if (gated) rho = e.gate[(((int64_t)b * (p.L - 1) + (loop - 1)) * p.Qn + (lq - loop * p.Qn)) * (p.Hq >> p.qsplit) +
                            ((h * p.G + (row - lq * p.G)) >> p.qsplit)];
    const int np = (c.y - c.x + 1) * e.kw;
    float m[kJoinRows], l[kJoinRows];
#pragma unroll
    for (int j = 0; j < kJoinRows; ++j) {
        m[j] = -1e30f;
        l[j] = 0.f;
    }
    for (int i = lane; i < np; i += 32) {                 // a piece per lane, its rows together
        const int64_t slot = slot_of(item, c.x + i / e.kw);
        const float2* src = (const float2*)e.ml + ((slot * p.hpc + hl) * e.kw + i % e.kw) * p.R + r0;
        float2 v[kJoinRows];
#pragma unroll
        for (int j = 0; j < kJoinRows; ++j) v[j] = r0 + j < p.R ? src[j] : make_float2(-1e30f, 0.f);
#pragma unroll
        for (int j = 0; j < kJoinRows; ++j) fold(m[j], l[j], v[j].x, v[j].y);
    }
    if (np > 1) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            if (o >= np) continue;                        // lanes from np on hold nothing
#pragma unroll
            for (int j = 0; j < kJoinRows; ++j)
                fold(m[j], l[j], __shfl_xor_sync(0xffffffffu, m[j], o), __shfl_xor_sync(0xffffffffu, l[j], o));
        }
    }
    if (gated) rho = 1.f / (1.f + expf(rho));             // 1 - sigmoid
    // lane 0 has the joined statistics (with one piece, alone); lane j takes row r0 + j
    float mj = 0.f, lj = 0.f;
#pragma unroll
    for (int j = 0; j < kJoinRows; ++j) {
        const float m0 = __shfl_sync(0xffffffffu, m[j], 0), l0 = __shfl_sync(0xffffffffu, l[j], 0);
        if (lane == j) {
            mj = m0;
            lj = l0;
        }
    }
    // a row without a key, or no row at all (the pitch may hold more than there are): 2^(score - inf) * 0
    if (lane < kJoinRows && row < e.row_pitch)            // the pitch ends within the last chunk of 8
        e.mc[(int64_t)id * e.row_pitch + row] = lj == 0.f ? make_float2(INFINITY, 0.f) : make_float2(mj, rho / lj);
}

constexpr int kAddThreads = 256;
constexpr int kAddRun = 128;                              // keys of a warp
constexpr int kAddBatch = 8;                              // loads in flight per lane

// Lengths, the line of the scores plan and this kernel's own line (runs of kAddRun keys of every head group) into shared
// memory; the latter's length. Waits for the kernel before. `tiles`: [B + 1], behind it `line` [B + 1] and `lens` [B].
__device__ __forceinline__ int add_plan(const EvictWeights& e, int32_t* s_tiles, uint32_t& flags) {
    const Params& p = e.p;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, groups = p.Hkv / e.hpg;
    int32_t *s_line = s_tiles + p.B + 1, *s_lens = s_line + p.B + 1;
    for (int b = tid; b < p.B; b += kAddThreads) {
        const int n = seq_len_clamped(p, b, flags);
        s_lens[b] = n;
        s_tiles[b + 1] = (p.Hkv / p.hpc) * line_len(p, scored_tiles(e, n));
        s_line[b + 1] = groups * ((n + kAddRun - 1) / kAddRun);
    }
    __syncthreads();
    if (wid < 2) {                                        // both prefixes, a warp each
        int32_t* sp = wid == 0 ? s_tiles : s_line;
        int32_t run = 0;
        if (lane == 0) sp[0] = 0;
        for (int b0 = 0; b0 < p.B; b0 += 32) {
            int32_t v = b0 + lane < p.B ? sp[b0 + lane + 1] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int32_t u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            if (b0 + lane < p.B) sp[b0 + lane + 1] = run + v;
            run += __shfl_sync(0xffffffffu, v, 31);
        }
    }
    __syncthreads();
    grid_dependency_wait();
    return s_line[p.B];
}

template <int LPK>
__global__ void __launch_bounds__(kAddThreads, 3) plt_evict_add(const __grid_constant__ EvictWeights e) {
    const Params& p = e.p;
    extern __shared__ int32_t smem_i[];
    const int groups = p.Hkv / e.hpg, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int32_t *s_tiles = smem_i, *s_line = s_tiles + p.B + 1, *s_lens = s_line + p.B + 1;
    uint32_t flags = 0;
    const int T = add_plan(e, smem_i, flags);
    const int64_t head = (int64_t)e.key_pitch << e.tile_shift;              // scores of a head's part of a tile
    // from the line's end: part of what the scores kernel wrote last is still in L2 (8 sequences of 32768 codes, 16 rows: 91
    // instead of 104 MB of the 134 read from HBM, the call 104 instead of 108 us)
    for (int pos = T - 1 - (int)(blockIdx.x * (kAddThreads / 32) + wid); pos >= 0; pos -= gridDim.x * (kAddThreads / 32)) {
        const int b = find_seq(s_line, p.B, pos);
        const int n = s_lens[b], runs = (n + kAddRun - 1) / kAddRun;
        const int o = pos - s_line[b], g = o / runs;
        constexpr int KPI = 32 / LPK, BATCHES = kAddRun / (KPI * kAddBatch);
        constexpr int U = BATCHES > 0 ? kAddBatch : kAddRun / KPI;          // keys of a lane's group in flight
        const int sub = lane & (LPK - 1), r0 = 4 * sub;
        const int gt = scored_tiles(e, n), scored = gt << e.tile_shift;     // keys that have scores (beyond a row's cutoff: -inf)
        float* w = e.weights + ((int64_t)b * groups + g) * e.weights_stride;
        const int64_t line = (int64_t)line_len(p, gt) * p.hpc * head;       // scores of a head line
        const float* first = e.scores + ((int64_t)s_tiles[b] + p.piece_cost) * p.hpc * head;
        for (int k0 = (o - g * runs) * kAddRun + lane / LPK, done = 0; done < kAddRun && k0 - lane / LPK < n; done += U * KPI, k0 += U * KPI) {
            float acc[U];
#pragma unroll
            for (int u = 0; u < U; ++u) acc[u] = 0.f;
            float old[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int key = k0 + u * KPI;
                old[u] = e.decay != 0.f && u % LPK == sub && key < n ? w[key] : 0.f;
            }
            if (r0 < e.row_pitch) {
                for (int h = g * e.hpg; h < (g + 1) * e.hpg; ++h) {
                    const int hg = h / p.hpc, hl = h - hg * p.hpc;
                    const float* s = first + hg * line + hl * head + r0;
                    const float2* mc = e.mc + ((int64_t)b * p.Hkv + h) * e.row_pitch + r0;
                    const float4 c01 = *(const float4*)mc, c23 = *(const float4*)(mc + 2);
                    float4 v[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int key = k0 + u * KPI;
                        v[u] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
                        // row (tile * hpc * TK + key % TK) of the head line
                        if (key < scored && key < n)
                            v[u] = *(const float4*)(s + ((int64_t)(key >> e.tile_shift) * ((p.hpc - 1) << e.tile_shift) + key) * e.row_pitch);
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        acc[u] = fmaf(fast_exp2(v[u].x - c01.x), c01.y, acc[u]);
                        acc[u] = fmaf(fast_exp2(v[u].y - c01.z), c01.w, acc[u]);
                        acc[u] = fmaf(fast_exp2(v[u].z - c23.x), c23.y, acc[u]);
                        acc[u] = fmaf(fast_exp2(v[u].w - c23.z), c23.w, acc[u]);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int i = 1; i < LPK; i <<= 1) acc[u] += __shfl_xor_sync(0xffffffffu, acc[u], i);
                const int key = k0 + u * KPI;
                if (u % LPK == sub && key < n) w[key] = e.decay != 0.f ? fmaf(e.decay, old[u], acc[u]) : acc[u];
            }
        }
    }
    if (flags) atomicOr(p.status, flags);
}

// After two passes over K: the sums over the rows are there for every KV head and key, and only the heads of a group and the
// old totals are left to add.
__global__ void __launch_bounds__(kAddThreads) plt_evict_fold(const __grid_constant__ EvictWeights e) {
    const Params& p = e.p;
    extern __shared__ int32_t smem_i[];
    const int groups = p.Hkv / e.hpg, lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int32_t *s_tiles = smem_i, *s_line = s_tiles + p.B + 1, *s_lens = s_line + p.B + 1;
    uint32_t flags = 0;
    const int T = add_plan(e, smem_i, flags);
    constexpr int U = kAddRun / 32;
    for (int pos = blockIdx.x * (kAddThreads / 32) + wid; pos < T; pos += gridDim.x * (kAddThreads / 32)) {
        const int b = find_seq(s_line, p.B, pos);
        const int n = s_lens[b], runs = (n + kAddRun - 1) / kAddRun;
        const int o = pos - s_line[b], g = o / runs, k0 = (o - g * runs) * kAddRun + lane;
        const int gt = scored_tiles(e, n), scored = gt << e.tile_shift;
        float* w = e.weights + ((int64_t)b * groups + g) * e.weights_stride;
        const int64_t head = (int64_t)e.key_pitch << e.tile_shift, line = (int64_t)line_len(p, gt) * p.hpc * head;
        const float* first = e.scores + ((int64_t)s_tiles[b] + p.piece_cost) * p.hpc * head;
        float acc[U], old[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = k0 + 32 * u;
            acc[u] = 0.f;
            old[u] = e.decay != 0.f && key < n ? w[key] : 0.f;
        }
        for (int h = g * e.hpg; h < (g + 1) * e.hpg; ++h) {
            const int hg = h / p.hpc, hl = h - hg * p.hpc;
            const float* s = first + hg * line + hl * head;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int key = k0 + 32 * u;
                if (key >= scored || key >= n) continue;
                const float* parts = s + ((int64_t)(key >> e.tile_shift) * ((p.hpc - 1) << e.tile_shift) + key) * e.key_pitch;
                if (e.key_pitch == 1) acc[u] += parts[0];
                else if (e.key_pitch == 2) {
                    const float2 v = *(const float2*)parts;
                    acc[u] += v.x + v.y;
                } else {
                    const float4 v = *(const float4*)parts;
                    acc[u] += (v.x + v.y) + (v.z + v.w);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int key = k0 + 32 * u;
            if (key < n) w[key] = e.decay != 0.f ? fmaf(e.decay, old[u], acc[u]) : acc[u];
        }
    }
    if (flags) atomicOr(p.status, flags);
}

}  // namespace

ScoreVariant score_variant(int D, int R, int Hkv, bool fp8, int max_batch) {
    ScoreVariant v;
    v.D = D;
    v.fp8 = fp8;
    // Above 16 rows K is streamed twice: the scores' way through the scratch (4 R bytes a key, written and read) costs more than
    // K's rows again. Once / twice, bf16, 64 ragged sequences: 8 rows 65 / 100 us, 16 rows 97 / 103, 24 rows 120 / 109, 32 rows
    // 157 / 110; E4M3, 8 x 32768: 16 rows 103 / 99, 20 rows 153 / 163, 28 rows 177 / 164, 32 rows 203 / 164. 64 rows, once with
    // 64 rows in a warp / twice with 16: bf16 423 / 165, E4M3 519 / 287.
    v.twice = R > 16;
    // At most 16 rows in a warp, so that 8 or 16 warps of an SM hold their queries in registers (64 rows, 32 / 16 in a warp: bf16
    // 180 / 165 us, E4M3 318 / 287).
    v.NT = R <= 8 ? 1 : 2;
    v.RS = R <= 16 ? 1 : (R <= 32 ? 2 : 4);
    v.HPC = Hkv % 4 == 0 ? 4 : (Hkv % 2 == 0 ? 2 : 1);
    v.KW = 4 / v.HPC;
    v.KS = 2;
    v.tile_keys = 16 * v.KW * v.KS;
    // two blocks per SM, at most 64 KB of loads in flight each (more only delays the first data)
    v.stages = 8;
    for (; v.stages > 2; --v.stages) {
        int bytes = 0;
        score_dispatch(0, v.twice ? kScoreStats : kScoreDump, v, nullptr, nullptr, max_batch, nullptr, &bytes);
        v.smem = (size_t)bytes;
        const size_t ring = (size_t)v.stages * v.HPC * v.tile_keys * D * (fp8 ? 1 : 2);
        if (ring <= 64 * 1024 && v.smem <= 110 * 1024) return v;
    }
    int bytes = 0;
    score_dispatch(0, v.twice ? kScoreStats : kScoreDump, v, nullptr, nullptr, max_batch, nullptr, &bytes);
    v.smem = (size_t)bytes;
    return v;
}

cudaError_t scores_prepare(const ScoreVariant& v, int* blocks_per_sm) {
    if (!v.twice) return score_dispatch(1, kScoreDump, v, nullptr, nullptr, 0, nullptr, blocks_per_sm);
    int stats = 0;
    const cudaError_t err = score_dispatch(1, kScoreStats, v, nullptr, nullptr, 0, nullptr, &stats);
    if (err != cudaSuccess) return err;
    const cudaError_t err2 = score_dispatch(1, kScoreSums, v, nullptr, nullptr, 0, nullptr, blocks_per_sm);
    if (stats < *blocks_per_sm) *blocks_per_sm = stats;
    return err2;
}

cudaError_t launch_scores(const ScoreVariant& v, const CUtensorMap& mapK, const EvictWeights& e, int grid, cudaStream_t stream) {
    return score_dispatch(2, v.twice ? kScoreStats : kScoreDump, v, &mapK, &e, grid, stream, nullptr);
}

cudaError_t launch_sums(const ScoreVariant& v, const CUtensorMap& mapK, const EvictWeights& e, int grid, cudaStream_t stream) {
    return score_dispatch(2, kScoreSums, v, &mapK, &e, grid, stream, nullptr);
}

size_t scores_f32_smem(int D, int R, int max_batch) {
    return D == 128 ? FCfg<128>::smem_bytes(R, max_batch) : FCfg<64>::smem_bytes(R, max_batch);
}

cudaError_t scores_f32_prepare(int D, int R, int max_batch, int* blocks_per_sm) {
    const void* fn = D == 128 ? (const void*)plt_evict_scores_f32<128> : (const void*)plt_evict_scores_f32<64>;
    const cudaError_t err = allow_max_dynamic_smem(fn);
    if (err != cudaSuccess) return err;
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks_per_sm, fn, kFThreads, scores_f32_smem(D, R, max_batch));
}

// Launched to overlap the end of the kernel before it in the stream; it waits before it touches anything but the lengths.
template <typename Fn>
static cudaError_t launch_overlapped(Fn fn, const EvictWeights& e, int grid, int threads, size_t smem, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fn, e);
}

cudaError_t launch_scores_f32(const EvictWeights& e, int grid, size_t smem, cudaStream_t stream) {
    return e.p.d == 128 ? launch_overlapped(plt_evict_scores_f32<128>, e, grid, kFThreads, smem, stream)
                        : launch_overlapped(plt_evict_scores_f32<64>, e, grid, kFThreads, smem, stream);
}

size_t evict_add_smem(int max_batch) { return (size_t)(3 * max_batch + 4) * 4; }

namespace {
// lanes per key: four rows each, a power of two
template <typename F>
cudaError_t with_lanes(bool twice, int key_pitch, F&& f) {
    if (twice) return f(plt_evict_fold);
    if (key_pitch <= 4) return f(plt_evict_add<1>);
    if (key_pitch <= 8) return f(plt_evict_add<2>);
    if (key_pitch <= 16) return f(plt_evict_add<4>);
    if (key_pitch <= 32) return f(plt_evict_add<8>);
    return f(plt_evict_add<16>);
}
}  // namespace

cudaError_t evict_add_prepare(bool twice, int key_pitch, size_t smem, int* blocks_per_sm) {
    return with_lanes(twice, key_pitch, [&](auto fn) {
        const cudaError_t err = allow_max_dynamic_smem((const void*)fn);
        return err != cudaSuccess ? err : cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks_per_sm, fn, kAddThreads, smem);
    });
}

cudaError_t launch_evict_join(const EvictWeights& e, cudaStream_t stream) {
    const int warps = e.p.B * e.p.Hkv * ((e.p.R + kJoinRows - 1) / kJoinRows);
    return launch_overlapped(plt_evict_join, e, (warps + kJoinThreads / 32 - 1) / (kJoinThreads / 32), kJoinThreads, 0, stream);
}

cudaError_t launch_evict_add(const EvictWeights& e, bool twice, int grid, size_t smem, cudaStream_t stream) {
    return with_lanes(twice, e.key_pitch, [&](auto fn) { return launch_overlapped(fn, e, grid, kAddThreads, smem, stream); });
}

}  // namespace plt

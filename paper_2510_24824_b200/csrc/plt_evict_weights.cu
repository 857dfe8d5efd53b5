// The rest of plt_cache_evict_weights: choice of the scores kernel's variant, the scores kernel for fp32 caches, and the
// kernel that turns scores into weights and adds them up.
#include "plt_common.cuh"
#include "plt_evict.h"
#include "plt_ptx.cuh"

namespace plt {

cudaError_t scores_bf16_d128(int op, const ScoreVariant&, const CUtensorMap*, const EvictWeights*, int, cudaStream_t, int*);
cudaError_t scores_bf16_d64(int op, const ScoreVariant&, const CUtensorMap*, const EvictWeights*, int, cudaStream_t, int*);
cudaError_t scores_e4m3(int op, const ScoreVariant&, const CUtensorMap*, const EvictWeights*, int, cudaStream_t, int*);

namespace {

cudaError_t score_dispatch(int op, const ScoreVariant& v, const CUtensorMap* map, const EvictWeights* e, int grid, cudaStream_t stream,
                           int* out) {
    if (v.fp8) return scores_e4m3(op, v, map, e, grid, stream, out);
    return v.D == 128 ? scores_bf16_d128(op, v, map, e, grid, stream, out) : scores_bf16_d64(op, v, map, e, grid, stream, out);
}

// ---- fp32 caches --------------------------------------------------------------------------------------------------
// Plain fp32 FMA (tensor-core formats would round the products). A tile of 32 keys in shared memory; warp = packed rows
// wid, wid + 8, ..; lane = key, so a row's statistics stay with the lane until the end of the piece.
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
        const int64_t tile0 = (int64_t)s_prefix[pc.b] + (int64_t)pc.hg * pc.sp.gt;
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
// weight of a key = sum over rows of 2^(score - m) * (rho / l), m and l joined over the pieces of the row's item. A block
// owns a run of 256-key tiles of one (sequence, head group): it joins the statistics of the group's rows into shared memory
// (one warp per row, lanes over the pieces), then one thread per key walks the rows of the group's heads. The rows of a key
// lie side by side, so the reads are whole sectors; the sum's order is the rows' order. Bound: L2 / HBM on the scores, and
// the exponentials (one per row and key).
constexpr int kAddThreads = kEvictAddKeys;
constexpr int kAddTiles = 4;

// Adds the weights of R rows of one head to the accumulators of kAddTiles keys; W rows per load.
template <int W>
__device__ __forceinline__ void add_rows(const float* s, const int64_t (&at)[kAddTiles], const float2* mc, int R, float (&acc)[kAddTiles]) {
    for (int r = 0; r < R; r += W) {
        float v[kAddTiles][W];
#pragma unroll
        for (int u = 0; u < kAddTiles; ++u) {
            if constexpr (W == 4) {
                const float4 x = *(const float4*)(s + at[u] + r);
                v[u][0] = x.x; v[u][1] = x.y; v[u][2] = x.z; v[u][3] = x.w;
            } else {
                const float2 x = *(const float2*)(s + at[u] + r);
                v[u][0] = x.x; v[u][1] = x.y;
            }
        }
#pragma unroll
        for (int j = 0; j < W; ++j) {
            if (r + j < R) {                               // the pitch may hold one row more than there are
                const float2 c = mc[r + j];
#pragma unroll
                for (int u = 0; u < kAddTiles; ++u) acc[u] = fmaf(fast_exp2(v[u][j] - c.x), c.y, acc[u]);
            }
        }
    }
}

__global__ void __launch_bounds__(kAddThreads) plt_evict_add(const __grid_constant__ EvictWeights e) {
    const Params &p = e.p, &pa = e.pa;
    extern __shared__ float2 smem_f2[];
    const int rows = pa.hpc * p.R;
    float2* s_mc = smem_f2;                               // [rows] (m, rho / l)
    int32_t* s_tiles = (int32_t*)(s_mc + rows);           // tile prefix of the scores plan
    int32_t* s_prefix = s_tiles + p.B + 1;
    int32_t* s_lens = s_prefix + p.B + 1;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    uint32_t flags = 0;
    build_prefix(p, s_tiles, flags);
    build_prefix(pa, s_prefix, flags, s_lens);
    const int64_t T = s_prefix[p.B];
    const int cta = blockIdx.x, nctas = evict_ctas(T, (int)gridDim.x, 1);
    const bool in_plan = cta < nctas;
    const int64_t lo = in_plan ? cta_begin(T, cta, nctas) : 0, hi = in_plan ? cta_begin(T, cta + 1, nctas) : 0;
    grid_dependency_wait();

    PieceWalk walk(pa, s_prefix, lo, hi, s_lens);
    Piece pc;
    while (walk.next(pc, flags)) {
        SeqPlan sp;
        seq_plan_n(p, pc.b, s_lens[pc.b], sp, flags);     // the scores plan of this sequence
        __syncthreads();
        for (int row = wid; row < rows; row += kAddThreads / 32) {
            const int hh = row / p.R, r = row - hh * p.R;
            const int h = pc.hg * pa.hpc + hh, hg = h / p.hpc, hl = h - hg * p.hpc;
            float m = -1e30f, l = 0.f;
            if (sp.gt > 0) {
                const int item = item_index(p, pc.b, hg, 0);
                const int2 c = *(const int2*)(p.item_blocks + 2 * item);
                const int np = (c.y - c.x + 1) * e.kw;
                for (int i = lane; i < np; i += 32) {
                    const int64_t slot = slot_of(item, c.x + i / e.kw);
                    const float2 v = *(const float2*)(e.ml + (((slot * p.hpc + hl) * e.kw + i % e.kw) * p.R + r) * 2);
                    const float mm = fmaxf(m, v.x);
                    l = l * fast_exp2(m - mm) + v.y * fast_exp2(v.x - mm);
                    m = mm;
                }
            }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
                const float mm = fmaxf(m, m2);
                l = l * fast_exp2(m - mm) + l2 * fast_exp2(m2 - mm);
                m = mm;
            }
            if (lane == 0) {
                const int lq = r / p.G, loop = lq / p.Qn;
                float rho = 1.f;
                if (e.gate != nullptr && loop > 0) {
                    const int hq = (h * p.G + (r - lq * p.G)) >> p.qsplit;
                    const float x = e.gate[(((int64_t)pc.b * (p.L - 1) + (loop - 1)) * p.Qn + (lq - loop * p.Qn)) * (p.Hq >> p.qsplit) + hq];
                    rho = 1.f / (1.f + expf(x));           // 1 - sigmoid(x)
                }
                s_mc[row] = make_float2(m, l == 0.f ? 0.f : rho / l);
            }
        }
        __syncthreads();
        const int n = pc.sp.cmax;                          // the length
        const int scored = sp.gt * p.tile_keys;            // keys that have scores (beyond a row's cutoff: -inf)
        float* w = e.weights + ((int64_t)pc.b * (p.Hkv / pa.hpc) + pc.hg) * e.weights_stride;
        for (int t = pc.t0; t < pc.t1; t += kAddTiles) {
            // kAddTiles keys of a thread, a tile apart: their loads are in flight together
            float acc[kAddTiles], old[kAddTiles];
            int key[kAddTiles];
            int64_t at[kAddTiles];                         // first score of the key for KV head 0 of the item's head line
#pragma unroll
            for (int u = 0; u < kAddTiles; ++u) {
                key[u] = (t + u) * kEvictAddKeys + tid;
                if (t + u >= pc.t1 || key[u] >= n) key[u] = -1;
                acc[u] = 0.f;
                old[u] = e.decay != 0.f && key[u] >= 0 ? w[key[u]] : 0.f;
                const int kk = key[u] >= 0 && key[u] < scored ? key[u] : 0;
                const int tile = kk / p.tile_keys;
                at[u] = ((int64_t)tile * p.hpc * p.tile_keys + (kk - tile * p.tile_keys)) * e.row_pitch;
            }
            if (scored > 0) {
                for (int hh = 0; hh < pa.hpc; ++hh) {
                    const int h = pc.hg * pa.hpc + hh, hg = h / p.hpc, hl = h - hg * p.hpc;
                    const float* s = e.scores + (((int64_t)s_tiles[pc.b] + (int64_t)hg * sp.gt) * p.hpc + hl) * p.tile_keys * e.row_pitch;
                    const float2* mc = s_mc + hh * p.R;
                    if ((e.row_pitch & 3) == 0) {
                        add_rows<4>(s, at, mc, p.R, acc);
                    } else {
                        add_rows<2>(s, at, mc, p.R, acc);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kAddTiles; ++u)
                if (key[u] >= 0) {
                    const float x = key[u] < scored ? acc[u] : 0.f;
                    w[key[u]] = e.decay != 0.f ? fmaf(e.decay, old[u], x) : x;
                }
        }
    }
    if (flags) atomicOr(p.status, flags);
}

}  // namespace

ScoreVariant score_variant(int D, int R, int Hkv, bool fp8, int max_batch) {
    ScoreVariant v;
    v.D = D;
    v.fp8 = fp8;
    const int nt = (R + 7) / 8;
    v.NT = nt <= 2 ? nt : (nt <= 4 ? 4 : 8);
    v.HPC = Hkv % 4 == 0 ? 4 : (Hkv % 2 == 0 ? 2 : 1);
    v.KW = 4 / v.HPC;
    v.KS = v.NT <= 4 ? 2 : 1;
    v.tile_keys = 16 * v.KW * v.KS;
    // two blocks per SM, at most 64 KB of loads in flight each (more only delays the first data)
    v.stages = 8;
    for (; v.stages > 2; --v.stages) {
        int bytes = 0;
        score_dispatch(0, v, nullptr, nullptr, max_batch, nullptr, &bytes);
        v.smem = (size_t)bytes;
        const size_t ring = (size_t)v.stages * v.HPC * v.tile_keys * D * (fp8 ? 1 : 2);
        if (ring <= 64 * 1024 && v.smem <= 110 * 1024) return v;
    }
    int bytes = 0;
    score_dispatch(0, v, nullptr, nullptr, max_batch, nullptr, &bytes);
    v.smem = (size_t)bytes;
    return v;
}

cudaError_t scores_prepare(const ScoreVariant& v, int* blocks_per_sm) {
    return score_dispatch(1, v, nullptr, nullptr, 0, nullptr, blocks_per_sm);
}

cudaError_t launch_scores(const ScoreVariant& v, const CUtensorMap& mapK, const EvictWeights& e, int grid, cudaStream_t stream) {
    return score_dispatch(2, v, &mapK, &e, grid, stream, nullptr);
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

size_t evict_add_smem(int rows, int max_batch) { return (size_t)rows * 8 + (size_t)(3 * max_batch + 4) * 4; }

cudaError_t evict_add_prepare(size_t smem, int* blocks_per_sm) {
    const cudaError_t err = allow_max_dynamic_smem((const void*)plt_evict_add);
    if (err != cudaSuccess) return err;
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks_per_sm, plt_evict_add, kAddThreads, smem);
}

cudaError_t launch_evict_add(const EvictWeights& e, int grid, size_t smem, cudaStream_t stream) {
    return launch_overlapped(plt_evict_add, e, grid, kAddThreads, smem, stream);
}

}  // namespace plt

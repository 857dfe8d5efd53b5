// Scores kernel of the attention-weight totals (plt_cache_evict_weights), caches of bf16 values or E4M3 codes.
//
// The total of a key needs every row's softmax denominator over the whole cache before its first weight is known. Up to 16
// packed rows this kernel streams K once, by TMA into a shared-memory ring like the decode step's main kernel, and leaves every
// score in a scratch array (kScoreDump), from which the add kernel makes the weights, once the pieces' statistics are joined:
// a row's score of a key is 4 bytes where the key's row of K is 2 d. With more rows the scratch would cost more than K, so K is
// streamed twice, first for the statistics (kScoreStats), then for the sums of the weights over the rows (kScoreSums: one float
// a key and share of the rows); the rule stands at score_variant. Bound: HBM (K); with E4M3 codes above 16 rows the
// instructions of 16 warps an SM (32 rows: issue slots 56 %, tensor pipe 41 %, DRAM 39 % busy), of which the conversion of the
// codes, repeated by every share of the rows, is the larger part.
// Measured: 8 rows, 64 ragged sequences of up to 8192 keys, 8 KV heads of 128 bf16 (284 MB of K): 52 us for this kernel, 65
// for the call; 32 rows there: 110 us, 64 rows 165. 16 rows, 8 x 32768 E4M3 codes in pages of 64: 67 us, the call 104.
//
// One producer warp; consumer warps in RS shares of the rows of four warps each. HPC * KW = 4 warps, each with KS 16-key slices
// of a tile for one KV head and the share's packed rows: S^T [16 keys x 8 NT] = K_slice . Q^T with the keys as the M dimension
// of mma.sync, K fragments by ldmatrix from the swizzled tile, query rows in registers. Row statistics are kept by each thread
// for its own keys (an online softmax with a reference that moves only when a score exceeds it by more than 2^8, no shuffles)
// and joined once per piece.
#pragma once
#include <cuda_bf16.h>

#include "plt_common.cuh"
#include "plt_evict.h"
#include "plt_ptx.cuh"

namespace plt {

constexpr uint64_t kScoreWaitNs = 2000000000ull;
constexpr float kScoreSlack = 8.f;
constexpr float kScoreNoMax = -1e30f;

// What a pass over K leaves: every score and the row statistics; the statistics alone; or, with the joined statistics at
// hand, the weights of every key summed over the rows.
enum ScoreMode { kScoreDump, kScoreStats, kScoreSums };

template <int D, int NT, int RS, int HPC, bool FP8>
struct ScoreCfg {
    static constexpr int ES = FP8 ? 1 : 2;
    static constexpr int NH = D * ES / 128;            // 128-byte pieces of a head row
    static constexpr int KW = 4 / HPC;                 // warps along the keys
    static constexpr int KS = 2;                       // 16-key slices per warp
    static constexpr int TK = 16 * KW * KS;
    static constexpr int CONSUMERS = 4 * RS;           // warps
    static constexpr int NTHREADS = (CONSUMERS + 1) * 32;
    static constexpr int PIECE_BYTES = 128 * TK * HPC; // one 128-byte piece of all rows of a tile
    static constexpr int STAGE_BYTES = NH * PIECE_BYTES;
    static constexpr int kMaxStages = 8;
    __host__ __device__ static constexpr size_t smem_bytes(int stages, int max_batch) {
        return 1024 + (size_t)stages * STAGE_BYTES + 2 * kMaxStages * 8 + (size_t)(2 * max_batch + 8) * 4;
    }
};

template <int D, int NT, int RS, int HPC, bool FP8, int MODE>
__global__ void __launch_bounds__(ScoreCfg<D, NT, RS, HPC, FP8>::NTHREADS, NT * RS <= 4 ? 2 : 1)
plt_evict_scores(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ EvictWeights e, const int stages) {
    using C = ScoreCfg<D, NT, RS, HPC, FP8>;
    const Params& p = e.p;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t* full_bar = (uint64_t*)(smem + (size_t)stages * C::STAGE_BYTES);
    uint64_t* empty_bar = full_bar + C::kMaxStages;
    int32_t* s_ctl = (int32_t*)(empty_bar + C::kMaxStages);   // [0] a wait ran out, [1] tiles issued
    int32_t* s_prefix = s_ctl + 2;
    int32_t* s_lens = s_prefix + p.B + 2;

    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    uint32_t flags = 0;
    bool ok = true;
    if (tid == 0) {
        s_ctl[0] = 0;
        s_ctl[1] = 0;
        for (int s = 0; s < stages; ++s) {
            mbar_init(&full_bar[s], 1);
            mbar_init(&empty_bar[s], C::CONSUMERS);
        }
        mbar_fence_init();
    }
    build_prefix(p, s_prefix, flags, s_lens);   // contains __syncthreads
    grid_dependency_wait();       // from here on caches and queries are read and the scratch (which the add kernel of an
                                  // earlier call may still read) is written
    grid_launch_dependents();     // the add kernel may set up; it waits for this grid before it reads the scratch
    const int64_t T = s_prefix[p.B];
    const int cta = blockIdx.x, nctas = evict_ctas(T, (int)gridDim.x, kEvictScoreTiles);
    const bool in_plan = cta < nctas;
    const int64_t lo = in_plan ? cta_begin(T, cta, nctas) : 0, hi = in_plan ? cta_begin(T, cta + 1, nctas) : 0;

    if (wid == C::CONSUMERS) {
        // =========================== producer warp (one lane issues) ==============================
        if (lane == 0 && lo < hi) {
            tma_prefetch_desc(&tmK);
            const uint64_t stream_once = l2_evict_first_policy();
            uint32_t it = 0, use = 0;
            int stage = 0;
            PieceWalk walk(p, s_prefix, lo, hi, s_lens);
            Piece pc;
            while (ok && walk.next(pc, flags)) {
                const int32_t* ptab = p.page_table + (int64_t)pc.b * p.max_pages;
                for (int t = pc.t0; t < pc.t1; ++t, ++it) {
                    if (use > 0) {
                        ok = mbar_wait_bounded(&empty_bar[stage], (use - 1) & 1, kScoreWaitNs);
                        if (!ok) {
                            flags |= kDevWaitTimeout;
                            break;
                        }
                    }
                    uint8_t* dst = smem + (size_t)stage * C::STAGE_BYTES;
                    mbar_expect_tx(&full_bar[stage], C::STAGE_BYTES);
                    // boxes of kbox keys (a divisor of the tile and of the page): [box][head][key][128 bytes]
                    for (int k = 0; k < C::TK; k += e.kbox) {
                        int c1 = t * C::TK + k, c3 = e.b0 + pc.b;
                        if (p.page_size > 0) {
                            const int pg = min(c1 / p.page_size, p.max_pages - 1);   // boxes behind the last key: any page
                            int page = ptab[pg];
                            if (page < 0 || page >= p.num_pool_pages) {
                                if (c1 < pc.sp.cmax) flags |= kDevPageIdClamped;
                                page = page < 0 ? 0 : p.num_pool_pages - 1;
                            }
                            c1 %= p.page_size;
                            c3 = page;
                        }
#pragma unroll
                        for (int hf = 0; hf < C::NH; ++hf)
                            tma_load_4d(dst + hf * C::PIECE_BYTES + k * HPC * 128, &tmK, &full_bar[stage], hf * (128 / C::ES), c1,
                                        pc.hg * HPC, c3, stream_once);
                    }
                    if (++stage == stages) {
                        stage = 0;
                        ++use;
                    }
                }
            }
            s_ctl[1] = (int32_t)it;
        }
    } else {
        // ================================= consumer warps =========================================
        const int slot4 = wid & 3, h_local = slot4 / C::KW, kw = slot4 % C::KW;
        const int rs = wid >> 2, rb = rs * NT * 8;   // this warp's rows: rb .. rb + 8 NT
        const int grp = lane >> 2, tq = lane & 3;
        const __nv_bfloat16* qg = (const __nv_bfloat16*)p.q;
        int lc[NT][2];   // loop of the row in the low byte (kMaxLoops: no row), newer tokens of the step above it
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = rb + nt * 8 + 2 * tq + j;
                const int lq = r / p.G;
                lc[nt][j] = r < p.R ? (lq / p.Qn) | ((p.Qn - 1 - lq % p.Qn) << 8) : kMaxLoops;
            }
        // byte offset of this warp's 16-key slices in a tile of kbox-key boxes
        int slice[C::KS];
#pragma unroll
        for (int ki = 0; ki < C::KS; ++ki) {
            const int k0 = (kw * C::KS + ki) * 16, box = k0 / e.kbox;
            slice[ki] = ((box * HPC + h_local) * e.kbox + (k0 - box * e.kbox)) * 128;
        }
        const int krow = (lane & 7) + ((lane >> 3) & 1) * 8;
        const uint32_t frag = (uint32_t)(krow * 128 + (((lane >> 4) ^ (krow & 7)) << 4));

        int stage = 0;
        uint32_t use = 0;
        int q_b = -1, q_hg = -1;
        uint32_t qb[D / 16][NT][2];
        PieceWalk walk(p, s_prefix, lo, hi, s_lens);
        Piece pc;
        while (walk.next(pc, flags)) {
            const int kvh = pc.hg * HPC + h_local;
            if (pc.b != q_b || pc.hg != q_hg) {
                q_b = pc.b;
                q_hg = pc.hg;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int r = rb + nt * 8 + grp;
                    const bool v = r < p.R;
                    const int lq = v ? r / p.G : 0;
                    const int64_t head_row = ((int64_t)pc.b * p.L * p.Qn + lq) * p.Hq + kvh * p.G + (v ? r - lq * p.G : 0);
                    const int64_t qrow = (head_row >> p.qsplit) * D;
                    const int zero_half = p.qsplit ? 1 - (int)(head_row & 1) : -1;
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        const bool useq = v && ks / (D / 32) != zero_half;
                        if constexpr (FP8) {
                            // a thread's K fragment holds d = 16 ks + 4 tq .. + 3 (pairs of codes move as 16-bit units); codes
                            // and bf16 queries are exact in f16 (queries: in its normal range, 2^-25 off below it)
                            uint2 u = make_uint2(0u, 0u);
                            if (useq) u = *(const uint2*)(qg + qrow + ks * 16 + 4 * tq);
                            qb[ks][nt][0] = pack_f16x2(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u));
                            qb[ks][nt][1] = pack_f16x2(__uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
                        } else {
                            qb[ks][nt][0] = useq ? *(const uint32_t*)(qg + qrow + ks * 16 + 2 * tq) : 0u;
                            qb[ks][nt][1] = useq ? *(const uint32_t*)(qg + qrow + ks * 16 + 2 * tq + 8) : 0u;
                        }
                    }
                }
            }
            float mref[NT][2], lsum[NT][2];   // reference and sum of the rows; kScoreSums: what the join left
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                mref[nt][0] = mref[nt][1] = kScoreNoMax;
                lsum[nt][0] = lsum[nt][1] = 0.f;
            }
            if constexpr (MODE == kScoreSums) {   // rows of the joined statistics lie as far apart as there are, rounded up to four
                const float2* mc = e.mc + ((int64_t)pc.b * p.Hkv + kvh) * e.row_pitch;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int r = rb + nt * 8 + 2 * tq + j;
                        const float2 c = r < p.R ? mc[r] : make_float2(INFINITY, 0.f);
                        mref[nt][j] = c.x;
                        lsum[nt][j] = c.y;
                    }
            }
            int cutr[NT][2], cmin = 0x7fffffff;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) cutr[nt][0] = cutr[nt][1] = 0;
#pragma unroll
            for (int l = 0; l < kMaxLoops; ++l)
                if (l < p.L) {
                    const int c = pc.sp.cut[l];
                    cmin = min(cmin, max(c - (p.Qn - 1), 0));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if ((lc[nt][j] & 0xff) == l) cutr[nt][j] = max(c - (lc[nt][j] >> 8), 0);
                }
            const float sc2 = FP8 ? p.scale_log2 * p.k_scale[kvh] : p.scale_log2;
            // the item's first tile on the line, behind its lead-in (whose places in the scratch stay empty)
            const int64_t tile0 = (int64_t)s_prefix[pc.b] + (int64_t)pc.hg * line_len(p, pc.sp.gt) + p.piece_cost;

            for (int t = pc.t0; t < pc.t1; ++t) {
                if (ok) {
                    ok = __all_sync(0xffffffffu, mbar_wait_bounded(&full_bar[stage], use & 1, kScoreWaitNs));   // what follows is the whole warp's
                    if (!ok) flags |= kDevWaitTimeout;
                }
                if (ok) {
                    const uint32_t sK = smem_u32(smem + (size_t)stage * C::STAGE_BYTES) + frag;
                    float s[C::KS][NT][4];
#pragma unroll
                    for (int ki = 0; ki < C::KS; ++ki)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) s[ki][nt][0] = s[ki][nt][1] = s[ki][nt][2] = s[ki][nt][3] = 0.f;
                    if constexpr (FP8) {
#pragma unroll
                        for (int j = 0; j < D / 32; ++j)
#pragma unroll
                            for (int ki = 0; ki < C::KS; ++ki) {
                                uint32_t r[4];
                                ldmatrix_x4((sK + slice[ki]) ^ (uint32_t)(j << 5), r[0], r[1], r[2], r[3]);
#pragma unroll
                                for (int c = 0; c < 2; ++c) {
                                    const uint32_t a[4] = {e4m3x2_to_f16x2(r[2 * c]), e4m3x2_to_f16x2(r[2 * c + 1]),
                                                           e4m3x2_to_f16x2(r[2 * c] >> 16), e4m3x2_to_f16x2(r[2 * c + 1] >> 16)};
#pragma unroll
                                    for (int nt = 0; nt < NT; ++nt) mma_f16_16816(s[ki][nt], a, qb[2 * j + c][nt][0], qb[2 * j + c][nt][1]);
                                }
                            }
                    } else {
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                            for (int ki = 0; ki < C::KS; ++ki) {
                                uint32_t a[4];
                                ldmatrix_x4(((sK + slice[ki]) ^ (uint32_t)((ks & 3) << 5)) + (uint32_t)((ks >> 2) * C::PIECE_BYTES), a[0],
                                            a[1], a[2], a[3]);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) mma_bf16_16816(s[ki][nt], a, qb[ks][nt][0], qb[ks][nt][1]);
                            }
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&empty_bar[stage]);   // the tile is in registers: the slot may be refilled
                    const int key0 = t * C::TK + kw * C::KS * 16 + grp;   // this thread's keys: key0 + 16 ki (+ 8)
                    const bool masked = t * C::TK + C::TK > cmin;
                    float* dst = e.scores + (((tile0 + t) * HPC + h_local) * C::TK + kw * C::KS * 16 + grp) * (int64_t)e.key_pitch + (MODE == kScoreSums ? rs : rb + 2 * tq);
                    float total[C::KS][2];
#pragma unroll
                    for (int ki = 0; ki < C::KS; ++ki) total[ki][0] = total[ki][1] = 0.f;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float mx = -INFINITY;
#pragma unroll
                            for (int ki = 0; ki < C::KS; ++ki)
#pragma unroll
                                for (int u = 0; u < 2; ++u) {
                                    float x = s[ki][nt][2 * u + j] * sc2;
                                    if (masked && key0 + 16 * ki + 8 * u >= cutr[nt][j]) x = -INFINITY;
                                    s[ki][nt][2 * u + j] = x;
                                    mx = fmaxf(mx, x);
                                }
                            if constexpr (MODE == kScoreSums) {
#pragma unroll
                                for (int ki = 0; ki < C::KS; ++ki)
#pragma unroll
                                    for (int u = 0; u < 2; ++u)
                                        total[ki][u] = fmaf(fast_exp2(s[ki][nt][2 * u + j] - mref[nt][j]), lsum[nt][j], total[ki][u]);
                            } else {
                                if (mx - mref[nt][j] > kScoreSlack) {
                                    lsum[nt][j] *= fast_exp2(mref[nt][j] - mx);
                                    mref[nt][j] = mx;
                                }
#pragma unroll
                                for (int ki = 0; ki < C::KS; ++ki)
                                    lsum[nt][j] += fast_exp2(s[ki][nt][j] - mref[nt][j]) + fast_exp2(s[ki][nt][2 + j] - mref[nt][j]);
                            }
                        }
                        if (MODE == kScoreDump && rb + nt * 8 + 2 * tq < e.key_pitch) {   // behind the last row: finite, or -inf
#pragma unroll
                            for (int ki = 0; ki < C::KS; ++ki)
#pragma unroll
                                for (int u = 0; u < 2; ++u)
                                    *(float2*)(dst + (int64_t)(16 * ki + 8 * u) * e.key_pitch + nt * 8) =
                                        make_float2(s[ki][nt][2 * u], s[ki][nt][2 * u + 1]);
                        }
                    }
                    if constexpr (MODE == kScoreSums) {   // the four threads that share a key
#pragma unroll
                        for (int ki = 0; ki < C::KS; ++ki)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                float x = total[ki][u];
                                x += __shfl_xor_sync(0xffffffffu, x, 1);
                                x += __shfl_xor_sync(0xffffffffu, x, 2);
                                if (tq == ((2 * ki + u) & 3)) dst[(16 * ki + 8 * u) * RS] = x;
                            }
                    }
                } else {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&empty_bar[stage]);
                }
                if (++stage == stages) {
                    stage = 0;
                    ++use;
                }
            }
            if constexpr (MODE == kScoreSums) continue;
            // ---- end of piece: the eight threads that share a row join their statistics --------------
            const int64_t slot = slot_of(item_index(p, pc.b, pc.hg, 0), cta);
            if (tid == 0) note_piece(p, pc, cta);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float m = mref[nt][j], l = lsum[nt][j];
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) {
                        const float m2 = __shfl_xor_sync(0xffffffffu, m, o), l2 = __shfl_xor_sync(0xffffffffu, l, o);
                        const float mm = fmaxf(m, m2);
                        l = l * fast_exp2(m - mm) + l2 * fast_exp2(m2 - mm);
                        m = mm;
                    }
                    if (grp == 0 && lc[nt][j] != kMaxLoops) {
                        const int64_t row = ((slot * HPC + h_local) * C::KW + kw) * p.R + rb + nt * 8 + 2 * tq + j;
                        *(float2*)(e.ml + row * 2) = make_float2(m, l);
                    }
                }
        }
    }
    if (flags) atomicOr(p.status, flags);
    if (flags & kDevWaitTimeout) s_ctl[0] = 1;
    __syncthreads();
    if (s_ctl[0] != 0 && tid == 0) {   // give every copy that was issued a bounded chance to land
        const uint32_t it = (uint32_t)s_ctl[1];
        const uint32_t filled = it < (uint32_t)stages ? it : (uint32_t)stages;
        for (uint32_t s = 0; s < filled; ++s) mbar_wait_bounded(&full_bar[s], ((it - 1 - s) / (uint32_t)stages) & 1, kScoreWaitNs);
    }
    __syncthreads();
}

}  // namespace plt

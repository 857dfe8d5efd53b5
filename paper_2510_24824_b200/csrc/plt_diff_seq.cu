// Prompt attention of differential heads (plt_diff_seq_attn_run) on the 5th-generation tensor cores.
//
// One thread block owns 128 consecutive rows t of one (sequence, loop, query head), for BOTH softmax maps of the head. Map x
// multiplies half x of the query and key rows: one of the two 128-byte swizzled halves of the tiles as TMA wrote them, so
// nothing is padded or copied; both maps multiply the same V tile.
//
//   S_x [128 rows x 64 keys] = Q_x [128 x 64] . K_x^T [64 x 64 keys]       x = 1, 2, for each half h of a 128-key tile
//   O_x [128 rows x 128]    += P_x [128 x 64] . V_half [64 x 128]          P in tensor memory (bf16, over S)
//
// The weights are rounded to bf16 for the second product, the operand type of its V; the denominators add them unrounded. That
// puts a map's result off by at most 2^-8 of the largest value it averages, as much as the output's own rounding.
//
// Tensor memory holds both accumulators (256 columns) and, for each map, the scores of two 64-key halves (256 columns). A
// softmax warp works on one half while the products on the other half of the same map run: the P of a half is consumed and
// the next tile's scores of that half are written behind it in the tensor core's own order. With whole 128-key score tiles
// the chain scores -> softmax -> P V -> next scores of a map was open at every link, and the two maps' chains alone filled
// 40 % of the exponential unit's time (5000 rows, 32 heads: 534 us; in this order, with an issuer for each map, 394 to 428 us on
// different devices, 718 to 779 TFLOP/s over the visible keys).
//
// The block owns both results of a row, so the epilogue takes y_1 - lambda y_2 and the norm over the head's 128 elements in
// fp32 from the two accumulators, and neither map reaches memory. Steps, masks and windows of loops 2..L are those of
// plt_seq_attn.cu: the tiles of the shared K/V, then the loop's own tiles scores only, then again with the second product,
// with the gate folded into the weights.
//
// Warp roles: warp 0 streams K and V tiles by TMA into a ring of 32 KB slots, warps 1 and 2 issue the products of map 1 and 2
// (one lane each; warp 1 owns tensor memory), warps 4-7 are the softmax of map 1, warps 8-11 of map 2 (thread = row =
// tensor-memory lane). The maps share nothing but the ring and may run two steps apart; they meet once, before the epilogue. Every
// wait on an mbarrier is bounded and reports through the status word. Bound: the exponentials, 2 x
// 128 x 128 per tile and block at 16 per cycle and SM (2048 cycles; the products take 1536). A tile takes 3440: a softmax warp is
// busy for 1436 of every half's 1720, 155 of the rest are waits for scores.
#include "plt_seq_util.cuh"

namespace plt {
namespace {

constexpr int kDRing = 6;                    // K/V ring slots
constexpr int HK = SK / 2;                   // keys of a half tile

// mbarriers; [x][h] = map x, half h
constexpr int DB_QFULL = 0;                  // query tile landed
constexpr int DB_FULL = 1;                   // + slot: tile landed
constexpr int DB_EMPTY = DB_FULL + kDRing;   // + slot: products reading the slot completed
constexpr int DB_SFULL = DB_EMPTY + kDRing;  // + 2 x + h: scores complete
constexpr int DB_PFULL = DB_SFULL + 4;       // + 2 x + h: softmax has read the scores (and written the weights)
constexpr int DB_PVD = DB_PFULL + 4;         // + 2 x + h: product with V completed
constexpr int DB_COUNT = DB_PVD + 4;

constexpr size_t kDiffSmem = 1024 + (size_t)(1 + kDRing) * kTileBytes + DB_COUNT * 8 + 64;

struct DiffPlan {
    int nG, l0, nL, total;   // tiles of the shared K/V; first own tile and their number (loops 2..L); steps nG + 2 nL
    // kind 0: shared K/V, 1: own K/V scores only, 2: own K/V with the second product
    __device__ __forceinline__ void step(int i, int& kind, int& tile) const {
        kind = i < nG ? 0 : (i < nG + nL ? 1 : 2);
        tile = i < nG ? i : l0 + (i - nG) - (kind == 2 ? nL : 0);
    }
};

// D[tmem] (+)= A * B with A in shared memory (ss) or tensor memory (ts); `accumulate` is a constant where it is inlined.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    if (accumulate)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    if (accumulate)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.eq.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "l"(b), "r"(idesc) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, 0, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "l"(b), "r"(idesc) : "memory");
}

// Weights of the 64 scores of a half row against the reference mref, packed bf16 into pk, their sum and the largest.
__device__ __forceinline__ void half_pass(uint32_t tS, int lim, bool full, float scale, float mref, uint32_t (&pk)[32], float& lsum,
                                          float& pbig) {
    const float2 sc2 = make_float2(scale, scale), nm2 = make_float2(-mref, -mref);
    float2 sum2 = make_float2(0.f, 0.f);
    uint32_t pmax = 0;
    uint32_t ra[32], rb[32];
    tmem_ld32(tS, ra);
    tmem_wait_ld();
    tmem_ld32(tS + 32, rb);
    if (full) global_chunk<true>(ra, 0, lim, sc2, nm2, &pk[0], sum2, pmax); else global_chunk<false>(ra, 0, lim, sc2, nm2, &pk[0], sum2, pmax);
    tmem_wait_ld();
    if (full) global_chunk<true>(rb, 1, lim, sc2, nm2, &pk[16], sum2, pmax); else global_chunk<false>(rb, 1, lim, sc2, nm2, &pk[16], sum2, pmax);
    lsum = sum2.x + sum2.y;
    pbig = fmaxf(__uint_as_float(pmax << 16), __uint_as_float(pmax & 0xffff0000u));
}

// Largest visible score of a half row.
__device__ __forceinline__ float half_max(uint32_t tS, int lim) {
    float mx = -INFINITY;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint32_t r[32];
        tmem_ld32(tS + c * 32, r);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (c * 32 + i < lim) mx = fmaxf(mx, __uint_as_float(r[i]));
    }
    return mx;
}

__global__ void __launch_bounds__(kSeqThreads, 1)
plt_diff_seq_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmKl,
                    const __grid_constant__ CUtensorMap tmVl, const __grid_constant__ SeqParams p) {
    extern __shared__ uint8_t seq_smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)seq_smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* q_smem = smem;                              // one tile; the epilogue's exchange buffer afterwards
    uint8_t* ring = smem + kTileBytes;                   // [kDRing][tile]
    uint64_t* bars = (uint64_t*)(ring + (size_t)kDRing * kTileBytes);
    int32_t* s_ctl = (int32_t*)(bars + DB_COUNT);        // [0] abort flag, [1] tensor-memory base, [2] loads issued
    volatile int* abort_flag = (volatile int*)s_ctl;
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;

    // ---- which rows: blocks with the most key tiles (the last rows of a sequence) come first in the grid ----
    int item = blockIdx.x;
    const int h = item % p.Hq; item /= p.Hq;
    const int l = item % p.L; item /= p.L;
    const int b = item % p.B; item /= p.B;
    const int r0 = (p.nqb - 1 - item) * SQ;
    uint32_t flags = 0;
    int n = p.seq_lens[b];
    if (n < 0 || n > p.T) {
        flags |= kDevSeqLenClamped;
        n = n < 0 ? 0 : p.T;
    }
    const int delta = p.delta[l], kvh = h / p.G;
    DiffPlan pl;
    {
        const int keys = r0 < n ? min(n, r0 + SQ) - delta : 0;
        pl.nG = keys > 0 ? (keys + SK - 1) / SK : 0;
        pl.l0 = pl.nL = 0;
        if (l > 0 && pl.nG > 0) {   // own keys: from the window start of the first row with a token to the last live row
            pl.l0 = max(delta, max(r0, delta) + 1 - p.w) / SK;
            pl.nL = (min(n, r0 + SQ) - 1) / SK - pl.l0 + 1;
        }
        pl.total = pl.nG + 2 * pl.nL;
    }

    if (pl.total == 0) {   // no row has a token: zeros, without tensor memory or barriers
        for (int i = tid; i < (min(r0 + SQ, p.T) - r0) * (SD / 8); i += kSeqThreads)
            *(uint4*)(p.out + ((((int64_t)b * p.L + l) * p.T + r0 + i / (SD / 8)) * p.Hq + h) * SD + i % (SD / 8) * 8) = make_uint4(0, 0, 0, 0);
        if (flags && tid == 0) atomicOr(p.status, flags);
        return;
    }
    if (tid == 0) {
        s_ctl[0] = 0;
        s_ctl[2] = 0;
        mbar_init(&bars[DB_QFULL], 1);
        for (int s = 0; s < kDRing; ++s) {
            mbar_init(&bars[DB_FULL + s], 1);
            mbar_init(&bars[DB_EMPTY + s], 2);   // both issuers
        }
        for (int s = 0; s < 4; ++s) {
            mbar_init(&bars[DB_SFULL + s], 1);
            mbar_init(&bars[DB_PFULL + s], 4);
            mbar_init(&bars[DB_PVD + s], 1);
        }
        mbar_fence_init();
    }
    if (wid == 1) tmem_alloc((uint32_t*)&s_ctl[1], 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = (uint32_t)s_ctl[1];
    // columns: scores of (x, h) at 128 x + 64 h (weights over the first 32 of them), O_x at 256 + 128 x

    if (wid == 0) {
        // =========================== TMA producer (one lane) ==============================================
        if (lane == 0) {
            tma_prefetch_desc(&tmQ);
            tma_prefetch_desc(&tmK);
            tma_prefetch_desc(&tmV);
            const uint64_t keep = l2_evict_first_policy();
            mbar_expect_tx(&bars[DB_QFULL], kTileBytes);
            for (int hf = 0; hf < 2; ++hf) tma_load_4d(q_smem + hf * kHalf, &tmQ, &bars[DB_QFULL], hf * 64, h, r0, b * p.L + l, keep);
            int slot = 0;
            uint32_t parity = 0, issued = 0;
            bool ok = true;
            for (int i = 0; i < pl.total && ok; ++i) {
                int kind, tile;
                pl.step(i, kind, tile);
                for (int which = 0; which < (kind == 1 ? 1 : 2) && ok; ++which) {
                    if (issued >= (uint32_t)kDRing) ok = seq_wait(&bars[DB_EMPTY + slot], parity ^ 1u, abort_flag);
                    if (!ok) break;
                    const CUtensorMap* m = kind == 0 ? (which == 0 ? &tmK : &tmV) : (which == 0 ? &tmKl : &tmVl);
                    const int c3 = kind == 0 ? b : b * (p.L - 1) + (l - 1);
                    uint8_t* dst = ring + (size_t)slot * kTileBytes;
                    mbar_expect_tx(&bars[DB_FULL + slot], kTileBytes);
                    for (int hf = 0; hf < 2; ++hf) tma_load_4d(dst + hf * kHalf, m, &bars[DB_FULL + slot], hf * 64, kvh, tile * SK, c3, keep);
                    ++issued;
                    if (++slot == kDRing) {
                        slot = 0;
                        parity ^= 1u;
                    }
                }
            }
            s_ctl[2] = (int32_t)issued;
        }
    } else if (wid <= 2) {
        // =========================== product issue: warp 1 + x for map x (whole warp walks, lane 0 issues) ==========
        // One lane's instruction stream is what bounds the issue (about 95 cycles a product with its descriptors and commits,
        // against 32 to 64 cycles of the tensor core), so each map has an issuer of its own.
        const int x = wid - 1;
        constexpr uint32_t idesc_qk = seq_instr_desc(SQ, HK, 0);
        constexpr uint32_t idesc_pv = seq_instr_desc(SQ, SD, 1);
        // descriptors of the first byte; a byte offset adds offset / 16 to the address field
        const uint64_t q_desc = seq_smem_desc(smem_u32(q_smem) + x * kHalf, 16, 1024);
        const uint64_t k_desc = seq_smem_desc(smem_u32(ring) + x * kHalf, 16, 1024);
        const uint64_t v_desc = seq_smem_desc(smem_u32(ring), kHalf, 1024);
        const uint32_t tS = tmem_base + x * 128, tO = tmem_base + 256 + x * 128;
        // waits as a warp; false once any wait of the block has run out
        auto wait = [&](int bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, seq_wait(&bars[bar], parity, abort_flag)); };
        auto issue_s = [&](int slot, int hh) {   // scores of half hh on the K tile in `slot`
            if (lane == 0) {
                const uint64_t kd = k_desc + (uint64_t)(slot * (kTileBytes / 16) + hh * (HK * 128 / 16));
#pragma unroll
                for (int kk = 0; kk < SD / 32; ++kk) mma_ss(tS + hh * HK, q_desc + kk * 2, kd + kk * 2, idesc_qk, kk > 0);
                umma_commit(&bars[DB_SFULL + 2 * x + hh]);
            }
            __syncwarp();
        };
        int slot = 0;                            // ring position of the next load to be used
        uint32_t parity = 0;
        auto advance = [&]() {
            if (++slot == kDRing) {
                slot = 0;
                parity ^= 1u;
            }
        };
        bool ok = wait(DB_QFULL, 0) && wait(DB_FULL + 0, 0);
        if (ok) {
            tc_fence_after_sync();
            issue_s(0, 0);
            issue_s(0, 1);
            if (lane == 0) umma_commit(&bars[DB_EMPTY + 0]);
            __syncwarp();
            advance();
        }
        bool o_started = false;
        for (int i = 0; i < pl.total && ok; ++i) {
            int kind, tile;
            pl.step(i, kind, tile);
            const int v_slot = slot;
            if (kind != 1) {
                ok = wait(DB_FULL + slot, parity);
                if (!ok) break;
                advance();
                // Rows of the V tile at or beyond the sequence's length may hold anything: zero them, so that a weight
                // of 0 times garbage cannot produce NaN (both issuers write the same zeros before their own products).
                const int vrow0 = max(n - tile * SK, 0);
                if (vrow0 < SK) {
                    uint8_t* v = ring + (size_t)v_slot * kTileBytes;
                    for (int idx = lane; idx < (SK - vrow0) * 16; idx += 32) {
                        const int row = vrow0 + idx / 16, ch = idx % 16;
                        *(uint4*)(v + (ch >> 3) * kHalf + row * 128 + (ch & 7) * 16) = make_uint4(0, 0, 0, 0);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                }
            }
            const bool next = i + 1 < pl.total;
            const int k_slot = slot;
            if (next) {
                ok = wait(DB_FULL + slot, parity);   // there since the step before, as a rule: the ring is six deep
                if (!ok) break;
                advance();
            }
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                if (ok) ok = wait(DB_PFULL + 2 * x + hh, (uint32_t)i & 1u);
                if (ok) {
                    tc_fence_after_sync();
                    if (kind != 1) {
                        if (lane == 0) {
                            const uint64_t vd = v_desc + (uint64_t)(v_slot * (kTileBytes / 16) + hh * (HK * 128 / 16));
#pragma unroll
                            for (int kk = 0; kk < HK / 16; ++kk) {
                                if (hh == 0 && kk == 0 && !o_started) mma_ts(tO, tS, vd, idesc_pv, false);
                                else mma_ts(tO, tS + hh * HK + kk * 8, vd + kk * (2048 / 16), idesc_pv, true);
                            }
                            umma_commit(&bars[DB_PVD + 2 * x + hh]);
                        }
                        __syncwarp();
                    }
                    // the next tile's scores of this half: behind the product that reads its weights, in order
                    if (next) issue_s(k_slot, hh);
                }
            }
            if (!ok) break;
            if (kind != 1) o_started = true;
            if (lane == 0) {
                if (kind != 1) umma_commit(&bars[DB_EMPTY + v_slot]);
                if (next) umma_commit(&bars[DB_EMPTY + k_slot]);
            }
            __syncwarp();
        }
    } else if (wid >= 4) {
        // =========================== softmax and epilogue ================================================
        const int x = (wid - 4) >> 2;                      // map
        const int wq = wid & 3;                            // lane quarter of tensor memory this warp may touch
        const int row = wq * 32 + lane;
        RowCtx rc;
        rc.t = r0 + row;
        rc.cut = max(0, min(rc.t, n - 1) + 1 - delta);
        rc.lo = max(delta, rc.t + 1 - p.w);
        rc.live = rc.t < n && rc.t + 1 - delta > 0;
        const uint32_t t_lane = tmem_base + ((uint32_t)(wq * 32) << 16);
        const uint32_t tO = t_lane + 256 + x * 128;
        const float scale = p.scale_log2;
        float d1 = 0.f, d2 = 0.f;                          // the learned factor of this head
        {
            const int lrow = p.tail.lambda_heads > 1 ? h * (SD / 2) : 0;
#pragma unroll
            for (int i = lane; i < SD / 2; i += 32) {
                d1 = fmaf(p.tail.lq1[lrow + i], p.tail.lk1[lrow + i], d1);
                d2 = fmaf(p.tail.lq2[lrow + i], p.tail.lk2[lrow + i], d2);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                d1 += __shfl_xor_sync(0xffffffffu, d1, o);
                d2 += __shfl_xor_sync(0xffffffffu, d2, o);
            }
        }
        const float lambda = expf(d1) - expf(d2) + p.tail.lambda_init;
        float gate = 0.f;
        if (l > 0 && rc.t < p.T) {
            const float z = p.gate[(((int64_t)b * (p.L - 1) + (l - 1)) * p.T + rc.t) * p.Hq + h];
            gate = 1.f / (1.f + __expf(-z));
        }
        float mref = kSeqNoMax, lg = 0.f;       // shared-K/V softmax: reference maximum (log2 units) and denominator
        float ml = -INFINITY, ll = 0.f;          // window softmax: exact maximum (log2 units) and denominator
        bool ok = true, o_scaled = false;
        uint32_t pv = 0;                         // steps with a second product before this one; of a half: + 1 once handed over
        // Waits until every product into O_x of the halves handed over so far has completed (`h1`: this step's first half is
        // among them). Collective over the warp.
        auto wait_products = [&](bool h1) {
            for (int hh = 0; hh < 2; ++hh) {
                const uint32_t count = pv + (hh == 0 && h1 ? 1u : 0u);
                if (count > 0 && ok) ok = seq_wait(&bars[DB_PVD + 2 * x + hh], (count - 1) & 1u, abort_flag);
            }
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after_sync();
        };
        for (int i = 0; i < pl.total && ok; ++i) {
            int kind, tile;
            pl.step(i, kind, tile);
            const bool full = tile * SK + SK <= r0 + 1 - delta && tile * SK + SK <= n;   // kind 0: no key masked for any row
#pragma unroll 1
            for (int hh = 0; hh < 2; ++hh) {
                ok = __all_sync(0xffffffffu, seq_wait(&bars[DB_SFULL + 2 * x + hh], (uint32_t)i & 1u, abort_flag));
                if (!ok) break;                  // the tensor-memory accesses below are collective over the warp
                tc_fence_after_sync();
                const uint32_t tS = t_lane + x * 128 + hh * HK;
                const int kbase = tile * SK + hh * HK;
                uint32_t pk[32];
                if (kind == 0) {
                    // ---- shared K/V: online softmax against the lazily updated reference ----------------
                    const int lim = rc.cut - kbase;
                    float lsum, pbig;
                    half_pass(tS, lim, full, scale, mref, pk, lsum, pbig);
                    if (__any_sync(0xffffffffu, rc.live && !(pbig <= kSeqBig))) {
                        // a weight of a live row beyond 2^8 of its reference: true maximum, rescale of this row of O once
                        // every product into it has completed, weights again
                        const float m_new = fmaxf(mref, half_max(tS, lim) * scale);
                        const float alpha = fast_exp2(mref - m_new);
                        mref = m_new;
                        lg *= alpha;
                        wait_products(hh == 1);
                        if (!ok) break;
                        if (pv > 0 || hh == 1) scale_o_row(tO, alpha);
                        half_pass(tS, lim, full, scale, mref, pk, lsum, pbig);
                    }
                    lg += lsum;
                } else {
                    if (!o_scaled) {
                        // O_x holds the unnormalised shared-K/V sum: make it (1 - g) * y_global (Eq. 2)
                        o_scaled = true;
                        wait_products(hh == 1);
                        if (!ok) break;
                        scale_o_row(tO, (rc.live && lg > 0.f) ? (1.f - gate) / lg : 0.f);
                    }
                    // own keys lo .. t of the row: columns [c_lo, c_hi] of the half
                    const int c_lo = rc.lo - kbase, c_hi = rc.t - kbase;
                    uint32_t r[32];
                    if (kind == 1) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            tmem_ld32(tS + c * 32, r);
                            tmem_wait_ld();
                            window_stats_chunk(r, c, c_lo, c_hi, scale, ml, ll);
                        }
                    } else {
                        // weights already normalised and gated: g * 2^(s - m) / l = 2^(s - m + log2(g / l))
                        const float beta = (rc.live && ll > 0.f) ? gate / ll : 0.f;
                        const float negm = beta > 0.f ? fast_log2(beta) - ml : -INFINITY;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            tmem_ld32(tS + c * 32, r);
                            tmem_wait_ld();
                            window_weights_chunk(r, c, c_lo, c_hi, make_float2(scale, scale), make_float2(negm, negm), &pk[c * 16]);
                        }
                    }
                }
                if (kind != 1) {
                    tmem_st32(tS, pk);
                    tmem_wait_st();
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars[DB_PFULL + 2 * x + hh]);
            }
            if (kind != 1) ++pv;
        }
        // ---- epilogue: both accumulators out of tensor memory ------------------------------------------------
        // Each map waits for its own last products only: a barrier's parity tells a phase from the one before it, and nothing
        // keeps the maps that close (the ring leaves them up to two steps apart). The block barrier then stands for both, and
        // for every product that reads the query tile, which the exchange buffer overwrites.
        wait_products(false);
        tc_fence_before_sync();                            // the other map's accumulator is read behind the barrier: its products,
        named_barrier_sync(1, 256);                        // and what its softmax warps stored to it, come before those loads
        tc_fence_after_sync();
        float* xch = (float*)q_smem;                       // [4][128]
        xch[x * SQ + row] = l == 0 ? (lg > 0.f ? 1.f / lg : 0.f) : 1.f;   // makes accumulator x of the row a finished result
        named_barrier_sync(1, 256);
        const float f1 = xch[row], f2 = -lambda * xch[SQ + row];
        // this thread's half of the row: columns [64 x, 64 x + 64)
        float y[SD / 2], ss = 0.f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint32_t ra[32], rb[32];
            if (ok) {
                tmem_ld32(t_lane + 256 + x * 64 + c * 32, ra);
                tmem_ld32(t_lane + 384 + x * 64 + c * 32, rb);
                tmem_wait_ld();
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float v = ok && rc.live ? fmaf(f2, __uint_as_float(rb[i]), f1 * __uint_as_float(ra[i])) : 0.f;
                y[c * 32 + i] = v;
                ss = fmaf(v, v, ss);
            }
        }
        float inv = 1.f;
        if (p.tail.gain != nullptr) {
            xch[2 * SQ + x * SQ + row] = ss;
            named_barrier_sync(1, 256);
            ss += xch[2 * SQ + (1 - x) * SQ + row];
            inv = (1.f - p.tail.lambda_init) / sqrtf(ss * (1.f / SD) + p.tail.eps);
        }
        if (rc.t < p.T) {
            __nv_bfloat16* dst = p.out + ((((int64_t)b * p.L + l) * p.T + rc.t) * p.Hq + h) * SD + x * 64;
#pragma unroll
            for (int i = 0; i < SD / 2; i += 8) {
                float g[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = inv * (p.tail.gain != nullptr ? p.tail.gain[x * 64 + i + j] : 1.f);
                uint4 v;
                v.x = pack_bf16x2(y[i] * g[0], y[i + 1] * g[1]);
                v.y = pack_bf16x2(y[i + 2] * g[2], y[i + 3] * g[3]);
                v.z = pack_bf16x2(y[i + 4] * g[4], y[i + 5] * g[5]);
                v.w = pack_bf16x2(y[i + 6] * g[6], y[i + 7] * g[7]);
                *(uint4*)(dst + i) = v;
            }
        }
    }
    if (flags && tid == 0) atomicOr(p.status, flags);
    tc_fence_before_sync();
    __syncthreads();
    if (tid == 0 && s_ctl[0] != 0) {
        atomicOr(p.status, kDevWaitTimeout);
        // give every copy that was issued a bounded chance to land before the block retires
        const uint32_t issued = (uint32_t)s_ctl[2];
        const uint32_t outstanding = issued < (uint32_t)kDRing ? issued : (uint32_t)kDRing;
        for (uint32_t k = 0; k < outstanding; ++k) {
            const uint32_t cnt = issued - 1 - k;
            mbar_wait_bounded(&bars[DB_FULL + cnt % kDRing], (cnt / kDRing) & 1u, kSeqWaitNs);
        }
        mbar_wait_bounded(&bars[DB_QFULL], 0, kSeqWaitNs);
    }
    __syncthreads();
    if (wid == 1) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, 512);
    }
}

}  // namespace

cudaError_t diff_seq_prepare() { return allow_max_dynamic_smem((const void*)plt_diff_seq_kernel); }

cudaError_t launch_diff_seq(const CUtensorMap maps[5], const SeqParams& p, unsigned grid, cudaStream_t stream) {
    plt_diff_seq_kernel<<<grid, kSeqThreads, kDiffSmem, stream>>>(maps[0], maps[1], maps[2], maps[3], maps[4], p);
    return cudaGetLastError();
}

}  // namespace plt

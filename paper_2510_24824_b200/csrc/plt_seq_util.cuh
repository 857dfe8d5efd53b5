// Pieces shared by the kernels of the sequence-shaped attention (queries as the M dimension of tcgen05.mma): tile geometry,
// kernel parameters, operand descriptors, tensor-memory accesses, bounded waits and the softmax on 32-column chunks of a row.
#pragma once
#include <cuda_bf16.h>

#include "plt_host.h"
#include "plt_ptx.cuh"

namespace plt {

constexpr int kSeqMaxLoops = 8;

struct SeqParams {
    const float* gate;          // [B, L-1, T, Hq]
    const int32_t* seq_lens;    // [B]
    __nv_bfloat16* out;         // [B, L, T, Hq, d]
    uint32_t* status;
    int32_t B, L, T, Hq, Hkv, G, w, nqb;   // nqb: row blocks per sequence (128 rows with paired heads, else 256)
    int32_t pair_heads, heads_per_grid;      // tiles of a block = two heads of one KV group; grid entries per (row block, loop)
    float scale_log2;
    int32_t delta[kSeqMaxLoops];
    DiffTail tail;              // differential heads only
};

namespace {

constexpr int SQ = 128;                    // query rows per tile
constexpr int SK = 128;                    // keys per tile
constexpr int SD = 128;                    // head dimension
constexpr int kTileBytes = SK * SD * 2;    // one Q, K or V tile
constexpr int kHalf = SK * 128;            // one 64-element half of a tile: [128 rows][128 bytes]
constexpr int kSeqThreads = 384;
constexpr float kSeqBig = 256.f;           // probabilities stay below 2^8 of their row's reference, else the slow path
constexpr float kSeqNoMax = -1e30f;
constexpr uint64_t kSeqWaitNs = 1000000000ull;

// Shared-memory matrix descriptor of tcgen05.mma (start address, leading / stride byte offsets in 16-byte units,
// descriptor version 1, 128-byte swizzle).
__device__ __forceinline__ uint64_t seq_smem_desc(uint32_t addr, uint32_t lbo_bytes, uint32_t sbo_bytes) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(lbo_bytes >> 4) << 16) | ((uint64_t)(sbo_bytes >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: fp32 accumulate, bf16 A and B, B majorness (0 = K-major, 1 = MN-major), N / 8, M / 16.
__host__ __device__ constexpr uint32_t seq_instr_desc(int M, int N, int b_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) |
           ((uint32_t)(M >> 4) << 24);
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc,
                                             uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// 32 consecutive 32-bit columns of this thread's lane
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
          "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
          "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// Bounded wait that also gives up as soon as another thread of the block has given up.
__device__ __noinline__ bool seq_wait_slow(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    const uint64_t t0 = global_timer_ns();
    uint32_t spins = 0;
    while (!mbar_try_wait(bar, parity)) {
        if ((++spins & 0x3fu) == 0) {
            if (*abort_flag) return false;
            if (global_timer_ns() - t0 > kSeqWaitNs) {
                *abort_flag = 1;
                return false;
            }
        }
    }
    return true;
}
__device__ __forceinline__ bool seq_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    if (mbar_test_wait(bar, parity)) return true;
    return seq_wait_slow(bar, parity, abort_flag);
}

// What a softmax thread knows about its row.
struct RowCtx {
    int t;            // row (decode step) index
    int cut;          // shared keys the row may see: max(0, t + 1 - delta)
    int lo;           // first own key of the window: max(delta, t + 1 - w)
    bool live;        // t < n_b and cut > 0
};

// 32 scores of a row -> probabilities against the reference: packed bf16 into pk[16], summed (fp32, two lanes) and
// their packed maximum tracked (bf16 bit patterns of non-negative numbers order like integers).
template <bool FULL>
__device__ __forceinline__ void global_chunk(const uint32_t (&r)[32], int c, int lim, float2 sc2, float2 nm2, uint32_t* pk,
                                             float2& sum2, uint32_t& pmax) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        float2 t = __ffma2_rn(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), sc2, nm2);
        if (!FULL) {
            if (c * 32 + i >= lim) t.x = -INFINITY;
            if (c * 32 + i + 1 >= lim) t.y = -INFINITY;
        }
        const float2 pr = make_float2(fast_exp2(t.x), fast_exp2(t.y));
        sum2 = __fadd2_rn(sum2, pr);
        const uint32_t h = pack_bf16x2(pr.x, pr.y);
        pk[i / 2] = h;
        asm("max.u16x2 %0, %0, %1;" : "+r"(pmax) : "r"(h));
    }
}

// Scores-only pass over a tile of the loop's own keys: folds the visible columns [c_lo, c_hi] of this thread's row into
// the window softmax's exact running maximum ml (log2 units) and denominator ll. Rows without a visible key keep
// ml = -inf, ll = 0. Every lane runs every load (they are collective over the warp).
__device__ __forceinline__ void window_stats_chunk(const uint32_t (&r)[32], int c, int c_lo, int c_hi, float scale, float& ml,
                                                   float& ll) {
    float t[32], cmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const int col = c * 32 + i;
        t[i] = (col >= c_lo && col <= c_hi) ? __uint_as_float(r[i]) * scale : -INFINITY;
        cmax = fmaxf(cmax, t[i]);
    }
    const float m_new = fmaxf(ml, cmax);
    const float m_use = m_new > -INFINITY ? m_new : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) sum += fast_exp2(t[i] - m_use);
    ll = ll * fast_exp2(ml - m_use) + sum;   // ml = -inf: the old denominator is 0 and stays 0
    ml = m_new;
}
// Second pass over the same tile: the weights 2^(s * scale + negm) of the visible columns (0 elsewhere), packed bf16.
__device__ __forceinline__ void window_weights_chunk(const uint32_t (&r)[32], int c, int c_lo, int c_hi, float2 sc2, float2 nm2,
                                                     uint32_t* pk) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        const int col = c * 32 + i;
        float2 t = __ffma2_rn(make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1])), sc2, nm2);
        if (!(col >= c_lo && col <= c_hi)) t.x = -INFINITY;
        if (!(col + 1 >= c_lo && col + 1 <= c_hi)) t.y = -INFINITY;
        pk[i / 2] = pack_bf16x2(fast_exp2(t.x), fast_exp2(t.y));
    }
}
// Multiplies this thread's row of O (128 fp32 columns) by f.
__device__ __forceinline__ void scale_o_row(uint32_t tO, float f) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint32_t r[32];
        tmem_ld32(tO + c * 32, r);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
        tmem_st32(tO + c * 32, r);
    }
    tmem_wait_st();
}

}  // namespace

// The kernel of differential heads (plt_diff_seq.cu).
cudaError_t diff_seq_prepare();
cudaError_t launch_diff_seq(const CUtensorMap maps[5], const SeqParams& p, unsigned grid, cudaStream_t stream);

}  // namespace plt

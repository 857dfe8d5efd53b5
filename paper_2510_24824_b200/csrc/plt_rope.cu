// Norm and rotation of queries and keys, with their way into the caches: a decode step and the rows of a prompt.
//
// d / 16 threads hold a head's row, 16 elements each: two 16-byte pieces whose elements are exactly the pairs that turn
// together (thread t < rotary_dim / 16 has pairs 8 t .. 8 t + 7 in both layouts), so a row is read once, normed by a shuffle
// over its threads, turned in registers and written once. The cosines and sines of a token are computed once for all its heads.
//
// An angle p f is taken in turns: f / 2 pi as a 64-bit fraction, multiplied by the position in integers, so that whole turns
// fall away exactly however far the position lies; the quarter turn is split off in integers too, and what is left (at most
// an eighth of a turn either way) goes to sincospif. Bound by reading and writing the rows.
#include "../../include/plt_rope.h"

#include <cuda_bf16.h>

#include <cmath>
#include <cstring>
#include <new>
#include <type_traits>

#include "plt_handle.h"
#include "plt_ptx.cuh"

using namespace plt;

namespace {

constexpr int kRopeThreads = 256;
constexpr int kSeqTokens = 8;         // rows of a prompt that a block takes
constexpr int kMaxPairs = 64;

thread_local char g_rope_error[512] = "";

}  // namespace

struct plt_rope : HandleBase {
    plt_rope_config cfg;
    int32_t delta[kMaxLoops];
    int rd, Qn;
    uint64_t* turns = nullptr;        // [rd / 2] fractions of a turn per position, in units of 2^-64
};

namespace {

struct RopeParams {
    const void *q, *k, *k_loc, *v;
    void *q_out, *k_out, *k_loc_out;  // k_out, k_loc_out: prompts only
    void *k_cache, *v_cache, *k_win, *v_win;
    int64_t q_stride, k_stride, v_stride;
    int64_t kv_stride_b, kv_stride_n, kv_stride_h;
    const float *q_gain, *k_gain, *k_scale, *v_scale, *w_gate, *b_gate;
    float* gate_out;
    const int32_t *seq_lens, *start, *prefix_lens, *page_table;
    const uint64_t* turns;
    uint32_t* status;
    int32_t B, L, Qn, Hq, Hkv, T, w, max_seq_len, page_size, max_pages, num_pool_pages, rd, interleaved;
    float factor, eps;
    int32_t delta[kMaxLoops];
};

// 16 elements of a row as fp32: two pieces of 8.
template <typename T>
__device__ __forceinline__ void load8(const T* src, float* x) {
    if constexpr (sizeof(T) == 2) {
        const uint4 v = *(const uint4*)src;
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
        const float4 a = *(const float4*)src, b = *((const float4*)src + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
}
__device__ __forceinline__ void store8(__nv_bfloat16* dst, const float* x) {
    *(uint4*)dst = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ void store8(float* dst, const float* x) {
    *(float4*)dst = make_float4(x[0], x[1], x[2], x[3]);
    *((float4*)dst + 1) = make_float4(x[4], x[5], x[6], x[7]);
}
// E4M3 codes of x / scale: fp32 division, nearest even, clamped to the largest finite magnitude.
__device__ __forceinline__ void store8_codes(uint8_t* dst, const float* x, float scale) {
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        unsigned short r;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(__fdiv_rn(x[2 * i + 1], scale)), "f"(__fdiv_rn(x[2 * i], scale)));
        c[i] = r;
    }
    *(uint2*)dst = make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}

// What a block knows about each of its tokens.
struct Token {
    int64_t cell;     // element where head 0 of its row starts in the cache (or window), or -1: not stored
    int64_t pos;      // its position, or -1: the row has no token
};

// Where position `slot` of sequence b lies in the shared cache, or -1.
__device__ __forceinline__ int64_t cache_cell(const RopeParams& p, int b, int64_t slot, uint32_t& flags) {
    if (p.page_size == 0) return (int64_t)b * p.kv_stride_b + slot * p.kv_stride_n;
    const int page = p.page_table[(int64_t)b * p.max_pages + slot / p.page_size];
    if (page < 0 || page >= p.num_pool_pages) {
        flags |= kDevPageIdClamped;
        return -1;
    }
    return (int64_t)page * p.kv_stride_b + (slot % p.page_size) * p.kv_stride_n;
}

// This thread's 16 elements of a row: the two pieces' offsets, and which of the pairs turn.
template <int D>
struct Lane {
    int t, o0, o1;
    bool turning, interleaved;
    __device__ __forceinline__ Lane(const RopeParams& p) {
        t = threadIdx.x % (D / 16);
        turning = t < p.rd / 16;
        interleaved = p.interleaved != 0;
        const bool halves = turning && !interleaved;
        o0 = (halves ? t : 2 * t) * 8;
        o1 = (halves ? t + p.rd / 16 : 2 * t + 1) * 8;
    }
};

// Norm (gain: the row's factors) and rotation (cs: the token's cosines and sines) of a row, in place.
template <int D>
__device__ __forceinline__ void norm_and_turn(float (&x)[16], const Lane<D>& ln, bool norm, const float* gain, float eps,
                                              const float2* cs) {
    if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
        for (int o = D / 32; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float inv = 1.f / sqrtf(ss * (1.f / D) + eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 g = *((const float4*)gain + i * (D / 16) + ln.t);
            x[4 * i] *= inv * g.x;
            x[4 * i + 1] *= inv * g.y;
            x[4 * i + 2] *= inv * g.z;
            x[4 * i + 3] *= inv * g.w;
        }
    }
    if (ln.turning) {
        float4 t4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t4[i] = *((const float4*)cs + i * (D / 16) + ln.t);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float c = (i & 1) ? t4[i / 2].z : t4[i / 2].x, s = (i & 1) ? t4[i / 2].w : t4[i / 2].y;
            if (ln.interleaved) {
                const float a = x[2 * i], b = x[2 * i + 1];
                x[2 * i] = fmaf(a, c, -(b * s));
                x[2 * i + 1] = fmaf(b, c, a * s);
            } else {
                const float a = x[i], b = x[i + 8];
                x[i] = fmaf(a, c, -(b * s));
                x[i + 8] = fmaf(b, c, a * s);
            }
        }
    }
}

// SEQ: rows of a prompt (TB of one loop of a sequence to a block), else one token of a step to a block.
template <typename T, bool FP8, int D, bool SEQ>
__global__ void __launch_bounds__(kRopeThreads, SEQ ? 4 : 2) plt_rope_kernel(const __grid_constant__ RopeParams p) {
    constexpr int TB = SEQ ? kSeqTokens : 1;
    constexpr int TPR = D / 16, RPB = kRopeThreads / TPR;      // threads of a row, rows of a pass
    using TD = typename std::conditional<FP8, uint8_t, T>::type;
    __shared__ Token s_tok[TB];
    __shared__ __align__(16) float2 s_cs[TB][kMaxPairs];
    __shared__ __align__(16) float s_gain[2][D];
    if (!SEQ) grid_launch_dependents();   // the attention's blocks may be set up meanwhile; they wait for this grid

    const int tid = threadIdx.x;
    int b, l, t0;                       // t0: first row of the prompt, or the token of the step
    if (SEQ) {
        b = blockIdx.y / p.L;
        l = blockIdx.y % p.L;
        t0 = blockIdx.x * TB;
    } else {
        t0 = blockIdx.x % p.Qn;
        l = (blockIdx.x / p.Qn) % p.L;
        b = blockIdx.x / (p.Qn * p.L);
    }
    uint32_t flags = 0;
    int n = p.seq_lens[b];
    int64_t before = p.prefix_lens != nullptr ? p.prefix_lens[b] : 0;
    if (before < 0) {
        flags |= kDevGroupClamped;
        before = 0;
    }
    if (SEQ) {
        if (n < 0 || n > p.T) {
            flags |= kDevSeqLenClamped;
            n = n < 0 ? 0 : p.T;
        }
    } else if (n < 0 || n > before + p.max_seq_len) {
        flags |= kDevSeqLenClamped;
        n = n < 0 ? 0 : (int)min(before + p.max_seq_len, (int64_t)0x7fffffff);
    }
    int64_t start = 0;
    if (SEQ && p.start != nullptr) {
        start = p.start[b];
        if (start < 0) {
            flags |= kDevGroupClamped;
            start = 0;
        }
    }
    if (SEQ && t0 >= n) {
        if (flags && tid == 0) atomicOr(p.status, flags);
        return;
    }
    if (tid < 2 * D) {
        const float* gain = tid < D ? p.q_gain : p.k_gain;
        // element e of a thread's 16 (pieces at o0 and o1): [e / 4][thread][e % 4]
        const int i = tid % D, e = i / (TPR * 4) * 4 + i % 4, owner = i / 4 % TPR;
        const bool halves = owner < p.rd / 16 && !p.interleaved;
        const int o = e < 8 ? (halves ? owner : 2 * owner) * 8 + e : (halves ? owner + p.rd / 16 : 2 * owner + 1) * 8 + e - 8;
        s_gain[tid / D][i] = gain != nullptr ? gain[o] : 1.f;
    }
    if (tid < TB) {
        Token tk;
        tk.cell = -1;
        if (SEQ) {
            const int t = t0 + tid;
            tk.pos = t < n ? start + t - p.delta[l] : -1;
            if (l == 0 && t < n && p.k_cache != nullptr) {
                const int64_t slot = start + t - before;
                if (slot >= p.max_seq_len) flags |= kDevSeqLenClamped;
                else if (slot >= 0) tk.cell = cache_cell(p, b, slot, flags);
            }
        } else {
            tk.pos = (int64_t)n - p.delta[l] - 1 - (p.Qn - 1 - t0);
            if (tk.pos >= 0) {
                if (l == 0) {
                    if (tk.pos >= before) tk.cell = cache_cell(p, b, tk.pos - before, flags);
                } else {
                    tk.cell = (((int64_t)b * (p.L - 1) + (l - 1)) * p.w + tk.pos % p.w) * p.Hkv * D;
                }
            }
        }
        if (tk.pos < 0) tk.pos = -1;
        s_tok[tid] = tk;
    }
    if (flags) atomicOr(p.status, flags);
    __syncthreads();

    // cosines and sines of the block's tokens
    const int pairs = p.rd / 2;
    for (int i = tid; i < TB * pairs; i += kRopeThreads) {
        const int tk = i / pairs, f = i - tk * pairs;
        const uint64_t turn = (uint64_t)s_tok[tk].pos * p.turns[f];      // whole turns fall off the top
        const int32_t x = (int32_t)((turn + (1ull << 31)) >> 32);        // 2^-32 turns, nearest
        const int32_t quarter = (int32_t)((uint32_t)x + (1u << 29)) >> 30;
        float s, c;
        sincospif((float)(int32_t)((uint32_t)x - ((uint32_t)quarter << 30)) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns
        const float cc = (quarter & 1) ? -s : c, ss = (quarter & 1) ? c : s;
        // pair k of a thread's 8: [k / 2][thread][k % 2], so that neighbouring threads read neighbouring words
        float2* const to = &s_cs[tk][((f % 8) / 2 * TPR + f / 8) * 2 + f % 2];
        *to = (quarter & 2) ? make_float2(-cc * p.factor, -ss * p.factor) : make_float2(cc * p.factor, ss * p.factor);
    }
    __syncthreads();

    const Lane<D> ln(p);
    const int r_in = tid / TPR;

    // ---- queries -----------------------------------------------------------------------------------------------
    const bool qnorm = p.q_gain != nullptr;
    {
        constexpr int U = sizeof(T) == 2 ? 2 : 1;      // rows whose loads are in flight together
        const int rows = TB * p.Hq;
        for (int r0 = 0; r0 < rows; r0 += RPB * U) {
            float x[U][16];
            int64_t at[U];
            bool live[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = r0 + u * RPB + r_in;
                const int tk = SEQ ? r / p.Hq : 0, h = r - tk * p.Hq;
                live[u] = r < rows && s_tok[r < rows ? tk : 0].pos >= 0;
                at[u] = -1;
                if (SEQ) {
                    at[u] = ((((int64_t)b * p.L + l) * p.T + t0 + tk) * p.Hq + h) * D;
                    if (live[u]) {
                        load8((const T*)p.q + at[u] + ln.o0, x[u]);
                        load8((const T*)p.q + at[u] + ln.o1, x[u] + 8);
                    }
                } else {
                    if (r < rows) at[u] = ((int64_t)blockIdx.x * p.Hq + h) * D;
                    if (live[u]) {
                        const T* src = (const T*)p.q + (int64_t)blockIdx.x * p.q_stride + (int64_t)h * D;
                        load8(src + ln.o0, x[u]);
                        load8(src + ln.o1, x[u] + 8);
                    }
                }
                if (!live[u])
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[u][i] = 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = r0 + u * RPB + r_in;
                const int tk = SEQ ? min(r / p.Hq, TB - 1) : 0;
                norm_and_turn<D>(x[u], ln, qnorm, s_gain[0], p.eps, s_cs[tk]);
                if (SEQ ? live[u] : at[u] >= 0) {
                    if (!live[u])
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[u][i] = 0.f;
                    store8((T*)p.q_out + at[u] + ln.o0, x[u]);
                    store8((T*)p.q_out + at[u] + ln.o1, x[u] + 8);
                }
                if (!SEQ && l > 0 && p.gate_out != nullptr) {
                    float dot = 0.f;
                    if (live[u]) {
                        const float* w = p.w_gate + (int64_t)r * D;
#pragma unroll
                        for (int i = 0; i < 16; ++i) dot = fmaf(w[i < 8 ? ln.o0 + i : ln.o1 + i - 8], x[u][i], dot);
                    }
#pragma unroll
                    for (int o = TPR / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
                    if (ln.t == 0 && r < rows) p.gate_out[((int64_t)b * (p.L - 1) + (l - 1)) * p.Hq + r] = dot + p.b_gate[r];
                }
            }
        }
    }

    // ---- keys, then values ---------------------------------------------------------------------------------------
    const bool knorm = p.k_gain != nullptr;
    const int rows = TB * p.Hkv;
    const int64_t head_stride = !SEQ && l > 0 ? D : p.kv_stride_h;
    TD* const k_to = (TD*)(!SEQ && l > 0 ? p.k_win : p.k_cache);
    TD* const v_to = (TD*)(!SEQ && l > 0 ? p.v_win : p.v_cache);
    const bool values = SEQ ? l == 0 && p.v_cache != nullptr : true;
    for (int r0 = 0; r0 < rows; r0 += RPB) {
        const int r = r0 + r_in;
        const int tk = SEQ ? min(r / p.Hkv, TB - 1) : 0, h = r - tk * p.Hkv;
        const Token tok = s_tok[tk];
        const bool live = r < rows && tok.pos >= 0, cached = live && tok.cell >= 0;
        float x[16], y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = y[i] = 0.f;
        int64_t at = 0;
        const T *ksrc, *vsrc;
        if (SEQ) {
            at = l == 0 ? (((int64_t)b * p.T + t0 + tk) * p.Hkv + h) * D
                        : ((((int64_t)b * (p.L - 1) + (l - 1)) * p.T + t0 + tk) * p.Hkv + h) * D;
            ksrc = (const T*)(l == 0 ? p.k : p.k_loc) + at;
            vsrc = (const T*)p.v + at;
        } else {
            ksrc = (const T*)p.k + (int64_t)blockIdx.x * p.k_stride + (int64_t)h * D;
            vsrc = (const T*)p.v + (int64_t)blockIdx.x * p.v_stride + (int64_t)h * D;
        }
        if (SEQ ? live : cached) {
            load8(ksrc + ln.o0, x);
            load8(ksrc + ln.o1, x + 8);
        }
        if (values && cached) {
            load8(vsrc + ln.o0, y);
            load8(vsrc + ln.o1, y + 8);
        }
        norm_and_turn<D>(x, ln, knorm, s_gain[1], p.eps, s_cs[tk]);
        if (SEQ && live) {
            T* const out = (T*)(l == 0 ? p.k_out : p.k_loc_out);
            if (out != nullptr) {
                store8(out + at + ln.o0, x);
                store8(out + at + ln.o1, x + 8);
            }
        }
        if (cached && (!SEQ || l == 0)) {
            TD* const kd = k_to + tok.cell + (int64_t)h * head_stride;
            TD* const vd = v_to + tok.cell + (int64_t)h * head_stride;
            if constexpr (FP8) {
                const float ks = p.k_scale[h], vs = p.v_scale[h];
                store8_codes(kd + ln.o0, x, ks);
                store8_codes(kd + ln.o1, x + 8, ks);
                store8_codes(vd + ln.o0, y, vs);
                store8_codes(vd + ln.o1, y + 8, vs);
            } else {
                store8(kd + ln.o0, x);
                store8(kd + ln.o1, x + 8);
                store8(vd + ln.o0, y);
                store8(vd + ln.o1, y + 8);
            }
        }
    }
}

plt_status rope_fail(plt_rope_t h, plt_status code, const char* what) { return handle_fail(h, g_rope_error, code, "%s", what); }

plt_status check_config(const plt_rope_config* c, int* rd) {
    if (!c) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "config is NULL");
    if (c->struct_size != sizeof(plt_rope_config))
        return handle_fail(nullptr, g_rope_error, PLT_ERR_INVALID_ARG, "config.struct_size %u != %zu", c->struct_size, sizeof *c);
    if (c->dtype != PLT_F32 && c->dtype != PLT_BF16) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "unknown dtype");
    if (c->kv_dtype != PLT_KV_SAME && c->kv_dtype != PLT_KV_E4M3) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "unknown kv_dtype");
    if (c->max_batch < 1 || c->L < 1 || c->Hq < 1 || c->Hkv < 1 || c->max_seq_len < 1 || c->w < 0 || c->page_size < 0 || c->q_len < 0)
        return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "non-positive size in config");
    if (c->max_batch > kMaxBatch) return rope_fail(nullptr, PLT_ERR_UNSUPPORTED, "max_batch above 4096");
    if (c->L > kMaxLoops) return rope_fail(nullptr, PLT_ERR_UNSUPPORTED, "L above 8");
    if (c->Hq % c->Hkv != 0) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "Hq is not a multiple of Hkv");
    if (c->Hq > 1024) return rope_fail(nullptr, PLT_ERR_UNSUPPORTED, "Hq above 1024");
    if (c->d != 64 && c->d != 128) return rope_fail(nullptr, PLT_ERR_UNSUPPORTED, "head dim (supported: 64, 128)");
    if (c->kv_dtype == PLT_KV_E4M3 && (c->dtype != PLT_BF16 || c->d != 128))
        return rope_fail(nullptr, PLT_ERR_UNSUPPORTED, "E4M3 caches need bf16 rows and head dim 128");
    if (c->L > 1 && c->w < 1) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "w must be >= 1 when L > 1");
    if (c->page_size % 16 != 0) return rope_fail(nullptr, PLT_ERR_UNSUPPORTED, "page_size is not a multiple of 16");
    if (c->q_len > 64 || (c->q_len > 1 && c->L > 1))
        return rope_fail(nullptr, PLT_ERR_UNSUPPORTED, "q_len above 64, or above 1 with several loops");
    if (c->loop_offset)
        for (int l = 0; l < c->L; ++l)
            if (c->loop_offset[l] < 0) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "loop_offset below 0");
    *rd = c->rotary_dim != 0 ? c->rotary_dim : c->d;
    if (*rd < 0 || *rd > c->d) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "rotary_dim outside [0, d]");
    if (*rd % 16 != 0) return rope_fail(nullptr, PLT_ERR_UNSUPPORTED, "rotary_dim is not a multiple of 16");
    if (c->layout != PLT_ROPE_HALF && c->layout != PLT_ROPE_INTERLEAVED) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "unknown layout");
    if (c->scaling < PLT_ROPE_PLAIN || c->scaling > PLT_ROPE_RAMP) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "unknown scaling");
    if (!(c->norm_eps > 0.f) || !std::isfinite(c->norm_eps)) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "norm_eps must be positive and finite");
    if (!std::isfinite(c->attn_factor)) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "attn_factor is not finite");
    if (c->inv_freq) {
        for (int i = 0; i < *rd / 2; ++i)
            if (!std::isfinite(c->inv_freq[i])) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "inv_freq is not finite");
        return PLT_OK;
    }
    if (!(c->theta > 1.0) || !std::isfinite(c->theta)) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "theta must be above 1 and finite");
    if (c->scaling != PLT_ROPE_PLAIN && (!(c->factor > 0.0) || !std::isfinite(c->factor)))
        return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "factor must be positive and finite");
    if (c->scaling >= PLT_ROPE_WAVELENGTH) {
        if (!(c->low > 0.0) || !(c->high > c->low) || !std::isfinite(c->high))
            return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "0 < low < high is needed");
        if (c->original_len < 1) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "original_len must be >= 1");
    }
    return PLT_OK;
}

double clamp01(double x) { return x < 0.0 ? 0.0 : x > 1.0 ? 1.0 : x; }

constexpr double kTwoPi = 6.283185307179586476925286766559;

void frequencies(const plt_rope_config* c, int rd, double* f) {
    if (c->inv_freq) {
        for (int i = 0; i < rd / 2; ++i) f[i] = c->inv_freq[i];
        return;
    }
    const double theta = c->scaling == PLT_ROPE_BASE ? c->theta * pow(c->factor, (double)rd / (rd - 2)) : c->theta;
    double first = 0.0, last = 0.0;
    if (c->scaling == PLT_ROPE_RAMP) {
        auto pair = [&](double t) { return rd * log(c->original_len / (t * kTwoPi)) / (2.0 * log(c->theta)); };
        first = fmax(floor(pair(c->high)), 0.0);
        last = fmin(ceil(pair(c->low)), (double)(rd - 1));
    }
    for (int i = 0; i < rd / 2; ++i) {
        const double g = pow(theta, -2.0 * i / rd);
        f[i] = g;
        if (c->scaling == PLT_ROPE_LINEAR) f[i] = g / c->factor;
        if (c->scaling == PLT_ROPE_WAVELENGTH) {
            const double s = clamp01((c->original_len * g / kTwoPi - c->low) / (c->high - c->low));
            f[i] = s * g + (1.0 - s) * g / c->factor;
        }
        if (c->scaling == PLT_ROPE_RAMP) {
            const double s = clamp01((i - first) / fmax(last - first, 0.001));
            f[i] = (1.0 - s) * g + s * g / c->factor;
        }
    }
}

// f radians a position as a fraction of a turn in units of 2^-64, nearest.
uint64_t turns_of(double f) {
    const long double turns = (long double)f / 6.283185307179586476925286766559005768L;
    const long double frac = turns - floorl(turns);                       // [0, 1]
    const long double x = rintl(frac * 18446744073709551616.0L);
    return x >= 18446744073709551616.0L ? 0 : (uint64_t)x;
}

// Strides of the shared cache; null, or what is wrong with them.
const char* cache_strides(const plt_rope_config& c, int64_t sb, int64_t sn, int64_t sh, RopeParams* p) {
    if (sb == 0 && sn == 0 && sh == 0) {
        sh = c.d;
        sn = (int64_t)c.Hkv * c.d;
        sb = (int64_t)(c.page_size > 0 ? c.page_size : c.max_seq_len) * sn;
    }
    const int64_t unit = c.kv_dtype == PLT_KV_E4M3 ? 16 : c.dtype == PLT_BF16 ? 8 : 4;
    if (sb <= 0 || sn <= 0 || sh <= 0 || sb % unit || sn % unit || sh % unit) return "kv strides must be positive multiples of 16 bytes";
    if (sh < c.d) return "kv_stride_h < d";
    if ((double)sb >= 1099511627776.0 || (double)sn >= 1099511627776.0 || (double)sh >= 1099511627776.0) return "kv stride of 2^40 elements or more";
    p->kv_stride_b = sb; p->kv_stride_n = sn; p->kv_stride_h = sh;
    return nullptr;
}

plt_status common(plt_rope_t h, int32_t batch, const int32_t* page_table, int32_t max_pages, int32_t num_pool_pages, bool cache,
                  const float* k_scale, const float* v_scale, RopeParams* p) {
    const plt_rope_config& c = h->cfg;
    if (cache && c.page_size > 0) {
        if (!page_table) return rope_fail(h, PLT_ERR_INVALID_ARG, "page_table is NULL for a paged cache");
        const int need = (c.max_seq_len + c.page_size - 1) / c.page_size;
        if (max_pages < need) return handle_fail(h, g_rope_error, PLT_ERR_CAPACITY, "max_pages %d < %d", max_pages, need);
        if (num_pool_pages < 1) return rope_fail(h, PLT_ERR_INVALID_ARG, "num_pool_pages < 1");
    }
    if (cache && c.kv_dtype == PLT_KV_E4M3 && (!k_scale || !v_scale))
        return rope_fail(h, PLT_ERR_INVALID_ARG, "k_scale and v_scale must not be NULL with E4M3 caches");
    p->page_table = page_table; p->max_pages = max_pages; p->num_pool_pages = num_pool_pages; p->page_size = c.page_size;
    p->k_scale = k_scale; p->v_scale = v_scale;
    p->turns = h->turns; p->status = h->status;
    p->B = batch; p->L = c.L; p->Qn = h->Qn; p->Hq = c.Hq; p->Hkv = c.Hkv; p->w = c.w; p->max_seq_len = c.max_seq_len;
    p->rd = h->rd; p->interleaved = c.layout == PLT_ROPE_INTERLEAVED;
    p->factor = c.attn_factor != 0.f ? c.attn_factor : 1.f;
    p->eps = c.norm_eps;
    for (int l = 0; l < kMaxLoops; ++l) p->delta[l] = h->delta[l];
    return PLT_OK;
}

template <bool SEQ>
plt_status launch(plt_rope_t h, const RopeParams& p, dim3 grid, cudaStream_t stream) {
    DeviceScope scope(h->device);
    if (scope.err != cudaSuccess) return handle_fail(h, g_rope_error, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    const plt_rope_config& c = h->cfg;
    if (c.kv_dtype == PLT_KV_E4M3) plt_rope_kernel<__nv_bfloat16, true, 128, SEQ><<<grid, kRopeThreads, 0, stream>>>(p);
    else if (c.dtype == PLT_BF16 && c.d == 128) plt_rope_kernel<__nv_bfloat16, false, 128, SEQ><<<grid, kRopeThreads, 0, stream>>>(p);
    else if (c.dtype == PLT_BF16) plt_rope_kernel<__nv_bfloat16, false, 64, SEQ><<<grid, kRopeThreads, 0, stream>>>(p);
    else if (c.d == 128) plt_rope_kernel<float, false, 128, SEQ><<<grid, kRopeThreads, 0, stream>>>(p);
    else plt_rope_kernel<float, false, 64, SEQ><<<grid, kRopeThreads, 0, stream>>>(p);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return handle_fail(h, g_rope_error, PLT_ERR_CUDA, "launching the kernel: %s", cudaGetErrorString(e));
    return PLT_OK;
}

}  // namespace

#define PLT_API __attribute__((visibility("default")))
extern "C" {

PLT_API plt_status plt_rope_frequencies(const plt_rope_config* config, double* out_freq) {
    int rd = 0;
    const plt_status s = check_config(config, &rd);
    if (s != PLT_OK) return s;
    if (!out_freq) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "out_freq is NULL");
    frequencies(config, rd, out_freq);
    return PLT_OK;
}

PLT_API plt_status plt_rope_create(const plt_rope_config* config, plt_rope_t* out_handle) {
    if (!out_handle) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "out_handle is NULL");
    *out_handle = nullptr;
    int rd = 0;
    plt_status s = check_config(config, &rd);
    if (s != PLT_OK) return s;
    double freq[kMaxPairs];
    frequencies(config, rd, freq);
    uint64_t turns[kMaxPairs] = {};
    for (int i = 0; i < rd / 2; ++i) {
        if (!std::isfinite(freq[i])) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "theta and factor give frequencies that are not finite");
        turns[i] = turns_of(freq[i]);
    }
    DeviceScope scope(config->device);
    if (scope.err != cudaSuccess) {
        (void)cudaGetLastError();
        return handle_fail(nullptr, g_rope_error, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    }
    s = check_device(config->device, g_rope_error, nullptr);
    if (s != PLT_OK) return s;
    plt_rope* h = new (std::nothrow) plt_rope();
    if (!h) return rope_fail(nullptr, PLT_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->cfg = *config;
    h->cfg.loop_offset = nullptr;
    h->cfg.inv_freq = nullptr;
    h->device = config->device;
    h->rd = rd;
    h->Qn = config->q_len > 1 ? config->q_len : 1;
    for (int l = 0; l < kMaxLoops; ++l) h->delta[l] = config->loop_offset && l < config->L ? config->loop_offset[l] : l;
    void* ws = nullptr;
    if (cudaMalloc(&ws, 256 + sizeof turns) != cudaSuccess) {
        (void)cudaGetLastError();
        delete h;
        return rope_fail(nullptr, PLT_ERR_OUT_OF_MEMORY, "cudaMalloc of the frequencies failed");
    }
    h->status = (uint32_t*)ws;
    h->turns = (uint64_t*)((char*)ws + 256);
    cudaError_t e = cudaMemset(ws, 0, 256);
    if (e == cudaSuccess) e = cudaMemcpy(h->turns, turns, sizeof turns, cudaMemcpyHostToDevice);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();   // another stream may run first
    if (e != cudaSuccess) {
        cudaFree(ws);
        delete h;
        return handle_fail(nullptr, g_rope_error, PLT_ERR_CUDA, "copying the frequencies: %s", cudaGetErrorString(e));
    }
    *out_handle = h;
    return PLT_OK;
}

PLT_API plt_status plt_rope_step(plt_rope_t h, const plt_rope_step_args* a, void* cuda_stream) {
    if (!h) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    if (!a) return rope_fail(h, PLT_ERR_INVALID_ARG, "args is NULL");
    if (a->struct_size != sizeof(plt_rope_step_args))
        return handle_fail(h, g_rope_error, PLT_ERR_INVALID_ARG, "args.struct_size %u != %zu", a->struct_size, sizeof *a);
    const plt_rope_config& c = h->cfg;
    if (a->batch < 0) return rope_fail(h, PLT_ERR_INVALID_ARG, "batch < 0");
    if (a->batch > c.max_batch) return handle_fail(h, g_rope_error, PLT_ERR_CAPACITY, "batch %d > max_batch %d", a->batch, c.max_batch);
    if (a->batch == 0) return PLT_OK;
    if (!a->q || !a->k_new || !a->v_new || !a->q_out || !a->k_cache || !a->v_cache || !a->seq_lens)
        return rope_fail(h, PLT_ERR_INVALID_ARG, "q, k_new, v_new, q_out, k_cache, v_cache and seq_lens must not be NULL");
    if (c.L > 1 && (!a->k_win || !a->v_win)) return rope_fail(h, PLT_ERR_INVALID_ARG, "k_win and v_win must not be NULL when L > 1");
    if ((a->w_gate == nullptr) != (a->gate_logits == nullptr) || (a->w_gate == nullptr) != (a->b_gate == nullptr))
        return rope_fail(h, PLT_ERR_INVALID_ARG, "w_gate, b_gate and gate_logits go together");
    if (misaligned(a->q, 16) || misaligned(a->k_new, 16) || misaligned(a->v_new, 16) || misaligned(a->q_out, 16) || misaligned(a->k_cache, 16) ||
        misaligned(a->v_cache, 16) || misaligned(a->k_win, 16) || misaligned(a->v_win, 16) || misaligned(a->w_gate, 16))
        return rope_fail(h, PLT_ERR_INVALID_ARG, "tensor base pointers must be 16-byte aligned");
    const uintptr_t words = (uintptr_t)a->q_gain | (uintptr_t)a->k_gain | (uintptr_t)a->seq_lens | (uintptr_t)a->prefix_lens | (uintptr_t)a->page_table |
                            (uintptr_t)a->k_scale | (uintptr_t)a->v_scale | (uintptr_t)a->b_gate | (uintptr_t)a->gate_logits;
    if (words & 3u) return rope_fail(h, PLT_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    RopeParams p;
    memset(&p, 0, sizeof p);
    const int64_t unit = c.dtype == PLT_BF16 ? 8 : 4, qw = (int64_t)c.Hq * c.d, kw = (int64_t)c.Hkv * c.d;
    p.q_stride = a->q_stride != 0 ? a->q_stride : qw;
    p.k_stride = a->k_stride != 0 ? a->k_stride : kw;
    p.v_stride = a->v_stride != 0 ? a->v_stride : kw;
    const int64_t rows_total = (int64_t)a->batch * c.L * h->Qn;
    if (p.q_stride % unit || p.k_stride % unit || p.v_stride % unit || p.q_stride < qw || p.k_stride < kw || p.v_stride < kw ||
        p.q_stride > ((int64_t)1 << 40) || p.k_stride > ((int64_t)1 << 40) || p.v_stride > ((int64_t)1 << 40))
        return rope_fail(h, PLT_ERR_INVALID_ARG, "row strides must be multiples of 16 bytes, at least a row and at most 2^40 elements");
    if (a->q_out == a->q && p.q_stride != qw && rows_total > 1)
        return rope_fail(h, PLT_ERR_INVALID_ARG, "q_out may be q only where q is dense");
    if (const char* bad = cache_strides(c, a->kv_stride_b, a->kv_stride_n, a->kv_stride_h, &p)) return rope_fail(h, PLT_ERR_INVALID_ARG, bad);
    const plt_status s = common(h, a->batch, a->page_table, a->max_pages, a->num_pool_pages, true, a->k_scale, a->v_scale, &p);
    if (s != PLT_OK) return s;
    p.q = a->q; p.k = a->k_new; p.v = a->v_new; p.q_out = a->q_out;
    p.k_cache = a->k_cache; p.v_cache = a->v_cache; p.k_win = a->k_win; p.v_win = a->v_win;
    p.q_gain = a->q_gain; p.k_gain = a->k_gain;
    p.w_gate = a->w_gate; p.b_gate = a->b_gate; p.gate_out = c.L > 1 ? a->gate_logits : nullptr;
    p.seq_lens = a->seq_lens; p.prefix_lens = a->prefix_lens;
    return launch<false>(h, p, dim3((unsigned)rows_total), (cudaStream_t)cuda_stream);
}

PLT_API plt_status plt_rope_seq(plt_rope_t h, const plt_rope_seq_args* a, void* cuda_stream) {
    if (!h) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    if (!a) return rope_fail(h, PLT_ERR_INVALID_ARG, "args is NULL");
    if (a->struct_size != sizeof(plt_rope_seq_args))
        return handle_fail(h, g_rope_error, PLT_ERR_INVALID_ARG, "args.struct_size %u != %zu", a->struct_size, sizeof *a);
    const plt_rope_config& c = h->cfg;
    if (a->batch < 0) return rope_fail(h, PLT_ERR_INVALID_ARG, "batch < 0");
    if (a->rows < 1) return rope_fail(h, PLT_ERR_INVALID_ARG, "rows < 1");
    if (a->batch > c.max_batch) return handle_fail(h, g_rope_error, PLT_ERR_CAPACITY, "batch %d > max_batch %d", a->batch, c.max_batch);
    if (h->delta[0] != 0) return rope_fail(h, PLT_ERR_UNSUPPORTED, "plt_rope_seq needs loop_offset[0] = 0");
    if (a->batch == 0) return PLT_OK;
    if (!a->q || !a->k_share || !a->q_out || !a->seq_lens) return rope_fail(h, PLT_ERR_INVALID_ARG, "q, k_share, q_out and seq_lens must not be NULL");
    if ((a->k_cache == nullptr) != (a->v_cache == nullptr)) return rope_fail(h, PLT_ERR_INVALID_ARG, "k_cache and v_cache go together");
    if (!a->k_cache && !a->k_share_out) return rope_fail(h, PLT_ERR_INVALID_ARG, "k_share_out or k_cache is needed");
    if (a->k_cache && !a->v_share) return rope_fail(h, PLT_ERR_INVALID_ARG, "v_share is NULL");
    if (c.L > 1 && (!a->k_loc || !a->k_loc_out)) return rope_fail(h, PLT_ERR_INVALID_ARG, "k_loc and k_loc_out must not be NULL when L > 1");
    if (misaligned(a->q, 16) || misaligned(a->k_share, 16) || misaligned(a->v_share, 16) || misaligned(a->k_loc, 16) || misaligned(a->q_out, 16) ||
        misaligned(a->k_share_out, 16) || misaligned(a->k_loc_out, 16) || misaligned(a->k_cache, 16) || misaligned(a->v_cache, 16))
        return rope_fail(h, PLT_ERR_INVALID_ARG, "tensor base pointers must be 16-byte aligned");
    const uintptr_t words = (uintptr_t)a->q_gain | (uintptr_t)a->k_gain | (uintptr_t)a->seq_lens | (uintptr_t)a->start | (uintptr_t)a->prefix_lens |
                            (uintptr_t)a->page_table | (uintptr_t)a->k_scale | (uintptr_t)a->v_scale;
    if (words & 3u) return rope_fail(h, PLT_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    RopeParams p;
    memset(&p, 0, sizeof p);
    if (a->k_cache)
        if (const char* bad = cache_strides(c, a->kv_stride_b, a->kv_stride_n, a->kv_stride_h, &p)) return rope_fail(h, PLT_ERR_INVALID_ARG, bad);
    const plt_status s = common(h, a->batch, a->page_table, a->max_pages, a->num_pool_pages, a->k_cache != nullptr, a->k_scale, a->v_scale, &p);
    if (s != PLT_OK) return s;
    p.q = a->q; p.k = a->k_share; p.v = a->v_share; p.k_loc = a->k_loc;
    p.q_out = a->q_out; p.k_out = a->k_share_out; p.k_loc_out = a->k_loc_out;
    p.k_cache = a->k_cache; p.v_cache = a->v_cache;
    p.q_gain = a->q_gain; p.k_gain = a->k_gain;
    p.seq_lens = a->seq_lens; p.start = a->start; p.prefix_lens = a->prefix_lens;
    p.T = a->rows;
    const dim3 grid((unsigned)((a->rows + kSeqTokens - 1) / kSeqTokens), (unsigned)(a->batch * c.L));
    return launch<true>(h, p, grid, (cudaStream_t)cuda_stream);
}

PLT_API plt_status plt_rope_check(plt_rope_t h, void* cuda_stream, uint32_t* out_bits) {
    if (!h) return rope_fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    return handle_check(h, g_rope_error, (cudaStream_t)cuda_stream, out_bits);
}

PLT_API plt_status plt_rope_destroy(plt_rope_t h) {
    if (!h) return PLT_OK;
    DeviceScope scope(h->device);
    cudaFree(h->status);
    delete h;
    return PLT_OK;
}

PLT_API const char* plt_rope_last_error(plt_rope_t h) { return h ? h->err : g_rope_error; }

}  // extern "C"

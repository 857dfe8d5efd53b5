// Norm and rotation of queries and keys, with their way into the caches: a decode step and the rows of a prompt.
//
// d / 16 threads hold a head's row, 16 elements each: the 8 pairs (a, b) that turn together, a from one 16-byte piece and b from
// another (halves) or both from the same two (interleaved), so a row is read once, normed by a shuffle over its threads, turned in
// registers (two pairs to an instruction) and written once. The cosines and sines of a token are computed once for all its heads.
//
// An angle p f is taken in turns: f / 2 pi as a 64-bit fraction, multiplied by the position in integers, so that whole turns
// fall away exactly however far the position lies; the quarter turn is split off in integers too, and what is left (at most
// an eighth of a turn either way) goes to sincospif.
//
// Prompts are bound by reading and writing the rows, with the instructions close behind: two of 8192 rows in two loops (32 and 8 heads
// of 128, normed, into a cache in pages) take 114.7 us for 738 MB, 6.4 TB/s; five short ragged ones in fp32 8.2 us, a start and a
// short row of blocks. A step is bound by latency: its rows are asked for before the lengths, the page and the cosines are known; one
// sequence takes 3.4 us, 256 of two loops with 8-bit caches 6.8.
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
constexpr int kMaxPairs = 64;

thread_local char g_rope_error[512] = "";

}  // namespace

struct plt_rope : HandleBase {
    plt_rope_config cfg;
    int32_t delta[kMaxLoops];
    int rd, Qn;
    int sms = 0;
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
    int32_t B, L, Qn, Hq, Hkv, T, w, max_seq_len, page_size, max_pages, num_pool_pages, rd;
    uint32_t q_reciprocal, k_reciprocal;   // ceil(2^32 / heads), or 0 for one head
    float factor, eps;
    int32_t delta[kMaxLoops];
};

// ---- a thread's 16 elements of a row ------------------------------------------------------------------------------------
// As loaded: two pieces of 8 elements.
template <typename T>
struct Raw {
    uint4 v[sizeof(T)];       // sizeof(T) = 2: one 16-byte vector for each piece; 4: two
};
template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T* row, int o0, int o1) {
    Raw<T> x;
    if constexpr (sizeof(T) == 2) {
        x.v[0] = *(const uint4*)(row + o0);
        x.v[1] = *(const uint4*)(row + o1);
    } else {
        x.v[0] = *(const uint4*)(row + o0);
        x.v[1] = *(const uint4*)(row + o0 + 4);
        x.v[2] = *(const uint4*)(row + o1);
        x.v[3] = *(const uint4*)(row + o1 + 4);
    }
    return x;
}
template <typename T>
__device__ __forceinline__ Raw<T> no_raw() {
    Raw<T> x;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) x.v[i] = make_uint4(0, 0, 0, 0);
    return x;
}

// As pairs, in fp32: {a[2 i], a[2 i + 1]} and {b[2 i], b[2 i + 1]}.
struct Pairs {
    float2 a[4], b[4];
};
template <typename T, bool INTER>
__device__ __forceinline__ Pairs pairs_of(const Raw<T>& x) {
    float e[16];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w[4] = {x.v[i].x, x.v[i].y, x.v[i].z, x.v[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                e[8 * i + 2 * k] = __uint_as_float(w[k] << 16);
                e[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[4 * i] = __uint_as_float(x.v[i].x);
            e[4 * i + 1] = __uint_as_float(x.v[i].y);
            e[4 * i + 2] = __uint_as_float(x.v[i].z);
            e[4 * i + 3] = __uint_as_float(x.v[i].w);
        }
    }
    Pairs y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y.a[i] = INTER ? make_float2(e[4 * i], e[4 * i + 2]) : make_float2(e[2 * i], e[2 * i + 1]);
        y.b[i] = INTER ? make_float2(e[4 * i + 1], e[4 * i + 3]) : make_float2(e[8 + 2 * i], e[8 + 2 * i + 1]);
    }
    return y;
}
// Element k of the row's two pieces, in the order of memory.
template <bool INTER>
__device__ __forceinline__ void elements_of(const Pairs& y, float (&e)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[INTER ? 4 * i : 2 * i] = y.a[i].x;
        e[INTER ? 4 * i + 2 : 2 * i + 1] = y.a[i].y;
        e[INTER ? 4 * i + 1 : 8 + 2 * i] = y.b[i].x;
        e[INTER ? 4 * i + 3 : 8 + 2 * i + 1] = y.b[i].y;
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
// A row into the cache (or window): as it is, or as codes.
template <bool FP8, typename TD>
__device__ __forceinline__ void store_cached(TD* row, int o0, int o1, const float (&e)[16], float scale) {
    if constexpr (FP8) {
        store8_codes(row + o0, e, scale);
        store8_codes(row + o1, e + 8, scale);
    } else {
        store8(row + o0, e);
        store8(row + o1, e + 8);
    }
}

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

// Where a thread's pieces lie in its row, and whether its pairs turn.
template <int D, bool INTER>
struct Lane {
    int t, o0, o1;
    bool turning;
    __device__ __forceinline__ Lane(const RopeParams& p, int thread) {
        t = thread % (D / 16);
        turning = t < p.rd / 16;
        const bool halves = turning && !INTER;
        o0 = (halves ? t : 2 * t) * 8;
        o1 = (halves ? t + p.rd / 16 : 2 * t + 1) * 8;
    }
    // row element of a[e] (e < 8) or b[e - 8]
    __device__ __forceinline__ int element(int e) const {
        if (INTER) return o0 + 2 * (e & 7) + (e >> 3);
        return e < 8 ? o0 + e : o1 + e - 8;
    }
};

// In shared memory: of each thread of a row, its 8 (cosine, sine) and its 16 gains, in 16-byte words of which neighbouring
// threads' are neighbours.
template <int D>
struct Turns {
    float4 w[4][D / 16];      // word i: c[2 i], c[2 i + 1], s[2 i], s[2 i + 1]
};
template <int D>
struct Gains {
    float4 w[4][D / 16];      // words 0, 1: of a; 2, 3: of b
};
template <int D, bool INTER>
__device__ __forceinline__ void fill_gains(const RopeParams& p, Gains<D>& to, const float* gain, int i) {   // i < D
    const Lane<D, INTER> owner(p, i / 16);
    ((float*)&to.w[i % 16 / 4][owner.t])[i % 4] = gain != nullptr ? gain[owner.element(i % 16)] : 1.f;
}
// Pair f of a token at position `pos`.
template <int D>
__device__ __forceinline__ void fill_turn(const RopeParams& p, Turns<D>& to, int64_t pos, int f) {
    const uint64_t turn = (uint64_t)pos * p.turns[f];                    // whole turns fall off the top
    const int32_t x = (int32_t)((turn + (1ull << 31)) >> 32);            // 2^-32 turns, nearest
    const int32_t quarter = (int32_t)((uint32_t)x + (1u << 29)) >> 30;
    float s, c;
    sincospif((float)(int32_t)((uint32_t)x - ((uint32_t)quarter << 30)) * 4.656612873077393e-10f, &s, &c);   // 2^-31: half turns
    const float cc = (quarter & 1) ? -s : c, ss = (quarter & 1) ? c : s, sign = (quarter & 2) ? -p.factor : p.factor;
    float* w = (float*)&to.w[f % 8 / 2][f / 8];
    w[f % 2] = cc * sign;
    w[2 + f % 2] = ss * sign;
}

__device__ __forceinline__ float2 times(float2 x, float2 y) { return __fmul2_rn(x, y); }

// Sum of squares over a row's threads.
template <int D>
__device__ __forceinline__ float row_squares(const Pairs& x) {
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s = __ffma2_rn(x.a[i], x.a[i], s);
        s = __ffma2_rn(x.b[i], x.b[i], s);
    }
    float ss = s.x + s.y;
#pragma unroll
    for (int o = D / 32; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    return ss;
}
// Norm by the row's sum of squares: the reciprocal root is the unit's, with one step of Newton's iteration (below a step of fp32).
template <int D>
__device__ __forceinline__ void norm_row(Pairs& x, float squares, float eps, const Gains<D>& g, int t) {
    const float m = fmaf(squares, 1.f / D, eps);
    float inv = rsqrtf(m);
    if (m <= 3.402823466e38f) inv = fmaf(0.5f * inv, fmaf(-m * inv, inv, 1.f), inv);
    const float2 i2 = make_float2(inv, inv);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 ga = g.w[i][t], gb = g.w[2 + i][t];
        x.a[2 * i] = times(x.a[2 * i], times(make_float2(ga.x, ga.y), i2));
        x.a[2 * i + 1] = times(x.a[2 * i + 1], times(make_float2(ga.z, ga.w), i2));
        x.b[2 * i] = times(x.b[2 * i], times(make_float2(gb.x, gb.y), i2));
        x.b[2 * i + 1] = times(x.b[2 * i + 1], times(make_float2(gb.z, gb.w), i2));
    }
}
template <int D>
__device__ __forceinline__ void turn_row(Pairs& x, const Turns<D>& cs, int t) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 w = cs.w[i][t];
        const float2 c = make_float2(w.x, w.y), s = make_float2(w.z, w.w), m = make_float2(-w.z, -w.w);
        const float2 a = x.a[i], b = x.b[i];
        x.a[i] = __ffma2_rn(a, c, times(b, m));
        x.b[i] = __ffma2_rn(b, c, times(a, s));
    }
}

// ---- a decode step: a block for each token of a loop of a sequence ---------------------------------------------------------
template <typename T, bool FP8, int D, bool INTER>
__global__ void __launch_bounds__(kRopeThreads, sizeof(T) == 2 ? 4 : 3) plt_rope_step_kernel(const __grid_constant__ RopeParams p) {
    constexpr int TPR = D / 16, RPB = kRopeThreads / TPR;      // threads of a row, rows of a pass
    constexpr int U = 2;                                       // passes whose loads are in flight together
    using TD = typename std::conditional<FP8, uint8_t, T>::type;
    __shared__ Turns<D> s_cs;
    __shared__ Gains<D> s_gain[2];
    grid_launch_dependents();   // the attention's blocks may be set up meanwhile; they wait for this grid
    const int tid = threadIdx.x, token = blockIdx.x;
    const int j = token % p.Qn, l = (token / p.Qn) % p.L, b = token / (p.Qn * p.L);
    const Lane<D, INTER> ln(p, tid);
    const int r_in = tid / TPR, rows = p.Hq + 2 * p.Hkv;       // queries, keys, values
    auto row_at = [&](int r) {
        if (r < p.Hq) return (const T*)p.q + (int64_t)token * p.q_stride + (int64_t)r * D;
        r -= p.Hq;
        if (r < p.Hkv) return (const T*)p.k + (int64_t)token * p.k_stride + (int64_t)r * D;
        return (const T*)p.v + (int64_t)token * p.v_stride + (int64_t)(r - p.Hkv) * D;
    };
    Raw<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = r_in + u * RPB < rows ? load_raw(row_at(r_in + u * RPB), ln.o0, ln.o1) : no_raw<T>();

    uint32_t flags = 0;
    int n = p.seq_lens[b];
    int64_t before = p.prefix_lens != nullptr ? p.prefix_lens[b] : 0;
    if (before < 0) {
        flags |= kDevGroupClamped;
        before = 0;
    }
    if (n < 0 || n > before + p.max_seq_len) {
        flags |= kDevSeqLenClamped;
        n = n < 0 ? 0 : (int)min(before + p.max_seq_len, (int64_t)0x7fffffff);
    }
    const int64_t pos = (int64_t)n - p.delta[l] - 1 - (p.Qn - 1 - j);
    int64_t cell = -1;                                         // element of the cache or window where the key's first head starts
    if (pos >= 0) {
        if (l > 0) cell = (((int64_t)b * (p.L - 1) + (l - 1)) * p.w + pos % p.w) * p.Hkv * D;
        else if (pos >= before) cell = cache_cell(p, b, pos - before, flags);
    }
    if (flags && tid == 0) atomicOr(p.status, flags);
    for (int i = tid; i < p.rd / 2; i += kRopeThreads) fill_turn<D>(p, s_cs, pos, i);
    if (tid < 2 * D) fill_gains<D, INTER>(p, s_gain[tid / D], tid < D ? p.q_gain : p.k_gain, tid % D);
    __syncthreads();

    const bool qnorm = p.q_gain != nullptr, knorm = p.k_gain != nullptr, gates = l > 0 && p.gate_out != nullptr;
    const int64_t head_stride = l > 0 ? D : p.kv_stride_h;
    TD* const k_to = (TD*)(l > 0 ? p.k_win : p.k_cache);
    TD* const v_to = (TD*)(l > 0 ? p.v_win : p.v_cache);
    for (int r0 = 0; r0 < rows; r0 += RPB * U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = r0 + u * RPB + r_in;
            Pairs x = pairs_of<T, INTER>(raw[u]);
            const int next = r + RPB * U;
            if (r0 + RPB * U < rows) raw[u] = next < rows ? load_raw(row_at(next), ln.o0, ln.o1) : no_raw<T>();
            const int kind = r < p.Hq ? 0 : r < p.Hq + p.Hkv ? 1 : r < rows ? 2 : 3;
            if (qnorm || knorm) {
                const float ss = row_squares<D>(x);
                if (kind == 0 ? qnorm : kind == 1 && knorm) norm_row<D>(x, ss, p.eps, s_gain[kind & 1], ln.t);
            }
            if (kind < 2 && ln.turning) turn_row<D>(x, s_cs, ln.t);
            float e[16];
            elements_of<INTER>(x, e);
            if (kind == 0) {
                if (pos < 0)
#pragma unroll
                    for (int i = 0; i < 16; ++i) e[i] = 0.f;
                T* const out = (T*)p.q_out + ((int64_t)token * p.Hq + r) * D;
                store8(out + ln.o0, e);
                store8(out + ln.o1, e + 8);
            } else if (kind < 3 && cell >= 0) {
                const int h = r - p.Hq - (kind == 2 ? p.Hkv : 0);
                store_cached<FP8>((kind == 1 ? k_to : v_to) + cell + (int64_t)h * head_stride, ln.o0, ln.o1, e,
                                  FP8 ? (kind == 1 ? p.k_scale : p.v_scale)[h] : 1.f);
            }
            if (gates) {
                float dot = 0.f;
                if (kind == 0 && pos >= 0) {
                    const float* w = p.w_gate + (int64_t)r * D;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float4 g = *(const float4*)(w + (i < 2 ? ln.o0 : ln.o1) + 4 * (i & 1));
                        dot = fmaf(g.x, e[4 * i], dot);
                        dot = fmaf(g.y, e[4 * i + 1], dot);
                        dot = fmaf(g.z, e[4 * i + 2], dot);
                        dot = fmaf(g.w, e[4 * i + 3], dot);
                    }
                }
#pragma unroll
                for (int o = TPR / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
                if (ln.t == 0 && kind == 0) p.gate_out[((int64_t)b * (p.L - 1) + (l - 1)) * p.Hq + r] = dot + p.b_gate[r];
            }
        }
    }
}

// ---- the rows of a prompt: a block for TB rows of a loop of a sequence -----------------------------------------------------------
template <typename T, bool FP8, int D, bool INTER, int TB>
__global__ void __launch_bounds__(kRopeThreads, 4) plt_rope_seq_kernel(const __grid_constant__ RopeParams p) {
    constexpr int TPR = D / 16, RPB = kRopeThreads / TPR;
    using TD = typename std::conditional<FP8, uint8_t, T>::type;
    __shared__ int64_t s_cell[TB];      // element where head 0 of the token's row starts in the cache, or -1: not stored
    __shared__ Turns<D> s_cs[TB];
    __shared__ Gains<D> s_gain[2];
    const int tid = threadIdx.x, b = blockIdx.y / p.L, l = blockIdx.y % p.L, t0 = blockIdx.x * TB;
    uint32_t flags = 0;
    int n = p.seq_lens[b];
    int64_t before = p.prefix_lens != nullptr ? p.prefix_lens[b] : 0, start = p.start != nullptr ? p.start[b] : 0;
    if (before < 0 || start < 0) {
        flags |= kDevGroupClamped;
        before = max(before, (int64_t)0);
        start = max(start, (int64_t)0);
    }
    if (n < 0 || n > p.T) {
        flags |= kDevSeqLenClamped;
        n = n < 0 ? 0 : p.T;
    }
    const int64_t first = start + t0 - p.delta[l];             // position of the block's first row
    const int hi = min(n - t0, TB), lo = first < 0 ? (int)min(-first, (int64_t)TB) : 0;     // its tokens [lo, hi)
    if (lo >= hi && !(l == 0 && hi > 0)) {
        if (flags && tid == 0) atomicOr(p.status, flags);
        return;
    }
    const bool cached = l == 0 && p.k_cache != nullptr;
    if (tid < TB) {
        int64_t cell = -1;
        if (cached && tid < hi) {
            const int64_t slot = start + t0 + tid - before;
            if (slot >= p.max_seq_len) flags |= kDevSeqLenClamped;
            else if (slot >= 0) cell = cache_cell(p, b, slot, flags);
        }
        s_cell[tid] = cell;
    }
    if (flags) atomicOr(p.status, flags);
    // the first queries are on their way while the tables are made
    constexpr int U = sizeof(T) == 2 ? 2 : 1;                  // rows whose loads are in flight together
    const Lane<D, INTER> ln(p, tid);
    const int r_in = tid / TPR, q_from = lo * p.Hq, q_to = hi * p.Hq;
    const int64_t q_base = (((int64_t)b * p.L + l) * p.T + t0) * p.Hq * D;
    const T* const q_in = (const T*)p.q + q_base;
    Raw<T> raws[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int r = q_from + u * RPB + r_in;
        raws[u] = r < q_to ? load_raw(q_in + r * D, ln.o0, ln.o1) : no_raw<T>();
    }
    if (tid < 2 * D) fill_gains<D, INTER>(p, s_gain[tid / D], tid < D ? p.q_gain : p.k_gain, tid % D);
    const int pairs = p.rd / 2;
    for (int i = tid; i < TB * pairs; i += kRopeThreads) {
        const int tk = i / pairs;
        fill_turn<D>(p, s_cs[tk], first + tk, i - tk * pairs);
    }
    __syncthreads();

    // A tensor's rows of the block lie one behind the other: row r is head r % heads of token r / heads (by a reciprocal; r and
    // heads are below 2^13 and 2^11).
    auto token_of = [](int r, uint32_t reciprocal) { return reciprocal == 0 ? r : (int)__umulhi((uint32_t)r, reciprocal); };

    // ---- queries -----------------------------------------------------------------------------------------------
    {
        const bool norm = p.q_gain != nullptr;
        T* const out = (T*)p.q_out + q_base;
        for (int r0 = q_from; r0 < q_to; r0 += RPB * U) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = r0 + u * RPB + r_in, tk = min(token_of(r, p.q_reciprocal), TB - 1);
                Pairs x = pairs_of<T, INTER>(raws[u]);
                if (norm) norm_row<D>(x, row_squares<D>(x), p.eps, s_gain[0], ln.t);
                if (ln.turning) turn_row<D>(x, s_cs[tk], ln.t);
                if (r < q_to) {
                    float e[16];
                    elements_of<INTER>(x, e);
                    store8(out + r * D + ln.o0, e);
                    store8(out + r * D + ln.o1, e + 8);
                }
            }
            if (r0 + RPB * U < q_to)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int r = r0 + (U + u) * RPB + r_in;
                    raws[u] = r < q_to ? load_raw(q_in + r * D, ln.o0, ln.o1) : no_raw<T>();
                }
        }
    }

    // ---- keys, and the first loop's values ------------------------------------------------------------------------
    const bool norm = p.k_gain != nullptr;
    const int64_t base = (l == 0 ? (int64_t)b * p.T + t0 : ((int64_t)b * (p.L - 1) + (l - 1)) * p.T + t0) * p.Hkv * D;
    const T* const k_in = (const T*)(l == 0 ? p.k : p.k_loc) + base;
    T* const k_out = (T*)(l == 0 ? p.k_out : p.k_loc_out);
    const int from = (l == 0 ? 0 : lo) * p.Hkv, to = hi * p.Hkv;
    for (int r0 = from; r0 < to; r0 += RPB) {
        const int r = r0 + r_in, tk = min(token_of(r, p.k_reciprocal), TB - 1);
        const Raw<T> raw = r < to ? load_raw(k_in + r * D, ln.o0, ln.o1) : no_raw<T>();
        const int64_t cell = cached && r < to ? s_cell[tk] : -1;
        Raw<T> values = no_raw<T>();
        if (cell >= 0) values = load_raw((const T*)p.v + base + r * D, ln.o0, ln.o1);
        Pairs x = pairs_of<T, INTER>(raw);
        if (norm) norm_row<D>(x, row_squares<D>(x), p.eps, s_gain[1], ln.t);
        if (ln.turning) turn_row<D>(x, s_cs[tk], ln.t);
        float e[16];
        elements_of<INTER>(x, e);
        if (k_out != nullptr && r < to) {
            store8(k_out + base + r * D + ln.o0, e);
            store8(k_out + base + r * D + ln.o1, e + 8);
        }
        if (cell >= 0) {
            const int h = r - tk * p.Hkv;
            const int64_t at = cell + (int64_t)h * p.kv_stride_h;
            store_cached<FP8>((TD*)p.k_cache + at, ln.o0, ln.o1, e, FP8 ? p.k_scale[h] : 1.f);
            elements_of<INTER>(pairs_of<T, INTER>(values), e);
            store_cached<FP8>((TD*)p.v_cache + at, ln.o0, ln.o1, e, FP8 ? p.v_scale[h] : 1.f);
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
    p->rd = h->rd;
    p->q_reciprocal = c.Hq > 1 ? (uint32_t)(((1ull << 32) + c.Hq - 1) / c.Hq) : 0;
    p->k_reciprocal = c.Hkv > 1 ? (uint32_t)(((1ull << 32) + c.Hkv - 1) / c.Hkv) : 0;
    p->factor = c.attn_factor != 0.f ? c.attn_factor : 1.f;
    p->eps = c.norm_eps;
    for (int l = 0; l < kMaxLoops; ++l) p->delta[l] = h->delta[l];
    return PLT_OK;
}

// Tokens of a block of a prompt.
//   - 32 where a token's queries and keys are so few bytes that a block's start counts, and the larger blocks still fill the device: 32
//     ragged prompts of up to 4096 rows of bf16 1 + 1 heads of 64 17.9 us against 45.3 with 8, 3 + 1 of 128 27.5 against 51.7, 8 + 2 of
//     128 44.1 against 54.8, 8 + 8 of 128 79.6 against 76.7; one prompt of 1000 rows of 3 + 1 heads of 128 6.0 against 4.3.
//   - 2 where blocks of 8 are few, since a block walks over its heads: one prompt of 60 rows, 32 + 8 heads of 128 in bf16 3.9 us against
//     7.3 with 8, of 300 rows 4.5 against 7.5; 1000 rows of 16 + 4 heads 6.3 against 5.3.
int tokens_of_block(const RopeParams& p, int row_bytes, int sms) {
    const int64_t prompts = (int64_t)p.B * p.L;
    if (prompts * ((p.T + 7LL) / 8) <= 64) return 2;
    return (p.Hq + p.Hkv) * row_bytes <= 2560 && prompts * ((p.T + 31LL) / 32) >= 3 * sms ? 32 : 8;
}

// A prompt's rows in blocks of TB tokens.
template <typename T, bool FP8, int D, bool INTER, int TB>
void launch_seq(const RopeParams& p, cudaStream_t stream) {
    const dim3 grid((unsigned)(((int64_t)p.T + TB - 1) / TB), (unsigned)(p.B * p.L));
    plt_rope_seq_kernel<T, FP8, D, INTER, TB><<<grid, kRopeThreads, 0, stream>>>(p);
}

template <typename T, bool FP8, int D, bool INTER>
void launch_one(bool seq, const RopeParams& p, int sms, cudaStream_t stream) {
    if (!seq) {
        plt_rope_step_kernel<T, FP8, D, INTER><<<p.B * p.L * p.Qn, kRopeThreads, 0, stream>>>(p);
        return;
    }
    const int tokens = tokens_of_block(p, D * (int)sizeof(T), sms);
    if (tokens == 32) launch_seq<T, FP8, D, INTER, 32>(p, stream);
    else if (tokens == 8) launch_seq<T, FP8, D, INTER, 8>(p, stream);
    else launch_seq<T, FP8, D, INTER, 2>(p, stream);
}

template <bool INTER>
void launch_type(const plt_rope_config& c, bool seq, const RopeParams& p, int sms, cudaStream_t stream) {
    if (c.kv_dtype == PLT_KV_E4M3) launch_one<__nv_bfloat16, true, 128, INTER>(seq, p, sms, stream);
    else if (c.dtype == PLT_BF16 && c.d == 128) launch_one<__nv_bfloat16, false, 128, INTER>(seq, p, sms, stream);
    else if (c.dtype == PLT_BF16) launch_one<__nv_bfloat16, false, 64, INTER>(seq, p, sms, stream);
    else if (c.d == 128) launch_one<float, false, 128, INTER>(seq, p, sms, stream);
    else launch_one<float, false, 64, INTER>(seq, p, sms, stream);
}

plt_status launch(plt_rope_t h, bool seq, const RopeParams& p, cudaStream_t stream) {
    DeviceScope scope(h->device);
    if (scope.err != cudaSuccess) return handle_fail(h, g_rope_error, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    if (h->cfg.layout == PLT_ROPE_INTERLEAVED) launch_type<true>(h->cfg, seq, p, h->sms, stream);
    else launch_type<false>(h->cfg, seq, p, h->sms, stream);
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
    int sms = 0;
    s = check_device(config->device, g_rope_error, &sms);
    if (s != PLT_OK) return s;
    plt_rope* h = new (std::nothrow) plt_rope();
    if (!h) return rope_fail(nullptr, PLT_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->cfg = *config;
    h->cfg.loop_offset = nullptr;
    h->cfg.inv_freq = nullptr;
    h->device = config->device;
    h->rd = rd;
    h->sms = sms;
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
    return launch(h, false, p, (cudaStream_t)cuda_stream);
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
    return launch(h, true, p, (cudaStream_t)cuda_stream);
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

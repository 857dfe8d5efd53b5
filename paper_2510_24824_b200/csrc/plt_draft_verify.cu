// Draft verification: how many of a sequence's drafted tokens stand, and the token behind them by inversion of the
// remaining distribution's running sum.
//
// Two or three launches, each set up while the one before it ends. (1) A warp for each sequence finds the number n of drafts that
// stand. (2) A warp for each chunk of 512 elements sums the chunk's weights in 64 bits, all its loads in flight at once, and
// leaves the sum; warps do not wait for one another. (3) A block for each sequence walks the sums to the chunk in which the
// running sum passes r * total, and that chunk (still in L2) to the token. The weights are never written. Where there are few
// chunks, latency counts and (2) does the work of (1) itself.
//
// Bound by reading one row of p and, after a refusal, one of q: 256 sequences of 131072 fp32 take 42 us (39.5 in a graph), 189 MB of p
// and q, which the copy rate would take 29.2 for: two more starts, and additions in 64 bits. One sequence of 32768 takes 5.5 us, which is two dependent launches; 48 copied drafts of 50257 bf16 7.8.
#include "../../include/plt_draft_verify.h"

#include <cuda_bf16.h>

#include <cstring>
#include <new>

#include "plt_handle.h"
#include "plt_ptx.cuh"

using namespace plt;

namespace {

constexpr int kVerifyThreads = 256;
template <typename T>
constexpr int kVecs = sizeof(T) == 4 ? 4 : 2;   // vectors of 16 bytes that a lane takes of a row's chunk: 16 elements
// Chunks of a multiprocessor up to which the sums' warps count the drafts that stand themselves (about as many as it holds warps),
// instead of a kernel before them: 64 chunks in all 5.5 us against 6.3, 4096 7.2 against 8.2, 8192 9.9 against 10.4; 16384 16.5 against
// 16.2, 65536 44.6 against 39.4.
constexpr int kAtOnce = 64;
constexpr int kMaxDrafts = 64;

thread_local char g_verify_error[512] = "";

}  // namespace

struct plt_draft_verify : HandleBase {
    plt_draft_verify_config cfg;
    double* sums = nullptr;      // [batch, chunks] of a call
    int2* stand = nullptr;       // [batch] drafts that stand, drafts there were
    int sms = 0;
};

namespace {

struct VerifyParams {
    const void* target;
    const void* draft;
    int64_t target_b, target_j, draft_b, draft_j;
    const int32_t* draft_tokens;
    const int32_t* draft_lens;
    const float* accept_u;
    const float* sample_u;
    int32_t* tokens;
    int32_t* num_accepted;
    const int32_t* seq_lens;
    int32_t* new_lens;
    double* sums;
    int2* stand;
    uint32_t* status;
    int32_t B, K, V, chunks;
};

template <typename T>
__device__ __forceinline__ float widen(T x) {
    if constexpr (sizeof(T) == 4) return x;
    else return __bfloat162float(x);
}

// One sequence's row of weights: p - q where that is above 0, or p, or p without the draft that was refused.
template <typename T>
struct Row {
    const T* p;
    const T* q;       // or null
    int without;      // index whose weight is 0, or -1
    // a - b where that is above 0 (and in fp32's range), else 0. The test is made in fp32, where a difference of two numbers that
    // differ never rounds to 0: 64-bit units are few.
    __device__ __forceinline__ double weight(float a, float b) const {
        const float d = a - b;
        const bool counts = d > 0.f && d <= 3.402823466e38f;
        return (double)(counts ? a : 0.f) - (double)(counts ? b : 0.f);
    }
    __device__ __forceinline__ double weight(float a) const { return (double)(a > 0.f && a <= 3.402823466e38f ? a : 0.f); }
    __device__ __forceinline__ double at(int i) const {
        if (i == without) return 0.0;
        return weight(widen(p[i]), q != nullptr ? widen(q[i]) : 0.f);
    }
};

// Largest thread for which `yes`, or -1.
__device__ __forceinline__ int last_thread(bool yes, int* s_last) {
    __syncthreads();
    if (threadIdx.x == 0) *s_last = -1;
    __syncthreads();
    const uint32_t m = __ballot_sync(0xffffffffu, yes);
    if ((threadIdx.x & 31) == 0 && m != 0) atomicMax(s_last, (int)threadIdx.x + 31 - __clz(m));
    __syncthreads();
    return *s_last;
}

// Elements of 16 bytes.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

template <typename T>
__device__ __forceinline__ void load_vec16(const T* src, float (&x)[kVec<T>]) {
    const uint4 v = __ldg((const uint4*)src);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Inclusive running sum over the block's threads, and the sum of all; s_warp: one double for each warp.
__device__ __forceinline__ double block_running_sum(double x, double* s_warp, double& total) {
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 31) s_warp[wid] = x;
    __syncthreads();
    double base = 0.0;
    total = 0.0;
#pragma unroll
    for (int w = 0; w < kVerifyThreads / 32; ++w) {
        if (w == wid) base = total;
        total += s_warp[w];
    }
    return base + x;
}

// Smallest thread for which `yes`, or kVerifyThreads.
__device__ __forceinline__ int first_thread(bool yes, int* s_first) {
    const int lane = threadIdx.x & 31;
    __syncthreads();
    if (threadIdx.x == 0) *s_first = kVerifyThreads;
    __syncthreads();
    const uint32_t m = __ballot_sync(0xffffffffu, yes);
    if (lane == 0 && m != 0) atomicMin(s_first, (int)threadIdx.x + __ffs(m) - 1);
    __syncthreads();
    return *s_first;
}

// Walks `n` numbers (value(i), i < n, none below 0) to the first whose running sum exceeds r times their total. Returns its
// index, or the last with a value above 0 where none does (-1: none has), `before`, the sum in front of it, and `total`. Each
// thread takes a run of consecutive numbers. All threads of the block call it and get the same answer. Only numbers above 0 are
// candidates: two running sums of the same numbers may differ by a rounding.
template <typename F>
__device__ int walk(int n, F value, double& before, double& total, double r, double* s_warp, int* s_first, double* s_base) {
    const int per = (n + kVerifyThreads - 1) / kVerifyThreads;
    const int lo = min((int)threadIdx.x * per, n), hi = min(lo + per, n);
    double own = 0.0;
    for (int i = lo; i < hi; ++i) own += value(i);
    const double upto = block_running_sum(own, s_warp, total);
    const double limit = r * total;
    int t = first_thread(own > 0.0 && upto > limit, s_first);
    if (t == kVerifyThreads) {
        t = last_thread(own > 0.0, s_first);
        if (t < 0) return -1;
    }
    __syncthreads();
    if ((int)threadIdx.x == t) {
        double run = upto - own, base = run;
        int found = lo;
        for (int i = lo; i < hi; ++i) {
            const double v = hi - lo == 1 ? own : value(i);
            if (v > 0.0) {
                found = i;
                base = run;
                run += v;
                if (run > limit) break;
            }
        }
        *s_first = found;
        *s_base = base;
    }
    __syncthreads();
    before = *s_base;
    return *s_first;
}

// (drafts that stand, drafts there were) of sequence b, by a whole warp.
template <typename T>
__device__ __forceinline__ int2 count_standing(const VerifyParams& p, int b, bool report) {
    const int lane = threadIdx.x & 31;
    uint32_t flags = 0;
    int len = p.K;
    if (p.draft_lens != nullptr) {
        len = p.draft_lens[b];
        if (len < 0 || len > p.K) {
            flags |= kDevSeqLenClamped;
            len = len < 0 ? 0 : p.K;
        }
    }
    int n = len;
#pragma unroll
    for (int h = 0; h < kMaxDrafts / 32; ++h) {
        const int j = h * 32 + lane;
        bool refused = false;
        if (j < len) {
            const int x = p.draft_tokens[(int64_t)b * p.K + j];
            const float u = p.accept_u[(int64_t)b * p.K + j];
            refused = true;
            if (x < 0 || x >= p.V) {
                flags |= kDevTokenRange;
            } else {
                const float pj = widen(((const T*)p.target)[b * p.target_b + j * p.target_j + x]);
                const float qj = p.draft != nullptr ? widen(((const T*)p.draft)[b * p.draft_b + j * p.draft_j + x]) : 1.f;
                refused = !((double)u * (double)qj < (double)pj);
            }
        }
        const uint32_t m = __ballot_sync(0xffffffffu, refused);
        if (m != 0) n = min(n, h * 32 + __ffs(m) - 1);
    }
    if (report && flags) atomicOr(p.status, flags);
    return make_int2(n, len);
}

// The row of weights that decides sequence b's next token.
template <typename T>
__device__ __forceinline__ Row<T> row_of(const VerifyParams& p, int b, int2 stand) {
    const bool cut = stand.x < stand.y;
    Row<T> row;
    row.p = (const T*)p.target + b * p.target_b + stand.x * p.target_j;
    row.q = cut && p.draft != nullptr ? (const T*)p.draft + b * p.draft_b + stand.x * p.draft_j : nullptr;
    row.without = cut && p.draft == nullptr ? p.draft_tokens[(int64_t)b * p.K + stand.x] : -1;
    return row;
}

// Elements of a chunk, and elements that the 16-byte grid puts in front of a row (chunk 0 starts there).
template <typename T>
constexpr int kChunk = 32 * kVecs<T> * kVec<T>;
template <typename T, bool VEC>
__device__ __forceinline__ int lead_of(const Row<T>& row) {
    return VEC ? (int)(((uintptr_t)row.p & 15) / sizeof(T)) : 0;
}

template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) plt_draft_verify_count(const __grid_constant__ VerifyParams p) {
    grid_launch_dependents();
    const int b = blockIdx.x * (kVerifyThreads / 32) + (threadIdx.x >> 5);
    if (b >= p.B) return;
    const int2 s = count_standing<T>(p, b, true);
    if ((threadIdx.x & 31) == 0) p.stand[b] = s;
}

template <typename T, bool VEC, bool COUNT>
__global__ void __launch_bounds__(kVerifyThreads, 5) plt_draft_verify_sums(const __grid_constant__ VerifyParams p) {
    constexpr int N = kVec<T>;
    grid_launch_dependents();
    const int b = blockIdx.y, lane = threadIdx.x & 31, chunk = blockIdx.x * (kVerifyThreads / 32) + (threadIdx.x >> 5);
    if (chunk >= p.chunks) return;
    int2 stand;
    if (COUNT) {
        stand = count_standing<T>(p, b, chunk == 0);
        if (chunk == 0 && lane == 0) p.stand[b] = stand;
    } else {
        grid_dependency_wait();
        stand = p.stand[b];
    }
    const Row<T> row = row_of<T>(p, b, stand);
    const int c0 = chunk * kChunk<T> - lead_of<T, VEC>(row);      // may be below 0
    double sum = 0.0;
    if constexpr (VEC) {
        // the row of q lies on the 16-byte grid as the row of p does
        auto load = [&](const T* from, int i, float (&x)[N]) {
            if (i >= 0 && i + N <= p.V) {
                load_vec16<T>(from + i, x);
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k) x[k] = i + k >= 0 && i + k < p.V ? widen(from[i + k]) : 0.f;
            }
        };
        float a[kVecs<T>][N];
        auto at = [&](int u) { return c0 + (u * 32 + lane) * N; };
#pragma unroll
        for (int u = 0; u < kVecs<T>; ++u) load(row.p, at(u), a[u]);
        if (row.q != nullptr) {
            float q[kVecs<T>][N];
#pragma unroll
            for (int u = 0; u < kVecs<T>; ++u) load(row.q, at(u), q[u]);
#pragma unroll
            for (int u = 0; u < kVecs<T>; ++u)
#pragma unroll
                for (int k = 0; k < N; ++k) sum += row.weight(a[u][k], q[u][k]);
        } else {
#pragma unroll
            for (int u = 0; u < kVecs<T>; ++u)
#pragma unroll
                for (int k = 0; k < N; ++k) sum += at(u) + k == row.without ? 0.0 : row.weight(a[u][k]);
        }
    } else {
        constexpr int U = 16;
        for (int v0 = 0; v0 < kChunk<T> / 32; v0 += U) {
            float a[U], q[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = c0 + (v0 + u) * 32 + lane;
                const bool in = i < p.V && i != row.without;
                a[u] = in ? widen(row.p[i]) : 0.f;
                q[u] = in && row.q != nullptr ? widen(row.q[i]) : 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) sum += row.weight(a[u], q[u]);
        }
    }
    sum = warp_sum(sum);
    if (lane == 0) p.sums[(int64_t)b * p.chunks + chunk] = sum;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kVerifyThreads) plt_draft_verify_pick(const __grid_constant__ VerifyParams p) {
    constexpr int N = kVec<T>;
    static_assert(kChunk<T> <= kVerifyThreads * N, "a thread takes one vector of the chunk");
    __shared__ double s_warp[kVerifyThreads / 32];
    __shared__ double s_base;
    __shared__ int s_pick;
    const int b = blockIdx.x, tid = threadIdx.x;
    const double r = (double)p.sample_u[b];
    grid_dependency_wait();
    const int2 stand = p.stand[b];
    const double* sums = p.sums + (int64_t)b * p.chunks;
    int token = -1;
    double before = 0.0, total = 0.0;
    const int c = walk(p.chunks, [&](int i) { return sums[i]; }, before, total, r, s_warp, &s_pick, &s_base);
    Row<T> row = row_of<T>(p, b, stand);
    if (total > 0.0) {
        const int first = c * kChunk<T> - lead_of<T, VEC>(row) + tid * N;
        double w[N], own = 0.0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            w[k] = tid < 32 * kVecs<T> && first + k >= 0 && first + k < p.V ? row.at(first + k) : 0.0;
            own += w[k];
        }
        double chunk_total;
        const double upto = before + block_running_sum(own, s_warp, chunk_total), limit = r * total;
        int t = first_thread(own > 0.0 && upto > limit, &s_pick);
        if (t == kVerifyThreads) t = last_thread(own > 0.0, &s_pick);
        __syncthreads();
        if (tid == t) {
            double run = upto - own;
            int found = -1;
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (w[k] > 0.0 && (found < 0 || !(run > limit))) {
                    found = first + k;
                    run += w[k];
                }
            s_pick = found;
        }
        __syncthreads();
        token = s_pick;
    } else if (stand.x < stand.y) {
        // p lies nowhere above q: the whole of p
        row.q = nullptr;
        row.without = -1;
        token = walk(p.V, [&](int i) { return row.at(i); }, before, total, r, s_warp, &s_pick, &s_base);
    }
    for (int j = tid; j <= p.K; j += kVerifyThreads)
        p.tokens[(int64_t)b * (p.K + 1) + j] = j < stand.x ? p.draft_tokens[(int64_t)b * p.K + j] : j == stand.x ? token : -1;
    if (tid == 0) {
        p.num_accepted[b] = stand.x;
        if (p.new_lens != nullptr) p.new_lens[b] = max(0, max(p.seq_lens[b], 0) - (p.K - stand.x));
        if (token < 0) atomicOr(p.status, kDevNoProbability);
    }
}

template <typename F>
cudaError_t launch(F fn, dim3 grid, bool overlap, const VerifyParams& p, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kVerifyThreads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = overlap ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, fn, p);
}

template <typename T, bool VEC>
cudaError_t launch_all(const VerifyParams& p, int sms, cudaStream_t stream) {
    constexpr int W = kVerifyThreads / 32;
    const dim3 grid((unsigned)((p.chunks + W - 1) / W), (unsigned)p.B);
    cudaError_t e;
    if ((int64_t)p.chunks * p.B <= (int64_t)kAtOnce * sms) {
        e = launch(plt_draft_verify_sums<T, VEC, true>, grid, false, p, stream);
    } else {
        e = launch(plt_draft_verify_count<T>, dim3((unsigned)((p.B + W - 1) / W)), false, p, stream);
        if (e == cudaSuccess) e = launch(plt_draft_verify_sums<T, VEC, false>, grid, true, p, stream);
    }
    if (e == cudaSuccess) e = launch(plt_draft_verify_pick<T, VEC>, dim3((unsigned)p.B), true, p, stream);
    return e;
}

plt_status verify_fail(plt_draft_verify_t h, plt_status code, const char* what) {
    return handle_fail(h, g_verify_error, code, "%s", what);
}

plt_status check_config(const plt_draft_verify_config* c) {
    if (!c) return verify_fail(nullptr, PLT_ERR_INVALID_ARG, "config is NULL");
    if (c->struct_size != sizeof(plt_draft_verify_config))
        return handle_fail(nullptr, g_verify_error, PLT_ERR_INVALID_ARG, "config.struct_size %u != %zu", c->struct_size, sizeof *c);
    if (c->dtype != PLT_F32 && c->dtype != PLT_BF16) return verify_fail(nullptr, PLT_ERR_INVALID_ARG, "unknown dtype");
    if (c->max_batch < 1 || c->max_drafts < 1 || c->vocab < 1) return verify_fail(nullptr, PLT_ERR_INVALID_ARG, "non-positive size in config");
    if (c->max_batch > kMaxBatch) return verify_fail(nullptr, PLT_ERR_UNSUPPORTED, "max_batch above 4096");
    if (c->max_drafts > kMaxDrafts) return verify_fail(nullptr, PLT_ERR_UNSUPPORTED, "max_drafts above 64");
    if (c->vocab > (1 << 24)) return verify_fail(nullptr, PLT_ERR_UNSUPPORTED, "vocab above 2^24");
    return PLT_OK;
}

// Chunks of a row that starts up to `lead` elements behind a place of the 16-byte grid.
int chunks_of(const plt_draft_verify_config* c, int lead) {
    const int chunk = c->dtype == PLT_F32 ? kChunk<float> : kChunk<__nv_bfloat16>;
    return (c->vocab + lead + chunk - 1) / chunk;
}

size_t workspace_of(const plt_draft_verify_config* c) {
    return (size_t)c->max_batch * (8u * (size_t)chunks_of(c, 7) + sizeof(int2)) + 256;
}

}  // namespace

#define PLT_API __attribute__((visibility("default")))
extern "C" {

PLT_API plt_status plt_draft_verify_workspace_bytes(const plt_draft_verify_config* config, size_t* out_bytes) {
    const plt_status s = check_config(config);
    if (s != PLT_OK) return s;
    if (!out_bytes) return verify_fail(nullptr, PLT_ERR_INVALID_ARG, "out_bytes is NULL");
    *out_bytes = workspace_of(config);
    return PLT_OK;
}

PLT_API plt_status plt_draft_verify_create(const plt_draft_verify_config* config, plt_draft_verify_t* out_handle) {
    if (!out_handle) return verify_fail(nullptr, PLT_ERR_INVALID_ARG, "out_handle is NULL");
    *out_handle = nullptr;
    plt_status s = check_config(config);
    if (s != PLT_OK) return s;
    DeviceScope scope(config->device);
    if (scope.err != cudaSuccess) {
        (void)cudaGetLastError();
        return handle_fail(nullptr, g_verify_error, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    }
    int sms = 0;
    s = check_device(config->device, g_verify_error, &sms);
    if (s != PLT_OK) return s;
    plt_draft_verify* h = new (std::nothrow) plt_draft_verify();
    if (!h) return verify_fail(nullptr, PLT_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->cfg = *config;
    h->device = config->device;
    h->sms = sms;
    const size_t bytes = workspace_of(config);
    void* ws = nullptr;
    if (cudaMalloc(&ws, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        delete h;
        return handle_fail(nullptr, g_verify_error, PLT_ERR_OUT_OF_MEMORY, "cudaMalloc of %zu workspace bytes failed", bytes);
    }
    h->status = (uint32_t*)ws;
    h->sums = (double*)((char*)ws + 256);
    h->stand = (int2*)(h->sums + (size_t)config->max_batch * chunks_of(config, 7));
    cudaError_t e = cudaMemset(ws, 0, bytes);
    if (e == cudaSuccess) e = cudaDeviceSynchronize();   // another stream may run first
    if (e != cudaSuccess) {
        cudaFree(ws);
        delete h;
        return handle_fail(nullptr, g_verify_error, PLT_ERR_CUDA, "clearing the workspace: %s", cudaGetErrorString(e));
    }
    *out_handle = h;
    return PLT_OK;
}

PLT_API plt_status plt_draft_verify_run(plt_draft_verify_t h, const plt_draft_verify_args* a, void* cuda_stream) {
    if (!h) return verify_fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    if (!a) return verify_fail(h, PLT_ERR_INVALID_ARG, "args is NULL");
    if (a->struct_size != sizeof(plt_draft_verify_args))
        return handle_fail(h, g_verify_error, PLT_ERR_INVALID_ARG, "args.struct_size %u != %zu", a->struct_size, sizeof *a);
    const plt_draft_verify_config& c = h->cfg;
    if (a->batch < 0) return verify_fail(h, PLT_ERR_INVALID_ARG, "batch < 0");
    if (a->batch > c.max_batch)
        return handle_fail(h, g_verify_error, PLT_ERR_CAPACITY, "batch %d > max_batch %d", a->batch, c.max_batch);
    if (a->batch == 0) return PLT_OK;
    if (!a->target_probs || !a->draft_tokens || !a->accept_u || !a->sample_u || !a->tokens || !a->num_accepted)
        return verify_fail(h, PLT_ERR_INVALID_ARG, "target_probs, draft_tokens, accept_u, sample_u, tokens and num_accepted must not be NULL");
    if ((a->seq_lens == nullptr) != (a->new_lens == nullptr))
        return verify_fail(h, PLT_ERR_INVALID_ARG, "seq_lens and new_lens go together");
    const int es = c.dtype == PLT_F32 ? 4 : 2;
    const uintptr_t words = (uintptr_t)a->draft_tokens | (uintptr_t)a->draft_lens | (uintptr_t)a->accept_u | (uintptr_t)a->sample_u |
                            (uintptr_t)a->tokens | (uintptr_t)a->num_accepted | (uintptr_t)a->seq_lens | (uintptr_t)a->new_lens;
    if ((words & 3u) || misaligned(a->target_probs, es) || misaligned(a->draft_probs, es))
        return verify_fail(h, PLT_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
    VerifyParams p;
    memset(&p, 0, sizeof p);
    p.target_b = a->target_stride_b; p.target_j = a->target_stride_j;
    p.draft_b = a->draft_stride_b; p.draft_j = a->draft_stride_j;
    if (p.target_b == 0 && p.target_j == 0) {
        p.target_j = c.vocab;
        p.target_b = (int64_t)(c.max_drafts + 1) * c.vocab;
    }
    if (p.draft_b == 0 && p.draft_j == 0) {
        p.draft_j = c.vocab;
        p.draft_b = (int64_t)c.max_drafts * c.vocab;
    }
    if (p.target_j < c.vocab || (a->batch > 1 && p.target_b < c.vocab) || (a->draft_probs && (p.draft_j < c.vocab || (a->batch > 1 && p.draft_b < c.vocab))))
        return verify_fail(h, PLT_ERR_INVALID_ARG, "strides of probabilities must be at least vocab elements");
    p.target = a->target_probs; p.draft = a->draft_probs;
    p.draft_tokens = a->draft_tokens; p.draft_lens = a->draft_lens; p.accept_u = a->accept_u; p.sample_u = a->sample_u;
    p.tokens = a->tokens; p.num_accepted = a->num_accepted; p.seq_lens = a->seq_lens; p.new_lens = a->new_lens;
    p.sums = h->sums; p.stand = h->stand; p.status = h->status;
    p.B = a->batch; p.K = c.max_drafts; p.V = c.vocab;
    // 16-byte loads where the rows of p and q that one sequence needs lie alike on the 16-byte grid: always without q
    // (chunks follow p's rows), else where both bases are aligned and all strides are whole vectors. Element by element 64 rows of
    // 32768 take 8.2 us instead of 7.2, 48 bf16 rows of 50257 8.6 instead of 7.8, 256 rows of 131072 40.5 instead of 39.4.
    const int unit = 16 / es;
    const bool vec = !a->draft_probs || (!misaligned(a->target_probs, 16) && !misaligned(a->draft_probs, 16) && p.target_b % unit == 0 &&
                                         p.target_j % unit == 0 && p.draft_b % unit == 0 && p.draft_j % unit == 0);
    const bool on_grid = !misaligned(a->target_probs, 16) && p.target_b % unit == 0 && p.target_j % unit == 0;
    const int lead = vec && !on_grid ? unit - 1 : 0;
    p.chunks = chunks_of(&c, lead);
    DeviceScope scope(h->device);
    if (scope.err != cudaSuccess) return handle_fail(h, g_verify_error, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (c.dtype == PLT_F32) e = vec ? launch_all<float, true>(p, h->sms, stream) : launch_all<float, false>(p, h->sms, stream);
    else e = vec ? launch_all<__nv_bfloat16, true>(p, h->sms, stream) : launch_all<__nv_bfloat16, false>(p, h->sms, stream);
    if (e != cudaSuccess) return handle_fail(h, g_verify_error, PLT_ERR_CUDA, "launching the kernels: %s", cudaGetErrorString(e));
    return PLT_OK;
}

PLT_API plt_status plt_draft_verify_check(plt_draft_verify_t h, void* cuda_stream, uint32_t* out_bits) {
    if (!h) return verify_fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    return handle_check(h, g_verify_error, (cudaStream_t)cuda_stream, out_bits);
}

PLT_API plt_status plt_draft_verify_destroy(plt_draft_verify_t h) {
    if (!h) return PLT_OK;
    DeviceScope scope(h->device);
    cudaFree(h->status);
    delete h;
    return PLT_OK;
}

PLT_API const char* plt_draft_verify_last_error(plt_draft_verify_t h) { return h ? h->err : g_verify_error; }

}  // extern "C"

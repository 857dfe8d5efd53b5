// Draft verification: how many of a sequence's drafted tokens stand, and the token behind them by inversion of the
// remaining distribution's running sum.
//
// One launch. A block takes one chunk of one sequence's vocabulary. It finds the number n of drafts that stand by itself (a
// warp reads the K pairs of probabilities), sums the chunk's weights in 64 bits and leaves the sum in the workspace; the
// sequence's last block to arrive walks the chunk sums to the chunk in which the running sum passes r * total, and that chunk
// (still in L2) to the token. The weights are never written. Bound by reading one row of p and one of q.
#include "../../include/plt_draft_verify.h"

#include <cuda_bf16.h>

#include <cstring>
#include <new>

#include "plt_handle.h"

using namespace plt;

namespace {

constexpr int kVerifyThreads = 256;
constexpr int kMinChunk = 2048, kMaxChunk = 16384;   // elements of a chunk: multiples of 8 * kVerifyThreads
constexpr int kOneWave = 592;                         // blocks that run at once (4 of 256 threads on each of 148 SMs)
constexpr int kMaxDrafts = 64;

thread_local char g_verify_error[512] = "";

}  // namespace

struct plt_draft_verify : HandleBase {
    plt_draft_verify_config cfg;
    double* sums = nullptr;      // [batch, chunks] of a call
    uint32_t* arrived = nullptr; // [max_batch] blocks of a sequence that have left their sum; 0 between calls
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
    uint32_t* arrived;
    uint32_t* status;
    int32_t K, V, chunk, chunks;
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
    int V;
    // a - b where that is finite and above 0, else 0. The test is made in fp32, where it is exact: 64-bit units are few.
    __device__ __forceinline__ double weight(float a, float b) const {
        const bool counts = a > b && a <= 3.402823466e38f && b >= -3.402823466e38f;
        return (double)(counts ? a : 0.f) - (double)(counts ? b : 0.f);
    }
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

// The same over the weights [first, last) of a row, at most kMaxChunk of them, with loads that lie together: a warp takes an
// eighth, its lanes N neighbouring weights at a time.
template <typename T>
__device__ int walk_row(const Row<T>& row, int first, int last, double before, double limit, double* s_warp, int* s_first) {
    constexpr int N = kVec<T>, STEPS = kMaxChunk / (kVerifyThreads * N);
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int per = (last - first + kVerifyThreads * N - 1) / (kVerifyThreads * N);   // steps of a warp, at most STEPS
    const int lo = first + wid * per * 32 * N + lane * N;
    double own[STEPS], sum = 0.0;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        own[s] = 0.0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int i = lo + s * 32 * N + k;
            if (s < per && i < last) own[s] += row.at(i);
        }
        sum += own[s];
    }
    sum = warp_sum(sum);
    __syncthreads();
    if (lane == 0) s_warp[wid] = sum;
    __syncthreads();
    int warp = -1;
    double base = before;
#pragma unroll
    for (int w = 0; w < kVerifyThreads / 32; ++w) {
        const double v = s_warp[w];
        if (v > 0.0) {
            if (warp >= 0) base += s_warp[warp];
            warp = w;
            if (base + v > limit) break;
        }
    }
    if (threadIdx.x == 0) *s_first = -1;
    __syncthreads();
    if (wid == warp) {
        // the step, then the lane, then the weight; `pick` is the last candidate seen where none passes the limit
        int pick = -1;
        double at_pick = 0.0;
        bool done = false;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s >= per || done) break;
            double upto = own[s];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double y = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += y;
            }
            const uint32_t any = __ballot_sync(0xffffffffu, own[s] > 0.0);
            const uint32_t past = __ballot_sync(0xffffffffu, own[s] > 0.0 && base + upto > limit);
            if (any != 0) {
                const int l = past != 0 ? __ffs(past) - 1 : 31 - __clz(any);
                pick = s * 32 + l;
                at_pick = base + __shfl_sync(0xffffffffu, upto - own[s], l);
                done = past != 0;
            }
            base += __shfl_sync(0xffffffffu, upto, 31);
        }
        if (pick >= 0 && lane == (pick & 31)) {
            const int i0 = first + wid * per * 32 * N + (pick >> 5) * 32 * N + lane * N;
            int found = -1;
            double run = at_pick;
            for (int k = 0; k < N && i0 + k < last; ++k) {
                const double v = row.at(i0 + k);
                if (v > 0.0) {
                    found = i0 + k;
                    run += v;
                    if (run > limit) break;
                }
            }
            *s_first = found;
        }
    }
    __syncthreads();
    return *s_first;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kVerifyThreads, 4) plt_draft_verify_kernel(const __grid_constant__ VerifyParams p) {
    __shared__ double s_warp[kVerifyThreads / 32];
    __shared__ double s_base;
    __shared__ int s_first, s_n, s_len;
    __shared__ bool s_last;
    const int b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;

    // ---- how many drafts stand ---------------------------------------------------------------------------------
    if (wid == 0) {
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
        if (lane == 0) {
            s_n = n;
            s_len = len;
        }
        if (blockIdx.x == 0 && flags) atomicOr(p.status, flags);
    }
    __syncthreads();
    const int n = s_n;
    const bool cut = n < s_len;
    Row<T> row;
    row.p = (const T*)p.target + b * p.target_b + n * p.target_j;
    row.q = cut && p.draft != nullptr ? (const T*)p.draft + b * p.draft_b + n * p.draft_j : nullptr;
    row.without = cut && p.draft == nullptr ? p.draft_tokens[(int64_t)b * p.K + n] : -1;
    row.V = p.V;

    // ---- the chunk's sum ----------------------------------------------------------------------------------------
    // With VEC, chunks are laid on the 16-byte grid of the row of p (the row of q lies alike): chunk 0 starts up to
    // kVec - 1 elements in front of the row. Each of a thread's sums takes the elements in a fixed order.
    constexpr int N = kVec<T>;
    const int lead = VEC ? (int)(((uintptr_t)row.p & 15) / sizeof(T)) : 0;
    const int c0 = (int)blockIdx.x * p.chunk - lead;          // may be below 0
    double sum = 0.0;
    if constexpr (VEC) {
        constexpr int U = 16 / N;         // vectors in flight: 16 elements of each row
        for (int i0 = c0 + tid * N; i0 < min(c0 + p.chunk, p.V); i0 += kVerifyThreads * N * U) {
            float a[U][N], q[U][N];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kVerifyThreads * N;
#pragma unroll
                for (int k = 0; k < N; ++k) a[u][k] = q[u][k] = 0.f;
                if (u * kVerifyThreads * N >= p.chunk) continue;     // the chunk's end (the same for the whole block)
                if (i >= 0 && i + N <= p.V) {
                    load_vec16<T>(row.p + i, a[u]);
                    if (row.q != nullptr) load_vec16<T>(row.q + i, q[u]);
                } else {
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        if (i + k >= 0 && i + k < p.V) {
                            a[u][k] = widen(row.p[i + k]);
                            if (row.q != nullptr) q[u][k] = widen(row.q[i + k]);
                        }
                }
                if (row.without >= i && row.without < i + N)
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        if (i + k == row.without) a[u][k] = 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < N; ++k) sum += row.weight(a[u][k], q[u][k]);
        }
    } else {
        constexpr int U = 16;
        for (int i0 = c0 + tid; i0 < min(c0 + p.chunk, p.V); i0 += kVerifyThreads * U) {
            float a[U], q[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kVerifyThreads;
                const bool in = i < min(c0 + p.chunk, p.V) && i != row.without;
                a[u] = in ? widen(row.p[i]) : 0.f;
                q[u] = in && row.q != nullptr ? widen(row.q[i]) : 0.f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) sum += row.weight(a[u], q[u]);
        }
    }
    sum = warp_sum(sum);
    if (lane == 0) s_warp[wid] = sum;
    __syncthreads();
    if (tid == 0) {
        double total = 0.0;
#pragma unroll
        for (int w = 0; w < kVerifyThreads / 32; ++w) total += s_warp[w];
        p.sums[(int64_t)b * p.chunks + blockIdx.x] = total;
        __threadfence();
        s_last = atomicAdd(&p.arrived[b], 1u) == (uint32_t)(p.chunks - 1);
    }
    __syncthreads();
    if (!s_last) return;

    // ---- the sequence's last block: the token --------------------------------------------------------------------
    __threadfence();
    const double* sums = p.sums + (int64_t)b * p.chunks;
    const double r = (double)p.sample_u[b];
    int token = -1;
    double before = 0.0, total = 0.0;
    const int c = walk(p.chunks, [&](int i) { return __ldcg(sums + i); }, before, total, r, s_warp, &s_first, &s_base);
    if (total > 0.0) {
        const int first = max(c * p.chunk - lead, 0), last = min((c + 1) * p.chunk - lead, p.V);
        token = walk_row(row, first, last, before, r * total, s_warp, &s_first);
    } else if (cut) {
        // p lies nowhere above q: the whole of p
        row.q = nullptr;
        row.without = -1;
        token = walk(p.V, [&](int i) { return row.at(i); }, before, total, r, s_warp, &s_first, &s_base);
    }
    for (int j = tid; j <= p.K; j += kVerifyThreads)
        p.tokens[(int64_t)b * (p.K + 1) + j] = j < n ? p.draft_tokens[(int64_t)b * p.K + j] : j == n ? token : -1;
    if (tid == 0) {
        p.num_accepted[b] = n;
        if (p.new_lens != nullptr) p.new_lens[b] = max(0, p.seq_lens[b] - (p.K - n));
        if (token < 0) atomicOr(p.status, kDevNoProbability);
        p.arrived[b] = 0;
    }
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

// Chunks of a row: of a length that lets all blocks of the batch run at once, or the longest. A row may start up to 7 elements
// behind a place of the 16-byte grid (`lead`).
int chunk_of(int batch, int vocab, int lead) {
    int chunk = kMinChunk;
    while (chunk < kMaxChunk && (int64_t)batch * ((vocab + lead + chunk - 1) / chunk) > kOneWave) chunk <<= 1;
    return chunk;
}

// Sums that any batch up to the largest leaves.
size_t sums_of(const plt_draft_verify_config* c) {
    const size_t most = (size_t)c->max_batch * ((c->vocab + 7 + kMaxChunk - 1) / kMaxChunk);
    return most > kOneWave ? most : kOneWave;
}

size_t workspace_of(const plt_draft_verify_config* c) {
    return 8u * sums_of(c) + 4u * (size_t)c->max_batch + 256;
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
    s = check_device(config->device, g_verify_error, nullptr);
    if (s != PLT_OK) return s;
    plt_draft_verify* h = new (std::nothrow) plt_draft_verify();
    if (!h) return verify_fail(nullptr, PLT_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->cfg = *config;
    h->device = config->device;
    const size_t bytes = workspace_of(config);
    void* ws = nullptr;
    if (cudaMalloc(&ws, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        delete h;
        return handle_fail(nullptr, g_verify_error, PLT_ERR_OUT_OF_MEMORY, "cudaMalloc of %zu workspace bytes failed", bytes);
    }
    h->status = (uint32_t*)ws;
    h->sums = (double*)((char*)ws + 256);
    h->arrived = (uint32_t*)(h->sums + sums_of(config));
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
    p.sums = h->sums; p.arrived = h->arrived; p.status = h->status;
    p.K = c.max_drafts; p.V = c.vocab;
    // 16-byte loads where the rows of p and q that one sequence needs lie alike on the 16-byte grid: always without q
    // (chunks follow p's rows), else where both bases are aligned and all strides are whole vectors.
    const int unit = 16 / es;
    const bool vec = !a->draft_probs || (!misaligned(a->target_probs, 16) && !misaligned(a->draft_probs, 16) && p.target_b % unit == 0 &&
                                         p.target_j % unit == 0 && p.draft_b % unit == 0 && p.draft_j % unit == 0);
    const bool on_grid = !misaligned(a->target_probs, 16) && p.target_b % unit == 0 && p.target_j % unit == 0;
    const int lead = vec && !on_grid ? unit - 1 : 0;
    p.chunk = chunk_of(a->batch, c.vocab, lead);
    p.chunks = (c.vocab + lead + p.chunk - 1) / p.chunk;
    DeviceScope scope(h->device);
    if (scope.err != cudaSuccess) return handle_fail(h, g_verify_error, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    const dim3 grid((unsigned)p.chunks, (unsigned)a->batch);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (c.dtype == PLT_F32) {
        if (vec) plt_draft_verify_kernel<float, true><<<grid, kVerifyThreads, 0, stream>>>(p);
        else plt_draft_verify_kernel<float, false><<<grid, kVerifyThreads, 0, stream>>>(p);
    } else {
        if (vec) plt_draft_verify_kernel<__nv_bfloat16, true><<<grid, kVerifyThreads, 0, stream>>>(p);
        else plt_draft_verify_kernel<__nv_bfloat16, false><<<grid, kVerifyThreads, 0, stream>>>(p);
    }
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return handle_fail(h, g_verify_error, PLT_ERR_CUDA, "launching the kernel: %s", cudaGetErrorString(e));
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

// Merge of a decode step with shared prefixes: for every row the partials of its group's prefix and of its own cache are joined
// by their references into one softmax, the window's likewise, and the gate mixes the two (Eq. 2). A block has 32 neighbouring rows
// of a KV head; what there is to know of them is found out once, by its first warp (with every thread for itself that took longer
// than the joining). A thread then holds 8 of a row's elements and a warp all 32 rows, so that the prefix's partials, which lie
// [d / 4][128 rows][4], are read 512 bytes at a time, those of four partials and the first of the own cache and of the window
// together. Where there are not many rows, four or sixteen warps work on each at the same time (two or fourteen take the prefix's
// partials in turn, one the own cache's, one the window's) and meet in shared memory. Everything up to the store is fp32, in an order
// that the plan and the batch alone decide. Bound by latency and by reading the partials (from L2): 3 to 5 us behind the last of them.
#include <cuda_bf16.h>

#include "plt_prefix.h"
#include "plt_ptx.cuh"

namespace plt {
namespace {

constexpr uint64_t kMergeWaitNs = 1000000000ull;

// Warps of a block that hold 8 elements each of the same 32 rows, and warps that share one such piece (1: none).
__host__ __device__ constexpr int merge_parts(int shares) { return shares == 1 ? 8 : shares == 4 ? 4 : 1; }

// N partials of a row, on their way: (reference, sum) and 8 elements each.
template <int N>
struct Parts {
    float2 ml[N];
    float4 v[N][2];
    // Partials k0 .. of `n`: part(k, ml, acc, step) says where partial k's (reference, sum) and its elements (two pieces of four,
    // `step` floats apart) lie.
    template <typename F>
    __device__ __forceinline__ void load(int k0, int n, F part) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            ml[u] = make_float2(-INFINITY, 0.f);
            v[u][0] = v[u][1] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (k0 + u < n) {
                const float2* m;
                const float* acc;
                int step;
                part(k0 + u, m, acc, step);
                ml[u] = *m;
                v[u][0] = *(const float4*)acc;
                v[u][1] = *(const float4*)(acc + step);
            }
        }
    }
    // Joins them into y, top and sum.
    __device__ __forceinline__ void join(float (&y)[8], float& top, float& sum) const {
        float m = top;
#pragma unroll
        for (int u = 0; u < N; ++u) m = fmaxf(m, ml[u].x);
        if (m == -INFINITY) return;              // nothing seen yet
        const float old = exp2f(top - m);
        top = m;
        sum *= old;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= old;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (ml[u].x == -INFINITY) continue;  // saw no key: what lies there was not written
            const float f = exp2f(ml[u].x - m);
            sum = fmaf(ml[u].y, f, sum);
            y[0] = fmaf(v[u][0].x, f, y[0]);
            y[1] = fmaf(v[u][0].y, f, y[1]);
            y[2] = fmaf(v[u][0].z, f, y[2]);
            y[3] = fmaf(v[u][0].w, f, y[3]);
            y[4] = fmaf(v[u][1].x, f, y[4]);
            y[5] = fmaf(v[u][1].y, f, y[5]);
            y[6] = fmaf(v[u][1].z, f, y[6]);
            y[7] = fmaf(v[u][1].w, f, y[7]);
        }
    }
};
// Joins the partials behind the `have` that have been joined.
template <int N, typename F>
__device__ __forceinline__ void join_rest(int have, int n, F part, float (&y)[8], float& top, float& sum) {
    for (int k = have; k < n; k += N) {
        Parts<N> more;
        more.load(k, n, part);
        more.join(y, top, sum);
    }
}

// What a block knows of each of its rows.
struct RowInfo {
    int64_t part[32];      // prefix: 128-row tile where the row's partials start
    float gate[32];
    int32_t n[32];         // prefix partials
    int32_t step[32];      // 128-row tiles from one to the next, and below that the row in the tile: step * 128 + row
    int32_t own[32];       // item of the own cache, or -1: no key
    int32_t window[32];    // item of the window, or -1
    int32_t at[32];        // the row among an item's
    int32_t out[32];       // row of the output, or -1: none; bit 30: the row has no token
};

// The partials of one item of the split-KV kernel for one row: the first one's row, and how many.
struct Item {
    int64_t row;
    int n;
};
__device__ __forceinline__ Item item_of(const Params& p, int item, int at) {
    const int2 c = item >= 0 ? *(const int2*)(p.item_blocks + 2 * item) : make_int2(0, -1);
    return {slot_of(max(item, 0), c.x) * p.hpc * p.R + at, c.y - c.x + 1};
}

template <int D, int SHARES>
__global__ void __launch_bounds__(merge_parts(SHARES) * SHARES * 32, 2) plt_prefix_merge(const __grid_constant__ Params p, const __grid_constant__ PrefixParams pp) {
    constexpr bool SPLIT = SHARES > 1;
    constexpr int PARTS = merge_parts(SHARES), OWN = SHARES - 2, WINDOW = SHARES - 1;      // shares 0 .. OWN - 1: the prefix's partials
    __shared__ RowInfo s;
    __shared__ float s_join[SPLIT ? SHARES - 1 : 1][10][SPLIT ? PARTS * 32 : 1];       // (reference, sum, 8 elements) of the other warps
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, share = SPLIT ? wid / PARTS : 0;
    const int part = blockIdx.z * PARTS + wid % PARTS;                        // elements 8 part .. 8 part + 7
    const int h = blockIdx.y;
    bool last = false;
    if (wid == 0) {
        // what the caller passed, and the plan, while the main kernel drains
        if (!acquire_word(pp.plan.ready, kMergeWaitNs)) atomicOr(pp.status, kDevWaitTimeout);
        if (lane == 0) last = atomicAdd(pp.plan.ready + 1, 1u) + 1 == gridDim.x * gridDim.y * gridDim.z;
        const int id = blockIdx.x * 32 + lane;
        const bool in = id < p.B * p.R;
        const int b = in ? small_div(id, p.R) : 0;
        const int r = in ? id - b * p.R : 0;
        const int lq = small_div(r, p.G), l = small_div(lq, p.Qn), newer = p.Qn - 1 - (lq - l * p.Qn), head = h * p.G + (r - lq * p.G);
        const PrefixPlan& plan = pp.plan;
        int group = -1, len = 0, begin = 0, end = 0;
        if (pp.groups > 0) {
            begin = plan.begin[0];
            end = plan.begin[pp.groups];
            if (b >= begin && b < end) {
                int lo = 0, hi = pp.groups;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1, at = plan.begin[mid];
                    if (at <= b) {
                        lo = mid;
                        begin = at;
                    } else {
                        hi = mid;
                        end = at;
                    }
                }
                group = lo;
                len = plan.len[lo];
            }
        }
        const int cut = row_sees(pp.seq_lens[b], (int64_t)len + p.max_seq_len, p.delta[l], newer), sees = min(cut, len);
        const int wl = l > 0 ? plan.win_lens[b * (p.L - 1) + l - 1] : 0;
        const bool has_own = in && plan.own_lens[b] - p.delta[l] > newer, has_window = in && cut > 0 && wl > 0;
        float gate = 0.f;
        if (l > 0) gate = 1.f / (1.f + expf(-p.gate_logits[(((int64_t)b * (p.L - 1) + (l - 1)) * p.Qn + (lq - l * p.Qn)) * p.Hq + head]));
        int64_t tile = 0;
        int count = 0, step = 1, row = 0;
        if (in && sees > 0) {
            const int rows = (end - begin) * p.R, nm = (rows + kPrefixRows - 1) / kPrefixRows;
            const int tiles = (len + kPrefixTile - 1) / kPrefixTile, chunk = *plan.chunk;
            const int lr = (b - begin) * p.R + r, m = lr / kPrefixRows, u = h * nm + m;
            if (chunk > 0) {
                count = small_div(tiles + chunk - 1, chunk);
                tile = plan.piece[group] + (int64_t)u * count;
            } else {
                const int T = plan.line[pp.groups], first = plan.line[group] + u * (tiles + kPrefixLead) + kPrefixLead;
                const int C = prefix_blocks(T, plan.chunk[1]), c0 = prefix_block_of(first, T, C);
                count = prefix_block_of(first + tiles - 1, T, C) - c0 + 1;
                tile = (int64_t)plan.unit[group] + u + c0;
            }
            // a unit of more than 128 rows has one tile for each half of them, else both tiles are partials of the same rows
            row = lr & 127;
            tile *= 2;
            if (rows - m * kPrefixRows > 128) {
                tile += (lr >> 7) & 1;
                step = 2;
            } else if (chunk > 0 && count == tiles) {
                step = 2;              // pieces of one key tile each: the first tile's
            } else {
                count *= 2;
            }
        }
        s.part[lane] = tile;
        s.n[lane] = count;
        s.step[lane] = step * 128 + row;
        s.gate[lane] = gate;
        s.out[lane] = in ? ((b * p.L * p.Qn + lq) * p.Hq + head) | (cut > 0 ? 0 : 1 << 30) : -1;
        const int hg = small_div(h, p.hpc), item = item_index(p, b, hg, 0);
        s.own[lane] = has_own ? item : -1;
        s.window[lane] = has_window ? item + 1 : -1;
        s.at[lane] = (h - hg * p.hpc) * p.R + r;
    }
    __syncthreads();
    grid_dependency_wait();
    if (last) pp.plan.ready[0] = pp.plan.ready[1] = 0;      // every block of the main kernel and of this one has acquired the plan

    // ---- one softmax over the prefix and the own keys, and the window's ---------------------------------------------------
    const bool does_own = !SPLIT || share == OWN, does_window = !SPLIT || share == WINDOW;
    const Item own = item_of(p, does_own ? s.own[lane] : -1, s.at[lane]), window = item_of(p, does_window ? s.window[lane] : -1, s.at[lane]);
    float y[8], z[8], top = -INFINITY, sum = 0.f, top_w = -INFINITY, sum_w = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = z[i] = 0.f;
    constexpr int EVERY = SPLIT ? OWN : 1;
    const int prefix_step = s.step[lane] >> 7, row = s.step[lane] & 127;
    const int64_t tile = s.part[lane] + share * prefix_step;
    const int n_prefix = !SPLIT || share < OWN ? (s.n[lane] - share + EVERY - 1) / EVERY : 0;
    auto of_prefix = [&](int k, const float2*& m, const float*& acc, int& apart) {
        const int64_t at = (tile + k * EVERY * prefix_step) * 128;
        m = (const float2*)(pp.ml + (at + row) * 2);
        acc = pp.acc + at * D + part * 2 * 512 + row * 4;
        apart = 512;
    };
    const int64_t next = (int64_t)p.hpc * p.R;               // rows between the partials of one item
    auto of_item = [&](const Item& it) {
        return [=, &p](int k, const float2*& m, const float*& acc, int& apart) {
            const int64_t at = it.row + k * next;
            m = (const float2*)(p.part_ml + at * 2);
            acc = p.part_acc + at * D + part * 8;
            apart = 4;
        };
    };
    if constexpr (SPLIT) {
        if (share < OWN) join_rest<2>(0, n_prefix, of_prefix, y, top, sum);
        if (does_own) join_rest<2>(0, own.n, of_item(own), y, top, sum);
        if (does_window) join_rest<1>(0, window.n, of_item(window), z, top_w, sum_w);
    } else {
        // the first partials of all three are on their way together
        Parts<4> of_p;
        Parts<1> of_o, of_w;
        of_p.load(0, n_prefix, of_prefix);
        of_o.load(0, own.n, of_item(own));
        of_w.load(0, window.n, of_item(window));
        of_p.join(y, top, sum);
        join_rest<4>(4, n_prefix, of_prefix, y, top, sum);
        of_o.join(y, top, sum);
        join_rest<4>(1, own.n, of_item(own), y, top, sum);
        of_w.join(z, top_w, sum_w);
        join_rest<1>(1, window.n, of_item(window), z, top_w, sum_w);
    }
    if (does_window) {
        const float f = sum_w > 0.f ? s.gate[lane] / sum_w : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= f;
    }
    if (SPLIT) {
        const int t = (wid % PARTS) * 32 + lane;
        if (share > 0) {
            s_join[share - 1][0][t] = top;
            s_join[share - 1][1][t] = sum;
#pragma unroll
            for (int i = 0; i < 8; ++i) s_join[share - 1][2 + i][t] = share == WINDOW ? z[i] : y[i];
        }
        __syncthreads();
        if (share > 0) return;
        float all = top;
#pragma unroll
        for (int o = 0; o < OWN; ++o) all = fmaxf(all, s_join[o][0][t]);
        if (all > -INFINITY) {
            const float own_f = exp2f(top - all);      // 0 for one that saw nothing
            sum *= own_f;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] *= own_f;
#pragma unroll
            for (int o = 0; o < OWN; ++o) {
                const float f = exp2f(s_join[o][0][t] - all);
                sum = fmaf(s_join[o][1][t], f, sum);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = fmaf(s_join[o][2 + i][t], f, y[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = s_join[WINDOW - 1][2 + i][t];
    }
    const int out = s.out[lane];
    if (out < 0) return;
    const float ig = sum > 0.f ? (1.f - s.gate[lane]) / sum : 0.f;
    const bool token = (out >> 30 & 1) == 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = token ? fmaf(y[i], ig, z[i]) : 0.f;
    uint4* dst = (uint4*)((__nv_bfloat16*)p.out + (int64_t)(out & ~(1 << 30)) * D + part * 8);
    *dst = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
}

}  // namespace

namespace {

template <int D, int SHARES>
cudaError_t launch(const Params& p, const PrefixParams& pp, bool overlap, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.B * p.R + 31) / 32), (unsigned)p.Hkv, (unsigned)(D / (8 * merge_parts(SHARES))));
    cfg.blockDim = dim3(merge_parts(SHARES) * SHARES * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = overlap ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, plt_prefix_merge<D, SHARES>, p, pp);
}

template <int D>
cudaError_t launch_for(const Params& p, const PrefixParams& pp, bool overlap, cudaStream_t stream) {
    // Four warps to a row as long as all run at once (32 on each multiprocessor): the step of two users 15.7 us against 16.4, drafts of
    // 21 sequences 21.9 against 22.7, 32 sequences of two loops 27.7 against 28.3; where they do not, 64 of two loops 40.2 against 36.2,
    // 128 of them 153 against 146. Sixteen where few units of long prefixes may have been cut into many pieces (one sequence of 2 heads
    // behind 12615 tokens 21.8 us against 29.0, 6 of 4 heads behind two prefixes of 32705 31.5 against 37.2; short prefixes lose half a
    // microsecond).
    const int64_t warps = (int64_t)(p.B * p.R + 31) / 32 * p.Hkv * (D / 8);
    const int pieces = min(pp.blocks / p.Hkv, (pp.max_prefix_len + kPrefixTile - 1) / kPrefixTile);      // of a unit, at most
    if (warps * 16 <= pp.blocks * 32 && pieces > 8) return launch<D, 16>(p, pp, overlap, stream);
    return warps * 4 <= pp.blocks * 32 ? launch<D, 4>(p, pp, overlap, stream) : launch<D, 1>(p, pp, overlap, stream);
}

}  // namespace

cudaError_t launch_prefix_merge(const Params& p, const PrefixParams& pp, bool overlap, cudaStream_t stream) {
    return p.d == 128 ? launch_for<128>(p, pp, overlap, stream) : launch_for<64>(p, pp, overlap, stream);
}

}  // namespace plt

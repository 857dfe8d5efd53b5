// Merge of a decode step with shared prefixes: for every row the partials of its group's prefix and of its own cache are joined
// by their references into one softmax, the window's likewise, and the gate mixes the two (Eq. 2). A thread holds 8 of a row's
// elements and a warp 32 neighbouring rows, so that the prefix's partials, which lie [d / 4][128 rows][4], are read 512 bytes at
// a time; the loads of four partials are in flight together. Everything up to the store is fp32. Bound by reading the partials
// (from L2) and by latency.
#include <cuda_bf16.h>

#include "plt_prefix.h"
#include "plt_ptx.cuh"

namespace plt {
namespace {

constexpr int kMergeBatch = 4;
constexpr int kMergeParts = 4;       // warps of a block: 8 elements each of the same 32 rows

// Joins `n` partials of a row into y, top and sum: part(k, ml, acc, step) says where partial k's (reference, sum) and its
// elements (two pieces of four, `step` floats apart) lie.
template <typename F>
__device__ __forceinline__ void join(int n, F part, float (&y)[8], float& top, float& sum) {
    for (int k0 = 0; k0 < n; k0 += kMergeBatch) {
        float2 ml[kMergeBatch];
        float4 v[kMergeBatch][2];
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) {
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
        float m = top;
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) m = fmaxf(m, ml[u].x);
        if (m == -INFINITY) continue;            // nothing seen yet
        const float old = exp2f(top - m);
        top = m;
        sum *= old;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= old;
#pragma unroll
        for (int u = 0; u < kMergeBatch; ++u) {
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
}

// The pieces of one item of the split-KV kernel for one row.
struct Own {
    int64_t row0, step;   // row of the first piece's partial, rows between pieces
    int n;
};
__device__ __forceinline__ Own own_pieces(const Params& p, int item, int hl, int r) {
    const int2 c = *(const int2*)(p.item_blocks + 2 * item);
    Own o;
    o.row0 = (slot_of(item, c.x) * p.hpc + hl) * p.R + r;
    o.step = (int64_t)p.hpc * p.R;
    o.n = c.y - c.x + 1;
    return o;
}

template <int D>
__global__ void __launch_bounds__(kMergeParts * 32, 6) plt_prefix_merge(const __grid_constant__ Params p, const __grid_constant__ PrefixParams pp) {
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, part = blockIdx.z * kMergeParts + (threadIdx.x >> 5);   // elements 8 part .. 8 part + 7
    const int h = blockIdx.y;
    const int64_t id = (int64_t)blockIdx.x * 32 + lane;
    const bool in = id < (int64_t)p.B * p.R;
    const int b = in ? (int)(id / p.R) : 0, r = in ? (int)(id - (int64_t)b * p.R) : 0;
    const int lq = r / p.G, l = lq / p.Qn, newer = p.Qn - 1 - lq % p.Qn, head = h * p.G + (r - lq * p.G);

    // what the caller passed and the plan, complete since before the main kernel let this one go
    int group = -1, len = 0;
    const PrefixPlan& plan = pp.plan;
    if (pp.groups > 0 && b >= plan.begin[0] && b < plan.begin[pp.groups]) {
        int lo = 0, hi = pp.groups;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (plan.begin[mid] <= b) lo = mid; else hi = mid;
        }
        group = lo;
        len = plan.len[lo];
    }
    const int n = (int)min((int64_t)pp.seq_lens[b], (int64_t)len + p.max_seq_len);
    const int cut = max(0, n - p.delta[l] - newer), sees = min(cut, len);
    const int own_cut = max(0, plan.own_lens[b] - p.delta[l] - newer);
    const int wl = l > 0 ? plan.win_lens[b * (p.L - 1) + l - 1] : 0;
    float gate = 0.f;
    if (l > 0) gate = 1.f / (1.f + expf(-p.gate_logits[(((int64_t)b * (p.L - 1) + (l - 1)) * p.Qn + (lq - l * p.Qn)) * p.Hq + head]));

    // the prefix's partials for this row: slots s0 .. s0 + ns - 1, tile x0 (or both)
    int64_t s0 = 0;
    int ns = 0, x0 = 0, row = 0;
    bool both = false;
    if (in && sees > 0) {
        const int rows = (plan.begin[group + 1] - plan.begin[group]) * p.R, nm = (rows + kPrefixRows - 1) / kPrefixRows;
        const int tiles = (len + kPrefixTile - 1) / kPrefixTile, chunk = *plan.chunk;
        const int lr = (b - plan.begin[group]) * p.R + r, m = lr / kPrefixRows, u = h * nm + m;
        if (chunk > 0) {
            ns = (tiles + chunk - 1) / chunk;
            s0 = plan.piece[group] + (int64_t)u * ns;
        } else {
            const int T = plan.line[pp.groups], first = plan.line[group] + u * (tiles + kPrefixLead) + kPrefixLead;
            const int C = prefix_blocks(T, pp.blocks), c0 = prefix_block_of(first, T, C);
            ns = prefix_block_of(first + tiles - 1, T, C) - c0 + 1;
            s0 = (int64_t)plan.unit[group] + u + c0;
        }
        row = lr & 127;
        both = rows - m * kPrefixRows <= 128;
        x0 = both ? 0 : (lr >> 7) & 1;
    }
    const int hg = h / p.hpc, hl = h - hg * p.hpc;

    grid_dependency_wait();
    Own og = {0, 0, 0}, ow = {0, 0, 0};
    if (in && own_cut > 0) og = own_pieces(p, item_index(p, b, hg, 0), hl, r);
    if (in && cut > 0 && wl > 0) ow = own_pieces(p, item_index(p, b, hg, 1), hl, r);

    // ---- one softmax over the prefix and the own keys ---------------------------------------------------------------
    float y[8], z[8], top = -INFINITY, sum = 0.f, top_w = -INFINITY, sum_w = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = z[i] = 0.f;
    join(both ? 2 * ns : ns, [&](int k, const float2*& m, const float*& acc, int& step) {
        const int64_t at = (both ? s0 * 2 + k : (s0 + k) * 2 + x0) * 128;
        m = (const float2*)(pp.ml + (at + row) * 2);
        acc = pp.acc + at * D + part * 2 * 512 + row * 4;
        step = 512;
    }, y, top, sum);
    join(og.n, [&](int k, const float2*& m, const float*& acc, int& step) {
        const int64_t at = og.row0 + k * og.step;
        m = (const float2*)(p.part_ml + at * 2);
        acc = p.part_acc + at * D + part * 8;
        step = 4;
    }, y, top, sum);
    // ---- the window -----------------------------------------------------------------------------------------------------
    join(ow.n, [&](int k, const float2*& m, const float*& acc, int& step) {
        const int64_t at = ow.row0 + k * ow.step;
        m = (const float2*)(p.part_ml + at * 2);
        acc = p.part_acc + at * D + part * 8;
        step = 4;
    }, z, top_w, sum_w);
    const float ig = sum > 0.f ? (1.f - gate) / sum : 0.f, il = sum_w > 0.f ? gate / sum_w : 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = cut > 0 ? fmaf(z[i], il, y[i] * ig) : 0.f;
    if (!in) return;
    uint4* dst = (uint4*)((__nv_bfloat16*)p.out + (((int64_t)b * p.L * p.Qn + lq) * p.Hq + head) * D + part * 8);
    *dst = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
}

}  // namespace

cudaError_t launch_prefix_merge(const Params& p, const PrefixParams& pp, bool overlap, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(((int64_t)p.B * p.R + 31) / 32), (unsigned)p.Hkv, (unsigned)(p.d / (8 * kMergeParts)));
    cfg.blockDim = dim3(kMergeParts * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = overlap ? 1 : 0;
    return p.d == 128 ? cudaLaunchKernelEx(&cfg, plt_prefix_merge<128>, p, pp) : cudaLaunchKernelEx(&cfg, plt_prefix_merge<64>, p, pp);
}

}  // namespace plt

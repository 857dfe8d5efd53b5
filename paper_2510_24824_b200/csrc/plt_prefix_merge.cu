// Merge of a decode step with shared prefixes: for every row the partials of its group's prefix and of its own cache are joined
// by their references into one softmax, the window's likewise, and the gate mixes the two (Eq. 2). A thread holds 16 of a row's
// elements and a warp 32 neighbouring rows, so that the prefix's partials, which lie [d / 4][128 rows][4], are read 512 bytes at
// a time. Everything up to the store is fp32. Bound by reading the partials (from L2) and by latency.
#include <cuda_bf16.h>

#include "plt_prefix.h"
#include "plt_ptx.cuh"

namespace plt {
namespace {

// Adds f times 16 elements that lie in four pieces of four, `step` floats apart.
__device__ __forceinline__ void add16(float (&y)[16], const float* src, int64_t step, float f) {
    float4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = *(const float4*)(src + k * step);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        y[4 * k] = fmaf(v[k].x, f, y[4 * k]);
        y[4 * k + 1] = fmaf(v[k].y, f, y[4 * k + 1]);
        y[4 * k + 2] = fmaf(v[k].z, f, y[4 * k + 2]);
        y[4 * k + 3] = fmaf(v[k].w, f, y[4 * k + 3]);
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
__global__ void __launch_bounds__(D * 2) plt_prefix_merge(const __grid_constant__ Params p, const __grid_constant__ PrefixParams pp) {
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;       // elements 16 part .. 16 part + 15
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

    // the prefix's pieces for this row: blocks c0 .. c1, tile x0 (and x1)
    int64_t unit = 0;
    int c0 = 0, c1 = -1, x0 = 0, x1 = 0, row = 0;
    if (in && sees > 0) {
        const int rows = (plan.begin[group + 1] - plan.begin[group]) * p.R, nm = (rows + kPrefixRows - 1) / kPrefixRows;
        const int tiles = (len + kPrefixTile - 1) / kPrefixTile, per = tiles + kPrefixLead;
        const int lr = (b - plan.begin[group]) * p.R + r, m = lr / kPrefixRows;
        const int64_t T = plan.line[pp.groups], first = plan.line[group] + (int64_t)(h * nm + m) * per + kPrefixLead;
        const int C = prefix_blocks(T, pp.blocks);
        c0 = prefix_block_of(first, T, C);
        c1 = prefix_block_of(first + tiles - 1, T, C);
        unit = plan.unit[group] + h * nm + m;
        row = lr & 127;
        const bool wide = rows - m * kPrefixRows > 128;
        x0 = wide ? (lr >> 7) & 1 : 0;
        x1 = wide ? x0 : 1;
    }
    const int hg = h / p.hpc, hl = h - hg * p.hpc;

    grid_dependency_wait();
    Own og = {0, 0, 0}, ow = {0, 0, 0};
    if (in && own_cut > 0) og = own_pieces(p, item_index(p, b, hg, 0), hl, r);
    if (in && cut > 0 && wl > 0) ow = own_pieces(p, item_index(p, b, hg, 1), hl, r);

    // ---- one softmax over the prefix and the own keys ---------------------------------------------------------------
    float top = -INFINITY;
    for (int c = c0; c <= c1; ++c)
        for (int x = x0; x <= x1; ++x) top = fmaxf(top, pp.ml[(((unit + c) * 2 + x) * 128 + row) * 2]);
    for (int i = 0; i < og.n; ++i) top = fmaxf(top, p.part_ml[(og.row0 + i * og.step) * 2]);
    float y[16], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = 0.f;
    if (top > -INFINITY) {
        for (int c = c0; c <= c1; ++c)
            for (int x = x0; x <= x1; ++x) {
                const int64_t at = ((unit + c) * 2 + x) * 128;
                const float2 ml = *(const float2*)(pp.ml + (at + row) * 2);
                if (ml.x == -INFINITY) continue;      // saw no key: its sums were not written
                const float f = exp2f(ml.x - top);
                sum = fmaf(ml.y, f, sum);
                add16(y, pp.acc + at * D + part * 4 * 512 + row * 4, 512, f);
            }
        for (int i = 0; i < og.n; ++i) {
            const int64_t at = og.row0 + i * og.step;
            const float2 ml = *(const float2*)(p.part_ml + at * 2);
            if (ml.x == -INFINITY) continue;
            const float f = exp2f(ml.x - top);
            sum = fmaf(ml.y, f, sum);
            add16(y, p.part_acc + at * D + part * 16, 4, f);
        }
    }
    const float ig = sum > 0.f ? (1.f - gate) / sum : 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] *= ig;
    // ---- the window -----------------------------------------------------------------------------------------------------
    if (ow.n > 0) {
        top = -INFINITY;
        sum = 0.f;
        for (int i = 0; i < ow.n; ++i) top = fmaxf(top, p.part_ml[(ow.row0 + i * ow.step) * 2]);
        if (top > -INFINITY) {
            for (int i = 0; i < ow.n; ++i) {
                const float2 ml = *(const float2*)(p.part_ml + (ow.row0 + i * ow.step) * 2);
                sum += ml.y * exp2f(ml.x - top);
            }
            const float il = sum > 0.f ? gate / sum : 0.f;
            for (int i = 0; i < ow.n; ++i) {
                const int64_t at = ow.row0 + i * ow.step;
                const float m = p.part_ml[at * 2];
                if (m > -INFINITY) add16(y, p.part_acc + at * D + part * 16, 4, exp2f(m - top) * il);
            }
        }
    }
    if (!in) return;
    if (cut == 0)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = 0.f;
    uint4* dst = (uint4*)((__nv_bfloat16*)p.out + (((int64_t)b * p.L * p.Qn + lq) * p.Hq + head) * D + part * 16);
    dst[0] = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]), pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
    dst[1] = make_uint4(pack_bf16x2(y[8], y[9]), pack_bf16x2(y[10], y[11]), pack_bf16x2(y[12], y[13]), pack_bf16x2(y[14], y[15]));
}

}  // namespace

cudaError_t launch_prefix_merge(const Params& p, const PrefixParams& pp, bool overlap, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(((int64_t)p.B * p.R + 31) / 32), (unsigned)p.Hkv);
    cfg.blockDim = dim3((unsigned)p.d * 2);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = overlap ? 1 : 0;
    return p.d == 128 ? cudaLaunchKernelEx(&cfg, plt_prefix_merge<128>, p, pp) : cudaLaunchKernelEx(&cfg, plt_prefix_merge<64>, p, pp);
}

}  // namespace plt

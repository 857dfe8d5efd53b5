// C ABI of cache eviction (plt_cache_evict.h): argument checks, workspace, the plan of the weights call and the launches.
#include "../../include/plt_cache_evict.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>

#include "plt_evict.h"

using namespace plt;

namespace {

thread_local char g_evict_create_error[512] = "";

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Scratch for scores: a batch whose scores at full length exceed this runs in several rounds of launches, each over a
// part of the batch. At 8 packed rows of d = 128 it holds the scores of 2 GB of keys. (Smaller parts, whose scores would stay in
// L2, cost more than they save: 8 sequences of 32768 codes, 16 rows, 104 us in one round, 122 us in parts of 72 MB, 145 us of 36.)
constexpr size_t kScoreScratch = (size_t)256 << 20;

struct EvictGeometry {
    int G, R, Qn, qsplit, hpg;   // packed rows per loop and token of a KV head (both maps), all packed rows
    bool bf16, fp8;
    ScoreVariant v;              // fp32: HPC, KW and tile_keys only
    int part;                    // sequences per round of launches
    size_t score_floats, ml_floats, mc_floats, items;
};

}  // namespace

struct plt_cache_evict {
    plt_cache_evict_config cfg;
    int32_t delta[kMaxLoops];
    int32_t min_delta = 0, max_delta = 0;
    EvictGeometry g;
    int sm_count = 0, score_grid = 0, add_grid = 0;
    size_t score_smem = 0, add_smem = 0;
    float scale_log2 = 0.f;
    float *scores = nullptr, *ml = nullptr, *mc = nullptr;
    int32_t* item_blocks = nullptr;
    uint32_t* status = nullptr;
    EncodeTiledFn encode = nullptr;
    char err[512];
};

namespace {

plt_status fail(plt_cache_evict_t h, plt_status code, const char* fmt, ...) {
    char* dst = h ? h->err : g_evict_create_error;
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(dst, 512, fmt, ap);
    va_end(ap);
    return code;
}

plt_status cuda_fail(plt_cache_evict_t h, const char* what, cudaError_t e) {
    return fail(h, PLT_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

int row_pitch(int rows) { return (rows + 3) & ~3; }
int key_pitch(const EvictGeometry& g) { return g.v.twice ? g.v.RS : row_pitch(g.R); }

plt_status check_config(const plt_cache_evict_config* c, EvictGeometry* g) {
    if (!c) return fail(nullptr, PLT_ERR_INVALID_ARG, "config is NULL");
    if (c->struct_size != sizeof(plt_cache_evict_config))
        return fail(nullptr, PLT_ERR_INVALID_ARG, "config.struct_size %u != %zu", c->struct_size, sizeof(plt_cache_evict_config));
    if (c->dtype != PLT_F32 && c->dtype != PLT_BF16) return fail(nullptr, PLT_ERR_INVALID_ARG, "unknown dtype %d", c->dtype);
    if (c->kv_dtype != PLT_KV_SAME && c->kv_dtype != PLT_KV_E4M3)
        return fail(nullptr, PLT_ERR_INVALID_ARG, "unknown kv_dtype %d", c->kv_dtype);
    if (c->max_batch < 1 || c->L < 1 || c->Hq < 1 || c->Hkv < 1 || c->max_seq_len < 1 || c->page_size < 0)
        return fail(nullptr, PLT_ERR_INVALID_ARG, "non-positive size in config");
    if (c->max_batch > kMaxBatch) return fail(nullptr, PLT_ERR_UNSUPPORTED, "max_batch %d > %d", c->max_batch, kMaxBatch);
    if (c->L > kMaxLoops) return fail(nullptr, PLT_ERR_UNSUPPORTED, "L %d > %d", c->L, kMaxLoops);
    if (c->max_seq_len > (1 << 24)) return fail(nullptr, PLT_ERR_UNSUPPORTED, "max_seq_len %d > 2^24", c->max_seq_len);
    if (c->Hq % c->Hkv != 0) return fail(nullptr, PLT_ERR_INVALID_ARG, "Hq %d is not a multiple of Hkv %d", c->Hq, c->Hkv);
    if (c->d != 64 && c->d != 128) return fail(nullptr, PLT_ERR_UNSUPPORTED, "head dim %d (supported: 64, 128)", c->d);
    g->bf16 = c->dtype == PLT_BF16;
    g->fp8 = c->kv_dtype == PLT_KV_E4M3;
    if (g->fp8 && (!g->bf16 || c->d != 128)) return fail(nullptr, PLT_ERR_UNSUPPORTED, "E4M3 caches need bf16 queries and head dim 128");
    if (c->q_len < 0) return fail(nullptr, PLT_ERR_INVALID_ARG, "q_len %d < 0", c->q_len);
    if (c->maps < 0 || c->maps > 2) return fail(nullptr, PLT_ERR_INVALID_ARG, "maps %d outside [0, 2]", c->maps);
    if (c->heads_per_group < 0) return fail(nullptr, PLT_ERR_INVALID_ARG, "heads_per_group %d < 0", c->heads_per_group);
    if (c->page_size % 16 != 0) return fail(nullptr, PLT_ERR_UNSUPPORTED, "page_size %d is not a multiple of 16", c->page_size);
    if (c->loop_offset)
        for (int l = 0; l < c->L; ++l)
            if (c->loop_offset[l] < 0) return fail(nullptr, PLT_ERR_INVALID_ARG, "loop_offset[%d] < 0", l);
    g->Qn = c->q_len > 1 ? c->q_len : 1;
    g->qsplit = c->maps == 2 ? 1 : 0;
    g->hpg = c->heads_per_group > 1 ? c->heads_per_group : 1;
    if (c->Hkv % g->hpg != 0)
        return fail(nullptr, PLT_ERR_INVALID_ARG, "heads_per_group %d does not divide Hkv %d", g->hpg, c->Hkv);
    const double rows = (double)c->L * g->Qn * (c->Hq / c->Hkv) * (1 + g->qsplit);
    if (rows > kMaxRows) return fail(nullptr, PLT_ERR_UNSUPPORTED, "maps * L * q_len * Hq/Hkv = %.0f packed rows > %d", rows, kMaxRows);
    // grids count blocks in 31 bits: compaction takes one for each sequence, head, cache and 64 bytes of a row and one more for
    // each group's totals, selection up to eight for each sequence and group
    const double pieces = c->d * (g->fp8 ? 1 : (g->bf16 ? 2 : 4)) / 64;
    if ((double)c->max_batch * c->Hkv * (2 * pieces + 8) >= 2147483647.0)
        return fail(nullptr, PLT_ERR_UNSUPPORTED, "max_batch %d * Hkv %d is more than a launch can count", c->max_batch, c->Hkv);
    g->G = (c->Hq / c->Hkv) << g->qsplit;
    g->R = c->L * g->Qn * g->G;
    if (g->bf16) {
        g->v = score_variant(c->d, g->R, c->Hkv, g->fp8, c->max_batch);
        if (g->v.smem > 227 * 1024) return fail(nullptr, PLT_ERR_UNSUPPORTED, "max_batch %d needs too much shared memory", c->max_batch);
    } else {
        g->v = ScoreVariant{c->d, 0, 1, 1, false, false, 1, 1, kEvictF32Keys, 0, scores_f32_smem(c->d, g->R, c->max_batch)};
    }
    const size_t tiles = ((size_t)c->max_seq_len + g->v.tile_keys - 1) / g->v.tile_keys + kEvictPieceCost;
    const size_t per = tiles * g->v.tile_keys * c->Hkv * key_pitch(*g);       // floats of a sequence's scores or sums
    size_t part = kScoreScratch / 4 / per;
    part = part < 1 ? 1 : (part > (size_t)c->max_batch ? (size_t)c->max_batch : part);
    g->part = (int)part;
    g->score_floats = part * per;
    // both plans' lines fit 31 bits
    if ((double)part * (c->Hkv / g->v.HPC) * tiles >= 2147483647.0)
        return fail(nullptr, PLT_ERR_UNSUPPORTED, "Hkv * max_seq_len too large for the tile plan");
    g->items = part * (c->Hkv / g->v.HPC) * 2;
    return PLT_OK;
}

size_t layout(const plt_cache_evict_config* c, EvictGeometry* g, int score_grid) {
    g->ml_floats = (g->items + score_grid) * g->v.HPC * g->v.KW * g->R * 2;
    g->mc_floats = (size_t)g->part * c->Hkv * row_pitch(g->R) * 2;
    g->ml_floats = (g->ml_floats + 3) & ~(size_t)3;       // the array behind is read 16 bytes at a time
    return (g->score_floats + g->ml_floats + g->mc_floats) * 4 + g->items * 8 + 256;
}

bool aligned(const void* p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

// Strides of a cache in elements (all 0: dense), checked as plt_decode_attn_run does.
plt_status cache_strides(plt_cache_evict_t h, int64_t& sb, int64_t& sn, int64_t& sh, int es) {
    const plt_cache_evict_config& c = h->cfg;
    if (sb == 0 && sn == 0 && sh == 0) {
        sh = c.d;
        sn = (int64_t)c.Hkv * c.d;
        sb = (int64_t)(c.page_size > 0 ? c.page_size : c.max_seq_len) * sn;
    }
    const int64_t unit = 16 / es;
    if (sb <= 0 || sn <= 0 || sh <= 0 || sb % unit || sn % unit || sh % unit)
        return fail(h, PLT_ERR_INVALID_ARG, "kv strides must be positive multiples of %lld elements", (long long)unit);
    if (sh < c.d) return fail(h, PLT_ERR_INVALID_ARG, "kv_stride_h %lld < d", (long long)sh);
    if ((double)sb * es >= 1099511627776.0 || (double)sn * es >= 1099511627776.0 || (double)sh * es >= 1099511627776.0)
        return fail(h, PLT_ERR_UNSUPPORTED, "kv stride of 2^40 bytes or more");
    return PLT_OK;
}

plt_status check_pages(plt_cache_evict_t h, const int32_t* page_table, int32_t max_pages, int32_t num_pool_pages) {
    const plt_cache_evict_config& c = h->cfg;
    if (c.page_size == 0) return PLT_OK;
    if (!page_table) return fail(h, PLT_ERR_INVALID_ARG, "page_table is NULL for a paged cache");
    const int need = (c.max_seq_len + c.page_size - 1) / c.page_size;
    if (max_pages < need) return fail(h, PLT_ERR_CAPACITY, "max_pages %d < %d", max_pages, need);
    if (num_pool_pages < 1) return fail(h, PLT_ERR_INVALID_ARG, "num_pool_pages %d < 1", num_pool_pages);
    return PLT_OK;
}

plt_status check_batch(plt_cache_evict_t h, int32_t batch) {
    if (batch < 0) return fail(h, PLT_ERR_INVALID_ARG, "batch %d < 0", batch);
    if (batch > h->cfg.max_batch) return fail(h, PLT_ERR_CAPACITY, "batch %d > max_batch %d", batch, h->cfg.max_batch);
    return PLT_OK;
}

plt_status check_totals(plt_cache_evict_t h, const void* weights, int64_t& stride) {
    if (!weights || !aligned(weights, 4)) return fail(h, PLT_ERR_INVALID_ARG, "weights must not be NULL and be 4-byte aligned");
    if (stride == 0) stride = h->cfg.max_seq_len;
    if (stride < h->cfg.max_seq_len)
        return fail(h, PLT_ERR_INVALID_ARG, "weights_stride %lld < max_seq_len %d", (long long)stride, h->cfg.max_seq_len);
    return PLT_OK;
}

plt_status encode_keys(plt_cache_evict_t h, CUtensorMap* map, const void* base, int64_t sb, int64_t sn, int64_t sh, int es, int64_t outer,
                       int kbox) {
    const plt_cache_evict_config& c = h->cfg;
    cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)(c.page_size > 0 ? c.page_size : c.max_seq_len), (cuuint64_t)c.Hkv, (cuuint64_t)outer};
    cuuint64_t strides[3] = {(cuuint64_t)(sn * es), (cuuint64_t)(sh * es), (cuuint64_t)(sb * es)};
    cuuint32_t box[4] = {(cuuint32_t)(128 / es), (cuuint32_t)kbox, (cuuint32_t)h->g.v.HPC, 1u};
    cuuint32_t estr[4] = {1u, 1u, 1u, 1u};
    const CUresult r = h->encode(map, es == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                                 const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(h, PLT_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d for the keys", (int)r);
    return PLT_OK;
}

plt_status create_on_device(plt_cache_evict* h) {
    const plt_cache_evict_config& c = h->cfg;
    EvictGeometry& g = h->g;
    cudaDeviceProp prop;
    cudaError_t e = cudaGetDeviceProperties(&prop, c.device);
    if (e != cudaSuccess) return cuda_fail(nullptr, "cudaGetDeviceProperties", e);
    if (prop.major != 10)
        return fail(nullptr, PLT_ERR_UNSUPPORTED, "device %d is sm_%d%d; this library is built for sm_100a only", c.device, prop.major,
                    prop.minor);
    h->sm_count = prop.multiProcessorCount;
    int blocks = 0;
    e = g.bf16 ? scores_prepare(g.v, &blocks) : scores_f32_prepare(c.d, g.R, c.max_batch, &blocks);
    if (e != cudaSuccess) return cuda_fail(nullptr, "preparing the scores kernel", e);
    if (blocks < 1) return fail(nullptr, PLT_ERR_UNSUPPORTED, "the scores kernel does not fit an SM");
    const int most = g.bf16 ? 2 : 4;
    h->score_grid = h->sm_count * (blocks < most ? blocks : most);
    h->score_smem = g.v.smem;
    h->add_smem = evict_add_smem(c.max_batch);
    e = evict_add_prepare(g.v.twice, key_pitch(g), h->add_smem, &blocks);
    if (e != cudaSuccess) return cuda_fail(nullptr, "preparing the add kernel", e);
    if (blocks < 1) return fail(nullptr, PLT_ERR_UNSUPPORTED, "the add kernel does not fit an SM");
    h->add_grid = h->sm_count * blocks;
    if (g.bf16) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
        if (e != cudaSuccess || !fn || qres != cudaDriverEntryPointSuccess)
            return fail(nullptr, PLT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
        h->encode = (EncodeTiledFn)fn;
    }
    const size_t bytes = layout(&c, &g, h->sm_count * (g.bf16 ? 2 : 4));
    void* ws = nullptr;
    e = cudaMalloc(&ws, bytes);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return fail(nullptr, PLT_ERR_OUT_OF_MEMORY, "cudaMalloc of %zu workspace bytes failed", bytes);
    }
    h->scores = (float*)ws;
    h->ml = h->scores + g.score_floats;
    h->mc = h->ml + g.ml_floats;
    h->item_blocks = (int32_t*)(h->mc + g.mc_floats);
    h->status = (uint32_t*)(h->item_blocks + 2 * g.items);
    e = cudaMemset(h->status, 0, 4);
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);   // before a call on a stream that does not wait for the default one
    if (e != cudaSuccess) {
        cudaFree(ws);
        return cuda_fail(nullptr, "cudaMemset", e);
    }
    return PLT_OK;
}

}  // namespace

#define PLT_API __attribute__((visibility("default")))
extern "C" {

PLT_API plt_status plt_cache_evict_workspace_bytes(const plt_cache_evict_config* config, size_t* out_bytes) {
    EvictGeometry g;
    const plt_status s = check_config(config, &g);
    if (s != PLT_OK) return s;
    if (!out_bytes) return fail(nullptr, PLT_ERR_INVALID_ARG, "out_bytes is NULL");
    int sms = 148;
    cudaDeviceProp prop;
    if (cudaGetDeviceProperties(&prop, config->device) == cudaSuccess) sms = prop.multiProcessorCount;
    else (void)cudaGetLastError();
    *out_bytes = layout(config, &g, sms * (g.bf16 ? 2 : 4));
    return PLT_OK;
}

PLT_API plt_status plt_cache_evict_create(const plt_cache_evict_config* config, plt_cache_evict_t* out_handle) {
    if (!out_handle) return fail(nullptr, PLT_ERR_INVALID_ARG, "out_handle is NULL");
    *out_handle = nullptr;
    EvictGeometry g;
    plt_status s = check_config(config, &g);
    if (s != PLT_OK) return s;
    DeviceScope scope(config->device);
    if (scope.err != cudaSuccess) return cuda_fail(nullptr, "cudaSetDevice", scope.err);
    plt_cache_evict* h = new (std::nothrow) plt_cache_evict();
    if (!h) return fail(nullptr, PLT_ERR_OUT_OF_MEMORY, "host allocation failed");
    h->cfg = *config;
    h->cfg.loop_offset = nullptr;
    h->g = g;
    for (int l = 0; l < kMaxLoops; ++l) {
        h->delta[l] = config->loop_offset && l < config->L ? config->loop_offset[l] : l;
        if (l < config->L && h->delta[l] > h->max_delta) h->max_delta = h->delta[l];
        if (l == 0 || (l < config->L && h->delta[l] < h->min_delta)) h->min_delta = h->delta[l];
    }
    const float scale = config->sm_scale > 0.f ? config->sm_scale : 1.0f / sqrtf((float)(config->d >> g.qsplit));
    h->scale_log2 = scale * 1.4426950408889634f;
    h->err[0] = 0;
    s = create_on_device(h);
    if (s != PLT_OK) {
        delete h;
        return s;
    }
    *out_handle = h;
    return PLT_OK;
}

PLT_API plt_status plt_cache_evict_weights(plt_cache_evict_t h, const plt_cache_evict_weights_args* a, void* cuda_stream) {
    if (!h) return fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    if (!a) return fail(h, PLT_ERR_INVALID_ARG, "args is NULL");
    if (a->struct_size != sizeof(plt_cache_evict_weights_args))
        return fail(h, PLT_ERR_INVALID_ARG, "args.struct_size %u != %zu", a->struct_size, sizeof(plt_cache_evict_weights_args));
    const plt_cache_evict_config& c = h->cfg;
    const EvictGeometry& g = h->g;
    plt_status s = check_batch(h, a->batch);
    if (s != PLT_OK || a->batch == 0) return s;
    if (!a->q || !a->k_cache || !a->seq_lens) return fail(h, PLT_ERR_INVALID_ARG, "q, k_cache and seq_lens must not be NULL");
    if (!aligned(a->q, 16) || !aligned(a->k_cache, 16)) return fail(h, PLT_ERR_INVALID_ARG, "q and k_cache must be 16-byte aligned");
    if (g.fp8 && !a->k_scale) return fail(h, PLT_ERR_INVALID_ARG, "k_scale must not be NULL with E4M3 caches");
    if (!(a->decay >= 0.f) || !std::isfinite(a->decay)) return fail(h, PLT_ERR_INVALID_ARG, "decay must be finite and not negative");
    int64_t ws = a->weights_stride, sb = a->kv_stride_b, sn = a->kv_stride_n, sh = a->kv_stride_h;
    s = check_totals(h, a->weights, ws);
    const int es = g.fp8 ? 1 : (g.bf16 ? 2 : 4);
    if (s == PLT_OK) s = cache_strides(h, sb, sn, sh, es);
    if (s == PLT_OK) s = check_pages(h, a->page_table, a->max_pages, a->num_pool_pages);
    if (s != PLT_OK) return s;
    DeviceScope scope(c.device);
    if (scope.err != cudaSuccess) return cuda_fail(h, "cudaSetDevice", scope.err);

    EvictWeights e;
    memset(&e, 0, sizeof e);
    e.kw = g.v.KW;
    e.kbox = g.v.tile_keys;
    if (c.page_size > 0)
        while (c.page_size % e.kbox != 0) e.kbox >>= 1;    // 16 divides every page
    e.row_pitch = row_pitch(g.R);
    e.key_pitch = key_pitch(g);
    while ((1 << e.tile_shift) < g.v.tile_keys) ++e.tile_shift;
    e.hpg = g.hpg;
    e.min_delta = h->min_delta;
    e.scores = h->scores;
    e.ml = h->ml;
    e.mc = (float2*)h->mc;
    e.weights_stride = ws;
    e.decay = a->decay;
    CUtensorMap map;
    if (g.bf16) {
        s = encode_keys(h, &map, a->k_cache, sb, sn, sh, es, c.page_size > 0 ? a->num_pool_pages : a->batch, e.kbox);
        if (s != PLT_OK) return s;
    }
    Params& p = e.p;
    p.k_cache = a->k_cache;
    p.k_scale = a->k_scale;
    p.item_blocks = h->item_blocks;
    p.status = h->status;
    p.kv_stride_b = sb; p.kv_stride_n = sn; p.kv_stride_h = sh;
    p.L = c.L; p.Hq = c.Hq << g.qsplit; p.Hkv = c.Hkv; p.G = g.G; p.R = g.R; p.d = c.d;
    p.Qn = g.Qn; p.qsplit = g.qsplit;
    p.max_seq_len = c.max_seq_len; p.page_size = c.page_size; p.max_pages = a->max_pages; p.num_pool_pages = a->num_pool_pages;
    p.hpc = g.v.HPC;
    p.tile_keys = g.v.tile_keys;
    p.piece_cost = kEvictPieceCost;
    p.scale_log2 = h->scale_log2;
    for (int l = 0; l < kMaxLoops; ++l) p.delta[l] = h->delta[l];
    const int groups = c.Hkv / g.hpg;
    const size_t qrow = (size_t)c.L * g.Qn * c.Hq * c.d * (g.bf16 ? 2 : 4);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    for (int b0 = 0; b0 < a->batch; b0 += g.part) {
        e.b0 = b0;
        p.B = a->batch - b0 < g.part ? a->batch - b0 : g.part;
        p.q = (const char*)a->q + b0 * qrow;
        p.seq_lens = a->seq_lens + b0;
        p.page_table = c.page_size > 0 ? a->page_table + (int64_t)b0 * a->max_pages : nullptr;
        e.gate = a->gate_logits && c.L > 1 ? a->gate_logits + (int64_t)b0 * (c.L - 1) * g.Qn * c.Hq : nullptr;
        e.weights = a->weights + (int64_t)b0 * groups * ws;
        cudaError_t err = g.bf16 ? launch_scores(g.v, map, e, h->score_grid, stream)
                                 : launch_scores_f32(e, h->score_grid, h->score_smem, stream);
        if (err != cudaSuccess) return cuda_fail(h, "launching the scores kernel", err);
        err = launch_evict_join(e, stream);
        if (err != cudaSuccess) return cuda_fail(h, "launching the join kernel", err);
        if (g.v.twice) err = launch_sums(g.v, map, e, h->score_grid, stream);
        if (err != cudaSuccess) return cuda_fail(h, "launching the sums kernel", err);
        err = launch_evict_add(e, g.v.twice, h->add_grid, h->add_smem, stream);
        if (err != cudaSuccess) return cuda_fail(h, "launching the add kernel", err);
    }
    return PLT_OK;
}

PLT_API plt_status plt_cache_evict_select(plt_cache_evict_t h, const plt_cache_evict_select_args* a, void* cuda_stream) {
    if (!h) return fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    if (!a) return fail(h, PLT_ERR_INVALID_ARG, "args is NULL");
    if (a->struct_size != sizeof(plt_cache_evict_select_args))
        return fail(h, PLT_ERR_INVALID_ARG, "args.struct_size %u != %zu", a->struct_size, sizeof(plt_cache_evict_select_args));
    const plt_cache_evict_config& c = h->cfg;
    plt_status s = check_batch(h, a->batch);
    if (s != PLT_OK || a->batch == 0) return s;
    if (!a->seq_lens || !a->keep || !a->new_lens) return fail(h, PLT_ERR_INVALID_ARG, "seq_lens, keep and new_lens must not be NULL");
    if (a->new_lens == a->seq_lens) return fail(h, PLT_ERR_INVALID_ARG, "new_lens and seq_lens must be different buffers");
    if (a->budget < 1 || a->budget > c.max_seq_len)
        return fail(h, PLT_ERR_INVALID_ARG, "budget %d outside [1, max_seq_len %d]", a->budget, c.max_seq_len);
    const int64_t least = (int64_t)h->max_delta + h->g.Qn - 1;   // positions that a row's cutoff counts from the end
    if (a->keep_first < 0 || a->keep_last < least || (int64_t)a->keep_first + a->keep_last > a->budget)
        return fail(h, PLT_ERR_INVALID_ARG, "keep_first %d, keep_last %d: not negative, keep_last >= %lld, together <= budget %d", a->keep_first,
                    a->keep_last, (long long)least, a->budget);
    int64_t ws = a->weights_stride;
    s = check_totals(h, a->weights, ws);
    if (s != PLT_OK) return s;
    DeviceScope scope(c.device);
    if (scope.err != cudaSuccess) return cuda_fail(h, "cudaSetDevice", scope.err);
    const SelectParams p = {a->weights, ws, a->seq_lens, a->keep, a->new_lens, h->status, c.Hkv / h->g.hpg, c.max_seq_len, a->budget,
                            a->keep_first, a->keep_last, h->sm_count};
    const cudaError_t err = launch_select(p, a->batch, (cudaStream_t)cuda_stream);
    if (err != cudaSuccess) return cuda_fail(h, "launching the selection kernel", err);
    return PLT_OK;
}

PLT_API plt_status plt_cache_evict_compact(plt_cache_evict_t h, const plt_cache_evict_compact_args* a, void* cuda_stream) {
    if (!h) return fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    if (!a) return fail(h, PLT_ERR_INVALID_ARG, "args is NULL");
    if (a->struct_size != sizeof(plt_cache_evict_compact_args))
        return fail(h, PLT_ERR_INVALID_ARG, "args.struct_size %u != %zu", a->struct_size, sizeof(plt_cache_evict_compact_args));
    const plt_cache_evict_config& c = h->cfg;
    plt_status s = check_batch(h, a->batch);
    if (s != PLT_OK || a->batch == 0) return s;
    if (!a->k_cache || !a->v_cache || !a->seq_lens || !a->keep || !a->new_lens)
        return fail(h, PLT_ERR_INVALID_ARG, "k_cache, v_cache, seq_lens, keep and new_lens must not be NULL");
    if (!aligned(a->k_cache, 16) || !aligned(a->v_cache, 16)) return fail(h, PLT_ERR_INVALID_ARG, "k_cache and v_cache must be 16-byte aligned");
    if (a->k_cache == a->v_cache) return fail(h, PLT_ERR_INVALID_ARG, "k_cache and v_cache must be different buffers");
    if (a->new_lens == a->seq_lens) return fail(h, PLT_ERR_INVALID_ARG, "new_lens and seq_lens must be different buffers");
    if (a->keep_stride < 1 || a->keep_stride > c.max_seq_len)
        return fail(h, PLT_ERR_INVALID_ARG, "keep_stride %d outside [1, max_seq_len %d]", a->keep_stride, c.max_seq_len);
    int64_t ws = a->weights_stride, sb = a->kv_stride_b, sn = a->kv_stride_n, sh = a->kv_stride_h;
    if (a->weights) s = check_totals(h, a->weights, ws);
    const int es = h->g.fp8 ? 1 : (h->g.bf16 ? 2 : 4);
    if (s == PLT_OK) s = cache_strides(h, sb, sn, sh, es);
    if (s == PLT_OK) s = check_pages(h, a->page_table, a->max_pages, a->num_pool_pages);
    if (s != PLT_OK) return s;
    DeviceScope scope(c.device);
    if (scope.err != cudaSuccess) return cuda_fail(h, "cudaSetDevice", scope.err);
    int shift = -1;
    if (c.page_size > 0 && (c.page_size & (c.page_size - 1)) == 0)
        while ((1 << ++shift) < c.page_size) {}
    const CompactParams p = {(char*)a->k_cache, (char*)a->v_cache, sb * es, sn * es, sh * es, a->page_table, a->seq_lens, a->keep,
                             a->new_lens, a->weights, ws, h->status, c.Hkv, h->g.hpg, c.d * es, c.max_seq_len, c.page_size, shift,
                             a->max_pages, a->num_pool_pages, a->keep_stride};
    const cudaError_t err = launch_compact(p, a->batch, (cudaStream_t)cuda_stream);
    if (err != cudaSuccess) return cuda_fail(h, "launching the compaction kernel", err);
    return PLT_OK;
}

PLT_API plt_status plt_cache_evict_check(plt_cache_evict_t h, void* cuda_stream, uint32_t* out_bits) {
    if (!h) return fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    DeviceScope scope(h->cfg.device);
    if (scope.err != cudaSuccess) return cuda_fail(h, "cudaSetDevice", scope.err);
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    uint32_t bits = 0;
    cudaError_t e = cudaMemcpyAsync(&bits, h->status, 4, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, 4, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e != cudaSuccess) return cuda_fail(h, "reading the device status word", e);
    if (out_bits) *out_bits = bits;
    if (bits == 0) return PLT_OK;
    return fail(h, PLT_ERR_DEVICE_CHECK, "device status 0x%x:%s%s%s%s", bits,
                (bits & PLT_DEV_SEQ_LEN_CLAMPED) ? " seq_lens entry out of range (clamped)" : "",
                (bits & PLT_DEV_PAGE_ID_CLAMPED) ? " page id out of range (clamped)" : "",
                (bits & PLT_DEV_WAIT_TIMEOUT) ? " a bounded wait ran out (totals invalid)" : "",
                (bits & PLT_DEV_KEEP_CLAMPED) ? " kept position or new length out of range (clamped)" : "");
}

PLT_API plt_status plt_cache_evict_destroy(plt_cache_evict_t h) {
    if (!h) return PLT_OK;
    {
        DeviceScope scope(h->cfg.device);
        if (h->scores) cudaFree(h->scores);
    }
    delete h;
    return PLT_OK;
}

PLT_API const char* plt_cache_evict_last_error(plt_cache_evict_t h) { return h ? h->err : g_evict_create_error; }

}  // extern "C"

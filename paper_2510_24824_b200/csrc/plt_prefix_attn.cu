// C ABI of the decode step with shared prefixes. The prefixes have a kernel of their own (plt_prefix_main.cu), which leaves the plan;
// the own caches and windows go through the decode step's kernels on the lengths in it, and plt_prefix_merge.cu joins both.
// Here: argument checks, the workspace and the tensor maps.
#include "../../include/plt_prefix_attn.h"

#include <cstring>
#include <new>

#include "plt_handle.h"
#include "plt_prefix.h"

using namespace plt;

namespace {

thread_local char g_prefix_error[512] = "";

}  // namespace

struct plt_prefix_attn : HandleBase {
    plt_decode_attn_t dec = nullptr;
    plt_prefix_attn_config cfg;
    int32_t delta[kMaxLoops];
    int G, R, Qn, blocks;
    PrefixPlan plan;
    float *acc = nullptr, *ml = nullptr;
};

namespace {

plt_status prefix_fail(plt_prefix_attn_t h, plt_status code, const char* what) { return handle_fail(h, g_prefix_error, code, "%s", what); }

// The decode step's message becomes this handle's.
plt_status from_decode(plt_prefix_attn_t h, plt_status s) {
    return handle_fail(h, g_prefix_error, s, "%s", plt_decode_attn_last_error(h ? h->dec : nullptr));
}

plt_status decode_config(const plt_prefix_attn_config* c, plt_decode_attn_config* d) {
    if (!c) return prefix_fail(nullptr, PLT_ERR_INVALID_ARG, "config is NULL");
    if (c->struct_size != sizeof(plt_prefix_attn_config))
        return handle_fail(nullptr, g_prefix_error, PLT_ERR_INVALID_ARG, "config.struct_size %u != %zu", c->struct_size, sizeof *c);
    if (c->dtype != PLT_BF16 && c->dtype != PLT_F32) return prefix_fail(nullptr, PLT_ERR_INVALID_ARG, "unknown dtype");
    if (c->dtype != PLT_BF16) return prefix_fail(nullptr, PLT_ERR_UNSUPPORTED, "shared prefixes need bf16 queries");
    if (c->max_prefix_len < 1 || c->max_groups < 1) return prefix_fail(nullptr, PLT_ERR_INVALID_ARG, "max_prefix_len and max_groups must be >= 1");
    if (c->max_prefix_len > (1 << 24)) return prefix_fail(nullptr, PLT_ERR_UNSUPPORTED, "max_prefix_len above 2^24");
    if (c->max_groups > kMaxGroups) return prefix_fail(nullptr, PLT_ERR_UNSUPPORTED, "max_groups above 1024");
    if (c->max_seq_len > 0x7fffffff - (1 << 24)) return prefix_fail(nullptr, PLT_ERR_UNSUPPORTED, "max_seq_len too large");
    memset(d, 0, sizeof *d);
    d->struct_size = sizeof *d;
    d->dtype = c->dtype; d->max_batch = c->max_batch; d->L = c->L; d->Hq = c->Hq; d->Hkv = c->Hkv; d->d = c->d;
    d->max_seq_len = c->max_seq_len; d->w = c->w; d->page_size = c->page_size; d->sm_scale = c->sm_scale; d->device = c->device;
    d->loop_offset = c->loop_offset; d->kernel_path = c->kernel_path; d->kv_dtype = c->kv_dtype; d->q_len = c->q_len;
    d->typical_seq_len = c->typical_seq_len;
    return PLT_OK;
}

// Units of a full batch: every group that has a sequence may end inside one. (The configuration has passed the decode step's checks.)
int64_t units_of(const plt_prefix_attn_config* c, int R) {
    const int groups = c->max_groups < c->max_batch ? c->max_groups : c->max_batch;
    return (int64_t)c->Hkv * (((int64_t)c->max_batch * R + kPrefixRows - 1) / kPrefixRows + groups);
}
int rows_of(const plt_prefix_attn_config* c) { return c->L * (c->q_len > 1 ? c->q_len : 1) * (c->Hq / c->Hkv); }

// The line of all units' key tiles and the rows of the output have to fit the kernels' whole numbers.
plt_status check_plan(const plt_prefix_attn_config* c) {
    const int R = rows_of(c);
    if ((double)units_of(c, R) * ((double)c->max_prefix_len / kPrefixTile + 1 + kPrefixLead) >= 2147483647.0 ||
        (double)c->max_batch * R * c->Hkv >= 1073741824.0)
        return prefix_fail(nullptr, PLT_ERR_UNSUPPORTED, "max_batch * max_prefix_len too large for the tile plan");
    return PLT_OK;
}

size_t plan_bytes(const plt_prefix_attn_config* c) {
    return 256 + 4 * ((size_t)5 * (c->max_groups + 1) + 3 + (size_t)c->max_batch * c->L);
}
size_t workspace_of(const plt_prefix_attn_config* c, int blocks) {
    const size_t slots = (size_t)units_of(c, rows_of(c)) + blocks;
    return ((plan_bytes(c) + 255) & ~(size_t)255) + slots * kPrefixRows * ((size_t)c->d + 2) * 4;
}

}  // namespace

#define PLT_API __attribute__((visibility("default")))
extern "C" {

PLT_API plt_status plt_prefix_attn_workspace_bytes(const plt_prefix_attn_config* config, size_t* out_bytes) {
    plt_decode_attn_config d;
    plt_status s = decode_config(config, &d);
    if (s != PLT_OK) return s;
    if (!out_bytes) return prefix_fail(nullptr, PLT_ERR_INVALID_ARG, "out_bytes is NULL");
    size_t own = 0;
    s = plt_decode_attn_workspace_bytes(&d, &own);
    if (s != PLT_OK) return from_decode(nullptr, s);
    s = check_plan(config);
    if (s != PLT_OK) return s;
    int sms = 148;
    cudaDeviceProp prop;
    if (cudaGetDeviceProperties(&prop, config->device) == cudaSuccess) sms = prop.multiProcessorCount;
    else (void)cudaGetLastError();
    *out_bytes = own + workspace_of(config, sms);
    return PLT_OK;
}

PLT_API plt_status plt_prefix_attn_create(const plt_prefix_attn_config* config, plt_prefix_attn_t* out_handle) {
    if (!out_handle) return prefix_fail(nullptr, PLT_ERR_INVALID_ARG, "out_handle is NULL");
    *out_handle = nullptr;
    plt_decode_attn_config d;
    plt_status s = decode_config(config, &d);
    if (s != PLT_OK) return s;
    size_t own = 0;
    s = plt_decode_attn_workspace_bytes(&d, &own);      // all of the decode step's checks, without a device
    if (s != PLT_OK) return from_decode(nullptr, s);
    const int R = rows_of(config);
    s = check_plan(config);
    if (s != PLT_OK) return s;
    DeviceScope scope(config->device);
    if (scope.err != cudaSuccess) {
        (void)cudaGetLastError();
        return handle_fail(nullptr, g_prefix_error, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    }
    int sms = 0;
    s = check_device(config->device, g_prefix_error, &sms);
    if (s != PLT_OK) return s;
    plt_prefix_attn* h = new (std::nothrow) plt_prefix_attn();
    if (!h) return prefix_fail(nullptr, PLT_ERR_OUT_OF_MEMORY, "host allocation failed");
    s = decode_create(&d, /*qsplit=*/0, &h->dec);
    if (s != PLT_OK) {
        delete h;
        return from_decode(nullptr, s);
    }
    h->cfg = *config;
    h->cfg.loop_offset = nullptr;
    h->device = config->device;
    for (int l = 0; l < kMaxLoops; ++l) h->delta[l] = config->loop_offset && l < config->L ? config->loop_offset[l] : l;
    h->G = config->Hq / config->Hkv;
    h->R = R;
    h->Qn = config->q_len > 1 ? config->q_len : 1;
    h->blocks = sms;
    const bool fp8 = config->kv_dtype == PLT_KV_E4M3;
    cudaError_t e = prefix_prepare(config->d, fp8);
    if (e != cudaSuccess) {
        plt_decode_attn_destroy(h->dec);
        delete h;
        return handle_fail(nullptr, g_prefix_error, PLT_ERR_CUDA, "preparing the prefix kernel: %s", cudaGetErrorString(e));
    }
    const size_t bytes = workspace_of(config, sms);
    char* ws = nullptr;
    if (cudaMalloc((void**)&ws, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        plt_decode_attn_destroy(h->dec);
        delete h;
        return handle_fail(nullptr, g_prefix_error, PLT_ERR_OUT_OF_MEMORY, "cudaMalloc of %zu workspace bytes failed", bytes);
    }
    h->status = (uint32_t*)ws;
    h->plan.ready = h->status + 1;
    int32_t* at = (int32_t*)(ws + 256);
    const int groups = config->max_groups + 1;
    h->plan.begin = at; at += groups;
    h->plan.len = at; at += groups;
    h->plan.line = at; at += groups;
    h->plan.unit = at; at += groups;
    h->plan.piece = at; at += groups;
    h->plan.chunk = at; at += 3;
    h->plan.own_lens = at; at += config->max_batch;
    h->plan.win_lens = at;
    h->acc = (float*)(ws + ((plan_bytes(config) + 255) & ~(size_t)255));
    h->ml = h->acc + ((size_t)units_of(config, R) + sms) * kPrefixRows * config->d;
    e = cudaMemset(ws, 0, plan_bytes(config));
    if (e == cudaSuccess) e = cudaDeviceSynchronize();   // another stream may run first
    if (e != cudaSuccess) {
        cudaFree(ws);
        plt_decode_attn_destroy(h->dec);
        delete h;
        return handle_fail(nullptr, g_prefix_error, PLT_ERR_CUDA, "clearing the workspace: %s", cudaGetErrorString(e));
    }
    *out_handle = h;
    return PLT_OK;
}

PLT_API plt_status plt_prefix_attn_run(plt_prefix_attn_t h, const plt_decode_attn_args* a, const plt_prefix_args* x, void* cuda_stream) {
    if (!h) return prefix_fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    if (!a) return prefix_fail(h, PLT_ERR_INVALID_ARG, "args is NULL");
    if (!x) return prefix_fail(h, PLT_ERR_INVALID_ARG, "prefix is NULL");
    if (x->struct_size != sizeof(plt_prefix_args))
        return handle_fail(h, g_prefix_error, PLT_ERR_INVALID_ARG, "prefix.struct_size %u != %zu", x->struct_size, sizeof *x);
    const plt_prefix_attn_config& c = h->cfg;
    if (x->num_groups < 0) return prefix_fail(h, PLT_ERR_INVALID_ARG, "num_groups < 0");
    if (x->num_groups > c.max_groups)
        return handle_fail(h, g_prefix_error, PLT_ERR_CAPACITY, "num_groups %d > max_groups %d", x->num_groups, c.max_groups);
    const bool fp8 = c.kv_dtype == PLT_KV_E4M3;
    const int es = fp8 ? 1 : 2;
    const int64_t unit = 16 / es;
    int64_t sg = x->stride_g, sn = x->stride_n, sh = x->stride_h;
    if (x->num_groups > 0) {
        if (!x->group_begin || !x->prefix_lens) return prefix_fail(h, PLT_ERR_INVALID_ARG, "group_begin and prefix_lens must not be NULL");
        if (misaligned(x->group_begin, 4) || misaligned(x->prefix_lens, 4) || misaligned(x->page_table, 4))
            return prefix_fail(h, PLT_ERR_INVALID_ARG, "a tensor is not aligned to its elements");
        if (c.page_size > 0) {
            if (!x->page_table) return prefix_fail(h, PLT_ERR_INVALID_ARG, "prefix.page_table is NULL for a paged cache");
            const int need = (c.max_prefix_len + c.page_size - 1) / c.page_size;
            if (x->max_pages < need) return handle_fail(h, g_prefix_error, PLT_ERR_CAPACITY, "prefix.max_pages %d < %d", x->max_pages, need);
        } else {
            if (!x->k_prefix || !x->v_prefix) return prefix_fail(h, PLT_ERR_INVALID_ARG, "k_prefix and v_prefix must not be NULL");
            if (misaligned(x->k_prefix, 16) || misaligned(x->v_prefix, 16))
                return prefix_fail(h, PLT_ERR_INVALID_ARG, "tensor base pointers must be 16-byte aligned");
            if (sg == 0 && sn == 0 && sh == 0) {
                sh = c.d;
                sn = (int64_t)c.Hkv * c.d;
                sg = (int64_t)c.max_prefix_len * sn;
            }
            if (sg <= 0 || sn <= 0 || sh <= 0 || sg % unit || sn % unit || sh % unit)
                return prefix_fail(h, PLT_ERR_INVALID_ARG, "prefix strides must be positive multiples of 16 bytes");
            if (sh < c.d) return prefix_fail(h, PLT_ERR_INVALID_ARG, "stride_h < d");
            if ((double)sg * es >= 1099511627776.0 || (double)sn * es >= 1099511627776.0 || (double)sh * es >= 1099511627776.0)
                return prefix_fail(h, PLT_ERR_UNSUPPORTED, "prefix stride of 2^40 bytes or more");
        }
    }
    DeviceScope scope(h->device);
    if (scope.err != cudaSuccess) return handle_fail(h, g_prefix_error, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    PrefixRun run;
    memset(&run, 0, sizeof run);
    PrefixParams& p = run.pp;
    run.fp8 = fp8;
    p.group_begin = x->group_begin; p.prefix_lens = x->prefix_lens; p.page_table = x->page_table;
    p.plan = h->plan; p.acc = h->acc; p.ml = h->ml; p.status = h->status;
    p.groups = x->num_groups; p.max_prefix_len = c.max_prefix_len; p.max_pages = x->max_pages; p.blocks = h->blocks;
    // Query rows by TMA where whole tokens make up a tile; by the softmax's threads two users take 16.1 us instead of 15.7, 64 sequences
    // of two loops 39.5 instead of 36.2.
    p.q_tma = 128 % h->G == 0;
    // Rates that the plan divides the multiprocessors by, read off batches of 21 to 96 sequences behind 1777 to 8192 tokens with 9 to
    // 138 multiprocessors left to the own caches: a key tile of 256 rows takes 1.9 us (8-bit caches 3.0) with the pass's start; of the
    // own caches a multiprocessor streams 80 bytes a nanosecond at up to 8 packed rows, and less where its products bound it: 50 at 16
    // and 24 at 32 (8-bit caches 36 at 16; with heads of 64 58 at 8; the others go on from these). Tiles of 1.5 us give the same times
    // within 1 %, of 1.3 us drafts lose (32 us instead of 20, both before probabilities had second terms; tiles of 2.1 us give the same times, of
    // 2.3 us the long prefixes lose, 208 instead of 149). With the multiprocessors divided and with one pass behind the other: 64
    // sequences of two loops 36.2 and 43.6 us, groups of 8-bit caches 42.8 and 49.2, drafts 21.9 and 27.2, 128 sequences behind 32768
    // tokens 146 and 164.
    p.tile_ns = fp8 ? 3000 : 1900;
    p.own_rate = h->R <= 8 ? 80 : h->R <= 16 ? (fp8 ? 36 : 50) : h->R <= 32 ? (fp8 ? 18 : 24) : (fp8 ? 9 : 12);
    if (c.d == 64) p.own_rate = p.own_rate * 7 / 10;
    p.token_bytes = 2 * c.Hkv * c.d * es;
    // keys of a TMA box: all of a tile, or as many as both tile and page are made of
    p.kbox = kPrefixTile;
    while (c.page_size > 0 && c.page_size % p.kbox != 0) p.kbox >>= 1;
    if (x->num_groups > 0 && c.page_size == 0) {
        plt_status s = decode_encode_rows(h->dec, &run.maps[0], x->k_prefix, es, c.d, c.max_prefix_len, c.Hkv, x->num_groups, sn, sh, sg, p.kbox);
        if (s == PLT_OK) s = decode_encode_rows(h->dec, &run.maps[1], x->v_prefix, es, c.d, c.max_prefix_len, c.Hkv, x->num_groups, sn, sh, sg, p.kbox);
        if (s != PLT_OK) return from_decode(h, s);
    }
    const plt_status s = decode_run_prefix(h->dec, a, &run, cuda_stream);
    return s == PLT_OK ? s : from_decode(h, s);
}

PLT_API plt_status plt_prefix_attn_check(plt_prefix_attn_t h, void* cuda_stream, uint32_t* out_bits) {
    if (!h) return prefix_fail(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    // both words: the plan and the prefixes' kernel set this handle's, the others the decode step's
    uint32_t own = 0, shared = 0;
    DeviceScope scope(h->device);
    plt_status s = handle_check(h, g_prefix_error, (cudaStream_t)cuda_stream, &shared);
    if (s != PLT_OK && s != PLT_ERR_DEVICE_CHECK) return s;
    const plt_status t = plt_decode_attn_check(h->dec, cuda_stream, &own);
    if (t != PLT_OK && t != PLT_ERR_DEVICE_CHECK) return from_decode(h, t);
    if (out_bits) *out_bits = own | shared;
    if (s != PLT_OK) return s;
    return t == PLT_OK ? t : from_decode(h, t);
}

PLT_API plt_status plt_prefix_attn_destroy(plt_prefix_attn_t h) {
    if (!h) return PLT_OK;
    DeviceScope scope(h->device);
    plt_decode_attn_destroy(h->dec);
    cudaFree(h->status);
    delete h;
    return PLT_OK;
}

PLT_API const char* plt_prefix_attn_last_error(plt_prefix_attn_t h) { return h ? h->err : g_prefix_error; }

}  // extern "C"

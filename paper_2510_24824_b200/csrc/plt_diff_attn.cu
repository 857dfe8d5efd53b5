// C ABI of differential attention: one decode step and whole prompts. The decode step runs on the main kernels of the plain
// attention, which take a query head as two packed rows (the halves of the row, the other half zero, so that one pass over a
// cache row serves both maps), with a merge kernel of its own that joins the maps (plt_reduce.cu); prompts have a kernel of
// their own (plt_diff_seq.cu). Here: argument checks and the parameters' struct.
#include "../../include/plt_diff_attn.h"

#include <cmath>
#include <cstring>
#include <new>

#include "plt_host.h"

using namespace plt;

struct plt_diff_attn {
    plt_decode_attn_t dec = nullptr;
    int32_t Hq;
    float lambda_init, eps;
};

struct plt_diff_seq_attn {
    plt_seq_attn_t seq = nullptr;
    int32_t Hq;
    float lambda_init, eps;
};

namespace {

const char* check_numbers(float lambda_init, float eps) {
    if (!std::isfinite(lambda_init)) return "lambda_init is not finite";
    if (!(eps > 0.f) || !std::isfinite(eps)) return "norm_eps must be positive and finite";
    return nullptr;
}

// null or what is wrong with the parameters
const char* make_tail(const plt_diff_weights* w, int Hq, float lambda_init, float eps, DiffTail* t) {
    if (!w) return "weights is NULL";
    if (w->struct_size != sizeof(plt_diff_weights)) return "weights.struct_size does not match";
    if (w->lambda_heads != 1 && w->lambda_heads != Hq) return "weights.lambda_heads must be 1 or Hq";
    if (!w->lambda_q1 || !w->lambda_k1 || !w->lambda_q2 || !w->lambda_k2) return "the lambda vectors must not be NULL";
    const uintptr_t bits = (uintptr_t)w->lambda_q1 | (uintptr_t)w->lambda_k1 | (uintptr_t)w->lambda_q2 |
                           (uintptr_t)w->lambda_k2 | (uintptr_t)w->norm_gain;
    if (bits & 3u) return "the lambda vectors and norm_gain must be 4-byte aligned";
    *t = DiffTail{w->lambda_q1, w->lambda_k1, w->lambda_q2, w->lambda_k2, w->norm_gain, w->lambda_heads, lambda_init, eps};
    return nullptr;
}

// The configuration of the decode step behind a differential handle: two rows for each query head.
plt_status decode_config(const plt_diff_attn_config* c, plt_decode_attn_config* d) {
    if (!c) return decode_error(nullptr, PLT_ERR_INVALID_ARG, "config is NULL");
    if (c->struct_size != sizeof(plt_diff_attn_config))
        return decode_error(nullptr, PLT_ERR_INVALID_ARG, "config.struct_size does not match plt_diff_attn_config");
    if (const char* bad = check_numbers(c->lambda_init, c->norm_eps)) return decode_error(nullptr, PLT_ERR_INVALID_ARG, bad);
    if (c->Hq < 1 || c->Hkv < 1 || c->L < 1) return decode_error(nullptr, PLT_ERR_INVALID_ARG, "non-positive size in config");
    if (c->Hq % c->Hkv != 0) return decode_error(nullptr, PLT_ERR_INVALID_ARG, "Hq is not a multiple of Hkv");
    const double rows = 2.0 * c->L * (c->q_len > 1 ? c->q_len : 1) * (c->Hq / c->Hkv);
    if (rows > kMaxRows)
        return decode_error(nullptr, PLT_ERR_UNSUPPORTED, "2 * L * q_len * Hq/Hkv packed rows exceed 64 (two for each differential head)");
    memset(d, 0, sizeof *d);
    d->struct_size = sizeof *d;
    d->dtype = c->dtype;
    d->max_batch = c->max_batch;
    d->L = c->L;
    d->Hq = 2 * c->Hq;
    d->Hkv = c->Hkv;
    d->d = c->d;
    d->max_seq_len = c->max_seq_len;
    d->w = c->w;
    d->page_size = c->page_size;
    d->sm_scale = c->sm_scale > 0.f ? c->sm_scale : (c->d > 0 ? 1.0f / sqrtf(0.5f * (float)c->d) : 0.f);
    d->device = c->device;
    d->loop_offset = c->loop_offset;
    d->kernel_path = c->kernel_path;
    d->kv_dtype = c->kv_dtype;
    d->q_len = c->q_len;
    d->typical_seq_len = c->typical_seq_len;
    return PLT_OK;
}

}  // namespace

#define PLT_API __attribute__((visibility("default")))
extern "C" {

PLT_API plt_status plt_diff_attn_workspace_bytes(const plt_diff_attn_config* config, size_t* out_bytes) {
    plt_decode_attn_config d;
    const plt_status s = decode_config(config, &d);
    return s != PLT_OK ? s : plt_decode_attn_workspace_bytes(&d, out_bytes);
}

PLT_API plt_status plt_diff_attn_create(const plt_diff_attn_config* config, plt_diff_attn_t* out_handle) {
    if (!out_handle) return decode_error(nullptr, PLT_ERR_INVALID_ARG, "out_handle is NULL");
    *out_handle = nullptr;
    plt_decode_attn_config d;
    plt_status s = decode_config(config, &d);
    if (s != PLT_OK) return s;
    plt_diff_attn* h = new (std::nothrow) plt_diff_attn();
    if (!h) return decode_error(nullptr, PLT_ERR_OUT_OF_MEMORY, "host allocation failed");
    DeviceScope scope(d.device);   // the caller's current device is put back
    s = decode_create(&d, /*qsplit=*/1, &h->dec);
    if (s != PLT_OK) {
        delete h;
        return s;
    }
    h->Hq = config->Hq;
    h->lambda_init = config->lambda_init;
    h->eps = config->norm_eps;
    *out_handle = h;
    return PLT_OK;
}

PLT_API plt_status plt_diff_attn_run(plt_diff_attn_t h, const plt_decode_attn_args* args, const plt_diff_weights* weights,
                                     void* cuda_stream) {
    if (!h) return decode_error(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    DiffTail tail;
    if (const char* bad = make_tail(weights, h->Hq, h->lambda_init, h->eps, &tail)) return decode_error(h->dec, PLT_ERR_INVALID_ARG, bad);
    DeviceScope scope(decode_device(h->dec));
    if (scope.err != cudaSuccess) return decode_error(h->dec, PLT_ERR_CUDA, cudaGetErrorString(scope.err));
    return decode_run(h->dec, args, &tail, cuda_stream);
}

PLT_API plt_status plt_diff_attn_step(plt_diff_attn_t h, const plt_decode_attn_args* args, const plt_decode_attn_step_args* step,
                                      const plt_diff_weights* weights, void* cuda_stream) {
    if (!h) return decode_error(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    DiffTail tail;
    if (const char* bad = make_tail(weights, h->Hq, h->lambda_init, h->eps, &tail)) return decode_error(h->dec, PLT_ERR_INVALID_ARG, bad);
    DeviceScope scope(decode_device(h->dec));
    if (scope.err != cudaSuccess) return decode_error(h->dec, PLT_ERR_CUDA, cudaGetErrorString(scope.err));
    return decode_step(h->dec, args, step, &tail, cuda_stream);
}

PLT_API plt_status plt_diff_attn_check(plt_diff_attn_t h, void* cuda_stream, uint32_t* out_bits) {
    if (!h) return decode_error(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    DeviceScope scope(decode_device(h->dec));
    if (scope.err != cudaSuccess) return decode_error(h->dec, PLT_ERR_CUDA, cudaGetErrorString(scope.err));
    return plt_decode_attn_check(h->dec, cuda_stream, out_bits);
}

PLT_API plt_status plt_diff_attn_destroy(plt_diff_attn_t h) {
    if (!h) return PLT_OK;
    {
        DeviceScope scope(decode_device(h->dec));
        plt_decode_attn_destroy(h->dec);
    }
    delete h;
    return PLT_OK;
}

PLT_API const char* plt_diff_attn_last_error(plt_diff_attn_t h) { return plt_decode_attn_last_error(h ? h->dec : nullptr); }

// ---- whole prompts ------------------------------------------------------------------------------------------------
PLT_API plt_status plt_diff_seq_attn_create(const plt_diff_seq_attn_config* c, plt_diff_seq_attn_t* out_handle) {
    if (!out_handle) return seq_error(nullptr, PLT_ERR_INVALID_ARG, "out_handle is NULL");
    *out_handle = nullptr;
    if (!c) return seq_error(nullptr, PLT_ERR_INVALID_ARG, "config is NULL");
    if (c->struct_size != sizeof(plt_diff_seq_attn_config))
        return seq_error(nullptr, PLT_ERR_INVALID_ARG, "config.struct_size does not match plt_diff_seq_attn_config");
    if (const char* bad = check_numbers(c->lambda_init, c->norm_eps)) return seq_error(nullptr, PLT_ERR_INVALID_ARG, bad);
    plt_seq_attn_config s;
    memset(&s, 0, sizeof s);
    s.struct_size = sizeof s;
    s.max_batch = c->max_batch;
    s.L = c->L;
    s.Hq = c->Hq;
    s.Hkv = c->Hkv;
    s.d = c->d;
    s.max_seq_len = c->max_seq_len;
    s.w = c->w;
    s.sm_scale = c->sm_scale;
    s.device = c->device;
    s.loop_offset = c->loop_offset;
    plt_diff_seq_attn* h = new (std::nothrow) plt_diff_seq_attn();
    if (!h) return seq_error(nullptr, PLT_ERR_OUT_OF_MEMORY, "host allocation failed");
    DeviceScope scope(c->device);
    const plt_status st = seq_create(&s, /*diff=*/true, &h->seq);
    if (st != PLT_OK) {
        delete h;
        return st;
    }
    h->Hq = c->Hq;
    h->lambda_init = c->lambda_init;
    h->eps = c->norm_eps;
    *out_handle = h;
    return PLT_OK;
}

PLT_API plt_status plt_diff_seq_attn_run(plt_diff_seq_attn_t h, const plt_seq_attn_args* args, const plt_diff_weights* weights,
                                         void* cuda_stream) {
    if (!h) return seq_error(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    DiffTail tail;
    if (const char* bad = make_tail(weights, h->Hq, h->lambda_init, h->eps, &tail)) return seq_error(h->seq, PLT_ERR_INVALID_ARG, bad);
    DeviceScope scope(seq_device(h->seq));
    if (scope.err != cudaSuccess) return seq_error(h->seq, PLT_ERR_CUDA, cudaGetErrorString(scope.err));
    return seq_run(h->seq, args, &tail, cuda_stream);
}

PLT_API plt_status plt_diff_seq_attn_check(plt_diff_seq_attn_t h, void* cuda_stream, uint32_t* out_bits) {
    if (!h) return seq_error(nullptr, PLT_ERR_INVALID_ARG, "handle is NULL");
    DeviceScope scope(seq_device(h->seq));
    if (scope.err != cudaSuccess) return seq_error(h->seq, PLT_ERR_CUDA, cudaGetErrorString(scope.err));
    return plt_seq_attn_check(h->seq, cuda_stream, out_bits);
}

PLT_API plt_status plt_diff_seq_attn_destroy(plt_diff_seq_attn_t h) {
    if (!h) return PLT_OK;
    {
        DeviceScope scope(seq_device(h->seq));
        plt_seq_attn_destroy(h->seq);
    }
    delete h;
    return PLT_OK;
}

PLT_API const char* plt_diff_seq_attn_last_error(plt_diff_seq_attn_t h) { return plt_seq_attn_last_error(h ? h->seq : nullptr); }

}  // extern "C"

/*
 * plt_diff_attn.h - C ABI of differential attention on the caches of plt_decode_attn.h, for NVIDIA B200 (sm_100a):
 * one decode step (plt_diff_attn_*) and every row of a prompt at once (plt_diff_seq_attn_*).
 *
 * A differential head takes the difference of two softmax maps.  The d elements of a query row and of a key row are two
 * halves of d / 2, one for each map; a value row is d wide and serves both:
 *
 *   y_m    = softmax(sm_scale * q_m K_m[0:cut]^T) V[0:cut],            m = 1, 2,   sm_scale = 1 / sqrt(d / 2)
 *   lambda = exp(lambda_q1 . lambda_k1) - exp(lambda_q2 . lambda_k2) + lambda_init      (learned vectors of d / 2)
 *   x      = y_1 - lambda y_2
 *   O      = (1 - lambda_init) * norm_gain * x / sqrt(mean(x^2) + norm_eps)             (mean over the head's d elements)
 *   O      = x                                                                          (norm_gain == NULL)
 *
 * Caches, pages, strides, lengths, loops with their cutoffs, windows and gates, multi-token steps and E4M3 codes are those
 * of plt_decode_attn.h: K and V have the same shape and size as for plain heads, and a query head h reads KV head
 * h / (Hq / Hkv).  With loops 2..L each map is mixed by the gate first (Eq. 2 is linear, so y_m = g * y_m,local +
 * (1 - g) * y_m,global), then the difference is taken.  Rows whose loop has no token yet are written as zeros.
 *
 * The K rows that a query row sees have to be finite in both halves (the decode step multiplies the half of the other map
 * by zero).
 *
 * Softmax statistics, both results, the factor, the difference and the norm are held in fp32; the output is rounded once.
 * All tensor pointers are DEVICE pointers owned by the caller.  No exception crosses this boundary; errors are plt_status
 * codes.  There is no CPU fallback.  The device of a handle is made current for the length of each call; the stream must
 * belong to it.
 */
#ifndef PLT_DIFF_ATTN_H
#define PLT_DIFF_ATTN_H

#include "plt_decode_attn.h"
#include "plt_seq_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The learned parameters of a layer, fp32, DEVICE pointers (4-byte aligned).  struct_size = sizeof(plt_diff_weights). */
typedef struct {
    uint32_t struct_size;
    int32_t lambda_heads;     /* rows of the four vectors: 1 (shared by the heads) or Hq */
    const float* lambda_q1;   /* [lambda_heads, d / 2] */
    const float* lambda_k1;
    const float* lambda_q2;
    const float* lambda_k2;
    const float* norm_gain;   /* [d], or NULL: no norm and no factor 1 - lambda_init */
} plt_diff_weights;

/* ---- one decode step --------------------------------------------------------------------------------------------- */

typedef struct plt_diff_attn* plt_diff_attn_t; /* opaque; owned by the library */

/*
 * Fixed at create.  struct_size = sizeof(plt_diff_attn_config).  Fields that plt_decode_attn_config has too mean the same
 * and have the same limits, except that a head takes two packed rows: 2 * L * q_len * (Hq / Hkv) <= 64.
 */
typedef struct {
    uint32_t struct_size;
    int32_t dtype;            /* plt_dtype */
    int32_t max_batch;
    int32_t L;
    int32_t Hq, Hkv, d;       /* differential query heads, KV heads, elements of a row (both halves): d in {64, 128} */
    int32_t max_seq_len;
    int32_t w;
    int32_t page_size;
    float sm_scale;           /* <= 0 selects 1/sqrt(d/2) */
    int32_t device;
    const int32_t* loop_offset;
    int32_t kernel_path;      /* plt_kernel_path; the rules count the packed rows */
    int32_t kv_dtype;         /* plt_kv_dtype */
    int32_t q_len;
    int32_t typical_seq_len;
    float lambda_init;        /* finite */
    float norm_eps;           /* > 0, finite */
} plt_diff_attn_config;

/* Validates the configuration and allocates the handle's workspace on config->device (the only call that allocates). */
plt_status plt_diff_attn_create(const plt_diff_attn_config* config, plt_diff_attn_t* out_handle);

/* Enqueues one decode step on `cuda_stream`: two kernels, the split-KV main kernel that streams every cached row once for
 * both maps, and the merge kernel that joins the splits, takes the difference and normalises.  Arguments, asynchrony,
 * capture and overlap as plt_decode_attn_run; `weights` is read by the merge kernel (under the terms that plt_decode_attn_run
 * states for gate_logits). */
plt_status plt_diff_attn_run(plt_diff_attn_t handle, const plt_decode_attn_args* args, const plt_diff_weights* weights,
                             void* cuda_stream);

/* The pre-step of plt_decode_attn_step (cache append, window rings, gate linear on a head's whole query row) and then the
 * attention: three kernels. */
plt_status plt_diff_attn_step(plt_diff_attn_t handle, const plt_decode_attn_args* args, const plt_decode_attn_step_args* step,
                              const plt_diff_weights* weights, void* cuda_stream);

/* Synchronises `cuda_stream`, reads the device status word (PLT_DEV_* bits) and clears it, as plt_decode_attn_check. */
plt_status plt_diff_attn_check(plt_diff_attn_t handle, void* cuda_stream, uint32_t* out_bits);

/* Frees the handle.  NULL is accepted. */
plt_status plt_diff_attn_destroy(plt_diff_attn_t handle);

/* Message for the last non-OK status of this handle (or of the last failed create when handle == NULL). */
const char* plt_diff_attn_last_error(plt_diff_attn_t handle);

/* Device bytes plt_diff_attn_create would allocate (as plt_decode_attn_workspace_bytes). */
plt_status plt_diff_attn_workspace_bytes(const plt_diff_attn_config* config, size_t* out_bytes);

/* ---- a whole prompt ------------------------------------------------------------------------------------------------ */

typedef struct plt_diff_seq_attn* plt_diff_seq_attn_t; /* opaque; owned by the library */

/* Fixed at create.  struct_size = sizeof(plt_diff_seq_attn_config).  Fields as plt_seq_attn_config (bf16, d = 128 = two
 * halves of 64, Hq % Hkv == 0, L <= 8). */
typedef struct {
    uint32_t struct_size;
    int32_t max_batch;
    int32_t L;
    int32_t Hq, Hkv, d;
    int32_t max_seq_len;
    int32_t w;
    float sm_scale;           /* <= 0 selects 1/sqrt(d/2) */
    int32_t device;
    const int32_t* loop_offset;
    float lambda_init;        /* finite */
    float norm_eps;           /* > 0, finite */
} plt_diff_seq_attn_config;

plt_status plt_diff_seq_attn_create(const plt_diff_seq_attn_config* config, plt_diff_seq_attn_t* out_handle);

/* Enqueues the differential attention of every row of every sequence on `cuda_stream`: ONE kernel.  Row t of loop l is what
 * plt_diff_attn_run computes at cache length t + 1 (with plt_seq_attn.h's rule for the windows).  Arguments as
 * plt_seq_attn_run; rows without a token and rows at or beyond the length are written as zeros. */
plt_status plt_diff_seq_attn_run(plt_diff_seq_attn_t handle, const plt_seq_attn_args* args, const plt_diff_weights* weights,
                                 void* cuda_stream);
plt_status plt_diff_seq_attn_check(plt_diff_seq_attn_t handle, void* cuda_stream, uint32_t* out_bits);
plt_status plt_diff_seq_attn_destroy(plt_diff_seq_attn_t handle);
const char* plt_diff_seq_attn_last_error(plt_diff_seq_attn_t handle);

#ifdef __cplusplus
}
#endif
#endif /* PLT_DIFF_ATTN_H */

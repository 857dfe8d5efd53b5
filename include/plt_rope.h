/*
 * plt_rope.h - C ABI of what happens to queries and keys between their projections and the attention, for NVIDIA B200
 * (sm_100a): a norm for each head and the rotation by position in one pass, together with the way of the rows into the caches
 * of plt_decode_attn.h.  Two forms: a decode step (plt_rope_step) and every row of a prompt (plt_rope_seq).
 *
 * For a row x of d elements (one head of a query or a key) at position p:
 *
 *   x' = gain * x / sqrt(mean(x^2) + norm_eps)                                    (where a gain is given; else x' = x)
 *   (a, b) -> attn_factor * (a cos(p f_i) - b sin(p f_i),  b cos(p f_i) + a sin(p f_i))        i = 0 .. rotary_dim / 2 - 1
 *
 * on the pairs (x'[i], x'[i + rotary_dim / 2]) (PLT_ROPE_HALF) or (x'[2 i], x'[2 i + 1]) (PLT_ROPE_INTERLEAVED) of the first
 * rotary_dim elements; the others stay x'.  The frequencies f_i (radians a position) come from theta and the scaling:
 *
 *   g_i = theta^(-2 i / rotary_dim)
 *   PLT_ROPE_PLAIN        f_i = g_i
 *   PLT_ROPE_LINEAR       f_i = g_i / factor
 *   PLT_ROPE_BASE         f_i = (theta * factor^(rotary_dim / (rotary_dim - 2)))^(-2 i / rotary_dim)
 *   PLT_ROPE_WAVELENGTH   f_i = s g_i + (1 - s) g_i / factor,  s = clamp((original_len g_i / (2 pi) - low) / (high - low), 0, 1)
 *   PLT_ROPE_RAMP         f_i = (1 - s) g_i + s g_i / factor,  s = clamp((i - first) / max(last - first, 0.001), 0, 1) with
 *                         first = max(floor(c(high)), 0), last = min(ceil(c(low)), rotary_dim - 1),
 *                         c(t) = rotary_dim log(original_len / (2 pi t)) / (2 log theta)
 *
 * or from the caller (inv_freq).  Angles are taken modulo a turn in 64-bit integers, to 2^-32 of a turn at any position (for
 * frequencies of up to a turn a position; faster ones lose in proportion), and rounded to fp32 then; norm, rotation and gates are held in fp32 (a row to be normed has to have a sum of squares below 2^128),
 * and each result is rounded once, to the type it is stored in (E4M3: the code nearest to value / scale[head]).
 *
 * All tensor pointers are DEVICE pointers owned by the caller unless a comment says "host".  No exception crosses this
 * boundary; errors are plt_status codes.  There is no CPU fallback.  The device of a handle is made current for the length of
 * each call; the stream must belong to it.  A call launches ONE kernel, allocates nothing, does not synchronise and can be
 * captured in a CUDA graph.
 */
#ifndef PLT_ROPE_H
#define PLT_ROPE_H

#include "plt_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct plt_rope* plt_rope_t; /* opaque; owned by the library */

typedef enum { PLT_ROPE_HALF = 0, PLT_ROPE_INTERLEAVED = 1 } plt_rope_layout;
typedef enum {
    PLT_ROPE_PLAIN = 0, PLT_ROPE_LINEAR = 1, PLT_ROPE_BASE = 2, PLT_ROPE_WAVELENGTH = 3, PLT_ROPE_RAMP = 4
} plt_rope_scaling;

/*
 * Fixed at create.  struct_size = sizeof(plt_rope_config).  Fields that plt_decode_attn_config has too mean the same.
 * Supported: d in {64, 128} (E4M3 codes: 128, with dtype PLT_BF16); Hq % Hkv == 0; L <= 8; max_batch <= 4096;
 * page_size a multiple of 16; rotary_dim a multiple of 16; q_len <= 64, and 1 when L > 1 (windows of several tokens a step
 * hold their entries in age order, which is the caller's work).
 */
typedef struct {
    uint32_t struct_size;
    int32_t dtype;            /* plt_dtype of q, k, v and (PLT_KV_SAME) the caches */
    int32_t kv_dtype;         /* plt_kv_dtype of the caches and windows */
    int32_t max_batch;
    int32_t L, Hq, Hkv, d;
    int32_t max_seq_len;      /* capacity of the shared cache per sequence, in tokens */
    int32_t w;                /* window capacity; may be 0 only if L == 1 */
    int32_t page_size;        /* 0: contiguous */
    int32_t device;
    const int32_t* loop_offset; /* host, L entries; NULL: delta_l = l-1.  Copied at create. */
    int32_t q_len;            /* query tokens per loop of one step; 0 or 1: one */
    int32_t rotary_dim;       /* elements of a head that turn, from the first; 0: all d */
    int32_t layout;           /* plt_rope_layout */
    int32_t scaling;          /* plt_rope_scaling */
    int32_t original_len;     /* PLT_ROPE_WAVELENGTH and PLT_ROPE_RAMP: positions trained on, >= 1 */
    float norm_eps;           /* > 0, finite */
    float attn_factor;        /* finite; 0: 1 */
    double theta;             /* > 1, finite */
    double factor;            /* > 0, finite (all but PLT_ROPE_PLAIN) */
    double low, high;         /* PLT_ROPE_WAVELENGTH and PLT_ROPE_RAMP: turns over original_len, 0 < low < high */
    const double* inv_freq;   /* host, rotary_dim / 2 finite values, or NULL.  Copied at create; theta and scaling are not read
                                 then */
} plt_rope_config;

/*
 * One decode step.  Loop l of sequence b serves, as its token j (oldest first), position
 * p = seq_lens[b] - delta_l - 1 - (q_len - 1 - j); nothing is stored where p < 0, and the query's row is zero there.
 *   - q_out[b, l, j, h] = the query's row at p;
 *   - loop 1: the key's row at p and the value's row go to position p - prefix_lens[b] of the shared cache (positions below 0
 *     lie in a prefix that is shared, and are not stored);
 *   - loops 2..L: they go to slot p mod w of that loop's window;
 *   - gate_logits[b, l-2, h] = sum_j w_gate[h, j] * (the query's row in fp32)[j] + b_gate[h].
 * That is plt_decode_attn_step's pre-step for queries and keys that have not been normed and rotated yet;
 * plt_decode_attn_run, plt_diff_attn_run or plt_prefix_attn_run follow it.
 */
typedef struct {
    uint32_t struct_size;
    int32_t batch;
    const void* q;                 /* [B, L, q_len, Hq, d]; rows (b, l, j) q_stride elements apart, 16-byte aligned */
    const void* k_new;             /* [B, L, q_len, Hkv, d], likewise */
    const void* v_new;
    int64_t q_stride, k_stride, v_stride; /* 0: dense; multiples of 16 bytes, so that one fused projection may hold all three */
    const float* q_gain;           /* [d] fp32, or NULL: queries are not normed */
    const float* k_gain;           /* [d] fp32, or NULL: keys are not normed */
    void* q_out;                   /* [B, L, q_len, Hq, d] dense; may be q where q is dense */
    void* k_cache;                 /* as plt_decode_attn_args; both are written */
    void* v_cache;
    int64_t kv_stride_b, kv_stride_n, kv_stride_h;
    const int32_t* seq_lens;       /* [B] tokens of each sequence, the prefix and this step's counted; values outside
                                      [0, prefix + max_seq_len] are clamped and flagged (PLT_DEV_SEQ_LEN_CLAMPED) */
    const int32_t* prefix_lens;    /* [B] tokens in front of this cache's first one, or NULL: 0; values below 0 are clamped and
                                      flagged (PLT_DEV_GROUP_CLAMPED) */
    const int32_t* page_table;
    int32_t max_pages, num_pool_pages;
    void* k_win;                   /* [B, L-1, w, Hkv, d]; both are written (NULL allowed when L == 1) */
    void* v_win;
    const float* k_scale;          /* PLT_KV_E4M3 only */
    const float* v_scale;
    const float* w_gate;           /* [Hq, d] fp32, or NULL (with gate_logits): no gates; 16-byte aligned */
    const float* b_gate;           /* [Hq] fp32 */
    float* gate_logits;            /* [B, L-1, Hq] fp32 */
} plt_rope_step_args;

/*
 * Every row of a prompt (or of a part of one).  Row t of sequence b stands at position start[b] + t (loop l's queries and own
 * keys: - delta_l); rows t >= seq_lens[b], and rows of loops whose position is below 0, are neither read nor written.
 *   - q_out, k_share_out, k_loc_out: the rows as plt_seq_attn_run takes them;
 *   - where k_cache is given, row t of k_share (turned) and of v_share also goes to position
 *     start[b] + t - prefix_lens[b] of the decode step's shared cache; positions outside [0, max_seq_len) are left out, those
 *     beyond it flagged (PLT_DEV_SEQ_LEN_CLAMPED).
 * Needs delta_1 = 0.
 */
typedef struct {
    uint32_t struct_size;
    int32_t batch;
    int32_t rows;                  /* T: rows per sequence in every tensor, >= 1 */
    const void* q;                 /* [B, L, T, Hq, d], all tensors dense and 16-byte aligned */
    const void* k_share;           /* [B, T, Hkv, d] */
    const void* v_share;           /* [B, T, Hkv, d]; read only where v_cache is given */
    const void* k_loc;             /* [B, L-1, T, Hkv, d] (NULL allowed when L == 1) */
    void* q_out;                   /* outputs may be the inputs */
    void* k_share_out;             /* NULL allowed where k_cache is given */
    void* k_loc_out;
    const float* q_gain;
    const float* k_gain;
    const int32_t* seq_lens;       /* [B] rows of each sequence; values outside [0, T] are clamped and flagged
                                      (PLT_DEV_SEQ_LEN_CLAMPED) */
    const int32_t* start;          /* [B] position of row 0, or NULL: 0; values below 0 are clamped and flagged
                                      (PLT_DEV_GROUP_CLAMPED) */
    const int32_t* prefix_lens;    /* as above */
    void* k_cache;                 /* as above, or NULL (with v_cache) */
    void* v_cache;
    int64_t kv_stride_b, kv_stride_n, kv_stride_h;
    const int32_t* page_table;
    int32_t max_pages, num_pool_pages;
    const float* k_scale;
    const float* v_scale;
} plt_rope_seq_args;

/* Validates the configuration and puts the frequencies on config->device (the only call that allocates). */
plt_status plt_rope_create(const plt_rope_config* config, plt_rope_t* out_handle);

/* The rotary_dim / 2 frequencies of a configuration in radians a position (host; no device needed). */
plt_status plt_rope_frequencies(const plt_rope_config* config, double* out_freq);

plt_status plt_rope_step(plt_rope_t handle, const plt_rope_step_args* args, void* cuda_stream);
plt_status plt_rope_seq(plt_rope_t handle, const plt_rope_seq_args* args, void* cuda_stream);

/* Synchronises `cuda_stream`, reads the device status word and clears it (PLT_DEV_* bits), as plt_decode_attn_check.  A row
 * whose page id is outside the pool is not stored (PLT_DEV_PAGE_ID_CLAMPED). */
plt_status plt_rope_check(plt_rope_t handle, void* cuda_stream, uint32_t* out_bits);

/* Frees the handle. NULL is accepted. The caller makes sure no call is in flight. */
plt_status plt_rope_destroy(plt_rope_t handle);

/* Message for the last non-OK status of this handle (or of the last failed create when handle == NULL). */
const char* plt_rope_last_error(plt_rope_t handle);

#ifdef __cplusplus
}
#endif
#endif /* PLT_ROPE_H */

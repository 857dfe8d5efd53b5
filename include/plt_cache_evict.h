/*
 * plt_cache_evict.h - C ABI of eviction from the shared cache by accumulated attention weight, for NVIDIA B200 (sm_100a).
 *
 * A shared first-loop cache that outgrows its budget loses the positions that the queries attend least.  Three calls, each
 * on the caller's own buffers, on the caches of plt_decode_attn.h (contiguous with strides or in pages, like q or E4M3
 * codes):
 *
 *   plt_cache_evict_weights   adds to a running total the weight that a step's queries give every cached position
 *   plt_cache_evict_select    picks the positions to keep under a budget: the first and the last ones always, the rest by
 *                             their totals
 *   plt_cache_evict_compact   moves the kept rows of K and V (and their totals) to the front of the cache, in place
 *
 * The KV heads are kept in groups of heads_per_group: the heads of a group share one total and one set of positions, the
 * groups are independent (1: every head its own positions; Hkv: whole tokens).  All groups of a sequence keep the same
 * number, so the sequence has one new length, which the caller passes on as seq_lens; the attention does not depend on
 * which positions a head's rows came from.  The kept positions stay in order, and the last ones are always among them, so
 * that the causal offsets of loops 2..L keep their meaning.
 *
 * All tensor pointers are DEVICE pointers owned by the caller unless a comment says "host".  No exception crosses this
 * boundary; errors are plt_status codes.  There is no CPU fallback.  The device of a handle is made current for the length
 * of each call; the stream must belong to it.  Calls on the same handle must be stream-ordered (they share the workspace);
 * none of them allocates or synchronises, and all can be captured in a CUDA graph (a call that a capture replays has fixed
 * addresses; lengths, positions and totals are read on the device).  plt_cache_evict_weights reads seq_lens while the kernel
 * before it in the stream finishes, under the terms that plt_decode_attn_run states; the other two are ordinary launches.
 */
#ifndef PLT_CACHE_EVICT_H
#define PLT_CACHE_EVICT_H

#include "plt_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct plt_cache_evict* plt_cache_evict_t; /* opaque; owned by the library */

/* Further bits of the device status word. */
#define PLT_DEV_KEEP_CLAMPED 16u    /* a kept position was outside [its slot, seq_lens[b]), or a new length outside
                                       [0, min(keep_stride, seq_lens[b])] */

/*
 * Fixed at create.  struct_size = sizeof(plt_cache_evict_config).  Fields that plt_decode_attn_config has too mean the same.
 * Supported: d in {64, 128} (E4M3 codes: 128, with dtype PLT_BF16); Hq % Hkv == 0; maps * L * q_len * (Hq / Hkv) <= 64 packed
 * query rows per KV head; L <= 8; max_batch <= 4096; page_size a multiple of 16; max_seq_len <= 2^24.
 */
typedef struct {
    uint32_t struct_size;
    int32_t dtype;            /* plt_dtype of q and (PLT_KV_SAME) the caches */
    int32_t kv_dtype;         /* plt_kv_dtype */
    int32_t max_batch;
    int32_t L, Hq, Hkv, d;
    int32_t max_seq_len;      /* capacity of the shared cache per sequence, in tokens */
    int32_t page_size;        /* 0: contiguous */
    float sm_scale;           /* <= 0 selects 1/sqrt(d / maps) */
    int32_t device;
    const int32_t* loop_offset; /* host, L entries delta_l >= 0; NULL: delta_l = l-1.  Copied at create. */
    int32_t q_len;            /* query tokens per loop of one plt_cache_evict_weights call; 0 or 1: one */
    int32_t maps;             /* 0 or 1: one softmax for each head; 2: differential heads (plt_diff_attn.h, with what it says
                                 of K's values), the weights of both maps count */
    int32_t heads_per_group;  /* KV heads that share totals and positions; 0 or 1: none; divides Hkv */
} plt_cache_evict_config;

/*
 * Totals after a step.  For every sequence b, group g and position n < N_b = seq_lens[b]:
 *
 *   weights[b, g, n] = decay * weights[b, g, n] + sum over the group's KV heads, their query heads, loops, tokens and maps of
 *                      rho * softmax(sm_scale * q K[0:cut]^T)[n]
 *
 * with the cutoffs of plt_decode_attn_run (cut = max(0, N_b - delta_l - (q_len - 1 - token)); a position that a row does not
 * see gets nothing from it).  rho = 1, or, where gate_logits is given, 1 - sigmoid(gate) for the rows of loops 2..L: the
 * share that Eq. 2 gives the shared cache.  Scores, softmax and totals are fp32 (with E4M3 caches the products take the
 * queries in f16, which holds bf16 values exactly between 2^-14 and 65504).  K rows that a query row sees have to be finite.  The sums' order depends on nothing but the
 * configuration and the lengths, so results repeat bit for bit.
 */
typedef struct {
    uint32_t struct_size;
    int32_t batch;
    const void* q;                 /* [B, L, q_len, Hq, d], 16-byte aligned */
    const void* k_cache;           /* as plt_decode_attn_args, 16-byte aligned */
    int64_t kv_stride_b, kv_stride_n, kv_stride_h;
    const int32_t* seq_lens;       /* [B]; values outside [0, max_seq_len] are clamped and flagged */
    const int32_t* page_table;     /* [B, max_pages] (paged only); ids outside the pool are clamped and flagged */
    int32_t max_pages, num_pool_pages;
    const float* k_scale;          /* PLT_KV_E4M3 only */
    const float* gate_logits;      /* [B, L-1, q_len, Hq] fp32, or NULL */
    float* weights;                /* [B, Hkv / heads_per_group] rows, weights_stride apart; positions >= N_b stay as they are */
    int64_t weights_stride;        /* elements between rows; 0: max_seq_len */
    float decay;                   /* >= 0, finite; 0: the old totals are not read (they may hold anything) */
} plt_cache_evict_weights_args;

/*
 * Positions to keep.  For every sequence b and group g: all of [0, N_b) if N_b <= budget, else exactly `budget` positions:
 * [0, keep_first), [N_b - keep_last, N_b), and of the others those with the largest weights; of equal weights (0 and -0 are
 * equal) the lowest position; NaN counts as less than every number.  keep[b, g, 0 .. new_lens[b]) holds them in ascending
 * order, the rest of the row -1.
 */
typedef struct {
    uint32_t struct_size;
    int32_t batch;
    const float* weights;          /* as above */
    int64_t weights_stride;
    const int32_t* seq_lens;       /* [B] */
    int32_t budget;                /* 1 <= budget <= max_seq_len */
    int32_t keep_first;            /* >= 0; keep_first + keep_last <= budget */
    int32_t keep_last;             /* >= the largest delta_l + q_len - 1 */
    int32_t* keep;                 /* [B, Hkv / heads_per_group, budget] */
    int32_t* new_lens;             /* [B] min(N_b, budget); not the same buffer as seq_lens */
} plt_cache_evict_select_args;

/*
 * Compaction in place.  For every sequence b, group g, KV head h of the group and slot i < new_lens[b]:
 *   K[b, i, h] = K[b, keep[b, g, i], h],  V likewise,  weights[b, g, i] = weights[b, g, keep[b, g, i]],
 * all from the values before the call; weights[b, g, new_lens[b] .. seq_lens[b]) = 0 (the next tokens start there).  K and V
 * rows from new_lens[b] on stay as they are.  Positions have to be ascending (as plt_cache_evict_select writes them): one
 * below its slot or not below seq_lens[b] is clamped and flagged.  No page may belong to two sequences, and the rows of the
 * cache must not overlap.  A row that would come from or go to a page outside the pool stays where it is (flagged).  Rows in front of the first dropped position stay where they are, all kept ones behind it move.
 */
typedef struct {
    uint32_t struct_size;
    int32_t batch;
    void* k_cache;                 /* as plt_decode_attn_args; both are written */
    void* v_cache;
    int64_t kv_stride_b, kv_stride_n, kv_stride_h;
    const int32_t* page_table;
    int32_t max_pages, num_pool_pages;
    const int32_t* seq_lens;       /* [B] the lengths before */
    const int32_t* keep;           /* [B, Hkv / heads_per_group, keep_stride] */
    int32_t keep_stride;           /* the budget of the select call; 1 <= keep_stride <= max_seq_len */
    const int32_t* new_lens;       /* [B] the lengths after */
    float* weights;                /* optional */
    int64_t weights_stride;
} plt_cache_evict_compact_args;

/* Validates the configuration and allocates the handle's workspace on config->device (the only call that allocates): at most
 * about 256 MB, or what one sequence of max_seq_len tokens needs where that is more; select and compact use the status word alone. */
plt_status plt_cache_evict_create(const plt_cache_evict_config* config, plt_cache_evict_t* out_handle);

/* Device bytes plt_cache_evict_create would allocate for this configuration (no device needed; 148 SMs are assumed then). */
plt_status plt_cache_evict_workspace_bytes(const plt_cache_evict_config* config, size_t* out_bytes);

plt_status plt_cache_evict_weights(plt_cache_evict_t handle, const plt_cache_evict_weights_args* args, void* cuda_stream);
plt_status plt_cache_evict_select(plt_cache_evict_t handle, const plt_cache_evict_select_args* args, void* cuda_stream);
plt_status plt_cache_evict_compact(plt_cache_evict_t handle, const plt_cache_evict_compact_args* args, void* cuda_stream);

/* Synchronises `cuda_stream`, reads the device status word and clears it (PLT_DEV_* bits), as plt_decode_attn_check. */
plt_status plt_cache_evict_check(plt_cache_evict_t handle, void* cuda_stream, uint32_t* out_bits);

/* Frees the workspace. NULL is accepted. The caller makes sure no call is in flight. */
plt_status plt_cache_evict_destroy(plt_cache_evict_t handle);

/* Message for the last non-OK status of this handle (or of the last failed create when handle == NULL). */
const char* plt_cache_evict_last_error(plt_cache_evict_t handle);

#ifdef __cplusplus
}
#endif
#endif /* PLT_CACHE_EVICT_H */

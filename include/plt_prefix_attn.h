/*
 * plt_prefix_attn.h - C ABI of the decode-step attention of plt_decode_attn.h for a batch whose sequences share long prefixes
 * (a system prompt, a document, the prompt of many samples), for NVIDIA B200 (sm_100a).
 *
 * Consecutive sequences of the batch form groups; the sequences of group g share a prefix of P_g tokens, whose keys and values
 * are stored, and read, once.  Each sequence keeps what follows the prefix in a cache of its own:
 *
 *   token position   0 .. P_g - 1              in the prefix of the sequence's group
 *                    P_g .. seq_lens[b] - 1    at P_g .. of it: position n lies at n - P_g of the sequence's own cache
 *
 * Everything else is plt_decode_attn_run's: seq_lens count the prefix, loop l's token j sees
 * cut = max(0, seq_lens[b] - delta_l - (q_len - 1 - j)) positions, which may end inside the prefix; loops 2..L mix in their windows
 * by the gate; one softmax runs over prefix and own keys; rows without a token are zero.  Sequences behind the last group have
 * no prefix.  bf16 probabilities that hold a large share of a row's weight meet the values in two terms on the prefix too, so that
 * results keep the decode step's bounds wherever a token lies.
 *
 * All tensor pointers are DEVICE pointers owned by the caller.  No exception crosses this boundary; errors are plt_status
 * codes.  There is no CPU fallback.  The device of a handle is made current for the length of each call; the stream must
 * belong to it.  Calls on the same handle must be stream-ordered (they share the workspace); a run neither allocates nor
 * synchronises, and can be captured in a CUDA graph.
 */
#ifndef PLT_PREFIX_ATTN_H
#define PLT_PREFIX_ATTN_H

#include "plt_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct plt_prefix_attn* plt_prefix_attn_t; /* opaque; owned by the library */

/*
 * Fixed at create.  struct_size = sizeof(plt_prefix_attn_config).  Fields that plt_decode_attn_config has too mean the same and
 * have the same limits.  dtype is PLT_BF16 (the prefix's products run on the tensor cores).
 */
typedef struct {
    uint32_t struct_size;
    int32_t dtype;            /* PLT_BF16 */
    int32_t max_batch;
    int32_t L, Hq, Hkv, d;
    int32_t max_seq_len;      /* capacity of a sequence's own cache, in tokens */
    int32_t w;
    int32_t page_size;        /* 0: contiguous; > 0: own caches and prefixes lie in pages of one pool */
    float sm_scale;           /* <= 0 selects 1/sqrt(d) */
    int32_t device;
    const int32_t* loop_offset;
    int32_t kernel_path;      /* plt_kernel_path of the pass over the own caches */
    int32_t kv_dtype;         /* plt_kv_dtype of the own caches, the windows and the prefixes */
    int32_t q_len;
    int32_t typical_seq_len;
    int32_t max_prefix_len;   /* capacity of a prefix, in tokens; 1 .. 2^24 */
    int32_t max_groups;       /* 1 .. 1024 */
} plt_prefix_attn_config;

/*
 * The shared prefixes of a call.  struct_size = sizeof(plt_prefix_args).  Prefix rows below P_g have to be finite; the rest may
 * hold anything.  With E4M3 caches the prefix's products take the queries in f16, which holds bf16 values exactly between 2^-14
 * and 65504.
 */
typedef struct {
    uint32_t struct_size;
    int32_t num_groups;            /* 0 .. max_groups */
    const int32_t* group_begin;    /* [num_groups + 1]: group g is sequences group_begin[g] .. group_begin[g + 1] - 1 (may be
                                      empty); not falling, the first 0 or more, the last at most batch.  Sequences in front of
                                      the first and behind the last have no prefix */
    const int32_t* prefix_lens;    /* [num_groups] P_g */
    const void* k_prefix;          /* contiguous: [num_groups, max_prefix_len, Hkv, d]; in pages: ignored, the pool is
                                      plt_decode_attn_args' */
    const void* v_prefix;
    int64_t stride_g, stride_n, stride_h; /* contiguous: elements between prefixes, tokens, heads; all 0: dense */
    const int32_t* page_table;     /* [num_groups, max_pages] ids in the pool (paged only) */
    int32_t max_pages;             /* >= ceil(max_prefix_len / page_size) */
} plt_prefix_args;

/* Validates the configuration and allocates the handle's workspace on config->device (the only call that allocates). */
plt_status plt_prefix_attn_create(const plt_prefix_attn_config* config, plt_prefix_attn_t* out_handle);

/* Device bytes plt_prefix_attn_create would allocate (as plt_decode_attn_workspace_bytes). */
plt_status plt_prefix_attn_workspace_bytes(const plt_prefix_attn_config* config, size_t* out_bytes);

/* Enqueues one decode step on `cuda_stream`: the kernel over the prefixes (tcgen05.mma with the queries of a whole group as its
 * rows), the split-KV kernel over the own caches and windows, which runs beside it, and the merge; before them a small plan kernel
 * where there are more than 31 groups, or none.  seq_lens, win_lens and gate_logits are read under the terms that
 * plt_decode_attn_run states for the kernels after the call; the kernels before it may write anything. */
plt_status plt_prefix_attn_run(plt_prefix_attn_t handle, const plt_decode_attn_args* args, const plt_prefix_args* prefix,
                               void* cuda_stream);

/* Synchronises `cuda_stream`, reads the device status word (PLT_DEV_* bits) and clears it, as plt_decode_attn_check. */
plt_status plt_prefix_attn_check(plt_prefix_attn_t handle, void* cuda_stream, uint32_t* out_bits);

/* Frees the handle.  NULL is accepted. */
plt_status plt_prefix_attn_destroy(plt_prefix_attn_t handle);

/* Message for the last non-OK status of this handle (or of the last failed create when handle == NULL). */
const char* plt_prefix_attn_last_error(plt_prefix_attn_t handle);

#ifdef __cplusplus
}
#endif
#endif /* PLT_PREFIX_ATTN_H */

/*
 * plt_draft_verify.h - C ABI of draft verification, for NVIDIA B200 (sm_100a): which of the tokens that a small model (or a
 * copy from the prompt) drafted for a multi-token decode step stand, and the token that follows them.
 *
 * A step of plt_decode_attn.h with q_len = max_drafts + 1 computes, for each sequence b, the target's probabilities p_j after
 * each of its K_b drafted tokens x_0 .. x_{K_b - 1} (p_0: after the token before them).  With q_j the probabilities that x_j was
 * drawn from, and numbers u_j, r that are uniform in [0, 1):
 *
 *   x_j passes  <=>  u_j * q_j(x_j) < p_j(x_j)                        n = number of drafts in front of the first that does not
 *   weights     w = max(p_n - q_n, 0)   where a draft was refused (n < K_b); if they are all 0:  w = p_n
 *               w = p_{K_b}             where none was
 *   next token  the lowest v with  w(0) + .. + w(v) > r * (w(0) + .. + w(V - 1))
 *
 * so that what comes out is distributed as the target's own tokens are.  Drafts without probabilities (draft_probs == NULL)
 * were certain: q_j is 1 at x_j and 0 elsewhere.  Products, differences and sums are held in 64 bits; the order of the sums
 * depends on nothing but the sizes and the tensors' alignment, so results repeat bit for bit.
 *
 * Entries of w that are NaN, not above 0, or infinite as fp32 numbers count as 0.  Where rounding leaves no v (or r is NaN or not below 1), the
 * last v with a weight is taken; a row without any weight gives token -1 and PLT_DEV_NO_PROBABILITY.  A draft outside
 * [0, vocab) is refused and flagged with PLT_DEV_TOKEN_OUT_OF_RANGE.
 *
 * All tensor pointers are DEVICE pointers owned by the caller.  No exception crosses this boundary; errors are plt_status
 * codes.  There is no CPU fallback.  The device of a handle is made current for the length of each call; the stream must
 * belong to it.  Calls on the same handle must be stream-ordered (they share the workspace); a run neither allocates nor
 * synchronises and can be captured in a CUDA graph.
 */
#ifndef PLT_DRAFT_VERIFY_H
#define PLT_DRAFT_VERIFY_H

#include "plt_decode_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct plt_draft_verify* plt_draft_verify_t; /* opaque; owned by the library */

/* Further bits of the device status word. */
#define PLT_DEV_TOKEN_OUT_OF_RANGE 32u  /* a drafted token was outside [0, vocab) */
#define PLT_DEV_NO_PROBABILITY 64u      /* a row of probabilities had no entry above 0 */

/* Fixed at create.  struct_size = sizeof(plt_draft_verify_config).  max_batch <= 4096, max_drafts <= 64, vocab <= 2^24. */
typedef struct {
    uint32_t struct_size;
    int32_t dtype;          /* plt_dtype of the probabilities */
    int32_t max_batch;
    int32_t max_drafts;     /* K: drafts a sequence can have in one call, >= 1 */
    int32_t vocab;          /* V */
    int32_t device;         /* CUDA device ordinal */
} plt_draft_verify_config;

/* Per call.  struct_size = sizeof(plt_draft_verify_args).  Probabilities need the alignment of their type; rows and sequences
 * may lie any number of elements apart, `vocab` at least (the vocabulary itself is dense). */
typedef struct {
    uint32_t struct_size;
    int32_t batch;                  /* B, 0 <= B <= max_batch */
    const void* target_probs;       /* [B, K + 1, V]; rows behind a sequence's K_b + 1 are not read */
    int64_t target_stride_b;        /* elements between sequences and between rows; both 0: dense */
    int64_t target_stride_j;
    const void* draft_probs;        /* [B, K, V], or NULL */
    int64_t draft_stride_b;
    int64_t draft_stride_j;
    const int32_t* draft_tokens;    /* [B, K] */
    const int32_t* draft_lens;      /* [B] K_b, or NULL: K; values outside [0, K] are clamped and flagged
                                       (PLT_DEV_SEQ_LEN_CLAMPED) */
    const float* accept_u;          /* [B, K] u_j */
    const float* sample_u;          /* [B] r */
    int32_t* tokens;                /* [B, K + 1]: the n drafts that stand, the next token, then -1 */
    int32_t* num_accepted;          /* [B] n */
    const int32_t* seq_lens;        /* [B], or NULL (with new_lens): lengths that count all K + 1 tokens of the step */
    int32_t* new_lens;              /* [B] max(0, seq_lens - (K - n)): without the refused ones; may be seq_lens */
} plt_draft_verify_args;

/* Validates the configuration and allocates the handle's workspace on config->device (the only call that allocates). */
plt_status plt_draft_verify_create(const plt_draft_verify_config* config, plt_draft_verify_t* out_handle);

/* Device bytes plt_draft_verify_create would allocate for this configuration (no device needed). */
plt_status plt_draft_verify_workspace_bytes(const plt_draft_verify_config* config, size_t* out_bytes);

/* Enqueues the verification on `cuda_stream`: two kernels (three for a large batch), which read one row of p and (after a
 * refusal) one of q for each sequence. */
plt_status plt_draft_verify_run(plt_draft_verify_t handle, const plt_draft_verify_args* args, void* cuda_stream);

/* Synchronises `cuda_stream`, reads the device status word and clears it (PLT_DEV_* bits), as plt_decode_attn_check. */
plt_status plt_draft_verify_check(plt_draft_verify_t handle, void* cuda_stream, uint32_t* out_bits);

/* Frees the workspace. NULL is accepted. The caller makes sure no call is in flight. */
plt_status plt_draft_verify_destroy(plt_draft_verify_t handle);

/* Message for the last non-OK status of this handle (or of the last failed create when handle == NULL). */
const char* plt_draft_verify_last_error(plt_draft_verify_t handle);

#ifdef __cplusplus
}
#endif
#endif /* PLT_DRAFT_VERIFY_H */

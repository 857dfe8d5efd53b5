// Shared prefixes: what the host layer and the kernels of the prefix pass have in common.
#pragma once
#include "plt_host.h"

namespace plt {

constexpr int kMaxGroups = 1024;
constexpr int kPrefixRows = 256;      // packed query rows of a unit: two tiles of 128
constexpr int kPrefixTile = 128;      // keys of a tile
constexpr int kPrefixLead = 2;        // line positions that stand for starting and finishing a unit's piece, in tiles

// The plan of a call. A unit is (group, KV head, 256 packed rows); its key tiles are cut into pieces, one block each.
//   - Where all units can be cut into as many pieces as there are blocks (one each) without much loss, every unit of a group has
//     the same number of nearly equal pieces of at most `*chunk` tiles, and piece i is block i's and leaves its partial in slot i.
//   - Else (*chunk = 0) the units lie one after the other on a line of key tiles, each preceded by kPrefixLead positions, and the
//     line is cut into equal ranges, one for each block, which may hold several pieces; slot unit + block.
// The line for all calls measured 19.0 us against 15.7 (two users), 28.3 against 21.9 (21 sequences of drafts), 36.9 against 36.2 (64
// sequences of two loops), 157 against 146 (128 of them behind 32768 tokens), and 41.4 against 42.8 for three groups of 8-bit caches.
// Not every block need take part: the pass over the prefixes is bound by the tensor cores and its start, the one over the own caches
// by memory and its start, so that the plan may leave some multiprocessors to the latter, which then runs at the same time.
//
// The plan reaches the kernels behind by release and acquire (0.3 to 1 us a call): its writer releases `ready[0]`, the pass over the own caches and the merge
// acquire it before they read a word of the plan. (griddepcontrol.launch_dependents only lets them start: it makes nothing visible,
// and a griddepcontrol.wait would have them wait for the prefixes' products.) The merge's last block to pass by, counted in ready[1],
// sets both words back behind its griddepcontrol.wait, so that every call finds them 0.
struct PrefixPlan {
    uint32_t *ready;     // two words
    int32_t *begin;      // [groups + 1] first sequence of each group, clamped
    int32_t *len;        // [groups] tokens of each prefix, clamped; 0 where the group is empty
    int32_t *line;       // [groups + 1] first line position of each group's units
    int32_t *unit;       // [groups + 1] first unit of each group
    int32_t *piece;      // [groups + 1] first piece of each group's units (*chunk > 0)
    int32_t *chunk;      // three words: tiles of a chunk or 0, blocks that take part, blocks of the pass over the own caches
    int32_t *own_lens;   // [max_batch] tokens that each sequence holds itself
    int32_t *win_lens;   // [max_batch, L - 1] valid window slots of each loop
};

struct PrefixParams {
    const void* q;                 // [B, L, Qn, Hq, d] bf16
    const int32_t* seq_lens;       // [B], prefix counted
    const int32_t* win_lens;       // [B, L - 1] or null: as the caller gave them
    const int32_t* group_begin;    // as the caller gave them
    const int32_t* prefix_lens;
    const int32_t* page_table;     // [groups, max_pages]
    const float *k_scale, *v_scale;
    PrefixPlan plan;
    float* acc;                    // [slots][2 tiles][d / 4][128 rows][4]: unnormalised sums of p * V
    float* ml;                     // [slots][2 tiles][128 rows][2]: reference (log2 units; -inf: saw no key), sum of p
    uint32_t* status;
    int32_t groups, B, L, Qn, Hq, Hkv, G, R, d, w;
    int32_t max_seq_len, max_prefix_len, page_size, max_pages, num_pool_pages, kbox;
    int32_t blocks;                // of the prefix kernel
    int32_t own_per_sm;            // blocks of the pass over the own caches on a multiprocessor; 0: it runs behind this one
    int32_t own_rate;              // bytes a nanosecond that a multiprocessor streams of the own caches, about
    int32_t own_items;             // items of the own caches and windows (sequence, heads of a block)
    int32_t tile_ns;               // time of a key tile of 256 rows, about
    int32_t token_bytes;           // K and V rows of a token
    int32_t q_tma;                 // 1: query rows by TMA (the heads of a KV head divide 128)
    float scale_log2;
    int32_t delta[kMaxLoops];
};

// What a run needs of the prefixes: filled by the public entry point, completed by the decode step's run.
struct PrefixRun {
    PrefixParams pp;
    CUtensorMap maps[3];           // K, V of the prefixes, q
    bool fp8;
};

cudaError_t prefix_prepare(int d, bool fp8);
cudaError_t launch_prefix_plan(const PrefixParams& pp, cudaStream_t stream);
cudaError_t launch_prefix_main(const CUtensorMap maps[3], const PrefixParams& pp, bool fp8, cudaStream_t stream);
cudaError_t launch_prefix_merge(const Params& p, const PrefixParams& pp, bool overlap, cudaStream_t stream);

// plt_decode_attn_run with shared prefixes in front of the caches: `args` as the caller gave them.
plt_status decode_run_prefix(plt_decode_attn_t h, const plt_decode_attn_args* args, PrefixRun* prefix, void* cuda_stream);
// Encodes the map of a cache's rows: [outer][heads][keys][d] with strides in elements, boxes of `box_keys` keys of one head.
plt_status decode_encode_rows(plt_decode_attn_t h, CUtensorMap* map, const void* base, int es, int d, int64_t keys, int64_t heads,
                              int64_t outer, int64_t sn, int64_t sh, int64_t so, int box_keys);

// a / b for 0 <= a < 2^21 and b > 0: (a + 1/2) / b is at least 1 / 2 b away from a whole number, and off by less than 2^-22 of itself.
// (A division of whole numbers is a long piece of code, which a launch finds outside the instruction caches.)
__device__ __forceinline__ int small_div(int a, int b) { return (int)__fdividef((float)a + 0.5f, (float)b); }

// Keys (prefix and own) that a row sees of a sequence whose length was given as `given`, `capacity` at most: its loop lies delta
// behind, `newer` tokens of the step are younger. No difference leaves 32 bits, whatever lengths and offsets are.
__device__ __forceinline__ int row_sees(int given, int64_t capacity, int delta, int newer) {
    const int n = (int)min((int64_t)max(given, 0), capacity);
    return max(max(n - delta, 0) - newer, 0);
}

// Blocks that take part in a line of T positions: at least kPrefixMinLine positions each.
constexpr int kPrefixMinLine = 3;
__host__ __device__ inline int prefix_blocks(int T, int launched) {
    const int c = T / kPrefixMinLine;
    return c < 1 ? 1 : c < launched ? c : launched;
}
// First position of block c's range (T c / C, without its product) and the block that owns position `pos`.
__host__ __device__ inline int prefix_range(int T, int c, int C) { return T / C * c + T % C * c / C; }
__host__ __device__ inline int prefix_block_of(int pos, int T, int C) { return (int)((((int64_t)pos + 1) * C - 1) / T); }

}  // namespace plt

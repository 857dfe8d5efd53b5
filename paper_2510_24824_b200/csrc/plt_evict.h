// Host-side interface between the C ABI of cache eviction and its kernels.
#pragma once
#include "plt_host.h"

namespace plt {

// ---- attention weights ------------------------------------------------------------------------------------------
// The work of plt_cache_evict_weights is three or four kernels over one batch of sequences:
//   scores  streams K: for every packed row the maximum (log2 units) and the sum of exponentials over the block's piece of
//           the keys; up to 16 rows also all scores into a scratch array
//   join    joins the pieces' statistics
//   sums    above 16 rows: streams K again and leaves 2^(score - max) * rho / sum added up over the rows in the scratch array
//   add     up to 16 rows: adds 2^(score - max) * rho / sum over the rows of a head group to the totals; fold, above: adds
//           up the sums of a head group
struct EvictWeights {
    Params p;                  // plan, query rows, lengths, pages; w = 0, hpc and tile_keys of the scores kernel
    int32_t b0;                // first sequence of this launch (the pointers in p are shifted already, K's tensor map is not)
    int32_t kw;                // warps along the keys of a tile of the scores kernel (each leaves statistics of its own)
    int32_t kbox;              // keys per TMA box
    int32_t row_pitch;         // rows rounded up to a multiple of four
    int32_t key_pitch;         // floats of a key in the scratch: row_pitch scores, or (twice) sums over each share of the rows
    int32_t tile_shift;        // log2 of p.tile_keys
    int32_t hpg;               // KV heads of a group
    int32_t min_delta;         // smallest causal offset: positions below length - min_delta have scores
    float* scores;             // [place on p's line][head of the tile][key][key_pitch]
    float* ml;                 // [slot of p's plan][head][kw][R][2] maximum and sum of a piece
    float2* mc;                // [B][Hkv][row_pitch] maximum of a row and rho / sum (0 where there is no row or no key)
    float* weights;            // [B][Hkv / hpg] rows, weights_stride apart
    int64_t weights_stride;
    const float* gate;         // [B, L-1, Qn, Hq] or null
    float decay;
};

constexpr int kEvictF32Keys = 32;      // keys per tile of the fp32 scores kernel

// Blocks of a plan of T tiles: at least `least` tiles each.
__host__ __device__ inline int evict_ctas(int64_t T, int launched, int least) {
    int64_t c = T / least;
    if (c < 1) c = 1;
    return c < launched ? (int)c : launched;
}
constexpr int kEvictScoreTiles = 2;    // least tiles per block of the scores kernel
constexpr int kEvictPieceCost = 3;     // what starting and finishing an item costs a block of it, in tiles

struct ScoreVariant {
    int D, NT, RS, HPC;    // head dim (elements), 8-row groups of a warp, warps that share the rows, KV heads per block
    bool fp8;
    bool twice;            // K is streamed twice (statistics, then sums) instead of leaving its scores in the scratch
    int KW, KS, tile_keys; // derived: HPC * KW = 4 consumer warps for each share of the rows, KS 16-key slices each
    int stages;
    size_t smem;
};
ScoreVariant score_variant(int D, int R, int Hkv, bool fp8, int max_batch);
cudaError_t scores_prepare(const ScoreVariant& v, int* blocks_per_sm);
cudaError_t launch_scores(const ScoreVariant& v, const CUtensorMap& mapK, const EvictWeights& e, int grid, cudaStream_t stream);
cudaError_t launch_sums(const ScoreVariant& v, const CUtensorMap& mapK, const EvictWeights& e, int grid, cudaStream_t stream);
size_t scores_f32_smem(int D, int R, int max_batch);
cudaError_t scores_f32_prepare(int D, int R, int max_batch, int* blocks_per_sm);
cudaError_t launch_scores_f32(const EvictWeights& e, int grid, size_t smem, cudaStream_t stream);
cudaError_t launch_evict_join(const EvictWeights& e, cudaStream_t stream);
size_t evict_add_smem(int max_batch);
cudaError_t evict_add_prepare(bool twice, int key_pitch, size_t smem, int* blocks_per_sm);
cudaError_t launch_evict_add(const EvictWeights& e, bool twice, int grid, size_t smem, cudaStream_t stream);

// ---- selection ----------------------------------------------------------------------------------------------------
struct SelectParams {
    const float* weights;
    int64_t weights_stride;
    const int32_t* seq_lens;
    int32_t* keep;
    int32_t* new_lens;
    uint32_t* status;
    int32_t groups, max_seq_len, budget, keep_first, keep_last;
    int32_t sm_count;
};
cudaError_t launch_select(const SelectParams& p, int batch, cudaStream_t stream);

// ---- compaction ---------------------------------------------------------------------------------------------------
struct CompactParams {
    char *k, *v;                       // bytes
    int64_t stride_b, stride_n, stride_h;   // bytes
    const int32_t *page_table, *seq_lens, *keep, *new_lens;
    float* weights;
    int64_t weights_stride;
    uint32_t* status;
    int32_t Hkv, hpg, row_bytes, max_seq_len, page_size, page_shift /* log2 of a page that is a power of two, else -1 */;
    int32_t max_pages, num_pool_pages, keep_stride;
};
cudaError_t launch_compact(const CompactParams& p, int batch, cudaStream_t stream);

}  // namespace plt

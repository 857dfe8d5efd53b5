// Instantiates the scores kernel for one head dimension and cache type (PLT_SCORE_D, PLT_SCORE_FP8, PLT_SCORE_NAME): packed
// rows up to 8 or 16 (scores to the scratch), up to 32 or 64 (K twice), and 1, 2 or 4 KV heads per block.
#include "plt_evict_scores.cuh"

namespace plt {

namespace {

template <int NT, int RS, int HPC, int MODE>
cudaError_t score_op(int op, const ScoreVariant& v, const CUtensorMap* map, const EvictWeights* e, int grid, cudaStream_t stream,
                     int* out) {
    using C = ScoreCfg<PLT_SCORE_D, NT, RS, HPC, PLT_SCORE_FP8>;
    auto fn = plt_evict_scores<PLT_SCORE_D, NT, RS, HPC, PLT_SCORE_FP8, MODE>;
    if (op == 0) {   // geometry: shared memory for v.stages stages and the batch in `grid`
        *out = (int)C::smem_bytes(v.stages, grid);
        return cudaSuccess;
    }
    if (op == 1) {
        const cudaError_t err = allow_max_dynamic_smem((const void*)fn);
        if (err != cudaSuccess) return err;
        return cudaOccupancyMaxActiveBlocksPerMultiprocessor(out, fn, C::NTHREADS, v.smem);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(C::NTHREADS);
    cfg.dynamicSmemBytes = v.smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, fn, *map, *e, v.stages);
}

template <int NT, int RS, int HPC>
cudaError_t score_mode(int op, int mode, const ScoreVariant& v, const CUtensorMap* map, const EvictWeights* e, int grid,
                       cudaStream_t stream, int* out) {
    if constexpr (RS == 1) return score_op<NT, RS, HPC, kScoreDump>(op, v, map, e, grid, stream, out);
    else return mode == kScoreSums ? score_op<NT, RS, HPC, kScoreSums>(op, v, map, e, grid, stream, out)
                                   : score_op<NT, RS, HPC, kScoreStats>(op, v, map, e, grid, stream, out);
}

template <int NT, int RS>
cudaError_t score_heads(int op, int mode, const ScoreVariant& v, const CUtensorMap* map, const EvictWeights* e, int grid,
                        cudaStream_t stream, int* out) {
    if (v.HPC == 4) return score_mode<NT, RS, 4>(op, mode, v, map, e, grid, stream, out);
    if (v.HPC == 2) return score_mode<NT, RS, 2>(op, mode, v, map, e, grid, stream, out);
    return score_mode<NT, RS, 1>(op, mode, v, map, e, grid, stream, out);
}

}  // namespace

cudaError_t PLT_SCORE_NAME(int op, int mode, const ScoreVariant& v, const CUtensorMap* map, const EvictWeights* e, int grid,
                           cudaStream_t stream, int* out) {
    if (v.NT == 1) return score_heads<1, 1>(op, mode, v, map, e, grid, stream, out);
    if (v.RS == 1) return score_heads<2, 1>(op, mode, v, map, e, grid, stream, out);
    return v.RS == 2 ? score_heads<2, 2>(op, mode, v, map, e, grid, stream, out)
                     : score_heads<2, 4>(op, mode, v, map, e, grid, stream, out);
}

}  // namespace plt

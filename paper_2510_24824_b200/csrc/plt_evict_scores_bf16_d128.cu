#define PLT_SCORE_D 128
#define PLT_SCORE_FP8 false
#define PLT_SCORE_NAME scores_bf16_d128
#include "plt_evict_scores_inst.inl"

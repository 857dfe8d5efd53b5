#define PLT_SCORE_D 64
#define PLT_SCORE_FP8 false
#define PLT_SCORE_NAME scores_bf16_d64
#include "plt_evict_scores_inst.inl"

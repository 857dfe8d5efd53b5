#define PLT_SCORE_D 128
#define PLT_SCORE_FP8 true
#define PLT_SCORE_NAME scores_e4m3
#include "plt_evict_scores_inst.inl"

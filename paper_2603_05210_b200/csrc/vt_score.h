// Token scoring: host side (vt_score.cu, vt_score_grad.cu).
#pragma once

#include "vt_launch.h"

namespace vt {

struct ScoreCall {      // after validation, all pointers device
    const void* h;
    int64_t ldh;
    const void* W;
    const int32_t* tokens;      // null: no given tokens, every row is scored
    int M, d, V;
    float scale;
};
struct ScoreOut {
    float *logprobs, *entropy, *lse;     // each may be null
    int32_t* top_ids;
    float* top_logprobs;
    int k;
};

// A row counts as scored when it has a token inside the vocabulary, or when no tokens are given at all.
#ifdef __CUDACC__
__device__ __forceinline__ bool row_scored(const int32_t* tokens, int V, int m) {
    return tokens == nullptr || (unsigned)tokens[m] < (unsigned)V;
}
#endif

size_t score_workspace_bytes(int M, int d, int V, int k);
size_t score_backward_workspace_bytes(int M, int d, int V);
vt_status launch_score(const ScoreCall& c, const ScoreOut& o, void* workspace, size_t workspace_bytes, cudaStream_t st);   // checks the size itself
vt_status launch_score_backward(const ScoreCall& c, const float* lse, const float* entropy, const float* grad_logprobs,
                                const float* grad_entropy, void* grad_h, void* grad_W, void* workspace, cudaStream_t st);

}  // namespace vt

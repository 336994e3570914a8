// Gated feed-forward block: host side (vt_ffn.cu).
#pragma once

#include "vt_launch.h"

namespace vt {

struct FfnCall {       // after validation, all pointers device
    const void* x;
    int64_t ldx;
    const void *W_gate, *W_up, *W_down;
    int M, d, f, act;
};

size_t ffn_workspace_bytes(int M, int d, int f);
size_t ffn_backward_workspace_bytes(int M, int d, int f);
vt_status launch_ffn(const FfnCall& c, void* y, float* saved, void* workspace, cudaStream_t st);
vt_status launch_ffn_backward(const FfnCall& c, const float* saved, const void* grad_y, int64_t ld_grad_y, void* grad_x,
                              void* grad_W_gate, void* grad_W_up, void* grad_W_down, void* workspace, cudaStream_t st);

}  // namespace vt

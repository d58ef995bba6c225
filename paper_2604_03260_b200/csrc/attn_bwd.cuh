// What the entry points hand to the attention's backward pass.
#pragma once

#include "attn_common.cuh"

namespace focus {

struct AttnBwdArgs {
    focus_shape s;
    focus_tensor q, k, v, o, dO, dq, dk, dv;
    const uint32_t* mq;
    const uint32_t* mk;
    const char* tiles;        // nullptr = every causal pair
    focus_tiles_layout L;     // valid when tiles != nullptr
    const float* lse;
    float scale;              // resolved logit scale
    const float* g;           // training-time soft gate: assignments [batch, n, ld]; nullptr = no gate
    float lambda;
    float* dg;
    char* ws;
    int32_t* dev_status;
};

size_t attn_bwd_workspace_bytes(const focus_shape* s, bool gate);
int launch_attn_bwd(const AttnBwdArgs& a, cudaStream_t st);

}  // namespace focus

// Launchers of head_rotation.hip: the arguments as daf_attention.h has them, checked.
#pragma once
#include <hip/hip_runtime.h>

#include "daf_attention.h"

constexpr int kRotationMaxDim = 256;

int64_t daf_head_rotation_workspace_size(int64_t tokens, int head_dim);   // bytes, of the backward pass
hipError_t daf_launch_head_rotation(const daf_head_rotation_t& p, const daf_heads_t& q, const daf_heads_t& k, const daf_heads_t* v, const daf_heads_t& out_q,
                                    const daf_heads_t& out_k, const daf_heads_t* out_v, const int32_t* rows, int64_t out_rows, hipStream_t stream);
hipError_t daf_launch_head_rotation_backward(const daf_head_rotation_t& p, const daf_heads_t& q, const daf_heads_t& k, const daf_heads_t& grad_q,
                                             const daf_heads_t& grad_k, const daf_heads_t& out_grad_q, const daf_heads_t& out_grad_k, float* out_grad_q_weight,
                                             float* out_grad_k_weight, float* partial, hipStream_t stream);

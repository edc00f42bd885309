// Launchers of residual_norm.hip: the arguments as daf_block.h has them, checked.
#pragma once
#include <hip/hip_runtime.h>

#include "daf_block.h"

constexpr int64_t kResidualNormMaxCols = 16384;

int64_t daf_residual_norm_workspace_size(int64_t rows, int64_t cols, int64_t gate_groups);   // bytes, of the backward pass
hipError_t daf_launch_residual_norm(const daf_residual_norm_t& p, const void* residual, const void* z, void* out_residual, void* out_y,
                                    float* out_stats, hipStream_t stream);
hipError_t daf_launch_residual_norm_backward(const daf_residual_norm_t& p, const void* sum, const void* z, const float* stats, const void* grad_y,
                                             const void* grad_sum, void* out_grad_residual, void* out_grad_z,
                                             const daf_residual_norm_grads_t& grads, float* partial, hipStream_t stream);

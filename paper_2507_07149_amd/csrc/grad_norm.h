// Launcher of grad_norm.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "daf_block.h"

constexpr int kGradNormBlocks = 2048;            // eight workgroups on each of 256 compute units: partial sums in the workspace

hipError_t daf_launch_grad_norm(const daf_grad_item_t* items, int32_t n_items, bool clip, float max_norm, float* out_norm, double* partial,
                                hipStream_t stream);

// Launchers of gated_linear.hip: arguments checked, sizes of 1 and more.
#pragma once
#include <hip/hip_runtime.h>

#include "daf_block.h"

struct GatedSizes {
  int64_t m, n, k;
};
struct GatedLinear {
  GatedSizes sizes;
  int dtype, act;
  const void *x, *w_gate, *w_up;
  char* workspace;
};

void daf_gated_schedule(const GatedSizes& sizes, int product, daf_gated_schedule_t* out);   // a daf_gated_product_t
int64_t daf_gated_workspace_size(const GatedSizes& sizes, bool backward);      // bytes
hipError_t daf_launch_gated_linear(const GatedLinear& g, void* out_h, void* out_gate, void* out_up, hipStream_t stream);
hipError_t daf_launch_gated_linear_backward(const GatedLinear& g, const void* grad_h, const void* gate, const void* up, void* out_grad_x,
                                            void* out_grad_w_gate, void* out_grad_w_up, void* out_h, hipStream_t stream);
hipError_t daf_launch_clear(void* out, int64_t bytes, hipStream_t stream);     // a multiple of 2

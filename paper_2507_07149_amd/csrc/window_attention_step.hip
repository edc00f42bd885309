// Attention with a window and sinks for one query of each of many sequences (daf_window_attention_step).
#include "window_attention_device.h"

namespace {

template <int DT>
__global__ __launch_bounds__(kWave) void k_attention_step(const Attention a) {
  Sequence s = sequence_of(a, blockIdx.x);
  s.q_begin = blockIdx.x;
  s.queries = 1;
  attend_row<DT>(a, s, 0, blockIdx.y);
}

}  // namespace

int64_t daf_window_attention_step_workspace_size(int64_t sequences, int q_heads, int kv_heads, int head_dim, int64_t k_rows, int64_t window, int64_t sinks) {
  return 0;
}

hipError_t daf_launch_window_attention_step(const daf_window_attention_t& p, const AttentionTensors& t, char* workspace, hipStream_t stream) {
  if (p.q_rows == 0) return hipSuccess;
  const Attention a = attention_of(p, t);
  const dim3 grid((unsigned)p.sequences, (unsigned)p.q_heads);
  if (p.dtype == DAF_F16) k_attention_step<kF16><<<grid, kWave, 0, stream>>>(a);
  else k_attention_step<kBF16><<<grid, kWave, 0, stream>>>(a);
  return hipGetLastError();
}

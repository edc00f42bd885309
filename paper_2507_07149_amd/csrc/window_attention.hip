// Attention with a window and sinks, forward (daf_window_attention).
#include "window_attention_device.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave, kRows = 32;

template <int DT>
__global__ __launch_bounds__(kThreads) void k_window_attention(const Attention a, int tiles) {
  const Turn turn = turn_of_workgroup(tiles);
  const TileOf at = find_tile<kRows>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  for (int i = at.tile * kRows + threadIdx.x / kWave; i < min(s.queries, (at.tile + 1) * kRows); i += kWaves) attend_row<DT>(a, s, i, turn.head);
}

}  // namespace

hipError_t daf_launch_window_attention(const daf_window_attention_t& p, const AttentionTensors& t, hipStream_t stream) {
  if (p.q_rows == 0) return hipSuccess;
  const Attention a = attention_of(p, t);
  const int64_t tiles = most_tiles(p, kRows);
  const unsigned blocks = (unsigned)(tiles * p.q_heads);
  if (p.dtype == DAF_F16) k_window_attention<kF16><<<blocks, kThreads, 0, stream>>>(a, (int)tiles);
  else k_window_attention<kBF16><<<blocks, kThreads, 0, stream>>>(a, (int)tiles);
  return hipGetLastError();
}

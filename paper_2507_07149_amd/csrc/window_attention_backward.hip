// Attention with a window and sinks, backward (daf_window_attention_backward).
#include "window_attention_device.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave, kRows = 32;

struct Backward : Attention {
  Heads grad_out, grad_q, grad_k, grad_v;
  float* delta;                // [q_heads, rows]: sum of grad_out * out over the head
};

// delta: eight elements to a lane, head_dim / 8 lanes (of 16) to a row.
template <int DT>
__global__ __launch_bounds__(kThreads) void k_attention_delta(const Backward a) {
  const int64_t n = (int64_t)blockIdx.x * (kThreads / 16) + threadIdx.x / 16, row = n / a.q_heads;
  const int head = (int)(n % a.q_heads), d = threadIdx.x % 16 * 8;
  float sum = 0.0f;
  if (row < a.q_rows && d < a.dim) {
    float x[8], y[8];
    widen_unit<DT>(load_unit<DT>(a.out.at + row * a.out.token + head * a.out.head + d * 2), x);
    widen_unit<DT>(load_unit<DT>(a.grad_out.at + row * a.grad_out.token + head * a.grad_out.head + d * 2), y);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[i], y[i], sum);
  }
  sum += u2f(dpp<kDppXor1>(0u, f2u(sum)));
  sum += u2f(dpp<kDppXor2>(0u, f2u(sum)));
  sum += u2f(dpp<kDppHalfMirror>(0u, f2u(sum)));
  sum += u2f(dpp<kDppMirror>(0u, f2u(sum)));
  if (row < a.q_rows && d == 0) a.delta[(int64_t)head * a.q_rows + row] = sum;
}

// grad_q of one query by a wave, as attend_row.
template <int DT>
__device__ __forceinline__ void query_row(const Backward& a, const Sequence& s, int i, int head) {
  const int lane = threadIdx.x % kWave, low = window_begin(a, i);
  const int64_t row = (int64_t)s.q_begin + i;
  const char* const q = a.q.at + row * a.q.token + head * a.q.head;
  const char* const grad = a.grad_out.at + row * a.grad_out.token + head * a.grad_out.head;
  const char* const k = a.k.at + s.k_begin * a.k.token + head / a.group * a.k.head;
  const char* const v = a.v.at + s.k_begin * a.v.token + head / a.group * a.v.head;
  const float lse = a.lse[(int64_t)head * a.q_rows + row], delta = a.delta[(int64_t)head * a.q_rows + row];
  const int sinks = min(a.sinks, low), seen = sinks + i - low + 1;
  float lo = 0.0f, hi = 0.0f;
  for (int first = 0; first < seen; first += kWave) {
    const int n = first + lane, j = n < sinks ? n : low + n - sinks, count = min(seen - first, kWave);
    float grad_s = 0.0f;
    if (lane < count) {
      const float p = __builtin_amdgcn_exp2f((row_dot<DT>(q, k + j * a.k.token, a.dim) * a.scale - lse) * kLog2E);
      grad_s = p * (row_dot<DT>(grad, v + j * a.v.token, a.dim) - delta) * a.scale;
    }
    for (int t = 0; t < count; ++t) {
      const float weight = u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(grad_s), t));
      const Two x = load_two<DT>(k + __builtin_amdgcn_readlane(j, t) * a.k.token, a.dim);
      lo = __builtin_fmaf(weight, x.lo, lo);
      hi = __builtin_fmaf(weight, x.hi, hi);
    }
  }
  store_two<DT>(a.grad_q.at + row * a.grad_q.token + head * a.grad_q.head, a.dim, lo, hi);
}

// grad_k and grad_v of one key by a wave: a query to a lane.
template <int DT>
__device__ __forceinline__ void key_row(const Backward& a, const Sequence& s, int j, int kv_head) {
  const int lane = threadIdx.x % kWave;
  const int64_t row = (int64_t)s.k_begin + j;
  const char* const k = a.k.at + row * a.k.token + kv_head * a.k.head;
  const char* const v = a.v.at + row * a.v.token + kv_head * a.v.head;
  const int last = j < a.sinks ? s.queries - 1 : (int)min((int64_t)s.queries - 1, (int64_t)j + a.window - 1);
  float k_lo = 0.0f, k_hi = 0.0f, v_lo = 0.0f, v_hi = 0.0f;
  for (int head = kv_head * a.group; head < (kv_head + 1) * a.group; ++head) {
    const char* const q = a.q.at + s.q_begin * a.q.token + head * a.q.head;
    const char* const grad = a.grad_out.at + s.q_begin * a.grad_out.token + head * a.grad_out.head;
    const int64_t stat = (int64_t)head * a.q_rows + s.q_begin;
    for (int first = j; first <= last; first += kWave) {
      const int i = first + lane, count = min(last - first + 1, kWave);
      float p = 0.0f, grad_s = 0.0f;
      if (lane < count) {
        p = __builtin_amdgcn_exp2f((row_dot<DT>(q + i * a.q.token, k, a.dim) * a.scale - a.lse[stat + i]) * kLog2E);
        grad_s = p * (row_dot<DT>(grad + i * a.grad_out.token, v, a.dim) - a.delta[stat + i]) * a.scale;
      }
      for (int t = 0; t < count; ++t) {
        const float wp = u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(p), t)), ws = u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(grad_s), t));
        const Two x = load_two<DT>(q + (first + t) * a.q.token, a.dim), y = load_two<DT>(grad + (first + t) * a.grad_out.token, a.dim);
        k_lo = __builtin_fmaf(ws, x.lo, k_lo);
        k_hi = __builtin_fmaf(ws, x.hi, k_hi);
        v_lo = __builtin_fmaf(wp, y.lo, v_lo);
        v_hi = __builtin_fmaf(wp, y.hi, v_hi);
      }
    }
  }
  store_two<DT>(a.grad_k.at + row * a.grad_k.token + kv_head * a.grad_k.head, a.dim, k_lo, k_hi);
  store_two<DT>(a.grad_v.at + row * a.grad_v.token + kv_head * a.grad_v.head, a.dim, v_lo, v_hi);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void k_attention_grad_q(const Backward a, int tiles) {
  const Turn turn = turn_of_workgroup(tiles);
  const TileOf at = find_tile<kRows>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  for (int i = at.tile * kRows + threadIdx.x / kWave; i < min(s.queries, (at.tile + 1) * kRows); i += kWaves) query_row<DT>(a, s, i, turn.head);
}
template <int DT>
__global__ __launch_bounds__(kThreads) void k_attention_grad_kv(const Backward a, int tiles) {
  const Turn turn = turn_of_workgroup(tiles);
  const TileOf at = find_tile<kRows>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  for (int j = at.tile * kRows + threadIdx.x / kWave; j < min(s.keys, (at.tile + 1) * kRows); j += kWaves) key_row<DT>(a, s, j, turn.head);
}

}  // namespace

int64_t daf_window_attention_backward_workspace_size(int64_t rows, int q_heads, int kv_heads, int head_dim, int64_t sequences, int64_t window, int64_t sinks) {
  return rows * q_heads * (int64_t)sizeof(float);
}

hipError_t daf_launch_window_attention_backward(const daf_window_attention_t& p, const AttentionTensors& t, const AttentionGradients& g, char* workspace,
                                                hipStream_t stream) {
  if (p.q_rows == 0) return hipSuccess;
  Backward a = {};
  static_cast<Attention&>(a) = attention_of(p, t);
  a.grad_out = heads_of(g.grad_out, p.q_rows);
  a.grad_q = heads_of(g.grad_q, p.q_rows);
  a.grad_k = heads_of(g.grad_k, p.q_rows);
  a.grad_v = heads_of(g.grad_v, p.q_rows);
  a.delta = reinterpret_cast<float*>(workspace);
  const int64_t tiles = most_tiles(p, kRows);
  auto launch = [&](auto dt) {
    constexpr int kDT = decltype(dt)::value;
    k_attention_delta<kDT><<<(unsigned)((p.q_rows * p.q_heads + 15) / 16), kThreads, 0, stream>>>(a);
    k_attention_grad_q<kDT><<<(unsigned)(tiles * p.q_heads), kThreads, 0, stream>>>(a, (int)tiles);
    k_attention_grad_kv<kDT><<<(unsigned)(tiles * p.kv_heads), kThreads, 0, stream>>>(a, (int)tiles);
  };
  if (p.dtype == DAF_F16) launch(std::integral_constant<int, kF16>{});
  else launch(std::integral_constant<int, kBF16>{});
  return hipGetLastError();
}

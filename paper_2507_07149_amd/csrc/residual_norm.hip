// The norms, gate and residual sum between two blocks (daf_residual_norm) and their backward pass.
//
//   forward   p = post(z), s = r + scale * gate * p, y = pre(s)
//   backward  with u = (s - mean) * rstd, n = grad_y * pre_weight:
//               grad_s = grad_sum + rstd * (n - mean(n) - u * mean(n * u))          (mean(n) left out by RMS norms)
//               grad_pre_weight = sum over rows of grad_y * u, grad_pre_bias = sum of grad_y
//             with v = (z - post_mean) * post_rstd, d = scale * grad_s, A = sum of d * v, B = sum of d over the rows of a gate's row:
//               grad_gate = w A + b B, grad_post_weight = gate A, grad_post_bias = gate B   (two sums for three vectors),
//               grad_z = post_rstd * (n - mean(n) - v * mean(n v)) with n = d gate w;  or d gate, and grad_gate = sum of d * z, where z is
//               not normalized
//
// Bound by memory: four tensors forward, six backward.  So a row is read once and stays in registers, eight elements at a time, over
// both norms: a wave for rows of up to 1024 elements, a workgroup for longer ones.  Every thread keeps its columns for all
// rows that it meets, so that the vectors are loaded once and their gradients add up in registers; the workgroups' sums go through
// memory and are added by a second launch in a fixed order (no atomics: the same bits every time).
// 32768 x 4096 bfloat16: forward 201 us (1074 MB, 5.3 TB/s), backward with two norms and gates 329 us (1612 MB, 4.9 TB/s); a copy reaches 4.9.
// What is short is latency: 1576 x 768 forward 6 us, of which the launch is most.
// The residual sum and its gradient are read again after the block's products, y and grad_z at once: the first two are stored past the caches.  (With the
// quantize pass that reads y, and grad_z, behind it: 32768 x 4096 bfloat16 249 -> 242 us and 373 -> 366, 8192 x 4096 61.8 -> 60.8 and 101 -> 98.7; with all
// four stored so 258 and 374, 66 and 103.)
#include "block_common.h"
#include "residual_norm.h"

namespace {

struct Vectors {
  const char *pre_weight, *pre_bias, *post_weight, *post_bias, *gate;
};
struct Forward {
  const char *residual, *z;
  char *sum, *y;
  float4* stats;
  Vectors vectors;
  int32_t rows, cols, rows_per_gate;
  int32_t layer;
  float eps, scale;
};

// A value that is the same in all lanes, in a scalar register.
__device__ __forceinline__ float uniform(float v) { return u2f((uint32_t)__builtin_amdgcn_readfirstlane((int)f2u(v))); }

// The same elements, of which the compiler knows nothing: what a pass computes from them is computed again by the next one instead of being
// kept in registers in between.
template <int DT>
__device__ __forceinline__ Unit<DT> again(Unit<DT> u) {
#pragma unroll
  for (auto& q : u.q) asm volatile("" : "+v"(q));
  return u;
}

// The columns of thread `t` of the T that share a row: units t, t + T, ... of eight.  A column's place is the same in all rows.
//
// A unit that the row does not fill is loaded as the row's last eight elements and put right where it is used: every lane loads, without a
// branch that would hold the loads of the next row up (3879 x 4088 bfloat16 backward 85 us with such branches, 63 without; 3879 x 4096 61).
template <int DT, int T, int NV>
struct Columns {
  static constexpr int kBytes = ElemTraits<DT>::kBytes;
  static constexpr bool kFew = T == kWave;           // only here rows can have fewer than eight elements
  int32_t cols;
  int count[NV];                                     // elements of the unit that exist: 8 or more, 1 ... 7 at the end of the row, 0 or less
  __device__ __forceinline__ Columns(int t, int cols) : cols(cols) {
#pragma unroll
    for (int j = 0; j < NV; ++j) count[j] = cols - (j * T + t) * 8;
  }
  static __device__ __forceinline__ int64_t at(int t, int j) { return (int64_t)(j * T + t) * 8 * kBytes; }
  // What is to be settled before it is used.
  __device__ __forceinline__ Unit<DT> load(const char* row, int t, int j) const {
    if (kFew && cols < 8) return load_unit_part<DT>(row + at(t, j), count[j]);
    uint32_t place = (uint32_t)min((j * T + t) * 8, cols - 8) * kBytes;
    asm volatile("" : "+v"(place));                  // added to a scalar base by the load: no address is kept in registers
    return load_unit<DT>(row + place);
  }
  // Beyond the row's end: zeros, or (ZEROS false, where they are multiplied by zero later on) elements of the row, which are as finite as those that count.
  template <bool ZEROS = true>
  __device__ __forceinline__ Unit<DT> settled(const Unit<DT>& u, int j) const {
    if (count[j] >= 8 || (kFew && cols < 8)) return u;
    int n = count[j];
    asm volatile("" : "+v"(n));                      // not computed ahead of the rows
    return unit_from_row_end<DT, ZEROS>(u, n);
  }
  // v = `value` beyond the row's end.
  __device__ __forceinline__ void fill_end(float (&v)[8], int j, float value) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < count[j] ? v[e] : value;
  }
  __device__ __forceinline__ void load(Unit<DT> (&u)[NV], const char* row, int t) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) u[j] = load(row, t, j);
  }
  __device__ __forceinline__ void store(char* row, int t, int j, const Unit<DT>& u) const { store_unit_of<DT>(row + at(t, j), u, count[j]); }
  __device__ __forceinline__ void stream(char* row, int t, int j, const Unit<DT>& u) const {
    if (count[j] >= 8) stream_unit<DT>(row + at(t, j), u);
    else store_unit_part<DT>(row + at(t, j), u, count[j]);
  }
  template <bool ZEROS = true>
  __device__ __forceinline__ Unit<DT> at_once(const char* row, int t, int j) const {
    return settled<ZEROS>(load(row, t, j), j);
  }
  // A vector of parameters; where there is none, `otherwise` in its place (zero beyond the row's end in either case).
  __device__ __forceinline__ Unit<DT> vector_unit(const char* vector, int t, int j, float otherwise) const {
    if (vector != nullptr) return at_once(vector, t, j);
    if (otherwise == 0.0f) return Unit<DT>{};
    int n = count[j];
    asm volatile("" : "+v"(n));                      // made where it is used: not kept in registers from the start
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? otherwise : 0.0f;
    return narrow_unit<DT>(v);
  }
  __device__ __forceinline__ void load_vector(Unit<DT> (&u)[NV], const char* vector, int t, float otherwise) const {
#pragma unroll
    for (int j = 0; j < NV; ++j) u[j] = vector_unit(vector, t, j, otherwise);
  }
};

// Sums over the T threads of a row, for everybody.  The waves' sums go through LDS: lane l takes those of wave l mod kWaves, and
// they are added across the lanes.  Two copies of the exchange space in turn: one barrier each.
template <int T>
struct RowSums {
  static constexpr int kWaves = T / kWave;
  float2 (*space)[kWaves];
  int turn = 0;
  __device__ __forceinline__ float2 exchange(float2 mine, int t) {
    if constexpr (kWaves == 1) return mine;
    if ((t & (kWave - 1)) == 0) space[turn][t / kWave] = mine;
    __syncthreads();
    const float2 other = space[turn][t & (kWaves - 1)];
    turn ^= 1;
    return other;
  }
  static __device__ __forceinline__ float over_waves(float v) {
    if constexpr (kWaves > 1) v += u2f(dpp<kDppXor1>(0u, f2u(v)));
    if constexpr (kWaves > 2) v += u2f(dpp<kDppXor2>(0u, f2u(v)));
    if constexpr (kWaves > 4) v += u2f(dpp<kDppHalfMirror>(0u, f2u(v)));
    if constexpr (kWaves > 8) v += u2f(dpp<kDppMirror>(0u, f2u(v)));
    return v;
  }
  __device__ __forceinline__ float2 sum(float a, float b, int t) {
    const float2 s = exchange(make_float2(wave_sum(a), wave_sum(b)), t);
    return make_float2(over_waves(s.x), over_waves(s.y));
  }
};

// Elements of wave `w` of a row's threads.
template <int T, int NV>
__device__ __forceinline__ float wave_count(int w, int cols) {
  int c = 0;
#pragma unroll
  for (int j = 0; j < NV; ++j) c += min(max(cols - (j * T + w * kWave) * 8, 0), kWave * 8);
  return (float)c;
}

// Mean and 1 / sqrt(variance + eps) of a row whose elements the threads hold; elements beyond its end are zero.  The squares are taken
// around the mean of the wave's own elements and the waves' results joined afterwards: as exact as two passes, with one exchange.
template <int DT, int T, int NV>
__device__ __forceinline__ float2 row_statistics(const float (&v)[NV][8], const Columns<DT, T, NV>& columns, int cols, bool layer, float eps,
                                                 RowSums<T>& sums, int t) {
  float squares = 0.0f, total = 0.0f;
  if (!layer) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) squares = __builtin_fmaf(v[j][e], v[j][e], squares);
    const float2 s = sums.sum(squares, 0.0f, t);
    return make_float2(0.0f, 1.0f / __builtin_sqrtf(s.x / (float)cols + eps));
  }
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) total += v[j][e];
  total = wave_sum(total);
  const float own = wave_count<T, NV>(t / kWave, cols);
  const float own_mean = own > 0.0f ? total / own : 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = e < columns.count[j] ? v[j][e] - own_mean : 0.0f;
      squares = __builtin_fmaf(d, d, squares);
    }
  const float2 other = sums.exchange(make_float2(total, wave_sum(squares)), t);
  const float mean = RowSums<T>::over_waves(other.x) / (float)cols;
  const float n = wave_count<T, NV>(t & (RowSums<T>::kWaves - 1), cols);
  const float d = n > 0.0f ? other.x / n - mean : 0.0f;
  const float m2 = RowSums<T>::over_waves(__builtin_fmaf(n * d, d, other.y));
  return make_float2(mean, 1.0f / __builtin_sqrtf(m2 / (float)cols + eps));
}

constexpr int threads_of(int T) { return T < 128 ? 256 : T; }

// The scheduler moves no instruction across: units are worked on one after the other, which keeps the registers of one of them in use.
__device__ __forceinline__ void next_unit() { __builtin_amdgcn_sched_barrier(0); }
// What the registers hold.  Vectors stay in them, what is read does between the passes over a row (backward), and the next row is on its
// way while a row is worked on; not all of it in rows of more than 8192 elements, nor where binary32 columns leave no room: there vectors, and
// rows again, are loaded out of a cache.
template <int T, int NV>
constexpr bool longest() {
  return T * NV * 8 > 8192;
}
template <int DT, int T, int NV>
constexpr bool holds_vectors() {
  return !longest<T, NV>() && !(DT == kF32 && T == 512);
}
template <int DT, int T, int NV>
constexpr bool holds_rows() {
  return !(DT == kF32 && T >= 512);
}

template <int DT, int T, int NV, bool POST>
__global__ __launch_bounds__(threads_of(T)) void k_residual_norm(const Forward p) {
  using C = Columns<DT, T, NV>;
  constexpr bool HOLD = holds_rows<DT, T, NV>(), VECTORS = holds_vectors<DT, T, NV>();
  constexpr int kRows = threads_of(T) / T;                    // rows of a workgroup at a time
  __shared__ float2 space[2][T / kWave];
  const int t = threadIdx.x % T;
  const C columns(t, p.cols);
  RowSums<T> sums{space};
  const int64_t row_bytes = (int64_t)p.cols * ElemTraits<DT>::kBytes;
  const int64_t step = (int64_t)gridDim.x * kRows;

  Unit<DT> pre_w[NV], pre_b[NV], post_w[NV], post_b[NV], gate[NV];
  if constexpr (VECTORS) {
    columns.load_vector(pre_w, p.vectors.pre_weight, t, 1.0f);
    columns.load_vector(pre_b, p.vectors.pre_bias, t, 0.0f);
    if constexpr (POST) {
      columns.load_vector(post_w, p.vectors.post_weight, t, 1.0f);
      columns.load_vector(post_b, p.vectors.post_bias, t, 0.0f);
    }
    columns.load_vector(gate, p.vectors.gate, t, 1.0f);
  }
  auto held = [&](const Unit<DT> (&u)[NV], const char* vector, int j, float otherwise) {
    if constexpr (VECTORS) return again(u[j]);
    return columns.vector_unit(vector, t, j, otherwise);
  };
  int gate_row = 0;

  Unit<DT> next_r[NV], next_z[NV];
  int64_t row = (int64_t)blockIdx.x * kRows + (kRows > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / T) : 0);
  auto fetch = [&](int64_t of_row) {
    columns.load(next_r, p.residual + of_row * row_bytes, t);
    if (p.z != nullptr) columns.load(next_z, p.z + of_row * row_bytes, t);
  };
  if (HOLD && row < p.rows) fetch(row);
  for (; row < p.rows; row += step) {
    const int64_t at = row * row_bytes;
    Unit<DT> raw_r[NV], raw_z[NV];
    if constexpr (HOLD) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        raw_r[j] = columns.settled(next_r[j], j);
        raw_z[j] = columns.settled(next_z[j], j);
      }
      if (row + step < p.rows) fetch(row + step);
    }
    auto read = [&](const Unit<DT> (&u)[NV], const char* tensor, int j) {
      if constexpr (HOLD) return u[j];
      return columns.at_once(tensor + at, t, j);
    };
    float s[NV][8];
    float4 stats = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    bool finite = true;                                       // what the norm of z makes of the zeros beyond the row's end, before their weight of zero
    if (p.z != nullptr) {
      if (const int g = p.rows_per_gate < p.rows ? (int)row / p.rows_per_gate : 0; g != gate_row) {
        gate_row = g;
        if constexpr (VECTORS) columns.load_vector(gate, p.vectors.gate == nullptr ? nullptr : p.vectors.gate + g * row_bytes, t, 1.0f);
      }
#pragma unroll
      for (int j = 0; j < NV; ++j) widen_unit<DT>(read(raw_z, p.z, j), s[j]);
      if constexpr (POST) {
        const float2 st = row_statistics<DT, T, NV>(s, columns, p.cols, p.layer != 0, p.eps, sums, t);
        stats.x = st.x;
        stats.y = st.y;
        finite = __builtin_fabsf(uniform(st.x) * uniform(st.y)) < __builtin_inff();
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          float w[8], b[8];
          widen_unit<DT>(held(post_w, p.vectors.post_weight, j, 1.0f), w);
          widen_unit<DT>(held(post_b, p.vectors.post_bias, j, 0.0f), b);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[j][e] = __builtin_fmaf((s[j][e] - st.x) * st.y, w[e], b[e]);
          next_unit();
        }
      }
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float g[8], r[8];
        widen_unit<DT>(held(gate, p.vectors.gate == nullptr ? nullptr : p.vectors.gate + gate_row * row_bytes, j, 1.0f), g);
        widen_unit<DT>(read(raw_r, p.residual, j), r);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[j][e] = __builtin_fmaf(p.scale * g[e], s[j][e], r[e]);
        next_unit();
      }
      if (!finite) {                                          // (rows of values that are all large and almost the same)
#pragma unroll
        for (int j = 0; j < NV; ++j) columns.fill_end(s[j], j, 0.0f);
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) widen_unit<DT>(read(raw_r, p.residual, j), s[j]);
    }
    if (p.sum != nullptr) {
#pragma unroll
      for (int j = 0; j < NV; ++j) columns.stream(p.sum + at, t, j, narrow_unit<DT>(s[j]));
    }
    if (p.y != nullptr) {
      const float2 st = row_statistics<DT, T, NV>(s, columns, p.cols, p.layer != 0, p.eps, sums, t);
      stats.z = st.x;
      stats.w = st.y;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float w[8], b[8];
        widen_unit<DT>(held(pre_w, p.vectors.pre_weight, j, 1.0f), w);
        widen_unit<DT>(held(pre_b, p.vectors.pre_bias, j, 0.0f), b);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[j][e] = __builtin_fmaf((s[j][e] - st.x) * st.y, w[e], b[e]);
        columns.store(p.y + at, t, j, narrow_unit<DT>(s[j]));
        next_unit();
      }
    }
    if (p.stats != nullptr && t == 0) p.stats[row] = stats;
  }
}

struct Backward {
  const char *sum, *z, *grad_y, *grad_sum;
  const float4* stats;
  char *grad_residual, *grad_z;
  Vectors vectors;
  float* partial[5];                                 // of pre weight, pre bias, post weight, post bias, gate: one row of cols for every workgroup (the gate's
                                                     // may be the gradient itself)
  int32_t cols, rows_per_gate, rows_per_chunk, chunks_per_gate;
  int32_t layer;
  float scale;
};

// BIAS: the sums that biases need are kept too.
template <int DT, int T, int NV, bool POST, bool BIAS>
__global__ __launch_bounds__(threads_of(T)) void k_residual_norm_backward(const Backward p) {
  using C = Columns<DT, T, NV>;
  constexpr bool HOLD = !longest<T, NV>() && !(DT == kF32 && T == 1024);
  constexpr bool AHEAD = HOLD && !(DT == kF32 && T > 256);        // the next row is on its way while a row is worked on
  constexpr int kRows = threads_of(T) / T;
  __shared__ float2 space[2][T / kWave];
  __shared__ float columns_of[kRows > 1 ? kRows : 1][kRows > 1 ? T * NV * 8 : 1];
  const int t = threadIdx.x % T, sub = kRows > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / T) : 0;
  const C columns(t, p.cols);
  RowSums<T> sums{space};
  const int64_t row_bytes = (int64_t)p.cols * ElemTraits<DT>::kBytes;
  const float inv_cols = 1.0f / (float)p.cols;

  // A workgroup's rows: a chunk of those that share a row of the gate.
  const int group = blockIdx.x / p.chunks_per_gate, chunk = blockIdx.x % p.chunks_per_gate;
  const int64_t begin = (int64_t)group * p.rows_per_gate + (int64_t)chunk * p.rows_per_chunk;
  const int64_t end = min(begin + p.rows_per_chunk, (int64_t)(group + 1) * p.rows_per_gate);
  const char* const gate_row = p.vectors.gate == nullptr ? nullptr : p.vectors.gate + group * row_bytes;

  Unit<DT> pre_w[NV], post_w[NV], gate[NV];
  if constexpr (HOLD) {
    columns.load_vector(pre_w, p.vectors.pre_weight, t, 1.0f);
    if constexpr (POST) columns.load_vector(post_w, p.vectors.post_weight, t, 1.0f);
    columns.load_vector(gate, gate_row, t, 1.0f);
  }
  auto held = [&](const Unit<DT> (&u)[NV], const char* vector, int j) {
    if constexpr (HOLD) return again(u[j]);
    return columns.vector_unit(vector, t, j, 1.0f);
  };

  // Sums of grad_y * u, of grad_y; and of d * v (d * z), of d, which stay in LDS in the longest rows (a thread has its own places: no wait).
  constexpr bool IN_LDS = longest<T, NV>();
  __shared__ float post_lds[IN_LDS ? (BIAS ? 2 : 1) : 1][IN_LDS ? NV * 8 : 1][IN_LDS ? T : 1];
  float pre_a[NV][8], pre_sum[BIAS ? NV : 1][8], post_regs[IN_LDS ? 1 : (BIAS ? 2 : 1)][IN_LDS ? 1 : NV][8];
  auto post_at = [&](int which, int j, int e) -> float& {
    if constexpr (IN_LDS) return post_lds[which][j * 8 + e][t];
    else return post_regs[which][j][e];
  };
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      pre_a[j][e] = post_at(0, j, e) = 0.0f;
      if constexpr (BIAS) pre_sum[j][e] = post_at(1, j, e) = 0.0f;
    }

  Unit<DT> raw_y[NV], raw_s[NV], raw_gs[NV], raw_z[NV], next_y[NV], next_s[NV], next_gs[NV], next_z[NV];
  auto load = [&](int64_t row, Unit<DT> (&y)[NV], Unit<DT> (&s)[NV], Unit<DT> (&gs)[NV], Unit<DT> (&z)[NV]) {
    const int64_t at = row * row_bytes;
    if (p.grad_y != nullptr) {
      columns.load(y, p.grad_y + at, t);
      columns.load(s, p.sum + at, t);
    }
    if (p.grad_sum != nullptr) columns.load(gs, p.grad_sum + at, t);
    if (p.z != nullptr) columns.load(z, p.z + at, t);
  };
  if (AHEAD && begin + sub < end) load(begin + sub, next_y, next_s, next_gs, next_z);
  for (int64_t row = begin + sub; row < end; row += kRows) {
    const int64_t at = row * row_bytes;
    if constexpr (AHEAD) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        raw_y[j] = columns.settled(next_y[j], j);
        raw_s[j] = columns.template settled<false>(next_s[j], j);
        raw_gs[j] = columns.settled(next_gs[j], j);
        raw_z[j] = columns.template settled<false>(next_z[j], j);
      }
      if (row + kRows < end) load(row + kRows, next_y, next_s, next_gs, next_z);
    } else if constexpr (HOLD) {
      load(row, raw_y, raw_s, raw_gs, raw_z);
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        raw_y[j] = columns.settled(raw_y[j], j);
        raw_s[j] = columns.template settled<false>(raw_s[j], j);
        raw_gs[j] = columns.settled(raw_gs[j], j);
        raw_z[j] = columns.template settled<false>(raw_z[j], j);
      }
    }
    auto read = [&](const Unit<DT> (&u)[NV], const char* tensor, int j) {
      if constexpr (HOLD) return again(u[j]);
      return columns.at_once(tensor + at, t, j);
    };
    // z and the sum: what they are normalized to has to be finite beyond the row's end too, where it meets gradients and weights of zero.  (0 - mean) * rstd is
    // not in rows of values that are all large and almost the same.
    auto read_values = [&](const Unit<DT> (&u)[NV], const char* tensor, int j, float mean, float (&v)[8]) {
      if constexpr (HOLD) widen_unit<DT>(again(u[j]), v);
      else widen_unit<DT>(columns.template at_once<false>(tensor + at, t, j), v);
      if (C::kFew && p.cols < 8) columns.fill_end(v, j, mean);
    };
    const float4 of_row = p.stats[row];
    const float4 stats = make_float4(uniform(of_row.x), uniform(of_row.y), uniform(of_row.z), uniform(of_row.w));

    float2 mean = make_float2(0.0f, 0.0f);
    if (p.grad_y != nullptr) {
      float a = 0.0f, b = 0.0f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float dy[8], s[8], w[8];
        widen_unit<DT>(read(raw_y, p.grad_y, j), dy);
        read_values(raw_s, p.sum, j, stats.z, s);
        widen_unit<DT>(held(pre_w, p.vectors.pre_weight, j), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = (s[e] - stats.z) * stats.w, n = dy[e] * w[e];
          a += n;
          b = __builtin_fmaf(n, u, b);
          pre_a[j][e] = __builtin_fmaf(dy[e], u, pre_a[j][e]);
          if constexpr (BIAS) pre_sum[j][e] += dy[e];
        }
        next_unit();
      }
      mean = sums.sum(a, b, t);
      mean.x = p.layer ? mean.x * inv_cols : 0.0f;
      mean.y *= inv_cols;
    }
    float ds[NV][8];                                 // gradient of the sum
#pragma unroll
    for (int j = 0; j < NV; ++j) {
#pragma unroll
      for (int e = 0; e < 8; ++e) ds[j][e] = 0.0f;
      if (p.grad_sum != nullptr) widen_unit<DT>(read(raw_gs, p.grad_sum, j), ds[j]);
      next_unit();
      if (p.grad_y != nullptr) {
        float dy[8], s[8], w[8];
        widen_unit<DT>(read(raw_y, p.grad_y, j), dy);
        read_values(raw_s, p.sum, j, stats.z, s);
        widen_unit<DT>(held(pre_w, p.vectors.pre_weight, j), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = (s[e] - stats.z) * stats.w;
          ds[j][e] = __builtin_fmaf(stats.w, __builtin_fmaf(-u, mean.y, __builtin_fmaf(dy[e], w[e], -mean.x)), ds[j][e]);
        }
      }
      next_unit();
      columns.stream(p.grad_residual + at, t, j, narrow_unit<DT>(ds[j]));
      next_unit();
    }
    if (p.z == nullptr) continue;
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      float z[8], g[8], w[8];
      read_values(raw_z, p.z, j, stats.x, z);
      widen_unit<DT>(held(gate, gate_row, j), g);
      if constexpr (POST) widen_unit<DT>(held(post_w, p.vectors.post_weight, j), w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = p.scale * ds[j][e];
        const float v = POST ? (z[e] - stats.x) * stats.y : z[e];
        post_at(0, j, e) = __builtin_fmaf(d, v, post_at(0, j, e));
        ds[j][e] = d * g[e];
        if constexpr (POST) {
          if constexpr (BIAS) post_at(1, j, e) += d;
          ds[j][e] *= w[e];
          a += ds[j][e];
          b = __builtin_fmaf(ds[j][e], v, b);
        }
      }
      if constexpr (!POST) columns.store(p.grad_z + at, t, j, narrow_unit<DT>(ds[j]));
      next_unit();
    }
    if constexpr (POST) {
      float2 m = sums.sum(a, b, t);
      m.x = p.layer ? m.x * inv_cols : 0.0f;
      m.y *= inv_cols;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float z[8];
        widen_unit<DT>(read(raw_z, p.z, j), z);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float v = (z[e] - stats.x) * stats.y;
          z[e] = stats.y * __builtin_fmaf(-v, m.y, ds[j][e] - m.x);
        }
        columns.store(p.grad_z + at, t, j, narrow_unit<DT>(z));
        next_unit();
      }
    }
  }

  // The workgroup's sums of one vector into its row of the partial sums.
  auto write = [&](float* partial, auto value) {
    if (partial == nullptr) return;
    float* const to = partial + (int64_t)blockIdx.x * p.cols;
    if constexpr (kRows > 1) {                       // its rows first
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) columns_of[sub][(j * T + t) * 8 + e] = value(j, e);
      __syncthreads();
      for (int c = threadIdx.x; c < p.cols; c += threads_of(T)) {
        float v = columns_of[0][c];
#pragma unroll
        for (int r = 1; r < kRows; ++r) v += columns_of[r][c];
        to[c] = v;
      }
    } else {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = value(j, e);
        store_unit_of<kF32>(reinterpret_cast<char*>(to + (j * T + t) * 8), narrow_unit<kF32>(v), columns.count[j]);
        next_unit();
      }
    }
  };
  write(p.partial[0], [&](int j, int e) { return pre_a[j][e]; });
  if constexpr (BIAS) write(p.partial[1], [&](int j, int e) { return pre_sum[j][e]; });
  // Vectors again, one element at a time: a few values per workgroup.
  auto element = [&](const char* vector, int j, int e, float otherwise) {
    const int c = (j * T + t) * 8 + e;
    if (vector == nullptr || c >= p.cols) return otherwise;
    if constexpr (DT == kF32) return reinterpret_cast<const float*>(vector)[c];
    else return widen16<DT>(reinterpret_cast<const uint16_t*>(vector)[c]);
  };
  if constexpr (POST) {
    write(p.partial[2], [&](int j, int e) { return element(gate_row, j, e, 1.0f) * post_at(0, j, e); });
    if constexpr (BIAS) write(p.partial[3], [&](int j, int e) { return element(gate_row, j, e, 1.0f) * post_at(1, j, e); });
    write(p.partial[4], [&](int j, int e) {
      const float of_weight = element(p.vectors.post_weight, j, e, 1.0f) * post_at(0, j, e);
      if constexpr (BIAS) return __builtin_fmaf(element(p.vectors.post_bias, j, e, 0.0f), post_at(1, j, e), of_weight);
      else return of_weight;
    });
  } else {
    write(p.partial[4], [&](int j, int e) { return post_at(0, j, e); });
  }
}

// The workgroups' sums added up: 32 columns on 32 x 32 threads, in a fixed order.  Workgroups: the vectors in turn, then the rows of the gate.
struct Totals {
  const float* partial[5];
  float* out[5];
  int32_t cols, blocks, chunks_per_gate;
  int32_t vectors;
  int32_t which[4];                                  // the vectors that are wanted, without the gate
};
constexpr int kTotalsSide = 32;
__global__ __launch_bounds__(kTotalsSide* kTotalsSide) void k_norm_totals(const Totals p) {
  __shared__ float sum[kTotalsSide][kTotalsSide + 1];
  const int x = threadIdx.x % kTotalsSide, y = threadIdx.x / kTotalsSide;
  const int tiles = (p.cols + kTotalsSide - 1) / kTotalsSide;
  const int c = (int)(blockIdx.x % tiles) * kTotalsSide + x, which = blockIdx.x / tiles;
  const bool of_gate = which >= p.vectors;
  const int v = of_gate ? 4 : p.which[which], gate_row = of_gate ? which - p.vectors : 0;
  const int first = gate_row * p.chunks_per_gate, last = of_gate ? first + p.chunks_per_gate : p.blocks;
  float s = 0.0f;
  if (c < p.cols) {
    const float* const from = p.partial[v] + c;
#pragma unroll 8
    for (int b = first + y; b < last; b += kTotalsSide) s += from[(int64_t)b * p.cols];
  }
  sum[y][x] = s;
  __syncthreads();
#pragma unroll
  for (int d = kTotalsSide / 2; d > 0; d >>= 1) {
    if (y < d) sum[y][x] += sum[y + d][x];
    __syncthreads();
  }
  if (y == 0 && c < p.cols) p.out[v][(int64_t)gate_row * p.cols + c] = sum[0][x];
}

__global__ __launch_bounds__(kEachThreads) void k_clear(float* out, int64_t n) {
  const int64_t i = element_of_thread();
  if (i < n) out[i] = 0.0f;
}

// How the backward pass cuts the rows: workgroups of whole chunks, no chunk over the end of a run of rows that share a row of the gate.
struct Chunks {
  int64_t rows_per_gate, rows_per_chunk, chunks_per_gate, blocks;
};
Chunks chunks_of(int64_t rows, int64_t cols, int64_t gate_groups) {
  const int64_t at_once = cols <= 512 ? 4 : 1;       // rows of a workgroup
  // Workgroups: one round of them, but no fewer rows to a workgroup than make up for its sums' way through memory, as long as the chip is full.
  // Microseconds at 1024 / 512 / 256 of them, bfloat16: 32768 x 4096 349 / 335 / 374, 8192 x 2048 53 / 48 / 64, 400 x 4096 18.6 / 18.7 / 16.1;
  // at 2048 / 1024 / 512, 4039 x 1001 binary32 58 / 43 / 48, 32768 x 768 90 / 129 / 211.
  const struct {
    int64_t cols, most, least, rows;
  } kinds[] = {{512, 1024, 1024, 4}, {1024, 2048, 768, 4}, {2048, 1024, 384, 16}, {4096, 512, 256, 16}, {kResidualNormMaxCols, 256, 256, 16}};
  int kind = 0;
  while (cols > kinds[kind].cols) ++kind;
  int64_t target = rows / kinds[kind].rows;
  if (target > kinds[kind].most) target = kinds[kind].most;
  if (target < kinds[kind].least) target = kinds[kind].least;
  Chunks c;
  c.rows_per_gate = rows / gate_groups;
  const int64_t most = (target + gate_groups - 1) / gate_groups;
  int64_t per = (c.rows_per_gate + most - 1) / most;
  c.rows_per_chunk = (per + at_once - 1) / at_once * at_once;
  c.chunks_per_gate = (c.rows_per_gate + c.rows_per_chunk - 1) / c.rows_per_chunk;
  c.blocks = c.chunks_per_gate * gate_groups;
  return c;
}

// A row's threads and units, by its length.  Forward two units to a thread are as good as one, and need fewer waves to agree; backward, with
// twice the tensors and the sums, one.
template <bool BACKWARD, class F>
hipError_t by_columns(int64_t cols, F&& f) {
  using std::integral_constant;
  using One = integral_constant<int, 1>;
  if (cols <= 512) return f(integral_constant<int, 64>{}, One{});
  if (cols <= 1024) return f(integral_constant<int, BACKWARD ? 128 : 64>{}, integral_constant<int, BACKWARD ? 1 : 2>{});
  if (cols <= 2048) return f(integral_constant<int, 256>{}, One{});
  if (cols <= 4096) return f(integral_constant<int, BACKWARD ? 512 : 256>{}, integral_constant<int, BACKWARD ? 1 : 2>{});
  if (cols <= 8192) return f(integral_constant<int, BACKWARD ? 1024 : 512>{}, integral_constant<int, BACKWARD ? 1 : 2>{});
  return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}
template <class F>
hipError_t by_type(int dtype, F&& f) {
  using std::integral_constant;
  if (dtype == DAF_F32) return f(integral_constant<int, kF32>{});
  if (dtype == DAF_F16) return f(integral_constant<int, kF16>{});
  return f(integral_constant<int, kBF16>{});
}

Vectors vectors_of(const daf_residual_norm_t& p) {
  auto c = [](const void* v) { return static_cast<const char*>(v); };
  return {c(p.pre_weight), c(p.pre_bias), c(p.post_weight), c(p.post_bias), c(p.gate)};
}

}  // namespace

hipError_t daf_launch_residual_norm(const daf_residual_norm_t& p, const void* residual, const void* z, void* out_residual, void* out_y,
                                    float* out_stats, hipStream_t stream) {
  if (p.rows == 0) return hipSuccess;
  Forward a = {};
  a.residual = static_cast<const char*>(residual);
  a.z = static_cast<const char*>(z);
  a.sum = static_cast<char*>(out_residual);
  a.y = static_cast<char*>(out_y);
  a.stats = reinterpret_cast<float4*>(out_stats);
  a.vectors = vectors_of(p);
  a.rows = (int32_t)p.rows;
  a.cols = (int32_t)p.cols;
  a.rows_per_gate = (int32_t)(p.rows / p.gate_groups);
  a.layer = p.kind == DAF_NORM_LAYER;
  a.eps = p.eps;
  a.scale = p.scale;
  return by_type(p.dtype, [&](auto type) {
    return by_columns<false>(p.cols, [&](auto row_threads, auto units) {
      constexpr int DT = decltype(type)::value, T = decltype(row_threads)::value, NV = decltype(units)::value;
      constexpr int kThreads = threads_of(T), kRows = kThreads / T;
      const int64_t blocks = (p.rows + kRows - 1) / kRows, resident = 256 * (2048 / kThreads);
      auto kernel = p.post && z != nullptr ? k_residual_norm<DT, T, NV, true> : k_residual_norm<DT, T, NV, false>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)(blocks < resident ? blocks : resident)), dim3(kThreads), 0, stream, a);
      return hipGetLastError();
    });
  });
}

int64_t daf_residual_norm_workspace_size(int64_t rows, int64_t cols, int64_t gate_groups) {
  if (rows == 0) return 0;
  return chunks_of(rows, cols, gate_groups).blocks * cols * 5 * (int64_t)sizeof(float);
}

hipError_t daf_launch_residual_norm_backward(const daf_residual_norm_t& p, const void* sum, const void* z, const float* stats, const void* grad_y,
                                             const void* grad_sum, void* out_grad_residual, void* out_grad_z,
                                             const daf_residual_norm_grads_t& grads, float* partial, hipStream_t stream) {
  float* const outs[5] = {grads.pre_weight, grads.pre_bias, grads.post_weight, grads.post_bias, grads.gate};
  if (p.rows == 0) {
    for (int v = 0; v < 5; ++v) {
      const int64_t n = p.cols * (v == 4 ? p.gate_groups : 1);
      if (outs[v] == nullptr) continue;
      hipLaunchKernelGGL(k_clear, blocks_for_each(n), dim3(kEachThreads), 0, stream, outs[v], n);
      if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
  }
  const Chunks c = chunks_of(p.rows, p.cols, p.gate_groups);
  Backward a = {};
  Totals totals = {};
  a.sum = static_cast<const char*>(sum);
  a.z = static_cast<const char*>(z);
  a.grad_y = static_cast<const char*>(grad_y);
  a.grad_sum = static_cast<const char*>(grad_sum);
  a.stats = reinterpret_cast<const float4*>(stats);
  a.grad_residual = static_cast<char*>(out_grad_residual);
  a.grad_z = static_cast<char*>(out_grad_z);
  a.vectors = vectors_of(p);
  a.cols = totals.cols = (int32_t)p.cols;
  a.rows_per_gate = (int32_t)c.rows_per_gate;
  a.rows_per_chunk = (int32_t)c.rows_per_chunk;
  a.chunks_per_gate = totals.chunks_per_gate = (int32_t)c.chunks_per_gate;
  a.layer = p.kind == DAF_NORM_LAYER;
  a.scale = p.scale;
  totals.blocks = (int32_t)c.blocks;
  // A row of the gate that one workgroup has is that workgroup's own sum: it goes where it belongs at once.  What is left to k_norm_totals are few rows
  // of the gate (chunks_of gives two workgroups to each only where there are fewer of them than workgroups to a round), whatever gate_groups is: a launch
  // ends below 2^32 threads.
  const bool gate_done = c.chunks_per_gate == 1;
  float* at = partial;
  for (int v = 0; v < 5; ++v) {
    if (outs[v] == nullptr) continue;
    if (v == 4 && gate_done) {
      a.partial[v] = outs[v];
      continue;
    }
    totals.partial[v] = a.partial[v] = at;
    totals.out[v] = outs[v];
    at += c.blocks * p.cols;
    if (v < 4) totals.which[totals.vectors++] = v;
  }
  const hipError_t e = by_type(p.dtype, [&](auto type) {
    return by_columns<true>(p.cols, [&](auto row_threads, auto units) {
      constexpr int DT = decltype(type)::value, T = decltype(row_threads)::value, NV = decltype(units)::value;
      const bool post = p.post && z != nullptr;
      const bool bias = grads.pre_bias != nullptr || grads.post_bias != nullptr || (post && p.post_bias != nullptr && grads.gate != nullptr);
      auto kernel = post ? (bias ? k_residual_norm_backward<DT, T, NV, true, true> : k_residual_norm_backward<DT, T, NV, true, false>)
                         : (bias ? k_residual_norm_backward<DT, T, NV, false, true> : k_residual_norm_backward<DT, T, NV, false, false>);
      hipLaunchKernelGGL(kernel, dim3((unsigned)c.blocks), dim3(threads_of(T)), 0, stream, a);
      return hipGetLastError();
    });
  });
  const int64_t sums = totals.vectors + (grads.gate != nullptr && !gate_done ? p.gate_groups : 0);
  if (e != hipSuccess || sums == 0) return e;
  const int64_t tiles = (p.cols + kTotalsSide - 1) / kTotalsSide;
  hipLaunchKernelGGL(k_norm_totals, dim3((unsigned)(tiles * sums)), dim3(kTotalsSide * kTotalsSide), 0, stream, totals);
  return hipGetLastError();
}

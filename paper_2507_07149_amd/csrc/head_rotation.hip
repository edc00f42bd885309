// Norms of heads and rotation by position (daf_head_rotation, daf_head_rotation_backward): one pass, memory bound.
//
//   n = x * rstd * w, rstd = 1 / sqrt(mean(x^2) + eps);  a' = a c - b s, b' = a s + b c
//   backward: dn = the rotation by minus the angle of the gradient; dx = rstd (dn w - u mean(dn w u)), dw = sum of dn u, u = x rstd
//
// A head is head_dim / 16 lanes (4, 8 or 16 of them), two units of eight elements to a lane, and both members of every pair are the lane's: with
// halves, lane l < rotary / 16 has units l and l + rotary / 16; what does not rotate follows by twos.  So nothing but the sum of squares (and of its gradient)
// crosses lanes, in DPP steps, and loads and stores are 16 bytes.  A wave works on one token, whose angles its lanes load once for all its heads.
// Measured (bfloat16, 32 + 8 heads of 128, 32768 tokens): 134 us, 5.0 TB/s; backward 207 us, 4.9 TB/s, of which the weights' sums are 5; binary32 263 and
// 394 us, 5.1 TB/s.  One token 2.9 us, two dependent loads.
#include <algorithm>
#include <type_traits>

#include "head_rotation.h"
#include "block_common.h"

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int64_t kMostBlocks = 1 << 23;        // in the first dimension of a launch, which has fewer than 2^32 threads

struct Heads {
  char* at;
  int64_t token, head;         // bytes
};
struct Rotation {
  int64_t tokens;
  uint32_t positions, out_rows;
  int q_heads, kv_heads, dim, rotating, norm;   // rotating: lanes of a head that rotate
  float eps;
  const char *q_weight, *k_weight;
  const float *cos, *sin;
  const int32_t *position, *rows;
};
struct Forward : Rotation {
  Heads q, k, v, out_q, out_k, out_v;           // v.at null: none
  int items;                                    // waves to a token
};
struct Backward : Rotation {
  Heads q, k, grad_q, grad_k, out_grad_q, out_grad_k;
  float* partial;                               // [workgroups][2][dim], or null
};

// (The same in all lanes, so that addresses of a token are the scalar unit's.)
__device__ __forceinline__ int wave_of_workgroup() { return __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); }

// The lane's two units of a head: where they begin (elements), whether they are there, and whether they rotate.
struct Place {
  int first, second;
  bool has_first, has_second, rotates;
};
template <bool PAIRS>
__device__ __forceinline__ Place place_of(int lane, int dim, int rotating) {
  Place p;
  p.rotates = lane < rotating;
  if (PAIRS || !p.rotates) {
    p.first = 16 * lane;
    p.second = p.first + 8;
  } else {
    p.first = 8 * lane;
    p.second = p.first + 8 * rotating;
  }
  p.has_first = p.first < dim && (PAIRS || p.rotates || lane < (dim + 15) / 16);
  p.has_second = p.second < dim;
  return p;
}

template <int DT>
struct Pair {
  Unit<DT> a, b;
};
template <int DT>
__device__ __forceinline__ Pair<DT> load_pair(const char* at, const Place& p) {
  constexpr int e = ElemTraits<DT>::kBytes;
  Pair<DT> r = {};
  if (p.has_first) r.a = load_unit<DT>(at + p.first * e);
  if (p.has_second) r.b = load_unit<DT>(at + p.second * e);
  return r;
}
template <int DT>
__device__ __forceinline__ void widen_pair(const Pair<DT>& u, float (&a)[8], float (&b)[8]) {
  widen_unit<DT>(u.a, a);
  widen_unit<DT>(u.b, b);
}
template <int DT>
__device__ __forceinline__ void store_pair(char* at, const Place& p, const float (&a)[8], const float (&b)[8]) {
  constexpr int e = ElemTraits<DT>::kBytes;
  if (p.has_first) store_unit<DT>(at + p.first * e, narrow_unit<DT>(a));
  if (p.has_second) store_unit<DT>(at + p.second * e, narrow_unit<DT>(b));
}
// The sum over the lanes of a head, in all of them.
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
  v += u2f(dpp<kDppXor1>(0u, f2u(v)));
  v += u2f(dpp<kDppXor2>(0u, f2u(v)));
  if constexpr (LANES >= 8) v += u2f(dpp<kDppHalfMirror>(0u, f2u(v)));
  if constexpr (LANES >= 16) v += u2f(dpp<kDppMirror>(0u, f2u(v)));
  return v;
}
// (The instruction for 1 / sqrt takes subnormal numbers for 0; eps may be 0.)
__device__ __forceinline__ float rstd_of(float squares, const Rotation& r) {
  const float v = squares / (float)r.dim + r.eps;
  const bool small = v < 0x1p-100f;
  return __builtin_amdgcn_rsqf(small ? v * 0x1p64f : v) * (small ? 0x1p32f : 1.0f);
}
// By the angle, or (BACK) by minus it.  PAIRS: neighbours in a unit, else member e of the first unit and of the second.
template <bool PAIRS, bool BACK>
__device__ __forceinline__ void rotate(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8]) {
  auto turn = [&](float& x, float& y, int i) {
    const float sine = BACK ? -s[i] : s[i], was = x;
    x = was * c[i] - y * sine;
    y = was * sine + y * c[i];
  };
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (PAIRS) {
      if (i < 4) turn(a[2 * i], a[2 * i + 1], i);
      else turn(b[2 * i - 8], b[2 * i - 7], i);
    } else {
      turn(a[i], b[i], i);
    }
  }
}
// (A token without a position has no row of them, and there may be no rows at all.)
__device__ __forceinline__ void load_angles(const Rotation& r, const Place& p, int lane, uint32_t position, float (&c)[8], float (&s)[8]) {
  const int64_t at = ((int64_t)position * r.rotating + lane) * 8;
  Unit<kF32> cu = {}, su = {};
  if (p.rotates && position < r.positions) {
    cu = load_unit<kF32>(reinterpret_cast<const char*>(r.cos + at));
    su = load_unit<kF32>(reinterpret_cast<const char*>(r.sin + at));
  }
  widen_unit<kF32>(cu, c);
  widen_unit<kF32>(su, s);
}
template <int DT>
__device__ __forceinline__ void load_weight(const char* w, const Place& p, float (&a)[8], float (&b)[8]) {
  Pair<DT> u = {};
  if (w != nullptr) u = load_pair<DT>(w, p);
  widen_pair<DT>(u, a, b);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a[i] = w != nullptr ? a[i] : 1.0f;
    b[i] = w != nullptr ? b[i] : 1.0f;
  }
}

// A wave takes every `items`-th set of 64 / LANES heads of a token.
template <int DT, int LANES, bool PAIRS>
__global__ __launch_bounds__(kThreads) void k_head_rotation(const Forward f) {
  constexpr int kSets = kWave / LANES;
  const int lane = threadIdx.x % LANES, set = threadIdx.x % kWave / LANES;
  const int64_t item = ((int64_t)blockIdx.y * kMostBlocks + blockIdx.x) * kWaves + wave_of_workgroup();
  const int64_t token = f.items == 1 ? item : (int64_t)((uint32_t)item / (uint32_t)f.items);
  if (token >= f.tokens) return;
  const Place p = place_of<PAIRS>(lane, f.dim, f.rotating);
  const uint32_t position = (uint32_t)f.position[token];
  const bool there = position < f.positions;
  const int64_t row = f.rows == nullptr ? token : (int64_t)(uint32_t)f.rows[token];
  const bool kept = row < (int64_t)f.out_rows;
  float c[8], s[8];
  load_angles(f, p, lane, position, c, s);
  const int with_k = f.q_heads + f.kv_heads, all = with_k + (f.v.at != nullptr ? f.kv_heads : 0);
  for (int h = (int)(item - token * f.items) * kSets + set; h < all; h += f.items * kSets) {
    const bool of_q = h < f.q_heads, of_k = !of_q && h < with_k;
    const int head = of_q ? h : of_k ? h - f.q_heads : h - with_k;
    char *from, *out;                                                   // (chosen by values: by reference the arguments would go through memory)
    int64_t from_token, from_head, out_token, out_head;
    if (of_q) from = f.q.at, from_token = f.q.token, from_head = f.q.head, out = f.out_q.at, out_token = f.out_q.token, out_head = f.out_q.head;
    else if (of_k) from = f.k.at, from_token = f.k.token, from_head = f.k.head, out = f.out_k.at, out_token = f.out_k.token, out_head = f.out_k.head;
    else from = f.v.at, from_token = f.v.token, from_head = f.v.head, out = f.out_v.at, out_token = f.out_v.token, out_head = f.out_v.head;
    const Pair<DT> x = load_pair<DT>(from + token * from_token + head * from_head, p);
    out += (of_q ? token : row) * out_token + head * out_head;
    const bool write = of_q || kept;
    if (!of_q && !of_k) {
      constexpr int e = ElemTraits<DT>::kBytes;
      if (write && p.has_first) store_unit<DT>(out + p.first * e, x.a);
      if (write && p.has_second) store_unit<DT>(out + p.second * e, x.b);
      continue;
    }
    float a[8], b[8];
    widen_pair<DT>(x, a, b);
    if (f.norm) {
      float wa[8], wb[8], squares = 0.0f;
      load_weight<DT>(of_q ? f.q_weight : f.k_weight, p, wa, wb);
#pragma unroll
      for (int i = 0; i < 8; ++i) squares = __builtin_fmaf(b[i], b[i], __builtin_fmaf(a[i], a[i], squares));
      const float rstd = rstd_of(head_sum<LANES>(squares), f);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] = a[i] * rstd * wa[i];
        b[i] = b[i] * rstd * wb[i];
      }
    }
    if (p.rotates) rotate<PAIRS, false>(a, b, c, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      a[i] = there ? a[i] : 0.0f;
      b[i] = there ? b[i] : 0.0f;
    }
    if (write) store_pair<DT>(out, p, a, b);
  }
}

// One kind of heads of a token; its part of the weight's gradient is added to da and db.
template <int DT, int LANES, bool PAIRS>
__device__ __forceinline__ void heads_backward(const Backward& f, const Heads& x_of, const Heads& grad, const Heads& out, int heads, const char* weight,
                                               int64_t token, uint32_t position, const Place& p, float (&da)[8], float (&db)[8]) {
  constexpr int kSets = kWave / LANES;
  const bool there = position < f.positions;
  const int set = threadIdx.x % kWave / LANES;
  for (int h = set; h < heads; h += kSets) {
    float ga[8], gb[8];
    Pair<DT> x = {};
    const Pair<DT> g = load_pair<DT>(grad.at + token * grad.token + h * grad.head, p);
    if (f.norm) x = load_pair<DT>(x_of.at + token * x_of.token + h * x_of.head, p);
    widen_pair<DT>(g, ga, gb);
    if (p.rotates) {                                                     // (loaded for every head: kept, they cost the kernel a wave)
      float c[8], s[8];
      load_angles(f, p, threadIdx.x % LANES, position, c, s);
      rotate<PAIRS, true>(ga, gb, c, s);
    }
    if (f.norm) {
      float a[8], b[8], squares = 0.0f;
      widen_pair<DT>(x, a, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) squares = __builtin_fmaf(b[i], b[i], __builtin_fmaf(a[i], a[i], squares));
      const float rstd = rstd_of(head_sum<LANES>(squares), f);
      float inner = 0.0f, wa[8], wb[8];
      load_weight<DT>(weight, p, wa, wb);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] *= rstd;
        b[i] *= rstd;
        const float ua = ga[i] * a[i], ub = gb[i] * b[i];
        if (there) {
          da[i] += ua;
          db[i] += ub;
        }
        ga[i] *= wa[i];
        gb[i] *= wb[i];
        inner = __builtin_fmaf(ub, wb[i], __builtin_fmaf(ua, wa[i], inner));
      }
      inner = head_sum<LANES>(inner) / (float)f.dim;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        ga[i] = (ga[i] - a[i] * inner) * rstd;
        gb[i] = (gb[i] - b[i] * inner) * rstd;
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      ga[i] = there ? ga[i] : 0.0f;
      gb[i] = there ? gb[i] : 0.0f;
    }
    store_pair<DT>(out.at + token * out.token + h * out.head, p, ga, gb);
  }
}

template <int DT, int LANES, bool PAIRS>
__global__ __launch_bounds__(kThreads, 4) void k_head_rotation_backward(const Backward f) {
  const int lane = threadIdx.x % LANES;
  const Place p = place_of<PAIRS>(lane, f.dim, f.rotating);
  float q[2][8] = {}, k[2][8] = {};
  for (int64_t token = (int64_t)blockIdx.x * kWaves + wave_of_workgroup(); token < f.tokens; token += (int64_t)gridDim.x * kWaves) {
    const uint32_t position = (uint32_t)f.position[token];
    heads_backward<DT, LANES, PAIRS>(f, f.q, f.grad_q, f.out_grad_q, f.q_heads, f.q_weight, token, position, p, q[0], q[1]);
    heads_backward<DT, LANES, PAIRS>(f, f.k, f.grad_k, f.out_grad_k, f.kv_heads, f.k_weight, token, position, p, k[0], k[1]);
  }
  if (f.partial == nullptr) return;
  // the workgroup's sums: a column's 256 / LANES lanes by as many threads as there are to a column, then those
  constexpr int kColumns = LANES * 16, kShares = kThreads / kColumns;
  __shared__ float sums[kThreads][17], shares[kShares][kColumns];
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
#pragma unroll
    for (int i = 0; i < 16; ++i) sums[threadIdx.x][i] = kind ? k[i >> 3][i & 7] : q[i >> 3][i & 7];
    __syncthreads();
    const int column = threadIdx.x % kColumns, l = column / 16, i = column % 16, share = threadIdx.x / kColumns;
    float v = 0.0f;
#pragma unroll
    for (int t = 0; t < kThreads / LANES / kShares; ++t) v += sums[(share * (kThreads / LANES / kShares) + t) * LANES + l][i];
    shares[share][column] = v;
    __syncthreads();
    if (share == 0) {
      v = 0.0f;
#pragma unroll
      for (int n = 0; n < kShares; ++n) v += shares[n][column];
      const Place of = place_of<PAIRS>(l, f.dim, f.rotating);
      if (i < 8 ? of.has_first : of.has_second)
        f.partial[((int64_t)blockIdx.x * 2 + kind) * f.dim + (i < 8 ? of.first + i : of.second + i - 8)] = v;
    }
  }
}

// Sums of the workgroups' parts: a workgroup to 16 columns of one weight, 64 threads to a column, each every 64th part, then one after the other.
constexpr int kSumThreads = 1024, kSumSlices = kSumThreads / 16;
__global__ __launch_bounds__(kSumThreads) void k_head_rotation_sums(const float* partial, int parts, int dim, float* out_q, float* out_k) {
  __shared__ float sums[kSumSlices][17];
  float* const out = blockIdx.y ? out_k : out_q;
  if (out == nullptr) return;
  const int column = blockIdx.x * 16 + threadIdx.x % 16, slice = threadIdx.x / 16;
  float v = 0.0f;
  if (column < dim) {
#pragma unroll 8
    for (int i = slice; i < parts; i += kSumSlices) v += partial[((int64_t)i * 2 + blockIdx.y) * dim + column];
  }
  sums[slice][threadIdx.x % 16] = v;
  __syncthreads();
  if (slice != 0 || column >= dim) return;
  v = 0.0f;
#pragma unroll
  for (int i = 0; i < kSumSlices; ++i) v += sums[i][threadIdx.x];
  out[column] = v;
}

Heads heads(const daf_heads_t& h, int es) { return {static_cast<char*>(h.at), h.token_stride * es, h.head_stride * es}; }

void fill(Rotation& r, const daf_head_rotation_t& p) {
  r.tokens = p.tokens;
  r.positions = (uint32_t)p.positions;
  r.q_heads = p.q_heads;
  r.kv_heads = p.kv_heads;
  r.dim = p.head_dim;
  r.rotating = p.rotary_dim / 16;
  r.norm = p.norm;
  r.eps = p.eps;
  r.q_weight = static_cast<const char*>(p.q_weight);
  r.k_weight = static_cast<const char*>(p.k_weight);
  r.cos = p.cos;
  r.sin = p.sin;
  r.position = p.position;
}

// `call` with the format, the lanes of a head and the pairing as constants.
template <class Call>
void with_form(const daf_head_rotation_t& p, Call call) {
  auto pairing = [&](auto dt, auto lanes) {
    if (p.pairing == DAF_ROTATE_PAIRS) call(dt, lanes, std::true_type{});
    else call(dt, lanes, std::false_type{});
  };
  auto lanes = [&](auto dt) {
    if (p.head_dim <= 64) pairing(dt, std::integral_constant<int, 4>{});
    else if (p.head_dim <= 128) pairing(dt, std::integral_constant<int, 8>{});
    else pairing(dt, std::integral_constant<int, 16>{});
  };
  if (p.dtype == DAF_F32) lanes(std::integral_constant<int, kF32>{});
  else if (p.dtype == DAF_F16) lanes(std::integral_constant<int, kF16>{});
  else lanes(std::integral_constant<int, kBF16>{});
}

// Workgroups of the backward pass: the parts that k_head_rotation_sums adds up.
int64_t backward_parts(int64_t tokens) { return std::min<int64_t>((tokens + kWaves - 1) / kWaves, 1024); }

}  // namespace

int64_t daf_head_rotation_workspace_size(int64_t tokens, int head_dim) { return backward_parts(tokens) * 2 * head_dim * (int64_t)sizeof(float); }

hipError_t daf_launch_head_rotation(const daf_head_rotation_t& p, const daf_heads_t& q, const daf_heads_t& k, const daf_heads_t* v, const daf_heads_t& out_q,
                                    const daf_heads_t& out_k, const daf_heads_t* out_v, const int32_t* rows, int64_t out_rows, hipStream_t stream) {
  if (p.tokens == 0) return hipSuccess;
  const int es = p.dtype == DAF_F32 ? 4 : 2;
  Forward f = {};
  fill(f, p);
  f.rows = rows;
  f.out_rows = (uint32_t)out_rows;
  f.q = heads(q, es);
  f.k = heads(k, es);
  f.out_q = heads(out_q, es);
  f.out_k = heads(out_k, es);
  if (v != nullptr) {
    f.v = heads(*v, es);
    f.out_v = heads(*out_v, es);
  }
  with_form(p, [&](auto dt, auto lanes, auto pairs) {
    constexpr int kSets = kWave / lanes.value;
    const int all = p.q_heads + p.kv_heads * (v != nullptr ? 2 : 1), sets = (all + kSets - 1) / kSets;
    f.items = p.tokens * sets <= 8192 ? sets : 1;
    const int64_t blocks = (p.tokens * f.items + kWaves - 1) / kWaves;
    const dim3 grid((unsigned)std::min(blocks, kMostBlocks), (unsigned)((blocks + kMostBlocks - 1) / kMostBlocks));
    k_head_rotation<dt.value, lanes.value, pairs.value><<<grid, kThreads, 0, stream>>>(f);
  });
  return hipGetLastError();
}

hipError_t daf_launch_head_rotation_backward(const daf_head_rotation_t& p, const daf_heads_t& q, const daf_heads_t& k, const daf_heads_t& grad_q,
                                             const daf_heads_t& grad_k, const daf_heads_t& out_grad_q, const daf_heads_t& out_grad_k, float* out_grad_q_weight,
                                             float* out_grad_k_weight, float* partial, hipStream_t stream) {
  const int es = p.dtype == DAF_F32 ? 4 : 2;
  const bool weights = out_grad_q_weight != nullptr || out_grad_k_weight != nullptr;
  const int64_t parts = backward_parts(p.tokens);
  if (parts > 0) {
    Backward f = {};
    fill(f, p);
    f.q = heads(q, es);
    f.k = heads(k, es);
    f.grad_q = heads(grad_q, es);
    f.grad_k = heads(grad_k, es);
    f.out_grad_q = heads(out_grad_q, es);
    f.out_grad_k = heads(out_grad_k, es);
    f.partial = weights ? partial : nullptr;
    with_form(p, [&](auto dt, auto lanes, auto pairs) {
      k_head_rotation_backward<dt.value, lanes.value, pairs.value><<<(unsigned)parts, kThreads, 0, stream>>>(f);
    });
  }
  if (weights)
    k_head_rotation_sums<<<dim3((unsigned)((p.head_dim + 15) / 16), 2), kSumThreads, 0, stream>>>(partial, (int)parts, p.head_dim, out_grad_q_weight,
                                                                                              out_grad_k_weight);
  return hipGetLastError();
}

// Shared by the operators of daf_block.h: eight elements of a tensor at a time, and sums over a wave.
#pragma once
#include "daf_device.h"

namespace {

using namespace daf;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Sixteen bytes at any element boundary: rows of an odd number of columns begin anywhere, and global memory takes such accesses whole.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ u32x4 load_any(const char* p) { return *reinterpret_cast<const u32x4_any*>(p); }
__device__ __forceinline__ void store_any(char* p, const u32x4& v) { *reinterpret_cast<u32x4_any*>(p) = v; }

// Eight elements as they lie in memory.
template <int DT>
struct Unit {
  static constexpr int kQuads = DT == kF32 ? 2 : 1;
  u32x4 q[kQuads];
};

template <int DT>
__device__ __forceinline__ Unit<DT> load_unit(const char* p) {
  Unit<DT> u;
#pragma unroll
  for (int i = 0; i < Unit<DT>::kQuads; ++i) u.q[i] = load_any(p + 16 * i);
  return u;
}
template <int DT>
__device__ __forceinline__ void store_unit(char* p, const Unit<DT>& u) {
#pragma unroll
  for (int i = 0; i < Unit<DT>::kQuads; ++i) store_any(p + 16 * i, u.q[i]);
}

// Only the first `count` (0 ... 7) elements; the others are zero.
template <int DT>
__device__ __forceinline__ Unit<DT> load_unit_part(const char* p, int count) {
  Unit<DT> u;
  if constexpr (DT == kF32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) u.q[e >> 2][e & 3] = e < count ? reinterpret_cast<const uint32_t*>(p)[e] : 0u;
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const uint32_t lo = e < count ? reinterpret_cast<const uint16_t*>(p)[e] : 0u;
      const uint32_t hi = e + 1 < count ? reinterpret_cast<const uint16_t*>(p)[e + 1] : 0u;
      u.q[0][e >> 1] = lo | (hi << 16);
    }
  }
  return u;
}
template <int DT>
__device__ __forceinline__ void store_unit_part(char* p, const Unit<DT>& u, int count) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (e >= count) continue;
    if constexpr (DT == kF32) reinterpret_cast<uint32_t*>(p)[e] = u.q[e >> 2][e & 3];
    else reinterpret_cast<uint16_t*>(p)[e] = (uint16_t)(u.q[0][e >> 1] >> (16 * (e & 1)));
  }
}
// `count` of 8 or more: all of them.  0 or less: none.
template <int DT>
__device__ __forceinline__ Unit<DT> load_unit_of(const char* p, int count) {
  if (count >= 8) return load_unit<DT>(p);
  return load_unit_part<DT>(p, count);
}
template <int DT>
__device__ __forceinline__ void store_unit_of(char* p, const Unit<DT>& u, int count) {
  if (count >= 8) store_unit<DT>(p, u);
  else store_unit_part<DT>(p, u, count);
}

template <int DT>
__device__ __forceinline__ void widen_unit(const Unit<DT>& u, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (DT == kF32) {
      v[e] = u2f(u.q[e >> 2][e & 3]);
    } else {
      const uint32_t d = u.q[0][e >> 1];
      if constexpr (DT == kBF16) v[e] = (e & 1) ? u2f(d & 0xFFFF0000u) : u2f(d << 16);
      else v[e] = widen16<kF16>((e & 1) ? (d >> 16) : (d & 0xFFFFu));
    }
  }
}

// Two binary32 values rounded (nearest even; NaN stays NaN) to the 16-bit format, low half first.
template <int DT>
__device__ __forceinline__ uint32_t narrow_pair(float lo, float hi) {
  if constexpr (DT == kBF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    const f16x2 v = {(_Float16)lo, (_Float16)hi};
    return __builtin_bit_cast(uint32_t, v);
  }
}
template <int DT>
__device__ __forceinline__ Unit<DT> narrow_unit(const float (&v)[8]) {
  Unit<DT> u;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    if constexpr (DT == kF32) {
      u.q[e >> 2][e & 3] = f2u(v[e]);
      u.q[e >> 2][(e & 3) + 1] = f2u(v[e + 1]);
    } else {
      u.q[0][e >> 1] = narrow_pair<DT>(v[e], v[e + 1]);
    }
  }
  return u;
}

// The sum over the wave, the same bits in every lane: by fours, rows of 16 and then rows in fixed order.
__device__ __forceinline__ float wave_sum(float v) {
  v += u2f(dpp<kDppXor1>(0u, f2u(v)));
  v += u2f(dpp<kDppXor2>(0u, f2u(v)));
  v += u2f(dpp<kDppHalfMirror>(0u, f2u(v)));
  v += u2f(dpp<kDppMirror>(0u, f2u(v)));
  v += u2f(dpp<kDppBcast15, 0xA>(0u, f2u(v)));
  v += u2f(dpp<kDppBcast31, 0xC>(0u, f2u(v)));
  return u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(v), 63));
}

}  // namespace

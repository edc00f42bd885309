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
// The same past the caches, for what is read again only after they have seen much else.
__device__ __forceinline__ void stream_any(char* p, const u32x4& v) { __builtin_nontemporal_store(v, reinterpret_cast<u32x4_any*>(p)); }
template <int DT>
__device__ __forceinline__ void stream_unit(char* p, const Unit<DT>& u) {
#pragma unroll
  for (int i = 0; i < Unit<DT>::kQuads; ++i) stream_any(p + 16 * i, u.q[i]);
}

// Only the first `count` (7 at most; none if it is not above 0) elements, as four, two and one of them; the others are zero.
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));
template <int DT>
__device__ __forceinline__ Unit<DT> load_unit_part(const char* p, int count) {
  Unit<DT> u = {};
  if (count <= 0) return u;
  const int pair = count & 4, single = count & 6;    // where the two, and the one, begin
  if constexpr (DT == kF32) {
    if (count & 4) u.q[0] = load_any(p);
    u32x2_any two = {0u, 0u};
    uint32_t one = 0u;
    if (count & 2) two = *reinterpret_cast<const u32x2_any*>(p + pair * 4);
    if (count & 1) one = *reinterpret_cast<const uint32_t*>(p + single * 4);
    const u32x4 rest = {(count & 2) ? two[0] : one, two[1], (count & 2) ? one : 0u, 0u};
    if (count & 4) u.q[1] = rest;
    else u.q[0] = rest;
  } else {
    u32x2_any four = {0u, 0u};
    uint32_t two = 0u, one = 0u;
    if (count & 4) four = *reinterpret_cast<const u32x2_any*>(p);
    if (count & 2) two = *reinterpret_cast<const u32_any*>(p + pair * 2);
    if (count & 1) one = *reinterpret_cast<const uint16_t*>(p + single * 2);
    const uint32_t lo = (count & 2) ? two : one, hi = (count & 2) ? one : 0u;
    u.q[0] = (count & 4) ? u32x4{four[0], four[1], lo, hi} : u32x4{lo, hi, 0u, 0u};
  }
  return u;
}
template <int DT>
__device__ __forceinline__ void store_unit_part(char* p, Unit<DT> u, int count) {
  if (count <= 0) return;
  if constexpr (DT == kF32) {
    if (count & 4) {
      store_any(p, u.q[0]);
      u.q[0] = u.q[1];
      p += 16;
    }
    if (count & 2) {
      *reinterpret_cast<u32x2_any*>(p) = u32x2_any{u.q[0][0], u.q[0][1]};
      u.q[0][0] = u.q[0][2];
      p += 8;
    }
    if (count & 1) *reinterpret_cast<uint32_t*>(p) = u.q[0][0];
  } else {
    u32x4& d = u.q[0];
    if (count & 4) {
      *reinterpret_cast<u32x2_any*>(p) = u32x2_any{d[0], d[1]};
      d[0] = d[2];
      d[1] = d[3];
      p += 8;
    }
    if (count & 2) {
      *reinterpret_cast<u32_any*>(p) = d[0];
      d[0] = d[1];
      p += 4;
    }
    if (count & 1) *reinterpret_cast<uint16_t*>(p) = (uint16_t)d[0];
  }
}
// The first `count` (1 ... 7; none if it is not above 0) elements of a unit, out of the row's last eight, which were loaded in its place.  The others
// are zero, or (ZEROS false) elements of the row's.
template <int DT, bool ZEROS = true>
__device__ __forceinline__ Unit<DT> unit_from_row_end(const Unit<DT>& u, int count) {
  Unit<DT> r = {};
  if (count <= 0) return ZEROS ? r : u;
  const int s = 8 - count;
  constexpr int kWords = Unit<DT>::kQuads * 4, kPerWord = 8 / kWords;
  uint32_t w[kWords];
#pragma unroll
  for (int i = 0; i < kWords; ++i) w[i] = u.q[i >> 2][i & 3];
  auto move_words = [&](bool really, auto by) {
    constexpr int kBy = decltype(by)::value;
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = !really ? w[i] : i + kBy < kWords ? w[i + kBy < kWords ? i + kBy : 0] : ZEROS ? 0u : w[i];
  };
  move_words((s & 4) != 0, std::integral_constant<int, 4 / kPerWord>{});
  move_words((s & 2) != 0, std::integral_constant<int, 2 / kPerWord>{});
  if constexpr (kPerWord == 1) {
    move_words((s & 1) != 0, std::integral_constant<int, 1>{});
  } else {
#pragma unroll
    for (int i = 0; i < kWords; ++i)
      w[i] = (s & 1) ? (w[i] >> 16) | (i + 1 < kWords ? w[i + 1 < kWords ? i + 1 : 0] << 16 : ZEROS ? 0u : w[i] & 0xFFFF0000u) : w[i];
  }
#pragma unroll
  for (int i = 0; i < kWords; ++i) r.q[i >> 2][i & 3] = w[i];
  return r;
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

// Launches of a thread to each of n elements (below 2^46).  One dimension of a launch has fewer than 2^32 threads: what is more goes into the second.
constexpr int kEachThreads = 256, kEachBlocks = 1 << 23;
inline dim3 blocks_for_each(int64_t n) {
  const int64_t blocks = (n + kEachThreads - 1) / kEachThreads;
  return dim3((unsigned)(blocks < kEachBlocks ? blocks : kEachBlocks), (unsigned)((blocks + kEachBlocks - 1) / kEachBlocks));
}
__device__ __forceinline__ int64_t element_of_thread() { return ((int64_t)blockIdx.y * kEachBlocks + blockIdx.x) * kEachThreads + threadIdx.x; }

}  // namespace

// The gated product of few rows (kGated, kGatedGrad): a token or a short batch, where reading Wg and Wu is all there is to it.
//
// A workgroup has 16 columns of h, its eight waves a part of l each, and their sums meet in LDS: one launch, no sums through memory, and as many
// workgroups as keep every memory channel busy.  W goes from memory straight into the registers that the matrix instruction takes it from
// (v_mfma_f32_16x16x32, its 16 rows of W against 16 of x), four instructions ahead; no element of it is read twice, so LDS would only be a detour.
// x comes out of the caches in the same way.  Rows may begin at any element, so that nothing is copied for the alignment either.
//
// Bound by the bytes of W: 1 x 11008 x 4096 bfloat16 35 to 36 us (180 MB, 5.0 to 5.1 TB/s; a copy moves 4.9); small ones by the launch, 2 x 248 x 656 4.0 us.
#pragma once
#include "gated_product.h"

namespace {

constexpr int kFewWaves = 8, kFewThreads = kFewWaves * kWave;

// MB: blocks of 16 rows.  COLS: 16 columns of h, Wg's rows and Wu's in a block each, or 8, both in one.
template <int DT, int KIND, int MB, int COLS>
__global__ __launch_bounds__(kFewThreads, 4) void k_gated_few_rows(const Product p) {
  constexpr int kWBlocks = COLS / 8, kOperands = kWBlocks + MB;          // of 16 rows of W, of x
  constexpr int kFewAhead = kOperands <= 2 ? 4 : 2;
  __shared__ float sums[kFewWaves][kWBlocks * MB][16 * 16];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int li = lane % 16, lg = lane / 16;
  const int64_t n0 = (int64_t)blockIdx.x * COLS;
  if (KIND == kGated && n0 >= p.n) return;                               // (columns that pad [da du])

  // The lane's rows, the last in place of those that do not exist: what they give is not used.
  const char* row[kOperands];
  const int64_t n = min(n0 + li % COLS, (int64_t)p.cols - 1);
  if constexpr (kWBlocks == 2) {
    row[0] = p.c[0] + n * p.c_pitch;
    row[1] = p.c[1] + n * p.c_pitch;
  } else {
    row[0] = (li < COLS ? p.c[0] : p.c[1]) + n * p.c_pitch;
  }
#pragma unroll
  for (int b = 0; b < MB; ++b) row[kWBlocks + b] = p.r + (int64_t)min(b * 16 + li, p.rows - 1) * p.r_pitch;

  const int steps = p.length / 32, begin = steps * wave / kFewWaves, end = steps * (wave + 1) / kFewWaves;   // whole instructions
  // The last values of l, wave 0's: a lane that the row does not fill loads the row's last eight and puts them right at the end.
  const int rest = p.length % 32, left = rest - lg * 8;
  u32x4 last[kOperands];
  if (wave == 0 && rest > 0) {
#pragma unroll
    for (int o = 0; o < kOperands; ++o) {
      if (p.length < 8) last[o] = load_unit_part<DT>(row[o] + lg * 16, left).q[0];
      else last[o] = load_any(row[o] + (int64_t)min(steps * 32 + lg * 8, p.length - 8) * 2);
    }
  }

  f32x4 acc[kWBlocks * MB] = {};
  auto multiply = [&](const u32x4 (&v)[kOperands]) {
#pragma unroll
    for (int w = 0; w < kWBlocks; ++w)
#pragma unroll
      for (int b = 0; b < MB; ++b) acc[w * MB + b] = mfma_16x16x32<DT>(v[w], v[kWBlocks + b], acc[w * MB + b]);
  };
  auto load = [&](u32x4 (&v)[kFewAhead][kOperands], int step) {
#pragma unroll
    for (int i = 0; i < kFewAhead; ++i)
#pragma unroll
      for (int o = 0; o < kWBlocks; ++o) v[i][o] = load_any(row[o] + ((int64_t)min(step + i, end - 1) * 32 + lg * 8) * 2);
    if (li < p.rows) {
#pragma unroll
      for (int i = 0; i < kFewAhead; ++i)
#pragma unroll
        for (int o = kWBlocks; o < kOperands; ++o) v[i][o] = load_any(row[o] + ((int64_t)min(step + i, end - 1) * 32 + lg * 8) * 2);
    }
  };
  if (begin < end) {
    u32x4 now[kFewAhead][kOperands], next[kFewAhead][kOperands];
    load(now, begin);
    for (int step = begin; step < end; step += kFewAhead) {
      if (step + kFewAhead < end) load(next, step + kFewAhead);
#pragma unroll
      for (int i = 0; i < kFewAhead; ++i)
        if (step + i < end) multiply(now[i]);
#pragma unroll
      for (int i = 0; i < kFewAhead; ++i)
#pragma unroll
        for (int o = 0; o < kOperands; ++o) now[i][o] = next[i][o];
    }
  }
  if (wave == 0 && rest > 0) {
    if (p.length >= 8 && left < 8) {
#pragma unroll
      for (int o = 0; o < kOperands; ++o) last[o] = unit_from_row_end<DT>(Unit<DT>{{last[o]}}, left).q[0];
    }
    multiply(last);
  }

  // A lane has rows 4 lg ... of W for row li of x.
#pragma unroll
  for (int b = 0; b < kWBlocks * MB; ++b) *reinterpret_cast<f32x4*>(&sums[wave][b][li * 16 + 4 * lg]) = acc[b];
  __syncthreads();
  if (threadIdx.x >= 16 * COLS * MB) return;
  const int m = threadIdx.x / COLS, c = threadIdx.x % COLS, at = m % 16 * 16 + c;
  const int64_t col = n0 + c;
  if (m >= p.rows) return;
  float a = 0.0f, u = 0.0f;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) {
    a += sums[w][m / 16][at];
    u += kWBlocks == 2 ? sums[w][(kWBlocks - 1) * MB + m / 16][at] : sums[w][m / 16][at + COLS];
  }
  auto store = [](char* to, int64_t element, float v) { reinterpret_cast<uint16_t*>(to)[element] = (uint16_t)narrow_pair<DT>(v, 0.0f); };
  const bool exists = col < p.n;
  float slope, f;
  by_activation(p.act, [&](auto act) { f = activate<decltype(act)::value, KIND == kGatedGrad>(a, slope); });
  if (exists && (KIND == kGated || p.out[0] != nullptr)) store(p.out[0], (int64_t)m * p.n + col, f * u);
  if constexpr (KIND == kGatedGrad) {                                    // (columns of [da du] that h does not have: zero)
    const float g = exists ? widen16<DT>(reinterpret_cast<const uint16_t*>(p.grad_h)[(int64_t)m * p.n + col]) : 0.0f;
    store(p.out[1], (int64_t)m * 2 * p.padded + col, exists ? g * u * slope : 0.0f);
    store(p.out[1], (int64_t)m * 2 * p.padded + p.padded + col, exists ? g * f : 0.0f);
  } else if (exists && p.out[1] != nullptr) {
    store(p.out[1], (int64_t)m * p.n + col, a);
    store(p.out[2], (int64_t)m * p.n + col, u);
  }
}

}  // namespace

// The products of gated_product.h in tiles of 256 x 256 on four waves of 128 x 128, for outputs of enough of them.
//
// What bounds them is the chip's power, and the LDS: a wave that multiplies 128 x 128 reads 8 + 8 operands of 32 values of l for 64 matrix instructions;
// eight waves of 64 x 128 read half as much again.  (kWeight, 8192 rows, 22016 x 4096, both operands transposed by the reads: 1292 us with eight waves,
// 1060 with four.)  The instruction is the one of 16 x 16 x 32: per product it moves half as much of the sums through registers as 32 x 32 x 16 does, and
// the clock rises by as much as that saves (forward 32768 x 11008 x 4096 4.52 -> 4.26 ms on one card).  The sums take 256 registers of a lane's 512, one wave
// to a SIMD, so nothing but this loop hides a latency:
//   - a step is 64 values of l, 32 KB of either operand (a unit); LDS holds five units, C and R of successive steps in turn;
//   - the operands of 32 values are read while the 64 matrix instructions of those before run;
//   - the one barrier of a step stands in front of its second half: all waves have read the step's units by then, and the next step's have
//     arrived.  Behind it the places of the step's units are free: R of the step after the next is fetched at once, the C after that in the first
//     half of the next step, so that a unit has a step to one and a half to arrive;
//   - a lane's offsets into an operand are made once; a load needs its place in LDS set and nothing else.
// Rows that run along l: 256 rows of 128 bytes, 16-byte piece p of row r at p ^ (r / 2 mod 8).  Across: 64 rows (one l) of 512 bytes, two to a load, the
// 64-byte piece q of row l at q ^ (l mod 4), its halves changing places with l / 8.
//
// 32768 x 11008 x 4096 bfloat16, forward: 4.02 to 4.28 ms, 1380 to 1470 TFLOP/s; the library's plain product of the same two matrices, without the activation, runs at 1498 to 1544.
// Handing the tiles out in the kernel, with the next tile's first loads under the end of this one, was 1 % slower (power again), rounds of 16 x 16
// tiles in place of 4 x 64 as well.
#pragma once
#include "gated_product.h"

namespace {

struct TileLarge {
  static constexpr int kRows = 256, kCols = 256, kWavesM = 2, kWavesN = 2, kMB = 4, kNB = 4, kWaves = 4, kThreads = 256;
};

// Workgroup -> tile of a launch.  Whole rounds of 256 workgroups: the s-th workgroup of a die d in round r takes position 256 r + 32 d + s (a patch of
// 4 x 8 tiles to a die); the rest keep their number.
__host__ __device__ inline int large_tile_of_workgroup(int id, int tiles) {
  constexpr int kRound = 256, kDies = 8;
  return id < tiles / kRound * kRound ? id / kRound * kRound + id % kDies * (kRound / kDies) + id % kRound / kDies : id;
}

constexpr int kUnit = 32768, kSlots = 5;

// sum += a b, in the sum's own registers.  (In assembly because the compiler gives such products other registers than their sums' and moves 256 of them
// about.  64 others lie between two products of a sum, and 32 cycles and more between the last of them and its reader.)
template <int DT>
__device__ __forceinline__ void add_16x16x32(f32x4& sum, const u32x4& a, const u32x4& b) {
  if constexpr (DT == kBF16) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(sum) : "v"(a), "v"(b));
  else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(sum) : "v"(a), "v"(b));
}

// Workgroup `id` of those that share a product's tiles and slices.
template <int DT, int KIND>
__device__ __forceinline__ void product_tile_large(const Product& p, int id, char* lds) {
  using S = TileLarge;
  constexpr bool kRAcross = rows_across(KIND), kCAcross = cols_across(KIND);
  constexpr int kSources = is_gated(KIND) ? 2 : 1;
  const int t = threadIdx.x, lane = t & (kWave - 1);
  const int uw = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = uw & 1, wn = uw >> 1;
  const int li = lane & 31, lg = lane >> 5;
  const Share share = p.slices == 1 ? Share{large_tile_of_workgroup(id, p.tiles), 0} : share_of_workgroup(id, p.tiles, p.slices);
  const int first = step_of_slice(p, share.slice), last = step_of_slice(p, share.slice + 1);   // steps of the workgroup
  const TileIndex tile = tile_at(p, share.pos);

  // ---- loads: eight of 1 KB per wave and unit, load i at (4 i + wave) KB.
  const bool second = KIND == kInput && first >= p.half;               // kInput: the slice begins in du Wu
  const int64_t line = (int64_t)(second ? first - p.half : first) * 64;  // the first value of l, in its half
  Feed<kCAcross, 8> c[kSources];
  Feed<kRAcross, 8> r;
  auto offsets = [&](auto& feed, uint32_t pitch, auto across, auto row_of_load) {
    feed.piece = (lane & 7) ^ ((lane >> 4) | ((uw & 1) << 2));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (decltype(across)::value)
        feed.off[i] = (uint32_t)(2 * (4 * i + uw) + lg) * pitch + (uint32_t)((lane & 31) ^ ((2 * (uw & 1) + lg) << 2) ^ ((i & 1) << 1)) * 16u;
      else
        feed.off[i] = (uint32_t)(row_of_load(i) + uw * 8 + (lane >> 3)) * pitch + (uint32_t)feed.piece * 16u;
    }
  };
  using CAcross = std::integral_constant<bool, kCAcross>;
  using RAcross = std::integral_constant<bool, kRAcross>;
  // A wave's 128 columns of C: two blocks of 32 rows of Wg and two of Wu, each of the same 64 columns of h; load i brings block i.
  constexpr int kOuterC = is_gated(KIND) ? 128 : 256;
  const int64_t n0 = (int64_t)tile.n * kOuterC, m0 = (int64_t)tile.m * 256;
#pragma unroll
  for (int w = 0; w < kSources; ++w) {
    const char* const base = second ? p.c[1] : p.c[w];
    c[w].begin(kCAcross ? base + line * p.c_pitch + n0 * 2 : base + n0 * p.c_pitch + line * 2, p.cols - n0, kOuterC, p.c_pitch, n0 * 2);
    offsets(c[w], (uint32_t)p.c_pitch, CAcross{}, [](int i) { return is_gated(KIND) ? (i >> 2) * 64 + (i & 1) * 32 : i * 32; });
  }
  r.begin(kRAcross ? p.r + line * p.r_pitch + m0 * 2 : p.r + m0 * p.r_pitch + (int64_t)first * 128, p.rows - m0, 256, p.r_pitch, m0 * 2);
  offsets(r, (uint32_t)p.r_pitch, RAcross{}, [](int i) { return i * 32; });
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds) + (uint32_t)uw * 1024u;
  auto exist = [&](bool of_c, int s) {                                   // from step s of the workgroup on
    const int at = first + s;
    if (at >= last) return 0;
    if (KIND == kInput) return of_c ? p.length - 64 * (at < p.half ? at : at - p.half) : 64;
    return p.length - 64 * at;
  };
  u32x4 c_buffer[kSources], r_buffer;
  auto open_c = [&](int s) {
    int64_t next = kCAcross ? 64 * p.c_pitch : 128;
    if (KIND == kInput && first + s + 1 == p.half) next = p.c[1] - p.c[0] - (int64_t)(p.half - 1) * next;
#pragma unroll
    for (int w = 0; w < kSources; ++w) c_buffer[w] = c[w].open(exist(true, s), (uint32_t)p.c_pitch, next);
  };
  auto open_r = [&](int s) { r_buffer = r.open(exist(false, s), (uint32_t)p.r_pitch, kRAcross ? 64 * p.r_pitch : 128); };
  auto fetch_c = [&](int i, int slot) {
    const int w = kSources == 2 ? (i >> 1) & 1 : 0;
    fetch_to_lds(lds0 + (uint32_t)(slot * kUnit + i * 4096), c[w].off[i], c_buffer[w]);
  };
  auto fetch_r = [&](int i, int slot) { fetch_to_lds(lds0 + (uint32_t)(slot * kUnit + i * 4096), r.off[i], r_buffer); };

  // ---- operand reads: a block of 16 rows, 32 values of l
  const int l16 = lane & 15, l8 = lane >> 4;
  // (across: the halves of 64 bytes change places with l / 8)
  const int tr_x = (lane >> 2) & 3, tr_at = (8 * l8 + (l16 >> 2)) * 512 + (lane & 3) * 8 + (l8 & 1) * 32;
  const char *pc[8], *pr[8];                                             // along: by half of a step (two of them); across: by block
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const int col = ((4 * (q & 1) + l8) ^ ((l16 >> 1) & 7)) << 4;
    pc[q] = lds + (kCAcross ? (tr_at ^ (q & 1) * 32) + (wn * 4 + (q / 2 ^ tr_x)) * 64 : (wn * 128 + l16) * 128 + col);
    pr[q] = lds + (kRAcross ? (tr_at ^ (q & 1) * 32) + (wm * 4 + (q / 2 ^ tr_x)) * 64 : (wm * 128 + l16) * 128 + col);
  }
  auto read = [&](const char* (&of)[8], int block, int half, int unit, auto across) {
    if constexpr (decltype(across)::value) {
      const char* const from = of[block] + unit + half * 16384;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(from)));
      const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(from + 2048)));
      return u32x4{lo.x, lo.y, hi.x, hi.y};
    } else {
      return *reinterpret_cast<const u32x4*>(of[half] + unit + block * 2048);
    }
  };

  QuarterBlocks acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[i][j].of[q >> 1][q & 1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  u32x4 a[2][8], b[2][8];                                                // of a step's halves

  // Units 0 ... 3: C and R of the first two steps.  Unit u lies in place u mod 5.
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    open_c(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) fetch_c(i, 2 * s);
    open_r(s);
#pragma unroll
    for (int i = 0; i < 8; ++i) fetch_r(i, 2 * s + 1);
  }
  wait_fetches_and_reads<16>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int j = 0; j < 8; ++j) a[0][j] = read(pc, j, 0, 0, CAcross{});
#pragma unroll
  for (int j = 0; j < 8; ++j) b[0][j] = read(pr, j, 0, kUnit, RAcross{});

  const int steps = last - first;
  int slot = 0;                                                          // of C of step s
  auto behind = [](int slot, int n) { return slot + n < kSlots ? slot + n : slot + n - kSlots; };
  for (int s = 0; s < steps; ++s) {
    const int c_here = slot * kUnit, r_here = behind(slot, 1) * kUnit, c_next = behind(slot, 2) * kUnit, r_next = behind(slot, 3) * kUnit;
    const int c_free = behind(slot, 4), r_free = slot;                   // places of C of step s + 2 and, behind the barrier, of its R
    open_c(s + 2);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (half == 1) {
        wait_fetches_and_reads<8>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        open_r(s + 2);
      }
      const int c_from = half == 0 ? c_here : c_next, r_from = half == 0 ? r_here : r_next, to = half ^ 1;
#pragma unroll
      for (int q = 0; q < 64; ++q) {
        const int nb = q >> 3, mb = q & 7;
        add_16x16x32<DT>(acc[mb >> 1][nb >> 1].of[mb & 1][nb & 1], a[half][nb], b[half][mb]);
        __builtin_amdgcn_sched_barrier(0);
        if ((q & 7) == 5) {
          if (half == 0) fetch_c(q >> 3, c_free);
          else fetch_r(q >> 3, r_free);
        }
        if ((q & 3) == 0) {
          if (q < 32) a[to][q >> 2] = read(pc, q >> 2, to, c_from, CAcross{});
          else b[to][(q >> 2) - 8] = read(pr, (q >> 2) - 8, to, r_from, RAcross{});
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    slot = behind(slot, 2);
  }
  wait_fetches_and_reads<0>();
  end_tile<DT, KIND, S>(p, share, tile, acc, wm, wn, li, lg);
}

template <int DT, int KIND>
__global__ __launch_bounds__(TileLarge::kThreads, 1) void k_gated_product_large(const Product p) {
  __shared__ __align__(1024) char lds[kSlots * kUnit];
  product_tile_large<DT, KIND>(p, (int)blockIdx.x, lds);
}

// Both gradients' products (k_gated_gradients).
template <int DT>
__global__ __launch_bounds__(TileLarge::kThreads, 1) void k_gated_gradients_large(const Product input, const Product weight, int weights_first) {
  __shared__ __align__(1024) char lds[kSlots * kUnit];
  const int id = (int)blockIdx.x, inputs = input.tiles * input.slices, weights = weight.tiles * weight.slices;
  if (weights_first ? id >= weights : id < inputs) product_tile_large<DT, kInput>(input, weights_first ? id - weights : id, lds);
  else product_tile_large<DT, kWeight>(weight, weights_first ? id : id - inputs, lds);
}

}  // namespace

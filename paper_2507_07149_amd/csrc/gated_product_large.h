// The products of gated_product.h in tiles of 256 x 256 on 8 waves, for outputs of enough of them (kWeight: gated_product_across.h).
//
// A 128 x 256 tile on four waves reads 96 KB of operands out of LDS and takes 48 KB in per step of 64 values of l: 1150 cycles at 128 bytes
// each, against 1024 cycles of matrix instructions.  Here it is 192 + 64 KB against 2048 cycles, and two waves to a SIMD.  LDS holds two steps
// only, so a step's operands are taken in by parts: four of C (the blocks nb of the two columns of waves) and two of R (the blocks mb of
// the four rows of waves), each loaded again as soon as it has been read, two to three half steps before it is waited for:
//   half 0 (blocks 0, 1 of C)  reads C1 C2 of s, R0 of s + 1;       loads R1 C0 of s + 2, C3 of s + 1
//   half 1 (blocks 2, 3)       reads C3 of s, C0 R1 of s + 1;       loads C1 C2 of s + 2, R0 of s + 3
// A part is overwritten in a half after the one that read it (the barrier between them follows a wait for the reads), and is read only
// behind a barrier that follows a wait for all but the last eight loads of every wave, those of the two last halves.
//
// C where it runs across is staged by blocks of 32 outputs here, rows of 64 bytes.  Registers are short (256, 128 of them sums): what
// lies outside an operand is cut off by the length of the buffer that a load is given, in scalar registers, and only the end of l of
// rows that run along it by the lanes' offsets.
#pragma once
#include "gated_product.h"

namespace {

struct TileLarge {
  static constexpr int kRows = 256, kCols = 256, kWavesM = 4, kWavesN = 2, kMB = 2, kNB = 4, kWaves = 8, kThreads = 512;
};
constexpr int kLargeOperand = 32768;                 // bytes of an operand's step

// Workgroup -> tile of a launch.  Whole rounds of 256 workgroups: the s-th workgroup of a die d in round r takes position 256 r + 32 d + s (a patch of
// 4 x 8 tiles to a die); the rest keep their number.
__host__ __device__ inline int large_tile_of_workgroup(int id, int tiles) {
  constexpr int kRound = 256, kDies = 8;
  return id < tiles / kRound * kRound ? id / kRound * kRound + id % kDies * (kRound / kDies) + id % kRound / kDies : id;
}

template <int DT, int KIND>
__global__ __launch_bounds__(TileLarge::kThreads, 2) void k_gated_product_large(const Product p) {
  using S = TileLarge;
  static_assert(!rows_across(KIND), "R runs along l");
  constexpr bool kCAcross = cols_across(KIND);
  __shared__ __align__(1024) char lds[4 * kLargeOperand];                // C of even and odd steps, R of even and odd steps
  const int t = threadIdx.x, lane = t & (kWave - 1);
  const int uw = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = uw & 3, wn = uw >> 2;
  const int li = lane & 31, lg = lane >> 5;
  const Share share = p.slices == 1 ? Share{large_tile_of_workgroup((int)blockIdx.x, p.tiles), 0} : share_of_workgroup((int)blockIdx.x, p.tiles, p.slices);
  const int first = step_of_slice(p, share.slice), last = step_of_slice(p, share.slice + 1);   // steps of the workgroup
  const TileIndex tile = tile_at(p, share.pos);
  const int64_t m0 = (int64_t)tile.m * S::kRows;

  // ---- loads: one of 1 KB per wave and part of C, two of R.
  // along: eight rows, piece (lane mod 8) ^ (row / 2 mod 8) of row lane / 8; odd: the second eight of sixteen.
  const int piece = (lane & 7) ^ (lane >> 4);
  const uint32_t c_pitch = (uint32_t)p.c_pitch, r_pitch = (uint32_t)p.r_pitch;
  const uint32_t along = (uint32_t)(lane >> 3) * (KIND == kInput ? r_pitch : c_pitch);
  const uint32_t off_even = along + (uint32_t)piece * 16u, off_odd = along + (uint32_t)(piece ^ 4) * 16u;
  // across: sixteen values of l, 64 bytes each.
  const uint32_t off_c = (uint32_t)(lane >> 2) * c_pitch + (uint32_t)(lane & 3) * 16u;

  struct Source {
    uint64_t at;
    uint32_t bytes;                                                      // that exist from there on
  };
  Source src_c[4], src_r[2][2];
  auto bytes_of = [](int64_t rows, int64_t pitch) { return (uint32_t)(rows <= 0 ? 0 : rows > 64 ? kNowhere : (uint64_t)(rows * pitch)); };
#pragma unroll
  for (int nb = 0; nb < 4; ++nb) {
    if constexpr (kCAcross) {
      const int64_t col = (int64_t)tile.n * 256 + (uw >> 2) * 128 + nb * 32;
      const bool second = KIND == kInput && first >= p.half;
      const int64_t line = (second ? first - p.half : first) * (int64_t)64 + (uw & 3) * 16;
      src_c[nb].at = reinterpret_cast<uint64_t>(p.c[second] + line * p.c_pitch + col * 2);
      src_c[nb].bytes = (uint32_t)(col * 2);                             // (before the place in its row: what is missing in the last one)
    } else {
      const int64_t row = (int64_t)tile.n * 128 + (uw >> 2) * 64 + (nb & 1) * 32 + (uw & 3) * 8;
      src_c[nb].at = reinterpret_cast<uint64_t>(p.c[nb >> 1] + row * p.c_pitch + (int64_t)first * 128);
      src_c[nb].bytes = bytes_of(p.cols - row, p.c_pitch);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int mb = i >> 1, j = i & 1, sub = (uw & 1) * 2 + j;
    const int64_t row = m0 + (uw >> 1) * 64 + mb * 32 + sub * 8;
    src_r[mb][j].at = reinterpret_cast<uint64_t>(p.r + row * p.r_pitch + (int64_t)first * 128);
    src_r[mb][j].bytes = bytes_of(p.rows - row, p.r_pitch);
  }
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds);
  const uint32_t dst_c = lds0 + (uint32_t)((uw >> 2) * 16384 + (uw & 3) * 1024), dst_r = lds0 + 2 * kLargeOperand + (uint32_t)((uw >> 1) * 8192 + (uw & 1) * 2048);
  auto load = [&](uint32_t dst, uint32_t off, uint64_t at, uint32_t bytes) {
    const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, bytes, 0x00020000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(dst), "v"(off), "s"(buffer) : "memory");
  };
  // Values of l that step `s` of the workgroup has.
  auto exist = [&](bool of_c, int s) {
    const int at = first + s;
    if (at >= last) return 0;
    if (KIND == kInput) return of_c ? p.length - 64 * (at < p.half ? at : at - p.half) : 64;
    return p.length - 64 * at;
  };
  // Of an operand across: `there` values of l from the load's first one on, the last of them in a row that ends the operand.
  auto across_bytes = [&](int there, uint32_t pitch, uint32_t col_bytes) {
    const uint32_t all = (uint32_t)there * pitch;
    return there >= 64 ? kNowhere : there > 0 && all > col_bytes ? all - col_bytes : 0u;
  };
  auto fetch_c = [&](int nb, int s) {
    const uint32_t dst = dst_c + (uint32_t)((s & 1) * kLargeOperand + nb * 4096);
    const int there = exist(true, s);
    if constexpr (kCAcross) {
      load(dst, off_c, src_c[nb].at, across_bytes(there - (uw & 3) * 16, c_pitch, src_c[nb].bytes));
      int64_t next = 64 * p.c_pitch;
      if (KIND == kInput && first + s + 1 == p.half) next = p.c[1] - p.c[0] - (int64_t)(p.half - 1) * next;
      src_c[nb].at += next;
    } else {
      const uint32_t off = (uw & 1) ? off_odd : off_even;
      load(dst, (piece ^ ((uw & 1) * 4)) * 8 < there ? off : kNowhere, src_c[nb].at, src_c[nb].bytes);
      src_c[nb].at += 128;
    }
  };
  auto fetch_r = [&](int mb, int j, int s) {
    const uint32_t dst = dst_r + (uint32_t)((s & 1) * kLargeOperand + mb * 4096 + j * 1024);
    const int there = exist(false, s);
    Source& from = src_r[mb][j];
    load(dst, (piece ^ (j * 4)) * 8 < there ? (j ? off_odd : off_even) : kNowhere, from.at, from.bytes);
    from.at += 128;
  };

  // ---- operand reads
  const char *pa[4], *pb[4];
  const int tr_at = (8 * lg + ((lane & 15) >> 2)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const int col = ((2 * ks + lg) ^ ((li >> 1) & 7)) << 4;
    pa[ks] = lds + wn * 16384 + (kCAcross ? tr_at + ks * 1024 : li * 128 + col);
    pb[ks] = lds + 2 * kLargeOperand + wm * 8192 + li * 128 + col;
  }
  auto read = [&](bool is_across, const char* at) {
    if (!is_across) return *reinterpret_cast<const u32x4*>(at);
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at + 256)));
    return u32x4{lo.x, lo.y, hi.x, hi.y};
  };
  auto read_c = [&](int nb, int ks, int parity) { return read(kCAcross, pa[ks] + parity * kLargeOperand + nb * 4096); };
  auto read_r = [&](int mb, int ks, int parity) { return read(false, pb[ks] + parity * kLargeOperand + mb * 4096); };

  f32x16 acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  u32x4 a[2][4], b[2][2][4];                         // a[nb mod 2][ks], b[step mod 2][mb][ks]
  fetch_r(0, 0, 0); fetch_r(0, 1, 0); fetch_r(1, 0, 0); fetch_r(1, 1, 0); fetch_c(0, 0);
  fetch_c(1, 0); fetch_c(2, 0); fetch_r(0, 0, 1); fetch_r(0, 1, 1);
  fetch_r(1, 0, 1); fetch_r(1, 1, 1); fetch_c(0, 1); fetch_c(3, 0);
  wait_fetches_and_reads<8>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    b[0][0][ks] = read_r(0, ks, 0);
    b[0][1][ks] = read_r(1, ks, 0);
    a[0][ks] = read_c(0, ks, 0);
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  fetch_c(1, 1); fetch_c(2, 1); fetch_r(0, 0, 2); fetch_r(0, 1, 2);
  wait_fetches_and_reads<8>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");

  // One step on the copies of parity P; two halves of sixteen matrix instructions, a barrier behind each.
  auto step = [&](auto parity, int s) {
    constexpr int P = decltype(parity)::value;
#pragma unroll
    for (int nb = 0; nb < 4; ++nb) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {                              // values of l 32 h ... of block nb
        acc[0][nb] = mfma16<DT>(a[nb & 1][2 * h], b[P][0][2 * h], acc[0][nb]);
        __builtin_amdgcn_sched_barrier(0);
        if (nb == 0) fetch_r(1, h, s + 2);
        else if (nb == 1) { if (h == 0) fetch_c(0, s + 2); else fetch_c(3, s + 1); }
        else if (nb == 2) fetch_c(1 + h, s + 2);
        else fetch_r(0, h, s + 3);
        __builtin_amdgcn_sched_barrier(0);
        a[(nb + 1) & 1][2 * h] = nb < 3 ? read_c(nb + 1, 2 * h, P) : read_c(0, 2 * h, P ^ 1);
        a[(nb + 1) & 1][2 * h + 1] = nb < 3 ? read_c(nb + 1, 2 * h + 1, P) : read_c(0, 2 * h + 1, P ^ 1);
        b[P ^ 1][nb >> 1][2 * (nb & 1) + h] = read_r(nb >> 1, 2 * (nb & 1) + h, P ^ 1);
        acc[1][nb] = mfma16<DT>(a[nb & 1][2 * h], b[P][1][2 * h], acc[1][nb]);
        acc[0][nb] = mfma16<DT>(a[nb & 1][2 * h + 1], b[P][0][2 * h + 1], acc[0][nb]);
        acc[1][nb] = mfma16<DT>(a[nb & 1][2 * h + 1], b[P][1][2 * h + 1], acc[1][nb]);
        // one operand's reads (two of a transposed one) in front of each of the three
        __builtin_amdgcn_sched_group_barrier(0x100, kCAcross ? 2 : 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, kCAcross ? 2 : 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (nb & 1) {
        wait_fetches_and_reads<8>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
      }
    }
  };
  const int steps = last - first;
  int s = 0;
  for (; s + 1 < steps; s += 2) {
    step(std::integral_constant<int, 0>{}, s);
    step(std::integral_constant<int, 1>{}, s + 1);
  }
  if (s < steps) step(std::integral_constant<int, 0>{}, s);
  wait_fetches_and_reads<0>();
  end_tile<DT, KIND, S>(p, share, tile, acc, wm, wn, li, lg);
}

}  // namespace

// The weights' gradients (kWeight of gated_product.h) in tiles of 256 x 256 on 8 waves: both operands run across the output.
//
// A slab of 32 values of l is 32 rows of 512 bytes of each operand, which the loads bring as they lie, two rows to an instruction; LDS holds five.
// Where the products whose operands run along l go through a step by blocks of 32 rows of C, this one goes by 16 values of l: all of a wave's
// six operands of 16 values are read while the eight matrix instructions of the 16 before run, half the registers, and one barrier for every 32.
// The 64-byte piece q of a slab's row l lies at place q ^ (l mod 4): the transposing reads take 64 bytes of four consecutive rows, which are then
// on different banks.
#pragma once
#include "gated_product_large.h"

namespace {

template <int DT>
__global__ __launch_bounds__(TileLarge::kThreads, 2) void k_gated_product_across(const Product p) {
  using S = TileLarge;
  constexpr int kSlab = 32, kRow = 512, kOperand = kSlab * kRow, kSlots = 5;
  __shared__ __align__(1024) char lds[kSlots * 2 * kOperand];            // C, R of each slab
  const int t = threadIdx.x, lane = t & (kWave - 1);
  const int uw = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = uw & 3, wn = uw >> 2;
  const int lg = lane >> 5;
  const Share share = p.slices == 1 ? Share{large_tile_of_workgroup((int)blockIdx.x, p.tiles), 0} : share_of_workgroup((int)blockIdx.x, p.tiles, p.slices);
  const int begin = step_of_slice(p, share.slice) * 64;                  // values of l of the workgroup
  const int end = min(step_of_slice(p, share.slice + 1) * 64, p.length);
  const TileIndex tile = tile_at(p, share.pos);

  // ---- loads: rows 2 uw, 2 uw + 1 of each half of a slab, of either operand.
  const uint32_t c_pitch = (uint32_t)p.c_pitch, r_pitch = (uint32_t)p.r_pitch;
  const int piece = (lane & 31) ^ ((2 * (uw & 1) + lg) << 2);
  const uint32_t off_c = (uint32_t)lg * c_pitch + (uint32_t)piece * 16u, off_r = (uint32_t)lg * r_pitch + (uint32_t)piece * 16u;
  const uint32_t col_c = (uint32_t)tile.n * kRow, col_r = (uint32_t)tile.m * kRow;   // bytes in front of the tile in a row
  uint64_t src_c = reinterpret_cast<uint64_t>(p.c[0] + ((int64_t)begin + 2 * uw) * p.c_pitch + col_c);
  uint64_t src_r = reinterpret_cast<uint64_t>(p.r + ((int64_t)begin + 2 * uw) * p.r_pitch + col_r);
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds);
  auto load = [&](uint32_t dst, uint32_t off, uint64_t at, int there, uint32_t pitch, uint32_t col) {
    // rows that exist from the load's first on; the last of them in the row that ends the operand
    const uint32_t all = (uint32_t)there * pitch, bytes = there >= 64 ? kNowhere : there > 0 && all > col ? all - col : 0u;
    const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, bytes, 0x00020000u};
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(dst), "v"(off), "s"(buffer) : "memory");
  };
  // Load i of slab `s` into slot `slot`.
  auto fetch = [&](int i, int s, int slot) {
    const int half = i & 1, there = end - begin - s * kSlab - half * 16 - 2 * uw;
    const uint32_t dst = lds0 + (uint32_t)(slot * 2 * kOperand + (half * 16 + 2 * uw) * kRow);
    if (i < 2) load(dst, off_c, src_c + (uint64_t)(half * 16) * c_pitch, there, c_pitch, col_c);
    else load(dst + kOperand, off_r, src_r + (uint64_t)(half * 16) * r_pitch, there, r_pitch, col_r);
    if (i == 1) src_c += (uint64_t)kSlab * c_pitch;
    if (i == 3) src_r += (uint64_t)kSlab * r_pitch;
  };

  // ---- operand reads: of 16 values of l, lane groups of 16 take four rows of 32 bytes
  const char *pc[4], *pr[2];
  const int x = (lane >> 2) & 3, at = (8 * lg + ((lane & 15) >> 2)) * kRow + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
#pragma unroll
  for (int nb = 0; nb < 4; ++nb) pc[nb] = lds + at + (wn * 4 + (nb ^ x)) * 64;
#pragma unroll
  for (int mb = 0; mb < 2; ++mb) pr[mb] = lds + kOperand + at + ((wm * 2 + mb) ^ x) * 64;
  auto read = [&](const char* from) {
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(from)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(from + 4 * kRow)));
    return u32x4{lo.x, lo.y, hi.x, hi.y};
  };

  f32x16 acc[2][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
  u32x4 a[2][4], b[2][2];                                                // of even and odd sixteens

#pragma unroll
  for (int slab = 0; slab < kSlots - 1; ++slab)
#pragma unroll
    for (int i = 0; i < 4; ++i) fetch(i, slab, slab);
  wait_fetches_and_reads<(kSlots - 2) * 4>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int nb = 0; nb < 4; ++nb) a[0][nb] = read(pc[nb]);
#pragma unroll
  for (int mb = 0; mb < 2; ++mb) b[0][mb] = read(pr[mb]);

  const int slabs = (end - begin + kSlab - 1) / kSlab;
  int slot = 0;
  for (int s = 0; s < slabs; ++s) {
    // Slab s + 1 has arrived for all, and nobody reads slab s - 1 any more: its place takes slab s + 4.
    wait_fetches_and_reads<(kSlots - 3) * 4>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int next = slot + 1 < kSlots ? slot + 1 : 0, free = slot > 0 ? slot - 1 : kSlots - 1;
    const int here = slot * 2 * kOperand, there = next * 2 * kOperand;
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int from = ks == 0 ? here + 16 * kRow : there;               // where the next sixteen lie
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int nb = q >> 1, mb = q & 1;
        acc[mb][nb] = mfma16<DT>(a[ks][nb], b[ks][mb], acc[mb][nb]);
        __builtin_amdgcn_sched_barrier(0);
        if (ks == 0 && (q & 1) == 0) fetch(q >> 1, s + kSlots - 1, free);
        if (q < 4) a[ks ^ 1][q] = read(pc[q] + from);
        else if (q < 6) b[ks ^ 1][q - 4] = read(pr[q - 4] + from);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    slot = next;
  }
  wait_fetches_and_reads<0>();
  end_tile<DT, kWeight, S>(p, share, tile, acc, wm, wn, lane & 31, lg);
}

}  // namespace

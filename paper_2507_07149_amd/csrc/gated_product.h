// The matrix products of the gated feed-forward block (gated_linear.hip): one kernel for all, in the tiles of `Tile`.
//
//   out[row, col] = sum over l of R[row, l] * C[col, l]        16-bit formats, binary32 accumulation (v_mfma_f32_32x32x16)
//
//   kGated      R = x, C = Wg and Wu in turns of 32 rows, so that a lane has a and u of the same outputs:   h = f(a) u
//   kGatedGrad  the same products again, with grad_h: da = grad_h u f'(a), du = grad_h f(a) (and h)
//   kInput      R = [da du], C = [Wg; Wu]^T:       grad_x = da Wg + du Wu
//   kWeight     R = [da du]^T, C = x^T:            grad_Wg = da^T x, grad_Wu = du^T x
//
// An operand whose rows run along l ("along": x, W, [da du] as rows) is staged as rows of 64 values of l, 128 bytes, with the 16-byte piece p of
// row r at place p ^ (r / 2 mod 8).  One whose rows run along the output ("across") is staged as it lies too, 64 outputs of one l to a row of
// 128 bytes, pieces at p ^ 4 (l / 2 mod 2), and transposed by the reads (ds_read_b64_tr_b16).  Both ways the loads move whole cache lines
// straight into LDS and neither they nor the reads meet bank conflicts; nothing is transposed in memory.
//
// What lies outside an operand is never read: such a lane's offset lies behind the end of the buffer that the load is given, and its place
// in LDS receives zeros.  So sizes need not be multiples of a tile, and what pads a tile adds 0 * 0 to the sums.
#pragma once
#include "block_common.h"
#include "linear_common.h"

namespace {

enum ProductKind { kGated, kGatedGrad, kInput, kWeight };
constexpr bool rows_across(int kind) { return kind == kWeight; }
constexpr bool cols_across(int kind) { return kind == kInput || kind == kWeight; }
constexpr bool is_gated(int kind) { return kind == kGated || kind == kGatedGrad; }

struct Product {
  const char *r, *c[2];          // c[1]: Wu where c[0] is Wg
  int64_t r_pitch, c_pitch;      // bytes of a row in memory
  int32_t rows, cols;            // of R and C that exist (kGated, kGatedGrad: of each of the two)
  int32_t length;                // of l: K; kInput: N, of each of the two halves; kWeight: M
  int32_t steps, half;           // of 64 values of l; kInput: in each of the two halves
  int32_t tiles_m, tiles_n, slices;
  float* partial;                // slices > 1: the tiles of every slice as the lanes have them
  // what becomes of the sums
  char *out[3];                  // kGated: h, a, u; kGatedGrad: h, [da du]; kInput: grad_x; kWeight: grad_Wg, grad_Wu.  h of kGatedGrad, a and u: may be null
  const char* grad_h;
  int64_t n;                     // columns of h
  int64_t padded;                // of da, a multiple of 64: [da du] is [rows, 2 padded], zero where da and du have no column
  int64_t k;                     // columns of grad_x and the weights
  int32_t act;
};

// `cols` of the tile are rows of C: kGated takes 32 of Wg and 32 of Wu for 32 columns of h.
template <int ROWS, int COLS, int WAVES_M, int WAVES_N, int STAGES>
struct Tile {
  static constexpr int kRows = ROWS, kCols = COLS, kWavesM = WAVES_M, kWavesN = WAVES_N, kStages = STAGES;
  static constexpr int kWaves = WAVES_M * WAVES_N, kThreads = kWaves * kWave;
  static constexpr int kMB = ROWS / WAVES_M / 32, kNB = COLS / WAVES_N / 32;            // blocks of 32 x 32 of a wave
  static constexpr int kStageBytes = (ROWS + COLS) * 128;                               // C's, then R's
  static constexpr int kLoadsC = COLS / 8 / kWaves, kLoadsR = ROWS / 8 / kWaves, kLoads = kLoadsC + kLoadsR;   // of 1 KB, per wave and step
  static_assert(kMB * WAVES_M * 32 == ROWS && kNB * WAVES_N * 32 == COLS, "tile shape");
  static_assert(kLoadsC * kWaves * 8 == COLS && kLoadsR * kWaves * 8 == ROWS && kWaves == 4, "loads of a wave");
  static_assert(kNB % 2 == 0 && COLS % 64 == 0, "pairs of blocks");
  static_assert(STAGES >= 3 && (STAGES - 1) * kLoads <= 63 && STAGES * kStageBytes <= 160 * 1024, "stages");
};

constexpr uint32_t kNowhere = 0x80000000u;           // an offset at the end of every buffer

// 64 lanes x 16 bytes from memory straight into LDS: lane l reads base + off, LDS byte lds + 16 l is written; zeros where off is kNowhere.
// (As load_to_lds: in assembly because the compiler would wait for it in front of the next LDS read, no register result.)
__device__ __forceinline__ void fetch_to_lds(uint32_t lds, uint32_t off, const char* base) {
  const uint64_t at = reinterpret_cast<uint64_t>(base);
  const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, kNowhere, 0x00020000u};   // untyped, 2^31 bytes
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds), "v"(off), "s"(buffer)
               : "memory");
}

template <int N>
__device__ __forceinline__ void wait_fetches_and_reads() {             // all but N loads into LDS, all LDS reads
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
__device__ __forceinline__ u32x4 read_across(const char* p) {          // four values of l, and the four behind them
  const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p)));
  const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(p + 512)));
  return u32x4{lo.x, lo.y, hi.x, hi.y};
}

// blockIdx -> tile and slice.  Every die (blockIdx mod 8) takes a run of consecutive tiles of panels of four tile rows, walked column by column, so
// that the workgroups that run together share operands in its cache; the slices of a tile are far apart.
struct Share {
  int tm, tn, slice;
};
__host__ __device__ inline Share share_of_workgroup(int id, int tiles_m, int tiles_n, int slices) {
  constexpr int kDies = 8, kPanel = 4;
  const int tiles = tiles_m * tiles_n, total = tiles * slices, each = total / kDies, more = total % kDies;
  const int die = id % kDies;
  const int pos = die * each + (die < more ? die : more) + id / kDies;
  const TileIndex t = tile_of_position(pos % tiles, tiles_m, tiles_n, kPanel);
  return {t.m, t.n, pos / tiles};
}

// ---- the activation ----
// f(a) and, where wanted, f'(a).
template <bool SLOPE>
__device__ __forceinline__ float activate(float a, int act, float& slope) {
  if (act == DAF_ACT_SILU || act == DAF_ACT_GELU_TANH) {
    // a p with p = 1 / (1 + exp(-v)): v = a, or 2 sqrt(2 / pi) (a + 0.044715 a^3) (0.5 (1 + tanh(v / 2)) is the same p)
    const bool silu = act == DAF_ACT_SILU;
    constexpr float kC = 1.5957691216057308f;
    const float v = silu ? a : kC * __builtin_fmaf(0.044715f * a * a, a, a);
    const float p = 1.0f / (1.0f + __expf(-v));
    if constexpr (SLOPE) {
      const float dv = silu ? 1.0f : kC * __builtin_fmaf(3.0f * 0.044715f * a, a, 1.0f), pq = p * (1.0f - p);
      slope = pq == 0.0f ? p : __builtin_fmaf(a * pq, dv, p);            // (far out the slope of p is 0 whatever dv has become)
    }
    return a * p;
  }
  if (act == DAF_ACT_GELU) {
    const float p = __builtin_fmaf(0.5f, erff(a * 0.70710678118654752f), 0.5f);
    if constexpr (SLOPE) slope = __builtin_fmaf(a * 0.3989422804014327f, __expf(-0.5f * a * a), p);
    return a * p;
  }
  if constexpr (SLOPE) slope = a > 0.0f ? 1.0f : 0.0f;
  return a <= 0.0f ? 0.0f : a;                                           // (NaN stays)
}

// ---- the end of a tile ----
// 16 consecutive elements of a row, of which `count` exist.
__device__ __forceinline__ void store_row16(char* to, const uint32_t (&v)[8], int64_t count) {
  if (count >= 16) {
    store_any(to, u32x4{v[0], v[1], v[2], v[3]});
    store_any(to + 16, u32x4{v[4], v[5], v[6], v[7]});
    return;
  }
#pragma unroll
  for (int e = 0; e < 16; ++e)
    if (e < count) reinterpret_cast<uint16_t*>(to)[e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
}
template <int DT>
__device__ __forceinline__ void store_block(char* out, int64_t at, const f32x16& v, int64_t count) {
  uint32_t packed[8];
  block_row<DT>(v, packed);
  store_row16(out + at * 2, packed, count);
}
// The lane's 16 values of a block: register r is column 8 (r / 4) + 4 (lane / 32) + r % 4; columns that do not exist are zero.
template <int DT>
__device__ __forceinline__ f32x16 load_block(const char* in, int64_t at, int64_t count, int lg) {
  typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
  f32x16 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int c = 8 * j + 4 * lg;
    u32x2 d = {0u, 0u};
    const char* const p = in + (at + c) * 2;
    if (c + 4 <= count) {
      d = *reinterpret_cast<const u32x2_any*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (c + e < count) d[e >> 1] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[e] << (16 * (e & 1));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * j + e] = widen16<DT>((d[e >> 1] >> (16 * (e & 1))) & 0xFFFFu);
  }
  return v;
}

template <int DT, int KIND, class S>
__device__ __forceinline__ void finish_tile(const Product& p, const f32x16 (&acc)[S::kMB][S::kNB], int64_t m0, int tn, int wm, int wn, int li, int lg) {
#pragma unroll
  for (int mb = 0; mb < S::kMB; ++mb) {
    const int64_t m = m0 + (wm * S::kMB + mb) * 32 + li;
    if (m >= p.rows) continue;
    if constexpr (is_gated(KIND)) {
#pragma unroll
      for (int b = 0; b < S::kNB / 2; ++b) {
        const f32x16 &a = acc[mb][b], &u = acc[mb][b + S::kNB / 2];
        const int64_t block = ((int64_t)tn * (S::kCols / 64) + wn * (S::kNB / 2) + b) * 32, n = block + 16 * lg;
        f32x16 h;
        if constexpr (KIND == kGated) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float unused;
            h[r] = activate<false>(a[r], p.act, unused) * u[r];
          }
          store_block<DT>(p.out[0], m * p.n + n, h, p.n - n);
          if (p.out[1] != nullptr) {
            store_block<DT>(p.out[1], m * p.n + n, a, p.n - n);
            store_block<DT>(p.out[2], m * p.n + n, u, p.n - n);
          }
        } else {
          const f32x16 g = load_block<DT>(p.grad_h, m * p.n + block, p.n - block, lg);
          f32x16 da, du;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float slope;
            const float f = activate<true>(a[r], p.act, slope);
            h[r] = f * u[r];
            da[r] = g[r] * u[r] * slope;
            du[r] = g[r] * f;
          }
          if (p.out[0] != nullptr) store_block<DT>(p.out[0], m * p.n + n, h, p.n - n);
          store_block<DT>(p.out[1], m * 2 * p.padded + n, da, p.padded - n);
          store_block<DT>(p.out[1], m * 2 * p.padded + p.padded + n, du, p.padded - n);
        }
      }
    } else {
      char* out = p.out[0];
      int64_t row = m;
      if constexpr (KIND == kWeight) {                                   // rows of da^T, then of du^T
        if (m >= p.padded) {
          row -= p.padded;
          out = p.out[1];
        }
        if (row >= p.n) continue;
      }
#pragma unroll
      for (int nb = 0; nb < S::kNB; ++nb) {
        const int64_t n = (int64_t)tn * S::kCols + (wn * S::kNB + nb) * 32 + 16 * lg;
        store_block<DT>(out, row * p.k + n, acc[mb][nb], p.k - n);
      }
    }
  }
}

// ---- the product ----
template <int DT, int KIND, class S, bool SLICED>
__global__ __launch_bounds__(S::kThreads, 1) void k_gated_product(const Product p) {
  constexpr int kMB = S::kMB, kNB = S::kNB, kStages = S::kStages;
  constexpr bool kRAcross = rows_across(KIND), kCAcross = cols_across(KIND);
  static_assert(!kRAcross || S::kRows % 64 == 0, "64 outputs to a row of LDS");
  __shared__ __align__(1024) char lds[kStages * S::kStageBytes];
  const int t = threadIdx.x, lane = t & (kWave - 1);
  const int uw = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = uw % S::kWavesM, wn = uw / S::kWavesM;
  const int li = lane & 31, lg = lane >> 5;

  const Share share = share_of_workgroup((int)blockIdx.x, p.tiles_m, p.tiles_n, p.slices);
  const int64_t m0 = (int64_t)share.tm * S::kRows;
  int first = 0, last = p.steps;
  if constexpr (SLICED) {
    first = (int)((int64_t)p.steps * share.slice / p.slices);
    last = (int)((int64_t)p.steps * (share.slice + 1) / p.slices);
  }

  // ---- loads.  Load i of a wave brings 1 KB: eight rows of 128 bytes of LDS, row lane / 8 of them at a lane.
  const int l_row = lane >> 3;
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds);
  const int along_piece = (lane & 7) ^ ((lane >> 4) | ((uw & 1) << 2));            // (row 8 L + lane / 8 with L odd where uw is)
  const int across_piece = (lane & 7) ^ (((lane >> 4) & 1) << 2);
  const char* src[S::kLoads];
  uint32_t off[S::kLoads];
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const bool of_c = i < S::kLoadsC, across = of_c ? kCAcross : kRAcross;
    const int load = (of_c ? i : i - S::kLoadsC) * S::kWaves + uw;                 // of the operand
    const int64_t pitch = of_c ? p.c_pitch : p.r_pitch;
    const char* base = of_c ? p.c[0] : p.r;
    int64_t line = first;                                                          // the step to begin with
    if (KIND == kInput && of_c && first >= p.half) {
      base = p.c[1];
      line -= p.half;
    }
    if (across) {
      const int64_t col = (of_c ? (int64_t)share.tn * S::kCols : m0) + load / 8 * 64;
      src[i] = base + (line * 64 + load % 8 * 8) * pitch + col * 2;
      off[i] = col + across_piece * 8 < (of_c ? p.cols : p.rows) ? (uint32_t)l_row * (uint32_t)pitch + (uint32_t)across_piece * 16u : kNowhere;
    } else {
      int64_t row = m0 + load * 8;
      if (of_c) {
        const int block = load / 4, in = block % kNB;                              // 32 rows; of a wave the first half Wg's, the others Wu's
        if (in >= kNB / 2) base = p.c[1];
        row = (int64_t)share.tn * (S::kCols / 2) + (block / kNB * (kNB / 2) + in % (kNB / 2)) * 32 + load % 4 * 8;
      }
      src[i] = base + row * pitch + line * 128;
      off[i] = row + l_row < (of_c ? p.cols : p.rows) ? (uint32_t)l_row * (uint32_t)pitch + (uint32_t)along_piece * 16u : kNowhere;
    }
  }
  // Values of l that step `s` has.
  auto exist = [&](bool of_c, int s) {
    if (s >= last) return 0;
    if (KIND == kInput) return of_c ? p.length - 64 * (s < p.half ? s : s - p.half) : 64;
    return p.length - 64 * s;
  };
  auto fetch = [&](int i, int s, int st, int exist_c, int exist_r) {
    const bool of_c = i < S::kLoadsC, across = of_c ? kCAcross : kRAcross;
    const int load = (of_c ? i : i - S::kLoadsC) * S::kWaves + uw, there = of_c ? exist_c : exist_r;
    const bool is = across ? l_row < there - load % 8 * 8 : along_piece * 8 < there;
    fetch_to_lds(lds0 + (uint32_t)(st * S::kStageBytes + (of_c ? 0 : S::kCols * 128) + load * 1024), is ? off[i] : kNowhere, src[i]);
    int64_t next = across ? 64 * (of_c ? p.c_pitch : p.r_pitch) : 128;
    if (KIND == kInput && of_c && s + 1 == p.half) next = p.c[1] - p.c[0] - (int64_t)(p.half - 1) * next;
    src[i] += next;
  };

  // ---- operand reads: lane li of a block takes eight values of l from 16 ks + 8 lg on.
  const char *pc[4], *pr[4], *tc[2], *tr[2];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) {
    const int col = ((2 * ks + lg) ^ ((li >> 1) & 7)) << 4;
    pc[ks] = lds + (wn * kNB * 32 + li) * 128 + col;
    pr[ks] = lds + (S::kCols + wm * kMB * 32 + li) * 128 + col;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {                                                    // even and odd blocks from the wave's first
    const int at = (8 * lg + ((lane & 15) >> 2)) * 128 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8, swapped = (lane >> 3) & 1;
    const int bc = wn * kNB, br = wm * kMB;
    tc[h] = lds + bc / 2 * 8192 + at + ((((bc & 1) ^ h) ^ swapped) << 6);
    tr[h] = lds + S::kCols * 128 + br / 2 * 8192 + at + ((((br & 1) ^ h) ^ swapped) << 6);
  }
  f32x16 acc[kMB][kNB];
#pragma unroll
  for (int i = 0; i < kMB; ++i)
#pragma unroll
    for (int j = 0; j < kNB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  u32x4 a[2][kNB][4], b[2][kMB][4];                                                // of even and odd steps
  constexpr int kReads = 4 * (kNB + kMB), kMfma = 4 * kNB * kMB;
  auto read = [&](int q, int parity, int st) {                                     // read q of a step: by l, C's blocks and then R's
    const int ks = q / (kNB + kMB), j = q % (kNB + kMB), at = st * S::kStageBytes;
    if (j < kNB) {
      if constexpr (kCAcross) a[parity][j][ks] = read_across(tc[j & 1] + at + j / 2 * 8192 + ks * 2048);
      else a[parity][j][ks] = *reinterpret_cast<const u32x4*>(pc[ks] + at + j * 4096);
    } else {
      const int i = j - kNB;
      if constexpr (kRAcross) b[parity][i][ks] = read_across(tr[i & 1] + at + i / 2 * 8192 + ks * 2048);
      else b[parity][i][ks] = *reinterpret_cast<const u32x4*>(pr[ks] + at + i * 4096);
    }
  };

#pragma unroll
  for (int st = 0; st < kStages; ++st) {
    const int exist_c = exist(true, first + st), exist_r = exist(false, first + st);
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) fetch(i, first + st, st, exist_c, exist_r);
  }
  wait_fetches_and_reads<(kStages - 1) * S::kLoads>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int q = 0; q < kReads; ++q) read(q, 0, 0);

  int st = 0;                                                                      // stage of step s
  auto step = [&](auto parity, int s) {
    constexpr int P = decltype(parity)::value;
    // Every wave has read step s out of its stage, and step s + 1 has arrived for all: kStages - 2 steps stay on their way.
    wait_fetches_and_reads<(kStages - 2) * S::kLoads>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    const int next = st + 1 < kStages ? st + 1 : 0;
    const int exist_c = exist(true, s + kStages), exist_r = exist(false, s + kStages);
#pragma unroll
    for (int q = 0; q < kMfma; ++q) {
      const int ks = q / (kNB * kMB), j = q % (kNB * kMB);
      acc[j / kNB][j % kNB] = mfma16<DT>(a[P][j % kNB][ks], b[P][j / kNB][ks], acc[j / kNB][j % kNB]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = q * S::kLoads / kMfma; i < (q + 1) * S::kLoads / kMfma; ++i) fetch(i, s + kStages, st, exist_c, exist_r);
#pragma unroll
      for (int r = q * kReads / kMfma; r < (q + 1) * kReads / kMfma; ++r) read(r, P ^ 1, next);
      __builtin_amdgcn_sched_barrier(0);
    }
    st = next;
  };
  int s = first;
  for (; s + 1 < last; s += 2) {
    step(std::integral_constant<int, 0>{}, s);
    step(std::integral_constant<int, 1>{}, s + 1);
  }
  if (s < last) step(std::integral_constant<int, 0>{}, s);
  wait_fetches_and_reads<0>();

  if constexpr (SLICED) {
    const int64_t tile = (int64_t)share.slice * p.tiles_m * p.tiles_n + (int64_t)share.tm * p.tiles_n + share.tn;
    float4* to = reinterpret_cast<float4*>(p.partial) + tile * (S::kRows * S::kCols / 4) + t;
#pragma unroll
    for (int mb = 0; mb < kMB; ++mb)
#pragma unroll
      for (int nb = 0; nb < kNB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x16& v = acc[mb][nb];
          to[((mb * kNB + nb) * 4 + j) * S::kThreads] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
  } else {
    finish_tile<DT, KIND, S>(p, acc, m0, share.tn, wm, wn, li, lg);
  }
}

// The slices of a tile added up, in order, and its end.
template <int DT, int KIND, class S>
__global__ __launch_bounds__(S::kThreads) void k_gated_join(const Product p) {
  const int t = threadIdx.x, lane = t & (kWave - 1), uw = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n, stride = tiles * (S::kRows * S::kCols / 4);
  const int tm = (int)(blockIdx.x / p.tiles_n), tn = (int)(blockIdx.x % p.tiles_n);
  const float4* const from = reinterpret_cast<const float4*>(p.partial) + (int64_t)blockIdx.x * (S::kRows * S::kCols / 4) + t;
  f32x16 acc[S::kMB][S::kNB];
#pragma unroll
  for (int mb = 0; mb < S::kMB; ++mb)
#pragma unroll
    for (int nb = 0; nb < S::kNB; ++nb)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[mb][nb][r] = 0.0f;
  for (int slice = 0; slice < p.slices; ++slice) {
#pragma unroll
    for (int mb = 0; mb < S::kMB; ++mb)
#pragma unroll
      for (int nb = 0; nb < S::kNB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float4 v = from[slice * stride + ((mb * S::kNB + nb) * 4 + j) * S::kThreads];
          acc[mb][nb][4 * j] += v.x;
          acc[mb][nb][4 * j + 1] += v.y;
          acc[mb][nb][4 * j + 2] += v.z;
          acc[mb][nb][4 * j + 3] += v.w;
        }
  }
  finish_tile<DT, KIND, S>(p, acc, (int64_t)tm * S::kRows, tn, uw % S::kWavesM, uw / S::kWavesM, lane & 31, lane >> 5);
}

}  // namespace

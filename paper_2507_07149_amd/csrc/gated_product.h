// The matrix products of the gated feed-forward block (gated_product.hip): one kernel for all, in the tiles of `Tile`.
//
//   out[row, col] = sum over l of R[row, l] * C[col, l]        16-bit formats, binary32 accumulation (v_mfma_f32_32x32x16; the largest tiles 16x16x32,
//                                                              which takes less power and, with twice the instructions, 3 to 5 % longer in the others)
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
#include "gated_linear.h"
#include "linear_common.h"

namespace {

constexpr bool rows_across(int kind) { return kind == kWeight; }
constexpr bool cols_across(int kind) { return kind == kInput || kind == kWeight; }
constexpr bool is_gated(int kind) { return kind == kGated || kind == kGatedGrad; }
using Product = GatedProduct;

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

// 64 lanes x 16 bytes from memory straight into LDS: lane l reads the buffer at off, LDS byte lds + 16 l is written; zeros where off is behind the
// buffer's end.  (As load_to_lds: in assembly because the compiler would wait for it in front of the next LDS read; no register result.  The
// buffer's four registers must not come out of the vector unit in the five cycles before, which the compiler does not see to here: they are made
// by the scalar unit, once for all loads of a step.)
__device__ __forceinline__ void fetch_to_lds(uint32_t lds, uint32_t off, const u32x4& buffer) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(off), "s"(buffer) : "memory");
}

// One operand on its way into LDS, 64 values of l at a time, in LOADS loads of a wave.
template <bool ACROSS, int LOADS>
struct Feed {
  uint64_t at;                   // of the next 64 (their tile's corner)
  uint32_t off[LOADS];           // of the lane, in each load
  uint32_t bytes;                // along: of the tile's rows that exist
  uint32_t col;                  // across: bytes in front of the tile in a row
  int piece;                     // along: of the lane in its row

  // `rows`: that exist from the tile's first on, of the `most` that a tile has.
  __device__ __forceinline__ void begin(const char* corner, int64_t rows, int64_t most, int64_t pitch, int64_t col_bytes) {
    at = reinterpret_cast<uint64_t>(corner);
    bytes = (uint32_t)(rows <= 0 ? 0 : rows >= most ? (int64_t)kNowhere : rows * pitch);
    col = (uint32_t)col_bytes;
  }
  // What the loads of the next 64 see, and on to those behind them.  `there`: values of l that exist from the first one on.
  __device__ __forceinline__ u32x4 open(int there, uint32_t pitch, int64_t next) {
    uint32_t length;
    if constexpr (ACROSS) {                                              // the last row in which values exist ends the operand
      const int left = there * (int)pitch - (int)col;                    // (of fewer than 128 rows: below 2^31)
      length = there >= 128 ? kNowhere : (uint32_t)max(left, 0);
    } else {
      length = there > 0 ? bytes : 0u;
      if (there < 64) {                                                  // its last values: the rows go on with others (later on nothing is seen at all)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) off[i] = piece * 8 < there ? off[i] : kNowhere;
      }
    }
    const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32), length, 0x00020000u};     // untyped
    at += (uint64_t)next;
    return buffer;
  }
};

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

// Tile `pos` of a launch -> its row and column of tiles.
__host__ __device__ inline TileIndex tile_at(const Product& p, int pos) {
  const int subs = p.sub_m * p.sub_n, sub = pos % subs;
  TileIndex t = tile_of_position(p.first + pos / subs, p.tiles_m, p.tiles_n, 4);
  t.m = t.m * p.sub_m + sub % p.sub_m;
  t.n = t.n * p.sub_n + sub / p.sub_m;
  return t;
}
// Workgroup -> tile and slice: every die (blockIdx mod 8) takes a run of consecutive tiles, so that the workgroups that run together share operands
// in its cache; the slices of a tile are far apart.
struct Share {
  int pos, slice;
};
__host__ __device__ inline Share share_of_workgroup(int id, int tiles, int slices) {
  constexpr int kDies = 8;
  const int total = tiles * slices, each = total / kDies, more = total % kDies;
  const int die = id % kDies;
  const int at = die * each + (die < more ? die : more) + id / kDies;
  return {at % tiles, at / tiles};
}

// ---- the activation ----
// The end of a tile is all vector work of its own: 64 or 128 activations to a lane at four cycles an instruction, while the matrix cores wait.  So exponentials and
// reciprocals are the hardware's (1 ulp; far out a rounding of the exponent's argument is up to 3e-5 of the result, where binary16 keeps 4.9e-4), and gelu takes
// its error function from the same exponential that its slope needs.
__device__ __forceinline__ float sigmoid(float v) {                      // 1 / (1 + exp(-v))
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * v));
}
// f(a) and, where wanted, f'(a).
template <int ACT, bool SLOPE>
__device__ __forceinline__ float activate(float a, float& slope) {
  if constexpr (ACT == DAF_ACT_SILU) {
    const float p = sigmoid(a), f = a * p;
    if constexpr (SLOPE) slope = __builtin_fmaf(f, 1.0f - p, p);
    return f;
  } else if constexpr (ACT == DAF_ACT_GELU_TANH) {
    // 0.5 (1 + tanh(v / 2)) = 1 / (1 + exp(-v)) with v = 2 sqrt(2 / pi) (a + 0.044715 a^3)
    constexpr float kC = 1.5957691216057308f;
    const float p = sigmoid(kC * __builtin_fmaf(0.044715f * a * a, a, a)), f = a * p;
    if constexpr (SLOPE) {
      const float dv = kC * __builtin_fmaf(3.0f * 0.044715f * a, a, 1.0f), q = f * (1.0f - p);
      slope = q == 0.0f ? p : __builtin_fmaf(q, dv, p);                  // (far out the slope of p is 0 whatever dv has become)
    }
    return f;
  } else if constexpr (ACT == DAF_ACT_GELU) {
    // a (1 - q) or, below zero, a q, with q = erfc(x) / 2, x = |a| / sqrt(2): far below zero q is all that the result is made of, so q has to be right
    // relative to itself.  q = t P(t) exp(-x^2) with t = 1 / (1 + 0.6 x), as erfc(x) exp(x^2) / t is smooth in t from 0 to 1; P is of degree 5, with the least
    // largest relative error over x of 0 ... 9.5 weighed by 1 + 3 x^2 (a linear program over its coefficients): 5.2e-7 (1 + 3 x^2).  Computed as
    // here 4e-7 off q at a = 0, and of q 1.1e-5 at -4, 3e-5 at -6 and 5e-5 at -10; binary16 keeps 4.9e-4, bfloat16 3.9e-3.
    const float x = __builtin_fabsf(a) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.6f, x, 1.0f));
    const float e = __builtin_amdgcn_exp2f(-1.4426950408889634f * x * x);
    float q = __builtin_fmaf(t, 0.059877953f, -0.23713051f);
    q = __builtin_fmaf(t, q, 0.25233790f);
    q = __builtin_fmaf(t, q, 0.076049743f);
    q = __builtin_fmaf(t, q, 0.18036656f);
    q = __builtin_fmaf(t, q, 0.16849846f) * t * e;
    const float p = a >= 0.0f ? 1.0f - q : q;
    if constexpr (SLOPE) slope = __builtin_fmaf(a * 0.3989422804014327f, e, p);
    return a * p;
  } else {
    if constexpr (SLOPE) slope = a > 0.0f ? 1.0f : 0.0f;
    return a <= 0.0f ? 0.0f : a;                                         // (NaN stays)
  }
}
// f with the activation as a constant.
template <class F>
__device__ __forceinline__ void by_activation(int act, F&& f) {
  switch (act) {
    case DAF_ACT_SILU: return f(std::integral_constant<int, DAF_ACT_SILU>{});
    case DAF_ACT_GELU: return f(std::integral_constant<int, DAF_ACT_GELU>{});
    case DAF_ACT_GELU_TANH: return f(std::integral_constant<int, DAF_ACT_GELU_TANH>{});
    default: return f(std::integral_constant<int, DAF_ACT_RELU>{});
  }
}

// ---- the end of a tile ----
// A 32 x 32 block of sums: lane li + 32 lg has row li, register r column 8 (r / 4) + 4 lg + r % 4.  Two swaps of half-waves to a unit of eight columns
// make that 8 lg ... and 16 + 8 lg ... of the row: a store then writes 32 consecutive bytes of each row.
template <int DT>
__device__ __forceinline__ void store_block(char* out, int64_t at, const f32x16& v, int64_t count, int lg) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    Unit<DT> u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 8 * half + 2 * h;
      const u32x2 s = __builtin_amdgcn_permlane32_swap(narrow_pair<DT>(v[r], v[r + 1]), narrow_pair<DT>(v[r + 4], v[r + 5]), false, false);
      u.q[0][h] = s.x;
      u.q[0][2 + h] = s.y;
    }
    const int c = 16 * half + 8 * lg;
    store_unit_of<DT>(out + (at + c) * 2, u, (int)(count - c < 8 ? count - c : 8));
  }
}
// The same backwards; columns that do not exist are zero.
template <int DT>
__device__ __forceinline__ void load_block(const char* in, int64_t at, int64_t count, int lg, Unit<DT> (&u)[2]) {
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int c = 16 * half + 8 * lg;
    u[half] = load_unit_of<DT>(in + (at + c) * 2, (int)(count - c < 8 ? count - c : 8));
  }
}
template <int DT>
__device__ __forceinline__ f32x16 block_of(const Unit<DT> (&u)[2]) {
  f32x16 v;
#pragma unroll
  for (int half = 0; half < 2; ++half)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 8 * half + 2 * h;
      const u32x2 s = __builtin_amdgcn_permlane32_swap(u[half].q[0][h], u[half].q[0][2 + h], false, false);
      v[r] = widen16<DT>(s.x & 0xFFFFu);
      v[r + 1] = widen16<DT>(s.x >> 16);
      v[r + 4] = widen16<DT>(s.y & 0xFFFFu);
      v[r + 5] = widen16<DT>(s.y >> 16);
    }
  return v;
}

// A block of sums for the vector unit.
__device__ __forceinline__ f32x16 block_sums(const f32x16& acc) { return acc; }
// A block of 32 x 32 as four of 16 x 16: [half of the rows][half of the columns], lane l has row l mod 16 and columns 4 (l / 16) ...  Two swaps, of 16
// and of 32 lanes, to two registers make it a block as above.  Where a wave has 256 sums they stay in accumulation registers until their block's turn:
// left to itself the compiler moves all of them at the end of the loop, through memory where they do not fit.
typedef float f32x4 __attribute__((ext_vector_type(4)));
struct QuarterBlocks {
  f32x4 of[2][2];
};
template <int DT>
__device__ __forceinline__ f32x4 mfma_16x16x32(const u32x4& a, const u32x4& b, const f32x4& c) {
  if constexpr (DT == kBF16) {
    typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
}

__device__ __forceinline__ f32x16 block_sums(const QuarterBlocks& acc) {
  f32x16 v;
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t x[2];
#pragma unroll
      for (int m = 0; m < 2; ++m) asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x[m]) : "a"(acc.of[m][n][i]));
      const u32x2 s = __builtin_amdgcn_permlane16_swap(x[0], x[1], false, false);
      const u32x2 w = __builtin_amdgcn_permlane32_swap(s.x, s.y, false, false);
      v[8 * n + i] = u2f(w.x);
      v[8 * n + 4 + i] = u2f(w.y);
    }
  return v;
}

// One row of a wave's blocks: block row `mb`.
// (sums: block_sums, or nothing where the sums come out of memory)
template <int DT, int KIND, class S, class B, class Sums>
__device__ __forceinline__ void finish_row(const Product& p, const B (&acc)[S::kNB], TileIndex tile, int mb, int wm, int wn, int li, int lg, Sums sums) {
  int64_t m = (int64_t)tile.m * S::kRows + (wm * S::kMB + mb) * 32 + li;
  const bool there = m < p.rows;                                         // (sums are made by all lanes: they change places among them)
  if constexpr (is_gated(KIND)) {
    constexpr int kH = S::kNB / 2;                                       // blocks of h to a row of blocks
    const int64_t n0 = ((int64_t)tile.n * (S::kCols / 64) + wn * kH) * 32;
    Unit<DT> g[kH][2];
    if (KIND == kGatedGrad && there) {
#pragma unroll
      for (int b = 0; b < kH; ++b) load_block<DT>(p.grad_h, m * p.n + n0 + 32 * b, p.n - n0 - 32 * b, lg, g[b]);
    }
#pragma unroll
    for (int b = 0; b < kH; ++b) {
      const f32x16 a = sums(acc[b]), u = sums(acc[b + kH]);
      if (!there) continue;
      const int64_t n = n0 + 32 * b, at = m * p.n + n;
      f32x16 h, da, du;
      if constexpr (KIND == kGatedGrad) du = block_of<DT>(g[b]);         // grad_h
      int kind_of_act = p.act;
      asm volatile("" : "+s"(kind_of_act));                              // a choice for this block alone: not one copy of all blocks for each activation
      by_activation(kind_of_act, [&](auto act) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          float slope;
          const float f = activate<decltype(act)::value, KIND == kGatedGrad>(a[r], slope);
          h[r] = f * u[r];
          if constexpr (KIND == kGatedGrad) {
            da[r] = du[r] * u[r] * slope;
            du[r] = du[r] * f;
          }
        }
      });
      if (KIND == kGated || p.out[0] != nullptr) store_block<DT>(p.out[0], at, h, p.n - n, lg);
      if constexpr (KIND == kGatedGrad) {
        if (n + 32 > p.n) {                                              // columns of [da du] that h does not have: zero, not 0 * infinity
          const int columns = (int)(p.n - n) - 4 * lg;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const bool exists = 8 * (r / 4) + r % 4 < columns;
            da[r] = exists ? da[r] : 0.0f;
            du[r] = exists ? du[r] : 0.0f;
          }
        }
        // (to 16 bits, as the products behind take them: half of a gradient's error, 0.0024 of its norm in bfloat16 where binary32 would leave 0.0017)
        store_block<DT>(p.out[1], m * 2 * p.padded + n, da, p.padded - n, lg);
        store_block<DT>(p.out[1], m * 2 * p.padded + p.padded + n, du, p.padded - n, lg);
      } else if (p.out[1] != nullptr) {
        store_block<DT>(p.out[1], at, a, p.n - n, lg);
        store_block<DT>(p.out[2], at, u, p.n - n, lg);
      }
      __builtin_amdgcn_sched_barrier(0);                                 // one block after the other: registers for one
    }
  } else {
    char* out = p.out[0];
    if constexpr (KIND == kWeight) {                                     // rows of da^T, then of du^T
      if (m >= p.padded) {
        m -= p.padded;
        out = p.out[1];
      }
    }
#pragma unroll
    for (int nb = 0; nb < S::kNB; ++nb) {
      const int64_t n = (int64_t)tile.n * S::kCols + (wn * S::kNB + nb) * 32;
      const f32x16 v = sums(acc[nb]);
      if (there && (KIND != kWeight || m < p.n)) store_block<DT>(out, m * p.k + n, v, p.k - n, lg);
    }
  }
}

// The sums of a tile as the lanes have them, 16 bytes each, for the join.
template <class S, class B>
__device__ __forceinline__ void write_partial(float* partial, int64_t tile, const B (&acc)[S::kMB][S::kNB]) {
  float4* const to = reinterpret_cast<float4*>(partial) + tile * (S::kRows * S::kCols / 4) + threadIdx.x;
#pragma unroll
  for (int mb = 0; mb < S::kMB; ++mb)
#pragma unroll
    for (int nb = 0; nb < S::kNB; ++nb) {
      const f32x16 v = block_sums(acc[mb][nb]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        to[((mb * S::kNB + nb) * 4 + j) * S::kThreads] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
    }
}

// The first step of a slice.  (The division is the vector unit's: back into a scalar register.)
__device__ __forceinline__ int step_of_slice(const Product& p, int slice) {
  return __builtin_amdgcn_readfirstlane(p.slices == 1 ? slice * p.steps : (int)((int64_t)p.steps * slice / p.slices));
}
template <int DT, int KIND, class S, class B>
__device__ __forceinline__ void end_tile(const Product& p, Share share, TileIndex tile, const B (&acc)[S::kMB][S::kNB], int wm, int wn, int li, int lg) {
  // (the last matrix instructions' sums are there for reads that the compiler does not see as such)
  if constexpr (S::kMB * S::kNB >= 16) asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
  if (p.slices > 1) return write_partial<S>(p.partial, (int64_t)share.slice * p.tiles + share.pos, acc);
#pragma unroll
  for (int mb = 0; mb < S::kMB; ++mb) finish_row<DT, KIND, S>(p, acc[mb], tile, mb, wm, wn, li, lg, [](const B& v) { return block_sums(v); });
}

// ---- the product ----
// Workgroup `id` of those that share a product's tiles and slices.
template <int DT, int KIND, class S>
__device__ __forceinline__ void product_tile(const Product& p, int id, char* lds) {
  constexpr int kMB = S::kMB, kNB = S::kNB, kStages = S::kStages;
  constexpr bool kRAcross = rows_across(KIND), kCAcross = cols_across(KIND);
  static_assert(!kRAcross || S::kRows % 64 == 0, "64 outputs to a row of LDS");
  const int t = threadIdx.x, lane = t & (kWave - 1);
  const int uw = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = uw % S::kWavesM, wn = uw / S::kWavesM;
  const int li = lane & 31, lg = lane >> 5;

  const Share share = share_of_workgroup(id, p.tiles, p.slices);
  const TileIndex tile = tile_at(p, share.pos);
  const int64_t m0 = (int64_t)tile.m * S::kRows;
  const int first = step_of_slice(p, share.slice), last = step_of_slice(p, share.slice + 1);

  // ---- loads.  Load i of a wave brings 1 KB, at (4 i + wave) KB of the operand: eight rows of 128 bytes of LDS, row lane / 8 of them at a lane.
  constexpr int kSources = is_gated(KIND) ? 2 : 1;
  const int l_row = lane >> 3;
  const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds) + (uint32_t)uw * 1024u;
  const bool second = KIND == kInput && first >= p.half;                           // kInput: the slice begins in du Wu
  const int64_t line = (int64_t)(second ? first - p.half : first) * 64;            // the first value of l, in its half
  Feed<kCAcross, S::kLoadsC> c[kSources];
  Feed<kRAcross, S::kLoadsR> r;
  auto offsets = [&](auto& feed, uint32_t pitch, auto across, auto row_of_load) {
    feed.piece = (lane & 7) ^ ((lane >> 4) | ((uw & 1) << 2));                     // (row 8 L + lane / 8 with L odd where uw is)
#pragma unroll
    for (int i = 0; i < (int)(sizeof(feed.off) / 4); ++i) {
      if constexpr (decltype(across)::value)
        feed.off[i] = (uint32_t)((i & 1) * 32 + uw * 8 + l_row) * pitch + (uint32_t)(i / 2 * 128 + ((lane & 7) ^ (((lane >> 4) & 1) << 2)) * 16);
      else
        feed.off[i] = (uint32_t)(row_of_load(i) + uw * 8 + l_row) * pitch + (uint32_t)feed.piece * 16u;
    }
  };
  using CAcross = std::integral_constant<bool, kCAcross>;
  using RAcross = std::integral_constant<bool, kRAcross>;
  // A load is 32 rows of C with those of the other waves: of a wave's blocks the first half Wg's, the others Wu's, of the same columns of h.
  constexpr int kOuterC = is_gated(KIND) ? S::kCols / 2 : S::kCols;
  const int64_t n0 = (int64_t)tile.n * kOuterC;
#pragma unroll
  for (int w = 0; w < kSources; ++w) {
    const char* const base = second ? p.c[1] : p.c[w];
    c[w].begin(kCAcross ? base + line * p.c_pitch + n0 * 2 : base + n0 * p.c_pitch + line * 2, p.cols - n0, kOuterC, p.c_pitch, n0 * 2);
    offsets(c[w], (uint32_t)p.c_pitch, CAcross{}, [](int i) { return (i / kNB * (kNB / 2) + i % (kNB / 2)) * 32; });
  }
  r.begin(kRAcross ? p.r + line * p.r_pitch + m0 * 2 : p.r + m0 * p.r_pitch + (int64_t)first * 128, p.rows - m0, S::kRows, p.r_pitch, m0 * 2);
  offsets(r, (uint32_t)p.r_pitch, RAcross{}, [](int i) { return i * 32; });
  // Values of l that exist from step `s` on.
  auto exist = [&](bool of_c, int s) {
    if (s >= last) return 0;
    if (KIND == kInput) return of_c ? p.length - 64 * (s < p.half ? s : s - p.half) : 64;
    return p.length - 64 * s;
  };
  u32x4 c_buffer[kSources], r_buffer;
  auto open = [&](int s) {
    int64_t next = kCAcross ? 64 * p.c_pitch : 128;
    if (KIND == kInput && s + 1 == p.half) next = p.c[1] - p.c[0] - (int64_t)(p.half - 1) * next;
#pragma unroll
    for (int w = 0; w < kSources; ++w) c_buffer[w] = c[w].open(exist(true, s), (uint32_t)p.c_pitch, next);
    r_buffer = r.open(exist(false, s), (uint32_t)p.r_pitch, kRAcross ? 64 * p.r_pitch : 128);
  };
  auto fetch = [&](int i, int st) {
    const bool of_c = i < S::kLoadsC;
    const int load = of_c ? i : i - S::kLoadsC, w = kSources == 2 && of_c && load % kNB >= kNB / 2 ? 1 : 0;
    const uint32_t dst = lds0 + (uint32_t)(st * S::kStageBytes + (of_c ? 0 : S::kCols * 128) + load * 4096);
    if (of_c) fetch_to_lds(dst, c[w].off[load], c_buffer[w]);
    else fetch_to_lds(dst, r.off[load], r_buffer);
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
    open(first + st);
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) fetch(i, st);
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
    open(s + kStages);
#pragma unroll
    for (int q = 0; q < kMfma; ++q) {
      const int ks = q / (kNB * kMB), j = q % (kNB * kMB);
      acc[j / kNB][j % kNB] = mfma16<DT>(a[P][j % kNB][ks], b[P][j / kNB][ks], acc[j / kNB][j % kNB]);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = q * S::kLoads / kMfma; i < (q + 1) * S::kLoads / kMfma; ++i) fetch(i, st);
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

  end_tile<DT, KIND, S>(p, share, tile, acc, wm, wn, li, lg);
}

template <int DT, int KIND, class S>
__global__ __launch_bounds__(S::kThreads, 1) void k_gated_product(const Product p) {
  __shared__ __align__(1024) char lds[S::kStages * S::kStageBytes];
  product_tile<DT, KIND, S>(p, (int)blockIdx.x, lds);
}

// grad_x and the weights' gradients, neither of which needs the other, side by side: one fills what the other leaves idle.  The workgroups that
// take longer come first.
template <int DT, class S>
__global__ __launch_bounds__(S::kThreads, 1) void k_gated_gradients(const Product input, const Product weight, int weights_first) {
  __shared__ __align__(1024) char lds[S::kStages * S::kStageBytes];
  const int id = (int)blockIdx.x, inputs = input.tiles * input.slices, weights = weight.tiles * weight.slices;
  if (weights_first ? id >= weights : id < inputs) product_tile<DT, kInput, S>(input, weights_first ? id - weights : id, lds);
  else product_tile<DT, kWeight, S>(weight, weights_first ? id : id - inputs, lds);
}

// A wave's part of a join: one block of 32 x 32, or those of a and u.
template <int KIND, class S>
struct JoinPart {
  static constexpr int kRows = S::kRows, kCols = S::kCols, kMB = S::kMB, kNB = is_gated(KIND) ? 2 : 1;
  static constexpr int kParts = S::kNB / kNB, kBlocks = kMB * kParts;    // workgroups to a tile
};
// The slices of a tile added up, in order, and its end: a workgroup for each block of its waves, eight slices on their way at a time.  (As few bytes
// to a workgroup as this: with a row of blocks to each, and two slices, 13 slices of 9 tiles took 12.6 us, now 4.8.)
template <int DT, int KIND, class S>
__device__ __forceinline__ void join_part(const Product& p, int id) {
  using J = JoinPart<KIND, S>;
  constexpr int kAhead = J::kNB == 1 ? 8 : 4;
  const int pos = id / J::kBlocks, mb = id % J::kBlocks / J::kParts, part = id % J::kParts;
  const int t = threadIdx.x, lane = t & (kWave - 1), uw = __builtin_amdgcn_readfirstlane(t >> 6);
  const int64_t stride = (int64_t)p.tiles * (S::kRows * S::kCols / 4);
  const float4* const from = reinterpret_cast<const float4*>(p.partial) + (int64_t)pos * (S::kRows * S::kCols / 4) + (mb * S::kNB + part) * 4 * S::kThreads + t;
  f32x16 acc[J::kNB] = {};
  for (int slice = 0; slice < p.slices; slice += kAhead) {
    float4 v[kAhead][J::kNB][4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int nb = 0; nb < J::kNB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          v[i][nb][j] = slice + i < p.slices ? from[(slice + i) * stride + (nb * J::kParts * 4 + j) * S::kThreads] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int nb = 0; nb < J::kNB; ++nb)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[nb][4 * j] += v[i][nb][j].x;
          acc[nb][4 * j + 1] += v[i][nb][j].y;
          acc[nb][4 * j + 2] += v[i][nb][j].z;
          acc[nb][4 * j + 3] += v[i][nb][j].w;
        }
  }
  finish_row<DT, KIND, J>(p, acc, tile_at(p, pos), mb, uw % S::kWavesM, uw / S::kWavesM * J::kParts + part, lane & 31, lane >> 5,
                          [](const f32x16& v) { return v; });
}
template <int DT, int KIND, class S>
__global__ __launch_bounds__(S::kThreads) void k_gated_join(const Product p) {
  join_part<DT, KIND, S>(p, (int)blockIdx.x);
}
template <int DT, class S>
__global__ __launch_bounds__(S::kThreads) void k_gated_join_gradients(const Product input, const Product weight) {
  const int inputs = input.tiles * JoinPart<kInput, S>::kBlocks;
  if ((int)blockIdx.x < inputs) join_part<DT, kInput, S>(input, (int)blockIdx.x);
  else join_part<DT, kWeight, S>(weight, (int)blockIdx.x - inputs);
}

}  // namespace

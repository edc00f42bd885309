// Tiles of attention with a window on the matrix cores: keys and values (or queries and gradients) in LDS, and the operands that come out of them.
//
// A tile is 32 or 64 rows of a head (128 in one case).  It lies in blocks of 32 elements, one after the other: 64 bytes of every row, row after row; the 16-byte
// piece p of a block's row r at place p ^ (r / 4 mod 4).  There are two ways to read it: along, where rows of the tile are rows of the product's left
// operand, eight elements of a row to a lane; and across, where its columns are, transposed by the reads (ds_read_b64_tr_b16).  Sixteen rows' pieces p lie in all
// 16 places of 256 bytes, and so do the 64 bytes of four rows that a quarter of a wave reads across, so neither way meets bank conflicts; and every
// operand of a tile lies at a constant distance from one of two places of a lane.
// Rows behind a sequence's end and elements behind head_dim arrive as zeros and are never read: their lane's offset lies behind the end of the
// buffer that the load is given.
//
// The products are v_mfma_f32_32x32x16.  A lane's column is lane mod 32; lg = lane / 32.  Its 16 results are rows 8 (r / 4) + 4 lg + r mod 4, and since
// a product does not care for the order of what it sums over, registers 8 c ... 8 c + 7 of a result, rounded, are the right operand of the next product
// over rows 16 c + {4 lg ... 4 lg + 3, 8 + 4 lg ... 8 + 4 lg + 3} as they are, if the left operand is read in that order: no exchange between lanes.
#pragma once
#include "linear_common.h"
#include "window_attention_device.h"

namespace {

constexpr int kTileRows = 64;                                            // of keys in LDS

template <int DP>
struct TileShape {                                                       // DP: head_dim, padded
  static constexpr int kSteps = DP / 16, kBlocks = DP / 32;
  static_assert(DP == 32 || DP == 64 || DP == 96 || DP == 128, "padded head_dim");
};
template <int DP>
constexpr int tile_bytes(int rows) { return rows * DP * 2; }

// 64 lanes x 16 bytes from a buffer straight into LDS, zeros where the offset is behind its end.  In assembly because the compiler would wait for it in
// front of the next LDS read; no register result.  (Five wait states: the buffer's registers may just have come out of the vector unit.)
__device__ __forceinline__ void fetch_piece(uint32_t lds, uint32_t off, const u32x4& buffer) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(lds), "v"(off), "s"(buffer) : "memory");
}
// The same, four bytes to a lane.
__device__ __forceinline__ void fetch_float(uint32_t lds, uint32_t off, const u32x4& buffer) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(lds), "v"(off), "s"(buffer) : "memory");
}
constexpr uint32_t kNowhere = 0x80000000u;           // an offset behind the end of every buffer

// A tile's way into LDS, shared by WAVES waves: 16 rows' 64 bytes of a block to a load.
template <int DP, int ROWS, int WAVES>
struct TileFeed {
  static constexpr int kParts = ROWS / 16, kAll = kParts * (DP / 32), kLoads = (kAll + WAVES - 1) / WAVES;     // loads of a tile; of a wave
  uint32_t off[kLoads];
  uint64_t first;                                                        // of the sequence's rows, this head
  uint32_t pitch, row_bytes;
  __device__ __forceinline__ void begin(const Heads& h, int64_t row, int head, int dim) {
    const int wave = WAVES == 1 ? 0 : threadIdx.x / kWave, lane = threadIdx.x % kWave;
    first = reinterpret_cast<uint64_t>(h.at) + (uint64_t)(row * h.token) + (uint64_t)(head * h.head);
    pitch = (uint32_t)h.token;
    row_bytes = (uint32_t)dim * 2;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int n = i * WAVES + wave, r = n % kParts * 16 + lane / 4;
      const uint32_t at = (uint32_t)(n / kParts) * 64 + (uint32_t)((lane & 3) ^ ((lane >> 4) & 3)) * 16;
      off[i] = at < row_bytes ? (uint32_t)r * pitch + at : kNowhere;
    }
  }
  // Rows `row` ... row + ROWS - 1 of the `rows` that there are, to LDS byte `lds`.
  __device__ __forceinline__ void fetch(uint32_t lds, int row, int rows) const {
    fetch_at(lds, first + (uint64_t)row * pitch, length_of(rows - row));
  }
  // The same for a wave that is alone with its tiles, in a workgroup of several (WAVES is 1).
  __device__ __forceinline__ void fetch_of_wave(uint32_t lds, int row, int rows) const {
    const uint64_t at = first + (uint64_t)row * pitch;
    const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32), length_of(rows - row), 0x00020000u};
#pragma unroll
    for (int i = 0; i < kLoads; ++i) fetch_piece(lds + (uint32_t)i * 1024, off[i], buffer);
  }
  __device__ __forceinline__ uint32_t length_of(int rows) const { return rows > 0 ? (uint32_t)(min(rows, ROWS) - 1) * pitch + row_bytes : 0u; }
  __device__ __forceinline__ void fetch_at(uint32_t lds, uint64_t at, uint32_t length) const {
    const int wave = uniform(threadIdx.x / kWave);
    const u32x4 buffer = {(uint32_t)at, (uint32_t)(at >> 32), length, 0x00020000u};      // untyped
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      if (kAll % WAVES == 0 || i * WAVES + wave < kAll) fetch_piece(lds + (uint32_t)(i * WAVES + wave) * 1024, off[i], buffer);
  }
};

// Tiles one after the other, with a jump in front of one of them and another length of the last: three additions to a tile, no multiplication.
template <int DP, int ROWS, int WAVES>
struct TileWalk : TileFeed<DP, ROWS, WAVES> {
  uint64_t at, step, jump;
  uint32_t whole, last;
  // from row `from` of `rows`; `over` rows are left out in front of the tile that says so; the last one begins at row `end`
  __device__ __forceinline__ void walk(int from, int over, int end, int rows) {
    at = this->first + (uint64_t)from * this->pitch;
    step = (uint64_t)ROWS * this->pitch;
    jump = (uint64_t)over * this->pitch;
    whole = this->length_of(ROWS);
    last = this->length_of(rows - end);
  }
  __device__ __forceinline__ void next(uint32_t lds, bool jumps, bool is_last) {
    at += jumps ? jump : 0;
    this->fetch_at(lds, at, is_last ? last : whole);
    at += step;
  }
};

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) char lds_char;
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Left operands out of a tile: along, rows 32 b ... 32 b + 31, elements 16 s + 8 lg ... + 7 of each.
template <int ROWS>
struct ReadAlong {
  const lds_char* at[2];                                                 // even and odd s
  __device__ __forceinline__ explicit ReadAlong(const lds_char* lds) {
    const int li = threadIdx.x & 31, lg = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int s = 0; s < 2; ++s) at[s] = lds + li * 64 + (((2 * s + lg) ^ ((li >> 2) & 3)) << 4);
  }
  __device__ __forceinline__ u32x4 read(int tile_at, int b, int s) const {
    return *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(at[s & 1] + (tile_at + (s >> 1) * (ROWS * 64) + b * 2048));
  }
};
// Across: columns 32 b ... 32 b + 31 of rows 16 c + {4 lg ... + 3, 8 + 4 lg ... + 3}.
template <int ROWS>
struct ReadAcross {
  const lds_char* at[2];                                                 // the first four rows, and the other four
  __device__ __forceinline__ explicit ReadAcross(const lds_char* lds) {
    const int lane = threadIdx.x % kWave, piece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = 8 * h + 4 * (lane >> 5) + ((lane & 15) >> 2);
      at[h] = lds + row * 64 + ((piece ^ ((row >> 2) & 3)) << 4) + (lane & 1) * 8;
    }
  }
  __device__ __forceinline__ u32x4 read(int tile_at, int b, int c) const {
    const int to = tile_at + b * (ROWS * 64) + c * 1024;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at[0] + to)));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(at[1] + to)));
    return u32x4{lo.x, lo.y, hi.x, hi.y};
  }
};

// The row of a result's register r in its block of 32 rows, less 4 lg.
__device__ __forceinline__ constexpr int row_of_register(int r) { return 8 * (r >> 2) + (r & 3); }
__device__ __forceinline__ int first_row() { return 4 * ((threadIdx.x >> 5) & 1); }

// Which rows of a result are seen, by their register's row alone, so that a tile has three numbers to a lane.
struct RowsSeen {
  int first, last, more;                                                 // rows first ... last, and those below `more`
  __device__ __forceinline__ bool at(int row) const { return row <= last && (row >= first || row < more); }
};
// Rows are keys from `key` on, for a query at `position`.
__device__ __forceinline__ RowsSeen keys_seen(const Attention& a, int position, int key) {
  const int begin = key + first_row();
  return {position - a.window + 1 - begin, position - begin, a.sinks - begin};
}

// A lane's column, worked out anew behind a loop that has no register for it.
__device__ __forceinline__ int column_again() {
  int lane = threadIdx.x;
  asm volatile("" : "+v"(lane));
  return lane & 31;
}
// Right operands straight from memory: column `row`, elements 16 s + 8 lg ... + 7; `flip`: with the other sign.
template <int DP>
__device__ __forceinline__ void load_columns(const char* row, int dim, bool flip, u32x4 (&q)[TileShape<DP>::kSteps]) {
  const int lg = (threadIdx.x >> 5) & 1;
  const uint32_t sign = flip ? 0x80008000u : 0u;
#pragma unroll
  for (int s = 0; s < TileShape<DP>::kSteps; ++s) {
    const int d = 16 * s + 8 * lg;
    u32x4 v = {0u, 0u, 0u, 0u};
    if (d < dim) v = *reinterpret_cast<const u32x4*>(row + d * 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) q[s][i] = v[i] ^ sign;
  }
}
// A block of 32 columns' results, times `by`, rounded, to rows of memory: lane li's column is row `row`, and its registers go by eights to
// elements 8 (2 g + lg) of the block.
template <int DT>
__device__ __forceinline__ void store_column_block(char* row, int block, int dim, bool write, const f32x16& o, float by) {
  int lane = threadIdx.x;
  asm volatile("" : "+v"(lane));                                         // (as column_again)
  const int lg = (lane >> 5) & 1;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    u32x2 half[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const int e = 8 * g + 2 * w;
      half[w] = __builtin_amdgcn_permlane32_swap(narrow_pair<DT>(o[e] * by, o[e + 1] * by), narrow_pair<DT>(o[e + 4] * by, o[e + 5] * by), false, false);
    }
    const int d = block * 32 + 8 * (2 * g + lg);
    const u32x4 v = {half[0].x, half[1].x, half[0].y, half[1].y};
    if (write && d < dim) *reinterpret_cast<u32x4*>(row + d * 2) = v;
  }
}
__device__ __forceinline__ float from_other_half(float v) { return u2f(other_half(f2u(v))); }

__device__ __forceinline__ void wait_tile() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
template <int N>
__device__ __forceinline__ void wait_but() {                             // all but the last N loads
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void tile_barrier() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

enum Seen { kNothing, kAll, kPart };

// Keys that the queries at positions `first` ... `last` see, as tiles of ROWS: the sinks' tiles in front of the window's, then those.
template <int ROWS>
struct KeyTiles {
  int sinks, low, count;
  __device__ __forceinline__ KeyTiles(const Attention& a, int first, int last) {
    low = window_begin(a, max(first, 0)) / ROWS;
    sinks = min((int)(((int64_t)a.sinks + ROWS - 1) / ROWS), low);
    count = last < 0 ? 0 : sinks + last / ROWS - low + 1;
  }
  __device__ __forceinline__ int key(int t) const { return (t < sinks ? t : low + t - sinks) * ROWS; }           // the first of tile t
  __device__ __forceinline__ int first_key() const { return sinks > 0 ? 0 : low * ROWS; }
  template <class Walk>
  __device__ __forceinline__ void walk(Walk& w, int keys) const { w.walk(first_key(), (low - sinks) * ROWS, key(count - 1), keys); }
};
// What queries at positions first ... last see of ROWS keys from `key` on, tile by tile: nothing, all, or a part (also where that takes longer to tell).
template <int ROWS>
struct KeyView {
  int begin, end, all_begin, all_end, sinks_all;
  __device__ __forceinline__ KeyView(const Attention& a, const KeyTiles<ROWS>& tiles, int first, int last) {
    sinks_all = a.sinks - ROWS;
    begin = a.sinks > tiles.low * ROWS ? 0 : first - a.window - ROWS + 2;      // (sinks go on into the window's tiles: any of them may be seen)
    end = last;
    all_begin = last - a.window + 1;
    all_end = first - ROWS + 1;
  }
  __device__ __forceinline__ Seen of(int t, int sinks, int key) const {
    if (t < sinks) return end < 0 ? kNothing : key <= sinks_all ? kAll : kPart;
    if (key < begin || key > end) return kNothing;
    return key >= all_begin && key <= all_end ? kAll : kPart;
  }
};
// What queries `query` ... query + 31 see of keys first ... last.
__device__ __forceinline__ Seen keys_seen_by(const Attention& a, int query, int first, int last) {
  const int end = query + 31;
  if (end < first || (query - a.window >= last && first >= a.sinks)) return kNothing;
  return query >= last && (end - a.window < first || last < a.sinks) ? kAll : kPart;
}

// Columns (bit li) in which a sum is infinite or NaN.  0 * x of what a column does not see is not 0 where x is infinite or NaN, so that such a column
// has to be done once more by itself, row by row.
template <int BLOCKS>
__device__ __forceinline__ uint32_t columns_to_do_again(const f32x16 (&o)[BLOCKS], bool mine) {
  float check = 0.0f;                                                    // NaN then
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) check = __builtin_fmaf(o[b][r], 0.0f, check);
  const uint64_t bad = __ballot(mine && !(check == 0.0f));
  return (uint32_t)bad | (uint32_t)(bad >> 32);
}

// Columns whose exponents of base 2 (the largest score's, or lse) are so far from 0 that what they are rounded by counts as a factor 2 of every exponential, and, farther
// still, leaves nothing of them or more than any format holds; kLowest too, which is less than all scores are.  They are done again, by scores' distances.
constexpr float kFarExponent = 0x1p24f;
__device__ __forceinline__ bool is_far(float exponent) { return !(fabsf(exponent) < kFarExponent); }
__device__ __forceinline__ uint32_t far_columns(float exponent, bool mine) {
  const uint64_t bad = __ballot(mine && is_far(exponent));
  return (uint32_t)bad | (uint32_t)(bad >> 32);
}

// Which queries from `query` on see a key, by their register's row.
struct QueriesSeen {
  int first, end;
  __device__ __forceinline__ bool at(int row) const { return row >= first && row < end; }
};
__device__ __forceinline__ QueriesSeen queries_seeing(const Attention& a, int key, int query) {
  const int begin = query + first_row();
  return {key - begin, key < a.sinks ? kTileRows : key + a.window - begin};
}

// Sums of four waves' blocks through LDS, OWN bytes of it to a wave, which it needs no more: block b of all goes to wave b, as its o[0].
template <int BLOCKS, int OWN>
__device__ __forceinline__ void add_up(char* lds, f32x16 (&o)[BLOCKS]) {
  static_assert(OWN >= BLOCKS * 4096, "a block is 4 KB");
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  const int lane = threadIdx.x % kWave, wave = uniform(threadIdx.x / kWave);
  lds_f32x4* const own = (lds_f32x4*)((lds_char*)lds + wave * OWN);
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int g = 0; g < 4; ++g) own[(b * 4 + g) * kWave + lane] = f32x4{o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]};
  __syncthreads();
  if (wave >= BLOCKS) return;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < 4; ++w) sum += ((const lds_f32x4*)((lds_char*)lds + w * OWN))[(wave * 4 + g) * kWave + lane];
#pragma unroll
    for (int r = 0; r < 4; ++r) o[0][4 * g + r] = sum[r];
  }
}
// Tiles of 32 queries, where they are so few that a workgroup's waves had better share the keys of 32 queries than have 32 queries each; else 0.  `tiles`: of
// 128 queries.  The waves' own tiles leave room for one workgroup to a compute unit with heads of 128, for two with heads of 64.  Measured, shared keys and own
// queries, one sequence, forward: 8 heads of 128, 256 rows 8.6 and 10.9 us, 1024 15.7 and 27.1, 2048 33.3 and 48.4, 4096 (not taken) 95 and 92; 12 heads of 64, 1024
// rows 13.3 and 20.0, 3300 51 and 58, 5000 (not taken) 106 and 98.  The backward pass: 1024 rows 54 and 67, 2048 102 and 117, 4096 (not taken) 242 and 231.
inline int64_t few_tiles(const daf_window_attention_t& p, int64_t tiles) {
  if (tiles * p.q_heads > (p.head_dim > 64 ? 160 : 320)) return 0;
  return p.q_rows / 32 + p.sequences;
}

// The maximum, by the one instruction that takes three of a product's results without making them canonical first; NaN if one is.
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The exponent's factor: base 2, and above 0 (a score of -infinity stays one).
__device__ __forceinline__ float exponent_factor(float scale) { return fmaxf(fabsf(scale) * kLog2E, 1e-45f); }
constexpr float kLowest = -3.0e38f;

}  // namespace

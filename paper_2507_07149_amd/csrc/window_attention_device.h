// What the kernels of attention with a window share: sequences and what a query sees, which tile a workgroup takes, and attention row by row.
#pragma once
#include "block_common.h"
#include "window_attention.h"

namespace {

struct Heads {
  char* at;
  int64_t token, head;         // bytes
};
struct Attention {
  Heads q, k, v, out;
  float* lse;
  const int32_t *q_starts, *k_starts, *k_lengths;
  int q_rows, k_rows, sequences;
  int window, sinks;           // window: kAttentionMostRows where there is none
  int q_heads, kv_heads, group, dim;
  float scale;
};
// (A stride by which nothing goes may be anything: then one that leads a tile's other rows out of its buffer.)
inline Heads heads_of(const daf_heads_t& h, int64_t rows) { return {static_cast<char*>(h.at), rows > 1 ? h.token_stride * 2 : 1 << 24, h.head_stride * 2}; }
inline Attention attention_of(const daf_window_attention_t& p, const AttentionTensors& t) {
  constexpr int64_t kMost = kAttentionMostRows;
  Attention a = {};
  a.q = heads_of(t.q, p.q_rows);
  a.k = heads_of(t.k, p.k_rows);
  a.v = heads_of(t.v, p.k_rows);
  a.out = heads_of(t.out, p.q_rows);
  a.lse = t.lse;
  a.q_starts = p.q_starts;
  a.k_starts = p.k_starts;
  a.k_lengths = p.k_lengths;
  a.q_rows = (int)p.q_rows;
  a.k_rows = (int)p.k_rows;
  a.sequences = (int)p.sequences;
  a.window = (int)(p.window == 0 || p.window > kMost ? kMost : p.window);
  a.sinks = (int)(p.sinks > kMost ? kMost : p.sinks);
  a.q_heads = p.q_heads;
  a.kv_heads = p.kv_heads;
  a.group = p.q_heads / p.kv_heads;
  a.dim = p.head_dim;
  a.scale = p.scale;
  return a;
}

// `call` with the format and head_dim padded to a multiple of 32 as constants.
template <class Call>
void with_padded_dim(const daf_window_attention_t& p, Call call) {
  auto padded = [&](auto dt) {
    if (p.head_dim <= 32) call(dt, std::integral_constant<int, 32>{});
    else if (p.head_dim <= 64) call(dt, std::integral_constant<int, 64>{});
    else if (p.head_dim <= 96) call(dt, std::integral_constant<int, 96>{});
    else call(dt, std::integral_constant<int, 128>{});
  };
  if (p.dtype == DAF_F16) padded(std::integral_constant<int, kF16>{});
  else padded(std::integral_constant<int, kBF16>{});
}

struct Sequence {
  int q_begin, queries, k_begin, keys;
  __device__ __forceinline__ int position(int i) const { return keys - queries + i; }    // of query i
};
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int within(int v, int lo, int hi) { return max(lo, min(v, hi)); }

// Queries of sequence b: where they begin and how many they are.
__device__ __forceinline__ void queries_of(const Attention& a, int b, int& begin, int& count) {
  if (a.q_starts == nullptr) {
    begin = 0;
    count = a.q_rows;
    return;
  }
  begin = within(a.q_starts[b], 0, a.q_rows);
  count = max(within(a.q_starts[b + 1], 0, a.q_rows) - begin, 0);
}
__device__ __forceinline__ Sequence sequence_of(const Attention& a, int b) {
  Sequence s;
  queries_of(a, b, s.q_begin, s.queries);
  s.k_begin = s.q_begin;
  s.keys = s.queries;
  if (a.k_starts != nullptr) {
    s.k_begin = within(a.k_starts[b], 0, a.k_rows);
    s.keys = within(a.k_lengths[b], 0, a.k_rows - s.k_begin);
  }
  s.q_begin = uniform(s.q_begin);
  s.queries = uniform(s.queries);
  s.k_begin = uniform(s.k_begin);
  s.keys = uniform(s.keys);
  return s;
}

// The first key of the window of a query at `position`, and whether key j is seen from there.
__device__ __forceinline__ int window_begin(const Attention& a, int position) { return max(0, position - a.window + 1); }   // (window at least 1)
__device__ __forceinline__ bool sees(const Attention& a, int position, int j) { return j <= position && (j > position - a.window || j < a.sinks); }

// Tile `pos` of all sequences' tiles of TILE queries (or keys), those with the most to do first: its sequence (-1: there is none) and tile.  What a tile
// has to do grows with its distance from its sequence's begin (queries; keys: from its end, LAST) until a window fits in.  So first come, sequence by
// sequence, the tiles that are `levels` or more away, then those of every sequence that are levels - 1 away, and so on.  Sequences are counted
// 64 at a time, a lane to each, so there is no list of tiles to be made in front of the launch; with thousands of them that takes most of the time (16 rows to each, 12 heads
// of 64: 1024 sequences 112 us, 4096 867, of which the search 540).
struct TileOf {
  int sequence, tile;
};
template <int TILE, bool LAST>
__device__ __forceinline__ TileOf find_tile(const Attention& a, int pos) {
  constexpr int kMostLevels = 32;
  const int lane = threadIdx.x % kWave, levels = min((a.window - 1) / TILE + 1, kMostLevels);
  for (int first = 0; first < a.sequences; first += kWave) {
    int begin = 0, length = 0;
    if (first + lane < a.sequences) queries_of(a, first + lane, begin, length);
    const int count = (int)(((int64_t)length + TILE - 1) / TILE), far = max(count - levels, 0);
    const int all = __builtin_amdgcn_readlane((int)wave_inclusive_sum((uint32_t)count), kWave - 1);
    if (pos >= all) {
      pos -= all;
      continue;
    }
    const int sum = (int)wave_inclusive_sum((uint32_t)far);              // of this lane and those before it
    auto tile = [&](int at, int level) {
      const int tiles = __builtin_amdgcn_readlane(count, at);
      return TileOf{first + at, LAST ? tiles - 1 - level : level};
    };
    const uint64_t behind = __ballot(sum > pos);
    if (behind != 0) {
      const int at = __builtin_ctzll(behind), before = __builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(far, at);
      return tile(at, __builtin_amdgcn_readlane(count, at) - 1 - (pos - before));
    }
    pos -= __builtin_amdgcn_readlane(sum, kWave - 1);
    for (int level = min(levels, all) - 1; level >= 0; --level) {
      const uint64_t there = __ballot(count > level);
      const int n = __builtin_popcountll(there);
      if (pos < n) {
        const bool me = ((there >> lane) & 1) != 0 && __builtin_popcountll(there & ((1ull << lane) - 1)) == pos;
        return tile(__builtin_ctzll(__ballot(me)), level);
      }
      pos -= n;
    }
  }
  return {-1, 0};
}
inline int64_t most_tiles(const daf_window_attention_t& p, int tile) {
  return p.q_starts == nullptr ? (p.q_rows + tile - 1) / tile : p.q_rows / tile + p.sequences;
}

// Workgroup -> head and tile.  A die (blockIdx mod 8) takes all the heads that share a key head, one after the other for every tile, so that the workgroups that run
// together read the same keys out of its cache; key heads go to dies evenly, and where dies share some, each takes every 2nd, 4th or 8th of their tiles, which come with the most to do
// first.  (Measured, against all tiles of a head one after the other, 32 on 8 heads of 128: 16x2048 rows, a window of 1024, 6 % less time; 1x32768, a window of 4096, 8 %.)
struct Turn {
  int head, tile;              // a tile that there is not: no turn
};
constexpr unsigned kDies = 8;
__host__ __device__ inline unsigned dies_of_head(unsigned kv_heads) { return kDies / min(kDies, kv_heads & (0u - kv_heads)); }     // that share one (or some)
inline unsigned workgroups_of(int64_t tiles, int kv_heads, int group) {
  const unsigned share = dies_of_head((unsigned)kv_heads), units = (unsigned)(tiles * kv_heads) / (kDies / share);       // of the dies that share them
  return (units + share - 1) / share * kDies * (unsigned)group;
}
__device__ __forceinline__ Turn turn_of_workgroup(int tiles, int kv_heads, int group) {
  const unsigned share = dies_of_head((unsigned)kv_heads), heads = (unsigned)kv_heads * share / kDies, die = blockIdx.x % kDies, n = blockIdx.x / kDies;
  const unsigned unit = n / (unsigned)group * share + die % share, head = unit / (unsigned)tiles;
  if (head >= heads) return {0, 0x7FFFFFFF};
  return {(int)((die / share * heads + head) * (unsigned)group + n % (unsigned)group), (int)(unit % (unsigned)tiles)};
}

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) v = fmaxf(v, __shfl_xor(v, d, kWave));
  return v;
}
template <int DT>
__device__ __forceinline__ float widen_one(uint32_t bits16) {
  if constexpr (DT == kBF16) return u2f(bits16 << 16);
  else return widen16<kF16>(bits16);
}
// The product of two rows of a head, times `scale`: of the factors one by one where it is below 1, so that a score is finite whose product alone is not.
template <int DT>
__device__ __forceinline__ float row_dot(const char* a, const char* b, int dim, float scale = 1.0f) {
  const bool first = fabsf(scale) < 1.0f;
  const float by = first ? scale : 1.0f;
  float sum = 0.0f;
  for (int d = 0; d < dim; d += 8) {
    float x[8], y[8];
    widen_unit<DT>(load_unit<DT>(a + d * 2), x);
    widen_unit<DT>(load_unit<DT>(b + d * 2), y);
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(x[i] * by, y[i], sum);
  }
  return first ? sum : sum * scale;
}
// Elements 2 lane and 2 lane + 1 of a row.
struct Two {
  float lo, hi;
};
template <int DT>
__device__ __forceinline__ Two load_two(const char* row, int dim) {
  const int lane = threadIdx.x % kWave;
  const uint32_t u = 2 * lane < dim ? reinterpret_cast<const uint32_t*>(row)[lane] : 0u;
  return {widen_one<DT>(u & 0xFFFFu), widen_one<DT>(u >> 16)};
}
template <int DT>
__device__ __forceinline__ void store_two(char* row, int dim, float lo, float hi) {
  const int lane = threadIdx.x % kWave;
  if (2 * lane < dim) reinterpret_cast<uint32_t*>(row)[lane] = narrow_pair<DT>(lo, hi);
}

// Whether nothing but NaN can come of a row any more (where a step's numbers have overflowed that is so for every row, after its first keys).
__device__ __forceinline__ bool all_nan(float lo, float hi, int dim) { return __all((lo != lo && hi != hi) || 2 * (int)(threadIdx.x % kWave) >= dim); }

// One query by a wave, 64 seen keys at a time: a key to a lane for the scores, two elements of the row to a lane for the sum.  Nothing that is not seen
// is read.  (What the tiles are checked against, and the way of rows whose tiles meet infinities or NaN: there 0 * v of an unseen key is not 0.)
template <int DT>
__device__ __forceinline__ void attend_row(const Attention& a, const Sequence& s, int i, int head) {
  const int lane = threadIdx.x % kWave, position = s.position(i), low = window_begin(a, position);
  const int64_t row = (int64_t)s.q_begin + i;
  const char* const q = a.q.at + row * a.q.token + head * a.q.head;
  const char* const k = a.k.at + s.k_begin * a.k.token + head / a.group * a.k.head;
  const char* const v = a.v.at + s.k_begin * a.v.token + head / a.group * a.v.head;
  const int sinks = position < 0 ? 0 : min(a.sinks, low), seen = position < 0 ? 0 : sinks + position - low + 1;
  float top = -INFINITY, total = 0.0f, lo = 0.0f, hi = 0.0f;
  for (int first = 0; first < seen; first += kWave) {
    const int n = first + lane, j = n < sinks ? n : low + n - sinks, count = min(seen - first, kWave);
    const float score = lane < count ? row_dot<DT>(q, k + j * a.k.token, a.dim, a.scale) : -INFINITY;
    const float new_top = fmaxf(top, wave_max(score)), base = new_top == -INFINITY ? 0.0f : new_top;
    const float shrink = top == -INFINITY ? (total == total ? 0.0f : total) : __builtin_amdgcn_exp2f((top - base) * kLog2E);
    const float p = lane < count ? __builtin_amdgcn_exp2f((score - base) * kLog2E) : 0.0f;
    top = new_top;
    total = total * shrink + wave_sum(p);
    lo *= shrink;
    hi *= shrink;
    for (int t = 0; t < count; ++t) {
      const float weight = u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(p), t));
      const Two x = load_two<DT>(v + __builtin_amdgcn_readlane(j, t) * a.v.token, a.dim);
      lo = __builtin_fmaf(weight, x.lo, lo);
      hi = __builtin_fmaf(weight, x.hi, hi);
    }
    if (total != total && all_nan(lo, hi, a.dim)) break;
  }
  const float by = seen > 0 ? 1.0f / total : 0.0f;
  store_two<DT>(a.out.at + row * a.out.token + head * a.out.head, a.dim, seen > 0 ? lo * by : 0.0f, seen > 0 ? hi * by : 0.0f);
  if (a.lse != nullptr && lane == 0) a.lse[(int64_t)head * a.q_rows + row] = seen > 0 ? top + __builtin_amdgcn_logf(total) * kLn2 : -INFINITY;
}

}  // namespace

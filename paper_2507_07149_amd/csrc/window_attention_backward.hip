// Attention with a window and sinks, backward (daf_window_attention_backward).
//
//   P = 2^(c s + n), dP = grad_out . v, dS = P (dP - delta);  grad_q = f dS k, grad_k = f dS^T q, grad_v = P^T grad_out / 2^8
//   c = scale log2(e), n = 8 - lse log2(e), delta = sum(grad_out * out), f = scale / 2^8
//
// Two kernels, each of which computes P and dS for itself: seven products instead of five, but no sum is shared between workgroups, and none goes through memory, but where
// far queries or pieces are split off (below): those leave sums in the workspace, which are added up in a fixed order.  k_attention_grad_q goes as the forward pass does, 32 queries to a wave as
// columns, over the keys; it also writes n and -delta of every query, for k_attention_grad_kv, where a wave has 32 keys as columns and goes over the
// queries that see them, head by head of those that share the keys.  The factor 2^8 keeps P and dS of long rows out of binary16's subnormal
// numbers; what leaves its range comes out as infinity, and such rows are done again in binary32, a wave to a row: 30 to 70 times as long as a pass without, where most are
// (binary16, 2x2048 rows, 8 on 2 heads of 128, a window of 1024: 137 us, with gradients 64 times as large 4.1 ms, 1024 times 9.9 ms).
//
// Sinks are seen by all queries behind them, the other keys by a window of them.  So the queries that see nothing but sinks of a sequence's first key tile
// are left to waves of their own (k_attention_grad_sinks), 64 or more to each; k_attention_sinks_sum adds their sums up in order, and
// k_attention_grad_kv adds those to its own.
//
// What bounds them: matrix products, exponentials and reads of LDS about evenly, with two waves to a SIMD, which is what the sums and operands of heads of 128 leave room for.  8 sequences of
// 2048 rows, 32 on 8 heads of 128, a window of 1024, 4 sinks: 834 us, 620 TFLOP/s of the formulas' five products; in a profile's run (822 us) grad_q 369 and grad_k, grad_v 408 (matrix cores 43 and 49 % busy at 2 GHz), sinks 45.
#include <algorithm>

#include "window_attention_tiles.h"

namespace {

constexpr int kWaves = 4, kColumns = 32, kRows = kWaves * kColumns;      // of a workgroup: queries (grad_q) or keys
constexpr int kAhead = 4, kAheadKv = 2;                                                // products' operands are read so many steps before
constexpr float kBoost = 8.0f, kUnboost = 1.0f / 256.0f;

struct Backward : Attention {
  Heads grad_out, grad_q, grad_k, grad_v;
  float *n, *minus_delta;      // [q_heads, rows]
  float* sums;                 // of far queries: [place, kv_heads, sink_blocks][grad_k, grad_v][32 keys][dim]; null: k_attention_grad_kv takes all queries
  int sink_blocks, far, chunk; // blocks of 32 keys with sinks; the first far query; far queries to a wave
  int64_t places;              // of waves' sums
  float* parts;                // of k_attention_grad_kv's pieces: [tiles, kv_heads, pieces][grad_k, grad_v][128 keys][dim]
  int pieces;                  // workgroups to a tile of keys, at most
};
constexpr int kSlots = 512, kLeastTurns = 4;      // pieces of all tiles, about; turns of a piece, at least

// Turns of a piece: of the turns of all tiles of all sequences, a 512th part.  (Sinks' far queries are left out: a tile that has more is cut into more
// turns than pieces of that size, if there are not enough of them.)
__device__ __forceinline__ int turns_of_piece(const Backward& a, int queries) {
  const int lane = threadIdx.x % kWave, most = (int)min(((int64_t)a.window + kRows - 2) / queries + 1, (int64_t)1 << 24), step = kRows / queries;
  float all = 0.0f;
  for (int first = 0; first < a.sequences; first += kWave) {
    int begin = 0, length = 0;
    if (first + lane < a.sequences) queries_of(a, first + lane, begin, length);
    const int n = (length + queries - 1) / queries, tiles = (length + kRows - 1) / kRows;
    const int full = max(0, min(tiles, (n - most + step - 1) / step));    // tiles that a whole window of queries sees
    all += (float)full * (float)most + (float)(tiles - full) * ((float)n - 0.5f * (float)step * (float)(tiles + full - 1));
  }
  return max(kLeastTurns, (int)fminf(wave_sum(all) * (float)a.q_heads * (1.0f / kSlots), 1e9f));
}

// What a tile of keys has to do: tiles of QUERIES queries from `begin` on, of each head that shares the keys.  Far queries, which see only sinks, are
// another kernel's if it has run (`split`).
struct KeyWork {
  int begin, end, query_tiles, turns, each;                              // each: turns to a piece
  bool split;
  __device__ __forceinline__ KeyWork(const Backward& a, const Sequence& s, int tile, int queries, bool pieces) {
    begin = tile * kRows;
    end = min(s.keys, begin + kRows);
    split = a.sums != nullptr && begin == 0 && s.queries > a.far;
    const int64_t window_end = (int64_t)end - 1 + a.window;
    const int last = split ? a.far - 1 : begin < a.sinks ? s.queries - 1 : (int)min((int64_t)s.queries, window_end) - 1;
    query_tiles = (last - begin) / queries + 1;
    turns = query_tiles * a.group;
    each = pieces ? max((turns - 1) / a.pieces + 1, turns_of_piece(a, queries)) : turns;
  }
};
template <int DP>
constexpr int kQueryTile = DP == 128 ? 32 : 64;
// Whether k_attention_grad_kv stores gradients itself of a tile that is one piece, among others that are more.  (With heads of 128 there are no registers for both ways.)
template <int DP>
constexpr bool kWholeTiles = DP < 128;

// Far queries of a sequence of `queries`: how many waves share them.
__device__ __forceinline__ int far_chunks(const Backward& a, int queries) { return queries > a.far ? (queries - a.far - 1) / a.chunk + 1 : 0; }
// The sequence and chunk of a wave's `place` (all sequences' chunks, one after the other), or the first place of a sequence (`of` not -1).
struct FarOf {
  int sequence, chunk, chunks;
};
__device__ __forceinline__ FarOf find_far(const Backward& a, int place, int of = -1) {
  const int lane = threadIdx.x % kWave;
  for (int first = 0, before = 0; first < a.sequences; first += kWave) {
    int begin = 0, length = 0;
    if (first + lane < a.sequences) queries_of(a, first + lane, begin, length);
    const int count = far_chunks(a, length);
    const int sum = (int)wave_inclusive_sum((uint32_t)count);
    const uint64_t behind = __ballot(of < 0 ? before + sum > place : first + lane == of);
    if (behind != 0) {
      const int at = __builtin_ctzll(behind), chunks = __builtin_amdgcn_readlane(count, at);
      return {first + at, (of < 0 ? place : 0) - (before + __builtin_amdgcn_readlane(sum, at) - chunks), chunks};
    }
    before += __builtin_amdgcn_readlane(sum, kWave - 1);
  }
  return {-1, 0, 0};
}
__device__ __forceinline__ float* far_sums(const Backward& a, int64_t place, int kv_head, int block) {
  place = max((int64_t)0, min(place, a.places - 1));                     // (sequences that overlap one another would have more)
  return a.sums + ((place * a.kv_heads + kv_head) * a.sink_blocks + block) * (2 * 32) * a.dim;
}

// n of a query; NaN where it is too far from 0 for P to come of it, so that its row, and the keys that it sees, are done again.
__device__ __forceinline__ float exponent_of(float lse) {
  const float n = __builtin_fmaf(-lse, kLog2E, kBoost);
  return is_far(n) ? __builtin_nanf("") : n;
}

// grad_q of one query by a wave, as attend_row.
template <int DT>
__device__ __forceinline__ void query_row(const Backward& a, const Sequence& s, int i, int head) {
  const int lane = threadIdx.x % kWave, low = window_begin(a, i);
  const int64_t row = (int64_t)s.q_begin + i;
  const char* const q = a.q.at + row * a.q.token + head * a.q.head;
  const char* const grad = a.grad_out.at + row * a.grad_out.token + head * a.grad_out.head;
  const char* const k = a.k.at + s.k_begin * a.k.token + head / a.group * a.k.head;
  const char* const v = a.v.at + s.k_begin * a.v.token + head / a.group * a.v.head;
  const float lse = a.lse[(int64_t)head * a.q_rows + row], delta = -a.minus_delta[(int64_t)head * a.q_rows + row];
  const int sinks = min(a.sinks, low), seen = sinks + i - low + 1;
  float lo = 0.0f, hi = 0.0f;
  for (int first = 0; first < seen; first += kWave) {
    const int n = first + lane, j = n < sinks ? n : low + n - sinks, count = min(seen - first, kWave);
    float grad_s = 0.0f;
    if (lane < count) {
      const float p = __builtin_amdgcn_exp2f((row_dot<DT>(q, k + j * a.k.token, a.dim, a.scale) - lse) * kLog2E);
      grad_s = p * (row_dot<DT>(grad, v + j * a.v.token, a.dim) - delta) * a.scale;
    }
    for (int t = 0; t < count; ++t) {
      const float weight = u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(grad_s), t));
      const Two x = load_two<DT>(k + __builtin_amdgcn_readlane(j, t) * a.k.token, a.dim);
      lo = __builtin_fmaf(weight, x.lo, lo);
      hi = __builtin_fmaf(weight, x.hi, hi);
    }
    if (all_nan(lo, hi, a.dim)) break;
  }
  store_two<DT>(a.grad_q.at + row * a.grad_q.token + head * a.grad_q.head, a.dim, lo, hi);
}

// grad_k and grad_v of one key by a wave: a query to a lane.
template <int DT>
__device__ __forceinline__ void key_row(const Backward& a, const Sequence& s, int j, int kv_head, bool of_k = true, bool of_v = true) {
  const int lane = threadIdx.x % kWave;
  const int64_t row = (int64_t)s.k_begin + j;
  const char* const k = a.k.at + row * a.k.token + kv_head * a.k.head;
  const char* const v = a.v.at + row * a.v.token + kv_head * a.v.head;
  const int last = j < a.sinks ? s.queries - 1 : (int)min((int64_t)s.queries - 1, (int64_t)j + a.window - 1);
  float k_lo = 0.0f, k_hi = 0.0f, v_lo = 0.0f, v_hi = 0.0f;
  bool over = false;
  for (int head = kv_head * a.group; head < (kv_head + 1) * a.group && !over; ++head) {
    const char* const q = a.q.at + s.q_begin * a.q.token + head * a.q.head;
    const char* const grad = a.grad_out.at + s.q_begin * a.grad_out.token + head * a.grad_out.head;
    const int64_t stat = (int64_t)head * a.q_rows + s.q_begin;
    for (int first = j; first <= last && !over; first += kWave) {
      const int i = first + lane, count = min(last - first + 1, kWave);
      float p = 0.0f, grad_s = 0.0f;
      if (lane < count) {
        p = __builtin_amdgcn_exp2f((row_dot<DT>(q + i * a.q.token, k, a.dim, a.scale) - a.lse[stat + i]) * kLog2E);
        grad_s = p * (row_dot<DT>(grad + i * a.grad_out.token, v, a.dim) + a.minus_delta[stat + i]) * a.scale;
      }
      for (int t = 0; t < count; ++t) {
        const float wp = u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(p), t)), ws = u2f((uint32_t)__builtin_amdgcn_readlane((int)f2u(grad_s), t));
        const Two x = load_two<DT>(q + (first + t) * a.q.token, a.dim), y = load_two<DT>(grad + (first + t) * a.grad_out.token, a.dim);
        k_lo = __builtin_fmaf(ws, x.lo, k_lo);
        k_hi = __builtin_fmaf(ws, x.hi, k_hi);
        v_lo = __builtin_fmaf(wp, y.lo, v_lo);
        v_hi = __builtin_fmaf(wp, y.hi, v_hi);
      }
      over = (!of_k || all_nan(k_lo, k_hi, a.dim)) && (!of_v || all_nan(v_lo, v_hi, a.dim));
    }
  }
  if (of_k) store_two<DT>(a.grad_k.at + row * a.grad_k.token + kv_head * a.grad_k.head, a.dim, k_lo, k_hi);
  if (of_v) store_two<DT>(a.grad_v.at + row * a.grad_v.token + kv_head * a.grad_v.head, a.dim, v_lo, v_hi);
}

template <int DT, int DP>
__global__ __launch_bounds__(kWaves * kWave, 2) void k_attention_grad_q(const Backward a, int tiles) {
  using S = TileShape<DP>;
  constexpr int kBytes = tile_bytes<DP>(kTileRows);
  __shared__ __attribute__((aligned(16))) char lds[4 * kBytes];        // keys, values; twice
  const Turn turn = turn_of_workgroup(tiles, a.kv_heads, a.group);
  const TileOf at = find_tile<kRows, false>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  const int begin = at.tile * kRows, end = min(s.queries, begin + kRows);
  const KeyTiles<kTileRows> keys(a, begin, end - 1);

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  const int kv_head = turn.head / a.group;
  TileWalk<DP, kTileRows, kWaves> k_walk, v_walk;
  k_walk.begin(a.k, s.k_begin, kv_head, a.dim);
  v_walk.begin(a.v, s.k_begin, kv_head, a.dim);
  auto fetch = [&](int t, int stage) {
    if (t == 0) {
      keys.walk(k_walk, s.keys);
      keys.walk(v_walk, s.keys);
    }
    const bool jumps = t == keys.sinks && t > 0, ends = t + 1 == keys.count;
    k_walk.next(lds0 + stage * kBytes, jumps, ends);
    v_walk.next(lds0 + (2 + stage) * kBytes, jumps, ends);
  };
  fetch(0, 0);

  const int wave = uniform(threadIdx.x / kWave), li = threadIdx.x & 31;
  const int first = begin + wave * kColumns, i = min(first + li, end - 1), last = min(first + kColumns, end) - 1;
  const int64_t row = (int64_t)s.q_begin + i, stat = (int64_t)turn.head * a.q_rows + row;
  const bool mine = first + li < end;
  u32x4 q[S::kSteps], grad[S::kSteps];
  load_columns<DP>(a.q.at + row * a.q.token + turn.head * a.q.head, a.dim, a.scale < 0.0f, q);
  load_columns<DP>(a.grad_out.at + row * a.grad_out.token + turn.head * a.grad_out.head, a.dim, false, grad);
  float delta = 0.0f;
  {
    u32x4 out[S::kSteps];
    load_columns<DP>(a.out.at + row * a.out.token + turn.head * a.out.head, a.dim, false, out);
#pragma unroll
    for (int x = 0; x < S::kSteps; ++x) {
      float u[8], v[8];
      widen_unit<DT>(Unit<DT>{{out[x]}}, u);
      widen_unit<DT>(Unit<DT>{{grad[x]}}, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = __builtin_fmaf(u[e], v[e], delta);
    }
    delta += from_other_half(delta);
  }
  const float c = exponent_factor(a.scale), n = exponent_of(a.lse[stat]);
  const KeyView<kTileRows> view(a, keys, first, first < end ? last : -1);
  const ReadAlong<kTileRows> along((lds_char*)lds);
  // P, times 2^8, times dP - delta of a block of 32 keys: dS
  auto block = [&](int at_keys, int at_values, int b, int key, Seen seen, f32x16& p) {
    f32x16 dp;
    u32x4 k[S::kSteps], v[S::kSteps];
    auto read = [&](int x) {
      k[x] = along.read(at_keys, b, x);
      v[x] = along.read(at_values, b, x);
    };
#pragma unroll
    for (int x = 0; x < kAhead && x < S::kSteps; ++x) read(x);
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = dp[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < S::kSteps; ++x) {
      if (x + kAhead < S::kSteps) read(x + kAhead);
      p = mfma16<DT>(k[x], q[x], p);
      dp = mfma16<DT>(v[x], grad[x], dp);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c, n)) * (dp[r] - delta);
    if (seen == kPart) {
      const RowsSeen rows = keys_seen(a, i, key + b * 32);
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = rows.at(row_of_register(r)) ? p[r] : 0.0f;
    }
  };
  // With few keys out is as large as a v, and its rounding, in delta, counts as much as that of dS (with n keys an n-th part of it).  There the sum of dS
  // over the keys, which is 0 but for that, says what delta is off.
  if (keys.count <= 2 || a.window < kTileRows) {
    float sum = 0.0f;
    for (int t = 0; t < keys.count; ++t) {
      const int stage = t & 1, key = keys.key(t);
      wait_tile();
      tile_barrier();
      if (t + 1 < keys.count) fetch(t + 1, 1 - stage);
      const Seen seen = view.of(t, keys.sinks, key);
      if (seen == kNothing) continue;
      for (int b = 0; b < 2; ++b) {
        f32x16 p;
        block(stage * kBytes, (2 + stage) * kBytes, b, key, seen, p);
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += p[r];
      }
    }
    sum += from_other_half(sum);
    if (sum == sum) delta = __builtin_fmaf(sum, kUnboost, delta);        // (else the row is done again, with this delta)
    if (keys.count > 2) {                                                // (two tiles are both there still)
      tile_barrier();
      fetch(0, 0);
    }
  }
  const bool kept = keys.count <= 2;
  if (mine && (threadIdx.x & 32) == 0) {
    a.n[stat] = n;
    a.minus_delta[stat] = -delta;
  }

  const ReadAcross<kTileRows> across((lds_char*)lds);
  f32x16 o[S::kBlocks];
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] = 0.0f;

  auto tile = [&](int key, Seen seen, auto stage_constant) {
    constexpr int kKeys = decltype(stage_constant)::value * kBytes, kValues = 2 * kBytes + kKeys;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x16 p;
      block(kKeys, kValues, b, key, seen, p);
      u32x4 w[2], k[2 * S::kBlocks];
      auto read = [&](int n) { k[n] = across.read(kKeys, n % S::kBlocks, 2 * b + n / S::kBlocks); };
#pragma unroll
      for (int n = 0; n < kAhead && n < 2 * S::kBlocks; ++n) read(n);
#pragma unroll
      for (int r = 0; r < 16; r += 2) w[r >> 3][(r & 7) >> 1] = narrow_pair<DT>(p[r], p[r + 1]);
#pragma unroll
      for (int n = 0; n < 2 * S::kBlocks; ++n) {
        if (n + kAhead < 2 * S::kBlocks) read(n + kAhead);
        o[n % S::kBlocks] = mfma16<DT>(k[n], w[n / S::kBlocks], o[n % S::kBlocks]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  int key = keys.first_key();
  auto turn_tile = [&](int t, auto stage_constant) {
    wait_tile();
    tile_barrier();
    if (t + 1 < keys.count && !kept) fetch(t + 1, 1 - decltype(stage_constant)::value);
    const Seen seen = view.of(t, keys.sinks, key);
    if (seen != kNothing) tile(key, seen, stage_constant);
    key = t + 1 == keys.sinks ? keys.low * kTileRows : key + kTileRows;
  };
  for (int t = 0; t < keys.count; t += 2) {
    turn_tile(t, std::integral_constant<int, 0>{});
    if (t + 1 < keys.count) turn_tile(t + 1, std::integral_constant<int, 1>{});
  }
  if (first >= end) return;
  const int query = first + column_again();
  uint32_t again = columns_to_do_again(o, query < end);
  char* const to = a.grad_q.at + ((int64_t)s.q_begin + min(query, end - 1)) * a.grad_q.token + turn.head * a.grad_q.head;
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b) store_column_block<DT>(to, b, a.dim, query < end, o[b], a.scale * kUnboost);
  if (again == 0) return;
  __threadfence_block();                                                 // (minus_delta, which the row reads, is this wave's own)
  while (again != 0) {
    const int x = __builtin_ctz(again);
    again &= again - 1;
    query_row<DT>(a, s, first + x, turn.head);
  }
}

// The same for few queries: 32 of them to a workgroup, whose waves take every fourth tile of 32 keys each, alone, and add their sums up at the end.
template <int DT, int DP>
__global__ __launch_bounds__(kWaves * kWave, 1) void k_attention_grad_q_few(const Backward a, int tiles) {
  using S = TileShape<DP>;
  constexpr int kKeys = 32, kTile = tile_bytes<DP>(kKeys), kStage = 2 * kTile, kOwn = 2 * kStage;
  __shared__ __attribute__((aligned(16))) char lds[kWaves * kOwn];        // of each wave: keys and values, twice; its sums in the end
  __shared__ float offs[kWaves][kColumns];
  __shared__ uint32_t bad;
  const Turn turn = turn_of_workgroup(tiles, a.kv_heads, a.group);
  const TileOf at = find_tile<kColumns, false>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  const int first = at.tile * kColumns, last = min(s.queries, first + kColumns) - 1;
  const KeyTiles<kKeys> keys(a, first, last);
  const int wave = uniform(threadIdx.x / kWave), li = threadIdx.x & 31, i = min(first + li, last);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds + (uint32_t)wave * kOwn;
  const int kv_head = turn.head / a.group;
  TileFeed<DP, kKeys, 1> k_feed, v_feed;
  k_feed.begin(a.k, s.k_begin, kv_head, a.dim);
  v_feed.begin(a.v, s.k_begin, kv_head, a.dim);
  auto fetch = [&](int t, int stage) {
    k_feed.fetch_of_wave(lds0 + stage * kStage, keys.key(t), s.keys);
    v_feed.fetch_of_wave(lds0 + stage * kStage + kTile, keys.key(t), s.keys);
  };
  if (wave < keys.count) fetch(wave, 0);

  const int64_t row = (int64_t)s.q_begin + i, stat = (int64_t)turn.head * a.q_rows + row;
  u32x4 q[S::kSteps], grad[S::kSteps];
  load_columns<DP>(a.q.at + row * a.q.token + turn.head * a.q.head, a.dim, a.scale < 0.0f, q);
  load_columns<DP>(a.grad_out.at + row * a.grad_out.token + turn.head * a.grad_out.head, a.dim, false, grad);
  float delta = 0.0f;
  {
    u32x4 out[S::kSteps];
    load_columns<DP>(a.out.at + row * a.out.token + turn.head * a.out.head, a.dim, false, out);
#pragma unroll
    for (int x = 0; x < S::kSteps; ++x) {
      float u[8], v[8];
      widen_unit<DT>(Unit<DT>{{out[x]}}, u);
      widen_unit<DT>(Unit<DT>{{grad[x]}}, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = __builtin_fmaf(u[e], v[e], delta);
    }
    delta += from_other_half(delta);
  }
  const float c = exponent_factor(a.scale), n = exponent_of(a.lse[stat]);
  const ReadAlong<kKeys> along((lds_char*)lds + wave * kOwn);
  const ReadAcross<kKeys> across((lds_char*)lds + wave * kOwn);
  const KeyView<kKeys> view(a, keys, first, last);
  f32x16 o[S::kBlocks];
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] = 0.0f;
  // dS of the wave's tile t, which is in `stage`; the next one is on its way meanwhile
  auto tile = [&](int t, int stage, f32x16& p) {
    const int at_keys = stage * kStage, at_values = at_keys + kTile;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                   // the next tile's place has been read
    if (t + kWaves < keys.count) {
      fetch(t + kWaves, 1 - stage);
      wait_but<2 * TileFeed<DP, kKeys, 1>::kLoads>();
    } else {
      wait_tile();
    }
    f32x16 dp;
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = dp[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < S::kSteps; ++x) {
      p = mfma16<DT>(along.read(at_keys, 0, x), q[x], p);
      dp = mfma16<DT>(along.read(at_values, 0, x), grad[x], dp);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], c, n)) * (dp[r] - delta);
    const int key = keys.key(t);
    if (view.of(t, keys.sinks, key) != kAll) {
      const RowsSeen rows = keys_seen(a, i, key);
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = rows.at(row_of_register(r)) ? p[r] : 0.0f;
    }
  };
  if (threadIdx.x == 0) bad = 0;
  if (keys.count <= 4 || a.window < kTileRows) {                         // (as k_attention_grad_q)
    float sum = 0.0f;
    int stage = 0;
    for (int t = wave; t < keys.count; t += kWaves, stage ^= 1) {
      f32x16 p;
      tile(t, stage, p);
#pragma unroll
      for (int r = 0; r < 16; ++r) sum += p[r];
    }
    sum += from_other_half(sum);
    if ((threadIdx.x & 32) == 0) offs[wave][li] = sum;
    __syncthreads();
    sum = (offs[0][li] + offs[1][li]) + (offs[2][li] + offs[3][li]);
    if (sum == sum) delta = __builtin_fmaf(sum, kUnboost, delta);
    if (keys.count > kWaves && wave < keys.count) fetch(wave, 0);        // (one tile is there still)
  }
  if (wave == 0 && first + li <= last && (threadIdx.x & 32) == 0) {
    a.n[stat] = n;
    a.minus_delta[stat] = -delta;
  }
  int stage = 0;
  for (int t = wave; t < keys.count; t += kWaves, stage ^= 1) {
    f32x16 p;
    tile(t, stage, p);
    u32x4 w[2];
#pragma unroll
    for (int r = 0; r < 16; r += 2) w[r >> 3][(r & 7) >> 1] = narrow_pair<DT>(p[r], p[r + 1]);
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int d = 0; d < S::kBlocks; ++d) o[d] = mfma16<DT>(across.read(stage * kStage, d, x), w[x], o[d]);
  }
  add_up<S::kBlocks, kOwn>(lds, o);
  const uint32_t mine = wave < S::kBlocks ? columns_to_do_again({o[0]}, first + li <= last) : 0u;
  if (mine != 0 && (threadIdx.x & 63) == 0) atomicOr(&bad, mine);
  if (wave < S::kBlocks)
    store_column_block<DT>(a.grad_q.at + row * a.grad_q.token + turn.head * a.grad_q.head, wave, a.dim, first + li <= last, o[0], a.scale * kUnboost);
  __threadfence_block();                                                 // (minus_delta, and rows that are done again)
  __syncthreads();
  uint32_t again = bad;
  for (int m = 0; again != 0; ++m) {
    const int x = __builtin_ctz(again);
    again &= again - 1;
    if (m % kWaves == wave) query_row<DT>(a, s, first + x, turn.head);
  }
}

// A wave's 32 keys as columns, and its sums.
template <int DT, int DP, bool V_IN_LDS>
struct KeyColumns {
  using S = TileShape<DP>;
  u32x4 k[S::kSteps], v[V_IN_LDS ? 1 : S::kSteps];
  f32x16 dk[S::kBlocks], dv[S::kBlocks];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] = 0.0f;
  }
};

// 32 queries of a tile in LDS against the wave's keys.  `values(x)`: v's columns.
template <int ROWS, int DT, int DP, bool V_IN_LDS, class Values>
__device__ __forceinline__ void queries_block(const Attention& a, KeyColumns<DT, DP, V_IN_LDS>& col, const ReadAlong<ROWS>& along, const ReadAcross<ROWS>& across,
                                              const lds_char* stats, int queries, int grads, int block, int query, int key, Seen seen, float c, Values values) {
  using S = TileShape<DP>;
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  const lds_f32x4* const stat = (const lds_f32x4*)(stats + ((threadIdx.x >> 5) & 1) * 16);      // n, and 256 bytes on -delta: rows 8 g + 4 lg ... + 3
  f32x16 p, dp;
  u32x4 q[S::kSteps], grad[S::kSteps], v[S::kSteps];
  auto read = [&](int x) {
    q[x] = along.read(queries, block, x);
    grad[x] = along.read(grads, block, x);
    v[x] = values(x);
  };
#pragma unroll
  for (int x = 0; x < kAheadKv && x < S::kSteps; ++x) read(x);
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x4 d = stat[16 + 2 * g];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      p[4 * g + r] = 0.0f;
      dp[4 * g + r] = d[r];
    }
  }
#pragma unroll
  for (int x = 0; x < S::kSteps; ++x) {
    if (x + kAheadKv < S::kSteps) read(x + kAheadKv);
    p = mfma16<DT>(q[x], col.k[x], p);
    dp = mfma16<DT>(grad[x], v[x], dp);
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x4 n = stat[2 * g];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int e = 4 * g + r;
      p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[e], c, n[r]));
      dp[e] *= p[e];
    }
  }
  if (seen == kPart) {
    const QueriesSeen rows = queries_seeing(a, key, query);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      p[e] = rows.at(row_of_register(e)) ? p[e] : 0.0f;
      dp[e] = rows.at(row_of_register(e)) ? dp[e] : 0.0f;
    }
  }
  u32x4 wp[2], ws[2], g[4 * S::kBlocks];
  constexpr int kProducts = 4 * S::kBlocks;                              // by 16 queries: of every block of elements, grad_v and grad_k
  auto read_across = [&](int n) { g[n] = across.read(n & 1 ? queries : grads, n / 2 % S::kBlocks, 2 * block + n / 2 / S::kBlocks); };
#pragma unroll
  for (int n = 0; n < kAheadKv && n < kProducts; ++n) read_across(n);
#pragma unroll
  for (int r = 0; r < 16; r += 2) {
    wp[r >> 3][(r & 7) >> 1] = narrow_pair<DT>(p[r], p[r + 1]);
    ws[r >> 3][(r & 7) >> 1] = narrow_pair<DT>(dp[r], dp[r + 1]);
  }
#pragma unroll
  for (int n = 0; n < kProducts; ++n) {
    if (n + kAheadKv < kProducts) read_across(n + kAheadKv);
    const int d = n / 2 % S::kBlocks, x = n / 2 / S::kBlocks;
    if (n & 1) col.dk[d] = mfma16<DT>(g[n], ws[x], col.dk[d]);
    else col.dv[d] = mfma16<DT>(g[n], wp[x], col.dv[d]);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// A float to a lane, zeros behind the first `count`.
__device__ __forceinline__ void fetch_floats(uint32_t lds, const float* from, int count) {
  const uint64_t at = reinterpret_cast<uint64_t>(from);
  const u32x4 buffer = {(uint32_t)uniform((int)(uint32_t)at), (uint32_t)uniform((int)(uint32_t)(at >> 32)), (uint32_t)uniform(count) * 4, 0x00020000u};
  fetch_float(lds, threadIdx.x % kWave * 4, buffer);
}

// Where a piece's sums go; and a lane's block of them, from its key's row on.
__device__ __forceinline__ float* part_of(const Backward& a, const Turn& turn, int tiles, int piece) {
  return a.parts + (((int64_t)turn.head * tiles + turn.tile) * a.pieces + piece) * (2 * kRows) * a.dim;
}
__device__ __forceinline__ void store_sums(float* to, int rows, int dim, int block, const f32x16& dk, const f32x16& dv) {
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int d = 32 * block + 8 * g;
    if (d + first_row() >= dim) continue;
    *reinterpret_cast<f32x4*>(to + d) = f32x4{dk[4 * g], dk[4 * g + 1], dk[4 * g + 2], dk[4 * g + 3]};
    *reinterpret_cast<f32x4*>(to + rows * dim + d) = f32x4{dv[4 * g], dv[4 * g + 1], dv[4 * g + 2], dv[4 * g + 3]};
  }
}

// PIECES: a.pieces workgroups at most share a tile's turns, and leave sums to k_attention_kv_sum (kWholeTiles).
template <int DT, int DP, bool PIECES>
__global__ __launch_bounds__(kWaves * kWave, 2) void k_attention_grad_kv(const Backward a, int tiles) {
  using S = TileShape<DP>;
  // With heads of 128 the registers hold k and both sums, but not v as well: it stays in LDS, and tiles of queries are half as large.
  constexpr bool kVInLds = DP == 128;
  constexpr int kQueries = kQueryTile<DP>, kTile = tile_bytes<DP>(kQueries), kStage = 2 * kTile + 512;      // queries, gradients, n and -delta
  __shared__ __attribute__((aligned(16))) char lds[2 * kStage + (kVInLds ? tile_bytes<DP>(kRows) : 0)];
  // (pieces of a tile far apart: neighbours go to different dies, and most tiles have few)
  const unsigned units = PIECES ? gridDim.x / (unsigned)a.pieces : 1u;
  const int piece = PIECES ? (int)(blockIdx.x / units) : 0, unit = PIECES ? (int)(blockIdx.x % units) : 0;
  const Turn turn = PIECES ? Turn{(int)((unsigned)unit / (unsigned)tiles), (int)((unsigned)unit % (unsigned)tiles)} : turn_of_workgroup(tiles, a.kv_heads, 1);
  const TileOf at = find_tile<kRows, true>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  const KeyWork work(a, s, at.tile, kQueries, PIECES);
  const int begin = work.begin, end = work.end, query_tiles = work.query_tiles;
  const int first_turn = PIECES ? piece * work.each : 0, turns = PIECES ? min(work.each, work.turns - first_turn) : work.turns;
  if (turns <= 0) return;
  const bool split = work.split;

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  const int wave = uniform(threadIdx.x / kWave), li = threadIdx.x & 31;
  TileWalk<DP, kQueries, kWaves> q_walk, grad_walk;
  const int first_head = turn.head * a.group;
  q_walk.begin(a.q, s.q_begin, first_head, a.dim);
  grad_walk.begin(a.grad_out, s.q_begin, first_head, a.dim);
  // A head's queries are walked round, from a tile whose number the length of the way divides: key tiles beside each other, whose windows are as long, then read the same
  // queries at the same time (8x2048 rows, 32 on 8 heads of 128, a window of 1024: 3 % less time for the backward pass).
  const int end_row = begin + (query_tiles - 1) * kQueries, skipped_heads = PIECES ? first_turn / query_tiles : 0,
            skipped = PIECES ? first_turn - skipped_heads * query_tiles : (query_tiles - begin / kQueries % query_tiles) % query_tiles;
  q_walk.walk(begin + skipped * kQueries, 0, end_row, s.queries);
  grad_walk.walk(begin + skipped * kQueries, 0, end_row, s.queries);
  q_walk.at += (uint64_t)skipped_heads * (uint64_t)a.q.head;
  grad_walk.at += (uint64_t)skipped_heads * (uint64_t)a.grad_out.head;
  int64_t stat = (int64_t)(first_head + skipped_heads) * a.q_rows + s.q_begin + begin + skipped * kQueries;
  int fetch_tile = skipped, of_head = PIECES ? skipped : 0;               // of_head: the tiles of this head that are behind
  auto fetch = [&](int stage) {                                          // the next tile
    const uint32_t to = lds0 + stage * kStage;
    const bool next_head = of_head == query_tiles;
    of_head = next_head ? 1 : of_head + 1;
    if (fetch_tile == query_tiles) {
      fetch_tile = 0;
      q_walk.at -= (uint64_t)query_tiles * q_walk.step;
      grad_walk.at -= (uint64_t)query_tiles * grad_walk.step;
      stat -= query_tiles * kQueries;
    }
    if (next_head) {
      q_walk.at += (uint64_t)a.q.head;
      grad_walk.at += (uint64_t)a.grad_out.head;
      stat += a.q_rows;
    }
    const bool ends = fetch_tile + 1 == query_tiles;
    q_walk.next(to, false, ends);
    grad_walk.next(to + kTile, false, ends);
    const int count = min(s.queries - begin - fetch_tile * kQueries, kQueries);
    if (wave == 0) fetch_floats(to + 2 * kTile, a.n + stat, count);
    if (wave == 1) fetch_floats(to + 2 * kTile + 256, a.minus_delta + stat, count);
    stat += kQueries;
    ++fetch_tile;
  };
  fetch(0);
  if constexpr (kVInLds) {
    TileFeed<DP, kRows, kWaves> v_feed;
    v_feed.begin(a.v, s.k_begin, turn.head, a.dim);
    v_feed.fetch(lds0 + 2 * kStage, begin, s.keys);
  }

  const int first = begin + wave * kColumns, j = min(first + li, end - 1), last = min(first + kColumns, end) - 1;
  const int64_t row = (int64_t)s.k_begin + j;
  KeyColumns<DT, DP, kVInLds> col;
  load_columns<DP>(a.k.at + row * a.k.token + turn.head * a.k.head, a.dim, a.scale < 0.0f, col.k);
  if constexpr (!kVInLds) load_columns<DP>(a.v.at + row * a.v.token + turn.head * a.v.head, a.dim, false, col.v);
  col.clear();
  const float c = exponent_factor(a.scale);
  const ReadAlong<kQueries> along((lds_char*)lds);
  const ReadAcross<kQueries> across((lds_char*)lds);
  const ReadAlong<kRows> v_along((lds_char*)lds + 2 * kStage + wave * 2048);
  auto values = [&](int x) {
    if constexpr (kVInLds) return v_along.read(0, 0, x);
    else return col.v[x];
  };

  int query_tile = skipped;
  auto turn_tile = [&](int t, auto stage_constant) {
    constexpr int kAt = decltype(stage_constant)::value * kStage;
    wait_tile();
    tile_barrier();
    if (t + 1 < turns) fetch(1 - decltype(stage_constant)::value);
    const int query = begin + query_tile * kQueries;
    if (++query_tile == query_tiles) query_tile = 0;
    if (first >= end) return;
#pragma unroll
    for (int b = 0; b < kQueries / 32; ++b) {
      const Seen seen = keys_seen_by(a, query + 32 * b, first, last);
      if (seen != kNothing)
        queries_block<kQueries, DT, DP, kVInLds>(a, col, along, across, (lds_char*)lds + kAt + 2 * kTile + b * 128, kAt, kAt + kTile, b, query + 32 * b, j, seen, c, values);
    }
  };
  for (int t = 0; t < turns; t += 2) {
    turn_tile(t, std::integral_constant<int, 0>{});
    if (t + 1 < turns) turn_tile(t + 1, std::integral_constant<int, 1>{});
  }
  if (first >= end) return;
  if (PIECES && (!kWholeTiles<DP> || work.turns > work.each)) {
    float* const parts = part_of(a, turn, tiles, piece) + (wave * kColumns + column_again()) * a.dim + first_row();
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) store_sums(parts, kRows, a.dim, b, col.dk[b], col.dv[b]);
    return;
  }
  if (split && first < a.sinks) {
    const FarOf far = find_far(a, 0, at.sequence);
    const float* const sums = far_sums(a, -far.chunk, turn.head, wave) + column_again() * a.dim + first_row();
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int d = 32 * b + 8 * g;
        if (d + first_row() >= a.dim) continue;
        const f32x4 k = *reinterpret_cast<const f32x4*>(sums + d), v = *reinterpret_cast<const f32x4*>(sums + 32 * a.dim + d);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          col.dk[b][4 * g + r] += k[r];
          col.dv[b][4 * g + r] += v[r];
        }
      }
  }
  const int to = first + column_again();
  const bool mine = to < end;
  const int64_t to_row = (int64_t)s.k_begin + min(to, end - 1);
  uint32_t again = columns_to_do_again(col.dk, mine) | columns_to_do_again(col.dv, mine);
  char* const to_k = a.grad_k.at + to_row * a.grad_k.token + turn.head * a.grad_k.head;
  char* const to_v = a.grad_v.at + to_row * a.grad_v.token + turn.head * a.grad_v.head;
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b) {
    store_column_block<DT>(to_k, b, a.dim, mine, col.dk[b], a.scale * kUnboost);
    store_column_block<DT>(to_v, b, a.dim, mine, col.dv[b], kUnboost);
  }
  while (again != 0) {
    const int x = __builtin_ctz(again);
    again &= again - 1;
    key_row<DT>(a, s, first + x, turn.head);
  }
}

// The sums of a tile's pieces, in order, and of its far queries: gridDim.y workgroups to its keys, for each of the two gradients.  What it takes is mostly a workgroup's
// way to its first load: fewer of them where there are many tiles.  Measured, with 2 and 8 workgroups, the whole backward pass: 4x1024 rows, 12 heads of 64, 90 and 109 us; 1x300
// rows, 8 on 2 heads of 128, 41 and 32.
template <int DT, int DP>
__global__ __launch_bounds__(kWaves * kWave) void k_attention_kv_sum(const Backward a, int tiles) {
  __shared__ uint32_t bad[kRows / 32];
  const Turn turn = {(int)(blockIdx.x / (unsigned)tiles), (int)(blockIdx.x % (unsigned)tiles)};
  const TileOf at = find_tile<kRows, true>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  const KeyWork work(a, s, at.tile, kQueryTile<DP>, true);
  const int share = kRows / gridDim.y, row = blockIdx.y * share, first = work.begin + row, keys = min(work.end - first, share), of_v = blockIdx.z;
  if (keys <= 0 || (kWholeTiles<DP> && work.turns <= work.each)) return;
  const int pieces = (work.turns - 1) / work.each + 1, quads = a.dim / 4;
  const float* const parts = part_of(a, turn, tiles, 0) + (of_v * kRows + row) * a.dim;
  // (a tile that has far queries begins at key 0)
  const float* const sums = work.split ? far_sums(a, -find_far(a, 0, at.sequence).chunk, turn.head, 0) + of_v * 32 * a.dim : nullptr;
  const float by = of_v ? kUnboost : a.scale * kUnboost;
  if (threadIdx.x < kRows / 32) bad[threadIdx.x] = 0;
  __syncthreads();
  for (int n = threadIdx.x; n < keys * quads; n += kWaves * kWave) {
    const int key = n / quads, d = (n - key * quads) * 4;
    const float* const from = parts + key * a.dim + d;
    f32x4 sum = *reinterpret_cast<const f32x4*>(from);
#pragma unroll 8
    for (int i = 1; i < pieces; ++i) sum += *reinterpret_cast<const f32x4*>(from + (int64_t)i * (2 * kRows) * a.dim);
    const int block = (row + key) / 32;
    if (work.split && block < a.sink_blocks) sum += *reinterpret_cast<const f32x4*>(sums + (block * 2 * 32 + (row + key) % 32) * a.dim + d);
    if (!(sum[0] * 0.0f + sum[1] * 0.0f + sum[2] * 0.0f + sum[3] * 0.0f == 0.0f)) atomicOr(&bad[key / 32], 1u << key % 32);
    u32x2 out;
    out.x = narrow_pair<DT>(sum[0] * by, sum[1] * by);
    out.y = narrow_pair<DT>(sum[2] * by, sum[3] * by);
    const int64_t to = (int64_t)s.k_begin + first + key;
    char* const grad = of_v ? a.grad_v.at + to * a.grad_v.token + turn.head * a.grad_v.head : a.grad_k.at + to * a.grad_k.token + turn.head * a.grad_k.head;
    *reinterpret_cast<u32x2*>(grad + d * 2) = out;
  }
  __threadfence_block();                                                 // (rows that are done again were written by other waves)
  __syncthreads();
  const int wave = uniform(threadIdx.x / kWave);
  for (int word = 0, n = 0; word * 32 < keys; ++word)
    for (uint32_t again = bad[word]; again != 0; ++n) {
      const int x = __builtin_ctz(again);
      again &= again - 1;
      if (n % kWaves == wave) key_row<DT>(a, s, first + word * 32 + x, turn.head, of_v == 0, of_v != 0);
    }
}

// A wave, alone: 32 keys of a sequence's first tile, some of them sinks, and a chunk of far queries of all heads that share them, 32 at a time, two tiles on
// their way into LDS.
template <int DT, int DP>
__global__ __launch_bounds__(kWave, 1) void k_attention_grad_sinks(const Backward a) {
  using S = TileShape<DP>;
  constexpr int kQueries = 32, kTile = tile_bytes<DP>(kQueries), kStage = 2 * kTile + 512;
  __shared__ __attribute__((aligned(16))) char lds[2 * kStage];
  const int units = a.kv_heads * a.sink_blocks, place = (int)(blockIdx.x / (unsigned)units), unit = (int)(blockIdx.x % (unsigned)units);
  const int kv_head = unit / a.sink_blocks, block = unit % a.sink_blocks;
  const FarOf at = find_far(a, place);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  const int begin = a.far + at.chunk * a.chunk, end = min(s.queries, begin + a.chunk);
  const int query_tiles = (end - begin - 1) / kQueries + 1, turns = query_tiles * a.group;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  TileWalk<DP, kQueries, 1> q_walk, grad_walk;
  const int first_head = kv_head * a.group;
  q_walk.begin(a.q, s.q_begin, first_head, a.dim);
  grad_walk.begin(a.grad_out, s.q_begin, first_head, a.dim);
  q_walk.walk(begin, 0, begin + (query_tiles - 1) * kQueries, end);
  grad_walk.walk(begin, 0, begin + (query_tiles - 1) * kQueries, end);
  q_walk.jump = (uint64_t)a.q.head - (uint64_t)query_tiles * q_walk.step;                      // on to the next head
  grad_walk.jump = (uint64_t)a.grad_out.head - (uint64_t)query_tiles * grad_walk.step;
  int64_t stat = (int64_t)first_head * a.q_rows + s.q_begin + begin;
  int fetch_tile = 0;
  auto fetch = [&](int stage) {                                          // the next tile
    const uint32_t to = lds0 + stage * kStage;
    const bool jumps = fetch_tile == query_tiles;
    fetch_tile = jumps ? 0 : fetch_tile;
    stat += jumps ? (int64_t)a.q_rows - query_tiles * kQueries : 0;
    q_walk.next(to, jumps, fetch_tile + 1 == query_tiles);
    grad_walk.next(to + kTile, jumps, fetch_tile + 1 == query_tiles);
    const int count = min(end - begin - fetch_tile * kQueries, kQueries);
    fetch_floats(to + 2 * kTile, a.n + stat, count);
    fetch_floats(to + 2 * kTile + 256, a.minus_delta + stat, count);
    stat += kQueries;
    ++fetch_tile;
  };
  fetch(0);
  const int li = threadIdx.x & 31, key = min(block * 32 + li, s.keys - 1);
  const int64_t row = (int64_t)s.k_begin + key;
  KeyColumns<DT, DP, false> col;
  load_columns<DP>(a.k.at + row * a.k.token + kv_head * a.k.head, a.dim, a.scale < 0.0f, col.k);
  load_columns<DP>(a.v.at + row * a.v.token + kv_head * a.v.head, a.dim, false, col.v);
  col.clear();
  const float c = exponent_factor(a.scale);
  const ReadAlong<kQueries> along((lds_char*)lds);
  const ReadAcross<kQueries> across((lds_char*)lds);
  auto values = [&](int x) { return col.v[x]; };
  const Seen seen = block * 32 + 31 < a.sinks ? kAll : kPart;
  int query_tile = 0;
  auto turn_tile = [&](int t, auto stage_constant) {
    constexpr int kAt = decltype(stage_constant)::value * kStage;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                   // the next tile's place has been read
    if (t + 1 < turns) {
      fetch(1 - decltype(stage_constant)::value);
      wait_but<2 * TileFeed<DP, kQueries, 1>::kLoads + 2>();
    } else {
      wait_tile();
    }
    const int query = begin + query_tile * kQueries;
    if (++query_tile == query_tiles) query_tile = 0;
    queries_block<kQueries, DT, DP, false>(a, col, along, across, (lds_char*)lds + kAt + 2 * kTile, kAt, kAt + kTile, 0, query, key, seen, c, values);
  };
  for (int t = 0; t < turns; t += 2) {
    turn_tile(t, std::integral_constant<int, 0>{});
    if (t + 1 < turns) turn_tile(t + 1, std::integral_constant<int, 1>{});
  }
  float* const sums = far_sums(a, place, kv_head, block) + column_again() * a.dim + first_row();
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b) store_sums(sums, 32, a.dim, b, col.dk[b], col.dv[b]);
}

// The sums of a sequence's chunks into the first one's place: four floats to a thread, 1024 to a workgroup.  `by_place`: gridDim.x counts places of chunks, not
// sequences, which may be more.
__global__ __launch_bounds__(256) void k_attention_sinks_sum(const Backward a, bool by_place) {
  const int units = a.kv_heads * a.sink_blocks, n = (int)(blockIdx.x / (unsigned)units), unit = (int)(blockIdx.x % (unsigned)units);
  const FarOf at = by_place ? find_far(a, n) : find_far(a, 0, n);
  if (at.sequence < 0 || (by_place && at.chunk != 0) || at.chunks < 2) return;
  const int place = by_place ? n : -at.chunk;
  const int e = (int)(blockIdx.y * 256 + threadIdx.x) * 4;
  if (e >= 2 * 32 * a.dim) return;
  float* const to = far_sums(a, place, unit / a.sink_blocks, unit % a.sink_blocks) + e;
  const int64_t step = (int64_t)units * (2 * 32) * a.dim;
  const int chunks = (int)min((int64_t)at.chunks, a.places - place);     // (of sequences that overlap one another only some have a place)
  f32x4 sum = *reinterpret_cast<const f32x4*>(to);
#pragma unroll 4
  for (int i = 1; i < chunks; ++i) sum += *reinterpret_cast<const f32x4*>(to + i * step);
  *reinterpret_cast<f32x4*>(to) = sum;
}

// How far queries are shared out, and the bytes of their sums.  Only where sinks are few: more of them are key tiles enough.
struct FarPlan {
  int sink_blocks, far, chunk;
  int64_t places, bytes;
};
constexpr int64_t kFarWaves = 1024, kMostFarBytes = (int64_t)1 << 29;
constexpr int kLeastChunk = 64;
int64_t first_far(int64_t window) { return (kRows - 1 + window + kTileRows - 1) / kTileRows * kTileRows; }      // a tile's other keys are out of sight there
int64_t far_bytes_of(int head_dim) { return 2 * 32 * head_dim * (int64_t)sizeof(float); }
FarPlan far_plan(int64_t rows, int kv_heads, int head_dim, int64_t sequences, int64_t window, int64_t sinks) {
  if (sinks == 0 || sinks > kRows || window == 0 || window >= rows) return {};
  const int64_t far = first_far(window);
  if (far >= rows) return {};
  // Two launches more.  Measured with and without, 32 on 8 heads of 128, a window of 1024: 3600 rows 296 and 304 us, 8192 527 and 1503, 32768 2126 and 6662;
  // 8 on 2 heads, a window of 100: 700 rows 55 and 37, 2000 71 and 80.
  if (rows < 3 * far) return {};
  FarPlan plan = {(int)((sinks + 31) / 32), (int)far, kLeastChunk, 0, 0};
  // (about as many waves as run at once: a sequence's first queries are not far; 8x2048 rows, a window of 1024: 64 queries to a wave 37 us, 128 39, of which their 147 MB are 30)
  const int64_t queries = std::max(rows - sequences * far, rows / 4);
  while (queries / plan.chunk * kv_heads * plan.sink_blocks > kFarWaves) plan.chunk *= 2;
  plan.places = rows / plan.chunk + std::min(sequences, rows / far);
  plan.bytes = plan.places * kv_heads * plan.sink_blocks * far_bytes_of(head_dim);
  return plan.bytes > kMostFarBytes ? FarPlan{} : plan;                  // (so many sequences may be long that there are tiles enough without)
}
// Into how many pieces the work of a tile of keys is cut at most.  Pieces cost the way of their sums, 128 KB for heads of 128, through memory and one more
// launch; they pay where the turns of the longest tile are more, by 8 (with heads of 128, whose turns are of 32 queries, by 4 and a 6th of the workgroups), than a 256th part of all turns, of which a sequence's begin has half.  Measured, with
// pieces and without, one sequence, 32 on 8 heads of 128: 2048 rows 211 and 344 us, 6000 1092 and 1233, 8192 2019 and 2001; with a window of 512: 1000 rows 89
// and 121, 2048 117 and 131, 3000 182 and 170, 6000 262 and 230; 12 heads of 64: 3300 rows 136 and 143, 5000 257 and 246, with a window of 256 64 and 44.
struct PiecePlan {
  int pieces;
  int64_t bytes;
};
constexpr int64_t kMostPieces = 32, kMostPieceBytes = (int64_t)256 << 20;
int64_t piece_bytes_of(int head_dim) { return 2 * kRows * head_dim * (int64_t)sizeof(float); }
int64_t turns_of(int64_t queries, int group, int head_dim) { return (queries + 63) / 64 * (head_dim > 96 ? 2 : 1) * group; }
PiecePlan piece_plan(int64_t rows, int64_t tiles, int q_heads, int kv_heads, int head_dim, int64_t window, int64_t sinks, bool far) {
  const bool whole = window == 0 || window >= rows;
  const int64_t queries = whole || (sinks > 0 && !far) ? rows : std::min(rows, window + kRows);
  const int group = q_heads / kv_heads;
  const int64_t turns = turns_of(queries, group, head_dim), workgroups = tiles * kv_heads;
  const int64_t each = turns_of(whole ? rows / 2 : std::min(rows, window + kRows) * (2 * rows - window) / (2 * rows), group, head_dim);
  if (turns - workgroups * each / 256 < (head_dim > 96 ? 4 + workgroups / 6 : 8)) return {1, 0};
  const int64_t bytes = workgroups * piece_bytes_of(head_dim);
  const int64_t pieces = std::min<int64_t>({(turns - 1) / kLeastTurns + 1, kMostPieceBytes / bytes, kMostPieces});
  return pieces < 2 ? PiecePlan{1, 0} : PiecePlan{(int)pieces, bytes * pieces};
}
int64_t stats_bytes(int64_t rows, int q_heads) { return (2 * rows * q_heads * (int64_t)sizeof(float) + 15) / 16 * 16; }

}  // namespace

int64_t daf_window_attention_backward_workspace_size(int64_t rows, int q_heads, int kv_heads, int head_dim, int64_t sequences, int64_t window, int64_t sinks) {
  const int64_t tiles = rows / kRows + sequences;                         // (as many as there can be, with q_starts or without)
  const FarPlan far = far_plan(rows, kv_heads, head_dim, sequences, window, sinks);
  return stats_bytes(rows, q_heads) + far.bytes + piece_plan(rows, tiles, q_heads, kv_heads, head_dim, window, sinks, far.places > 0).bytes;
}
// No less than that for these rows and sequences, nor for fewer: there are rules by which fewer have work cut into more pieces.
int64_t daf_window_attention_backward_workspace_bound(int64_t rows, int q_heads, int kv_heads, int head_dim, int64_t sequences, int64_t window, int64_t sinks) {
  const bool whole = window == 0 || window >= rows;
  int64_t far_bytes = 0;
  if (sinks > 0 && sinks <= kRows && !whole) {
    const int64_t far = first_far(window), units = kv_heads * ((sinks + 31) / 32);
    // (chunks of the rows: a 4th of the rows at least are counted when their size is chosen, for kFarWaves / units chunks of these or less)
    if (rows >= 3 * far) far_bytes = (std::min(rows / kLeastChunk, 4 * (kFarWaves / units + 1)) + std::min(sequences, rows / far)) * units * far_bytes_of(head_dim);
  }
  const int64_t turns = turns_of(whole || sinks > 0 ? rows : std::min(rows, window + kRows), q_heads / kv_heads, head_dim);
  const int64_t pieces = std::min<int64_t>((turns - 1) / kLeastTurns + 1, kMostPieces);
  const int64_t piece_bytes = pieces < 2 ? 0 : (rows / kRows + sequences) * kv_heads * piece_bytes_of(head_dim) * pieces;
  return stats_bytes(rows, q_heads) + std::min(far_bytes, kMostFarBytes) + std::min(piece_bytes, kMostPieceBytes);
}

hipError_t daf_launch_window_attention_backward(const daf_window_attention_t& p, const AttentionTensors& t, const AttentionGradients& g, char* workspace,
                                                hipStream_t stream) {
  if (p.q_rows == 0) return hipSuccess;
  Backward a = {};
  static_cast<Attention&>(a) = attention_of(p, t);
  a.grad_out = heads_of(g.grad_out, p.q_rows);
  a.grad_q = heads_of(g.grad_q, p.q_rows);
  a.grad_k = heads_of(g.grad_k, p.q_rows);
  a.grad_v = heads_of(g.grad_v, p.q_rows);
  a.n = reinterpret_cast<float*>(workspace);
  a.minus_delta = a.n + p.q_rows * p.q_heads;
  const FarPlan far = far_plan(p.q_rows, p.kv_heads, p.head_dim, p.sequences, p.window, p.sinks);
  if (far.places > 0) a.sums = reinterpret_cast<float*>(workspace + stats_bytes(p.q_rows, p.q_heads));
  a.sink_blocks = far.sink_blocks;
  a.far = far.far;
  a.chunk = far.chunk;
  a.places = far.places;
  const int64_t tiles = p.q_rows / kRows + p.sequences;
  const PiecePlan pieces = piece_plan(p.q_rows, tiles, p.q_heads, p.kv_heads, p.head_dim, p.window, p.sinks, far.places > 0);
  a.parts = reinterpret_cast<float*>(workspace + stats_bytes(p.q_rows, p.q_heads) + far.bytes);
  a.pieces = pieces.pieces;
  with_padded_dim(p, [&](auto dt, auto dp) {
    const int64_t few = few_tiles(p, tiles);
    if (few > 0) k_attention_grad_q_few<dt.value, dp.value><<<workgroups_of(few, p.kv_heads, a.group), kWaves * kWave, 0, stream>>>(a, (int)few);
    else k_attention_grad_q<dt.value, dp.value><<<workgroups_of(tiles, p.kv_heads, a.group), kWaves * kWave, 0, stream>>>(a, (int)tiles);
    if (far.places > 0) {
      const unsigned units = (unsigned)(far.places * p.kv_heads * far.sink_blocks);
      k_attention_grad_sinks<dt.value, dp.value><<<units, kWave, 0, stream>>>(a);
      const bool by_place = p.sequences > far.places;
      const unsigned sums = by_place ? units : (unsigned)(p.sequences * p.kv_heads * far.sink_blocks);
      k_attention_sinks_sum<<<dim3(sums, (unsigned)((p.head_dim * 64 + 1023) / 1024)), 256, 0, stream>>>(a, by_place);
    }
    const unsigned all = (unsigned)(tiles * p.kv_heads);
    if (a.pieces == 1) {
      k_attention_grad_kv<dt.value, dp.value, false><<<workgroups_of(tiles, p.kv_heads, 1), kWaves * kWave, 0, stream>>>(a, (int)tiles);
    } else {
      k_attention_grad_kv<dt.value, dp.value, true><<<all * (unsigned)a.pieces, kWaves * kWave, 0, stream>>>(a, (int)tiles);
      k_attention_kv_sum<dt.value, dp.value><<<dim3(all, all >= 256 ? 2 : all >= 128 ? 4 : 8, 2), kWaves * kWave, 0, stream>>>(a, (int)tiles);
    }
  });
  return hipGetLastError();
}

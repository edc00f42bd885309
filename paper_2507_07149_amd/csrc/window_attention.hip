// Attention with a window and sinks, forward (daf_window_attention).
//
//   s = q . k, p = 2^(c s - m), l = sum of p, o = sum of p v;  out = o / l, lse = (m + log2 l) ln 2        c = scale log2(e)
//
// A workgroup has 128 queries of a head, a wave 32 of them, and goes once over the 32-key tiles that they see, the next tile on its way into LDS meanwhile.
// Scores come out as keys x queries, so that a lane has a query: its maximum and sum need one exchange between two lanes, and p, rounded, is the next
// product's operand as it lies in the registers (window_attention_tiles.h); o is collected as elements x queries.  m follows the maximum only once it is more
// than 8 behind: o is then multiplied by 2^(m' - m), which few tiles need; p is at most 2^8 meanwhile.
// Only tiles at the edges of what a wave sees are masked, and those that it sees nothing of are left out.
// Tiles of 32 keys need 168 registers with heads of 128 (so many that three waves fit a SIMD): while one wave's exponentials run, the others' products do; tiles of 64 leave
// room for two waves, and were slower.  Rows whose scores lie beyond 2^24, or in whose products an infinity or NaN meets a 0, are done again row by row (attend_row).
// 16 sequences of 2048 rows, 32 on 8 heads of 128, a window of 1024: 488 us, 845 TFLOP/s; 32768 rows, a window of 4096: 1.86 ms, 1.11 PFLOP/s.  32768 rows of such heads
// take, whatever their sequences and windows, 98 us for their workgroups' begins and ends (queries in, rows out) and 55 ns for every tile of keys that a head's workgroups go over,
// which is 1.2 PFLOP/s for all 32 heads at 1.7 GHz, the clock that power leaves; tiles at the window's edges, of which a part is masked, take as long as others.
#include "window_attention_tiles.h"

namespace {

constexpr int kKeys = 32, kWaves = 4, kQueries = 32, kRows = kWaves * kQueries;
constexpr float kBehind = 8.0f;

template <int DT, int DP>
__global__ __launch_bounds__(kWaves * kWave, 3) void k_window_attention(const Attention a, int tiles) {
  using S = TileShape<DP>;
  constexpr int kBytes = tile_bytes<DP>(kKeys);
  __shared__ __attribute__((aligned(16))) char lds[4 * kBytes];        // keys, values; twice
  const Turn turn = turn_of_workgroup(tiles, a.kv_heads, a.group);
  const TileOf at = find_tile<kRows, false>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  const int begin = at.tile * kRows, end = min(s.queries, begin + kRows);
  const KeyTiles<kKeys> keys(a, s.position(begin), s.position(end - 1));

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  const int kv_head = turn.head / a.group;
  TileWalk<DP, kKeys, kWaves> k_walk, v_walk;
  k_walk.begin(a.k, s.k_begin, kv_head, a.dim);
  v_walk.begin(a.v, s.k_begin, kv_head, a.dim);
  keys.walk(k_walk, s.keys);
  keys.walk(v_walk, s.keys);
  auto fetch = [&](int t, int stage) {
    const bool jumps = t == keys.sinks && t > 0, last = t + 1 == keys.count;
    k_walk.next(lds0 + stage * kBytes, jumps, last);
    v_walk.next(lds0 + (2 + stage) * kBytes, jumps, last);
  };
  if (keys.count > 0) fetch(0, 0);

  // the wave's queries: a column to a lane (those behind the end are the last one again)
  const int wave = uniform(threadIdx.x / kWave), li = threadIdx.x & 31;
  const int first = begin + wave * kQueries, i = min(first + li, end - 1);
  const int position = s.position(i), first_position = s.position(first), last_position = s.position(min(first + kQueries, end) - 1);
  u32x4 q[S::kSteps];
  load_columns<DP>(a.q.at + ((int64_t)s.q_begin + i) * a.q.token + turn.head * a.q.head, a.dim, a.scale < 0.0f, q);
  const float c = exponent_factor(a.scale);
  const KeyView<kKeys> view(a, keys, first_position, first < end ? last_position : -1);

  const ReadAlong<kKeys> k_read((lds_char*)lds);
  const ReadAcross<kKeys> v_read((lds_char*)lds + 2 * kBytes);
  f32x16 o[S::kBlocks];
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] = 0.0f;
  float m = kLowest, l = 0.0f;

  auto tile = [&](int key, Seen seen, auto stage_constant) {
    constexpr int kStage = decltype(stage_constant)::value * kBytes;
    f32x16 p;
    u32x4 k[S::kSteps], v[2][S::kBlocks];
    constexpr int kAhead = 4;
#pragma unroll
    for (int x = 0; x < kAhead && x < S::kSteps; ++x) k[x] = k_read.read(kStage, 0, x);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < S::kSteps; ++x) {
      p = mfma16<DT>(k[x], q[x], p);
      if (x + kAhead < S::kSteps) k[x + kAhead] = k_read.read(kStage, 0, x + kAhead);
    }
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) v[0][b] = v_read.read(kStage, b, 0);
    __builtin_amdgcn_sched_barrier(0);
    if (seen == kPart) {
      const RowsSeen rows = keys_seen(a, position, key);
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = rows.at(row_of_register(r)) ? p[r] : -INFINITY;
    }
    float high[2] = {largest(p[0], p[1]), largest(p[2], p[3])};
#pragma unroll
    for (int r = 4; r < 16; r += 4) {
      high[0] = largest(largest(high[0], p[r]), p[r + 1]);
      high[1] = largest(largest(high[1], p[r + 2]), p[r + 3]);
    }
    float top = largest(high[0], high[1]);
    top = largest(top, from_other_half(top)) * c;
    if (__any(top > m + kBehind)) {
      const float to = fmaxf(m, top), shrink = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= shrink;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] *= shrink;
    }
    u32x4 w[2];
    float sum[2] = {0.0f, 0.0f};
    auto exponentials = [&](int h) {
#pragma unroll
      for (int x = 8 * h; x < 8 * h + 8; x += 2) {
        float e[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          e[y] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[x + y], c, -m));
          sum[y] += e[y];
        }
        w[h][(x & 7) >> 1] = narrow_pair<DT>(e[0], e[1]);
      }
    };
    exponentials(0);
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) v[1][b] = v_read.read(kStage, b, 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) o[b] = mfma16<DT>(v[0][b], w[0], o[b]);
    exponentials(1);
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) o[b] = mfma16<DT>(v[1][b], w[1], o[b]);
    l += sum[0] + sum[1];
  };
  int key = keys.first_key();
  auto turn_tile = [&](int t, auto stage_constant) {
    wait_tile();
    tile_barrier();
    if (t + 1 < keys.count) fetch(t + 1, 1 - decltype(stage_constant)::value);
    const Seen seen = view.of(t, keys.sinks, key);
    if (seen != kNothing) tile(key, seen, stage_constant);
    key = t + 1 == keys.sinks ? keys.low * kKeys : key + kKeys;
  };
  for (int t = 0; t < keys.count; t += 2) {
    turn_tile(t, std::integral_constant<int, 0>{});
    if (t + 1 < keys.count) turn_tile(t + 1, std::integral_constant<int, 1>{});
  }
  if (first >= end) return;
  l += from_other_half(l);
  const int query = first + column_again(), to_row = min(query, end - 1);
  const bool mine = query < end, any = s.position(to_row) >= 0;
  const int64_t row = (int64_t)s.q_begin + to_row;
  uint32_t again = columns_to_do_again(o, mine && any) | far_columns(m, mine && any);
  const float by = any ? 1.0f / l : 0.0f;
  char* const out = a.out.at + row * a.out.token + turn.head * a.out.head;
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b) {
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] = any ? o[b][r] : 0.0f;
    store_column_block<DT>(out, b, a.dim, mine, o[b], by);
  }
  if (a.lse != nullptr && mine && (threadIdx.x & 32) == 0)
    a.lse[(int64_t)turn.head * a.q_rows + row] = any ? (m + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  while (again != 0) {
    const int x = __builtin_ctz(again);
    again &= again - 1;
    attend_row<DT>(a, s, first + x, turn.head);
  }
}

// The same for few queries: 32 of them to a workgroup, whose waves take every fourth tile of keys each, alone, and join what they have at the end.
template <int DT, int DP>
__global__ __launch_bounds__(kWaves * kWave, 1) void k_window_attention_few(const Attention a, int tiles) {
  using S = TileShape<DP>;
  constexpr int kTile = tile_bytes<DP>(kKeys), kStage = 2 * kTile, kOwn = 2 * kStage;
  __shared__ __attribute__((aligned(16))) char lds[kWaves * kOwn];        // of each wave: keys and values, twice; its sums in the end
  __shared__ float tops[kWaves][kQueries], totals[kWaves][kQueries];
  __shared__ uint32_t bad;
  const Turn turn = turn_of_workgroup(tiles, a.kv_heads, a.group);
  const TileOf at = find_tile<kQueries, false>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  const int first = at.tile * kQueries, last = min(s.queries, first + kQueries) - 1;
  const KeyTiles<kKeys> keys(a, s.position(first), s.position(last));
  const int wave = uniform(threadIdx.x / kWave), li = threadIdx.x & 31, i = min(first + li, last), position = s.position(i);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds + (uint32_t)wave * kOwn;
  TileFeed<DP, kKeys, 1> k_feed, v_feed;
  k_feed.begin(a.k, s.k_begin, turn.head / a.group, a.dim);
  v_feed.begin(a.v, s.k_begin, turn.head / a.group, a.dim);
  auto fetch = [&](int t, int stage) {
    k_feed.fetch_of_wave(lds0 + stage * kStage, keys.key(t), s.keys);
    v_feed.fetch_of_wave(lds0 + stage * kStage + kTile, keys.key(t), s.keys);
  };
  if (wave < keys.count) fetch(wave, 0);
  const int64_t row = (int64_t)s.q_begin + i;
  u32x4 q[S::kSteps];
  load_columns<DP>(a.q.at + row * a.q.token + turn.head * a.q.head, a.dim, a.scale < 0.0f, q);
  const float c = exponent_factor(a.scale);
  const ReadAlong<kKeys> k_read((lds_char*)lds + wave * kOwn);
  const ReadAcross<kKeys> v_read((lds_char*)lds + wave * kOwn + kTile);
  const KeyView<kKeys> view(a, keys, s.position(first), s.position(last));
  f32x16 o[S::kBlocks];
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] = 0.0f;
  float m = kLowest, l = 0.0f;
  int stage = 0;
  for (int t = wave; t < keys.count; t += kWaves, stage ^= 1) {
    const int from = stage * kStage, key = keys.key(t);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                   // the next tile's place has been read
    if (t + kWaves < keys.count) {
      fetch(t + kWaves, 1 - stage);
      wait_but<2 * TileFeed<DP, kKeys, 1>::kLoads>();
    } else {
      wait_tile();
    }
    f32x16 p;
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < S::kSteps; ++x) p = mfma16<DT>(k_read.read(from, 0, x), q[x], p);
    if (view.of(t, keys.sinks, key) != kAll) {
      const RowsSeen rows = keys_seen(a, position, key);
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = rows.at(row_of_register(r)) ? p[r] : -INFINITY;
    }
    float top = p[0];
#pragma unroll
    for (int r = 1; r < 15; r += 2) top = largest(largest(top, p[r]), p[r + 1]);
    top = largest(top, p[15]);
    top = largest(top, from_other_half(top)) * c;
    if (__any(top > m + kBehind)) {
      const float to = fmaxf(m, top), shrink = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= shrink;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] *= shrink;
    }
    u32x4 w[2];
#pragma unroll
    for (int x = 0; x < 16; x += 2) {
      float e[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        e[y] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[x + y], c, -m));
        l += e[y];
      }
      w[x >> 3][(x & 7) >> 1] = narrow_pair<DT>(e[0], e[1]);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) o[b] = mfma16<DT>(v_read.read(from, b, x), w[x], o[b]);
  }
  // the waves' parts, all in terms of the largest m
  l += from_other_half(l);
  if ((threadIdx.x & 32) == 0) tops[wave][li] = m;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  const float high = fmaxf(fmaxf(tops[0][li], tops[1][li]), fmaxf(tops[2][li], tops[3][li])), shrink = __builtin_amdgcn_exp2f(m - high);
  if ((threadIdx.x & 32) == 0) totals[wave][li] = l * shrink;
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] *= shrink;
  add_up<S::kBlocks, kOwn>(lds, o);                                      // (with a barrier)
  l = (totals[0][li] + totals[1][li]) + (totals[2][li] + totals[3][li]);
  const bool mine = first + li <= last, any = position >= 0;
  if (wave < S::kBlocks) {
    const uint32_t again = columns_to_do_again({o[0]}, mine && any) | far_columns(high, mine && any);
    if (again != 0 && (threadIdx.x & 63) == 0) atomicOr(&bad, again);
#pragma unroll
    for (int r = 0; r < 16; ++r) o[0][r] = any ? o[0][r] : 0.0f;
    store_column_block<DT>(a.out.at + row * a.out.token + turn.head * a.out.head, wave, a.dim, mine, o[0], any ? 1.0f / l : 0.0f);
  }
  if (a.lse != nullptr && wave == 0 && mine && (threadIdx.x & 32) == 0)
    a.lse[(int64_t)turn.head * a.q_rows + row] = any ? (high + __builtin_amdgcn_logf(l)) * kLn2 : -INFINITY;
  __threadfence_block();                                                 // (rows that are done again)
  __syncthreads();
  uint32_t again = bad;
  for (int n = 0; again != 0; ++n) {
    const int x = __builtin_ctz(again);
    again &= again - 1;
    if (n % kWaves == wave) attend_row<DT>(a, s, first + x, turn.head);
  }
}

}  // namespace

hipError_t daf_launch_window_attention(const daf_window_attention_t& p, const AttentionTensors& t, hipStream_t stream) {
  if (p.q_rows == 0) return hipSuccess;
  const Attention a = attention_of(p, t);
  const int64_t tiles = most_tiles(p, kRows);
  const int64_t few = few_tiles(p, tiles);
  with_padded_dim(p, [&](auto dt, auto dp) {
    if (few > 0) k_window_attention_few<dt.value, dp.value><<<workgroups_of(few, p.kv_heads, a.group), kWaves * kWave, 0, stream>>>(a, (int)few);
    else k_window_attention<dt.value, dp.value><<<workgroups_of(tiles, p.kv_heads, a.group), kWaves * kWave, 0, stream>>>(a, (int)tiles);
  });
  return hipGetLastError();
}

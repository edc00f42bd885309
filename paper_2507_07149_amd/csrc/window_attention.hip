// Attention with a window and sinks, forward (daf_window_attention).
//
//   s = q . k, p = 2^(c s - m), l = sum of p, o = sum of p v;  out = o / l, lse = (m + log2 l) ln 2        c = scale log2(e)
//
// A workgroup has 128 queries of a head, a wave 32 of them, and goes once over the 64-key tiles that they see, the next tile on its way into LDS meanwhile.
// Scores come out as keys x queries, so that a lane has a query: its maximum and sum need one exchange between two lanes, and p, rounded, is the next
// product's operand as it lies in the registers (window_attention_tiles.h); o is collected as elements x queries.  m follows the maximum only once it is more
// than 8 behind: o is then multiplied by 2^(m' - m), which few tiles need; p is at most 2^8 meanwhile.
// Only tiles at the edges of what a wave sees are masked, and those that it sees nothing of are left out.
#include "window_attention_tiles.h"

namespace {

constexpr int kWaves = 4, kQueries = 32, kRows = kWaves * kQueries;
constexpr float kBehind = 8.0f;

template <int DT, int DP>
__global__ __launch_bounds__(kWaves * kWave, 2) void k_window_attention(const Attention a, int tiles) {
  using S = TileShape<DP>;
  __shared__ __attribute__((aligned(16))) char lds[4 * S::kBytes];        // keys, values; twice
  const Turn turn = turn_of_workgroup(tiles);
  const TileOf at = find_tile<kRows>(a, turn.tile);
  if (at.sequence < 0) return;
  const Sequence s = sequence_of(a, at.sequence);
  const int begin = at.tile * kRows, end = min(s.queries, begin + kRows);
  const KeyTiles keys(a, s.position(begin), s.position(end - 1));

  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  const int kv_head = turn.head / a.group;
  TileFeed<DP, kTileRows, kWaves> k_feed, v_feed;
  k_feed.begin(a.k, s.k_begin, kv_head, a.dim);
  v_feed.begin(a.v, s.k_begin, kv_head, a.dim);
  auto fetch = [&](int t, int stage) {
    k_feed.fetch(lds0 + stage * S::kBytes, keys.key(t), s.keys);
    v_feed.fetch(lds0 + (2 + stage) * S::kBytes, keys.key(t), s.keys);
  };
  if (keys.count > 0) fetch(0, 0);

  // the wave's queries: a column to a lane (those behind the end are the last one again)
  const int wave = uniform(threadIdx.x / kWave), li = threadIdx.x & 31;
  const int first = begin + wave * kQueries, i = min(first + li, end - 1);
  const int position = s.position(i), first_position = s.position(first), last_position = s.position(min(first + kQueries, end) - 1);
  const int64_t row = (int64_t)s.q_begin + i;
  u32x4 q[S::kSteps];
  load_columns<DP>(a.q.at + row * a.q.token + turn.head * a.q.head, a.dim, a.scale < 0.0f, q);
  const float c = exponent_factor(a.scale);

  const ReadAlong<DP> k_read((lds_char*)lds);
  const ReadAcross<DP> v_read((lds_char*)lds + 2 * S::kBytes);
  f32x16 o[S::kBlocks];
#pragma unroll
  for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] = 0.0f;
  float m = kLowest, l = 0.0f;

  auto tile = [&](int key, Seen seen, auto stage_constant) {
    constexpr int kStage = decltype(stage_constant)::value * S::kBytes;
    f32x16 p[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) p[b][r] = 0.0f;
#pragma unroll
      for (int x = 0; x < S::kSteps; ++x) p[b] = mfma16<DT>(k_read.read(kStage, b, x), q[x], p[b]);
    }
    if (seen == kPart) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) p[b][r] = sees(a, position, key + b * 32 + row_of_register(r)) ? p[b][r] : -INFINITY;
    }
    float top = p[0][0];
#pragma unroll
    for (int r = 1; r < 31; r += 2) top = largest(largest(top, p[r >> 4][r & 15]), p[(r + 1) >> 4][(r + 1) & 15]);
    top = largest(top, p[1][15]);
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
    u32x4 w[4];
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < 32; x += 2) {
      float e[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        e[y] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[x >> 4][(x & 15) + y], c, -m));
        sum[y] += e[y];
      }
      w[x >> 3][(x & 7) >> 1] = narrow_pair<DT>(e[0], e[1]);
    }
    l += sum[0] + sum[1];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) o[b] = mfma16<DT>(v_read.read(kStage, b, x), w[x], o[b]);
  };
  auto turn_tile = [&](int t, auto stage_constant) {
    wait_tile();
    tile_barrier();
    if (t + 1 < keys.count) fetch(t + 1, 1 - decltype(stage_constant)::value);
    const int key = keys.key(t);
    const Seen seen = first < end ? seen_of(a, first_position, last_position, key) : kNothing;
    if (seen != kNothing) tile(key, seen, stage_constant);
  };
  for (int t = 0; t < keys.count; t += 2) {
    turn_tile(t, std::integral_constant<int, 0>{});
    if (t + 1 < keys.count) turn_tile(t + 1, std::integral_constant<int, 1>{});
  }
  if (first >= end) return;

  l += from_other_half(l);
  const bool mine = first + li < end, any = position >= 0;
  uint32_t again = columns_to_do_again(o, mine && any);
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

}  // namespace

hipError_t daf_launch_window_attention(const daf_window_attention_t& p, const AttentionTensors& t, hipStream_t stream) {
  if (p.q_rows == 0) return hipSuccess;
  const Attention a = attention_of(p, t);
  const int64_t tiles = most_tiles(p, kRows);
  const unsigned blocks = (unsigned)(tiles * p.q_heads);
  with_padded_dim(p, [&](auto dt, auto dp) { k_window_attention<dt.value, dp.value><<<blocks, kWaves * kWave, 0, stream>>>(a, (int)tiles); });
  return hipGetLastError();
}

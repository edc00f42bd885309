// Attention with a window and sinks for one query of each of many sequences (daf_window_attention_step).
//
// What it costs is one read of the keys and values that are seen.  All heads that share a key head see the same of them: they are the columns of a wave's
// products, 32 at a time, and a wave goes alone (no barriers) over a piece of a sequence's tiles of 32 keys, two tiles on their way into LDS, 32 KB for heads
// of 128.  Tiles begin where what is seen begins (the sinks, then the window) and end where it ends, so nothing else is read.  Pieces are joined by
// k_attention_join: o and l of each, times 2^(2 c (m - the largest m)).  m is half the largest q . k, without the factor c: what m c is rounded by would be the exponent of
// the largest exponential, and where scores are large that is none that an exponential has.  (Half: the distance of two products may be none of binary32's numbers.)
// Measured (bfloat16, 32 on 8 heads of 128): 64 sequences of 8192 to 16384 tokens, a window of 4096: 211 us, 5.1 TB/s; one sequence of 8191 13.4 us, of which the join 3.9.
#include <algorithm>
#include <cfloat>

#include "window_attention_tiles.h"

namespace {

constexpr int kKeys = 32, kHeads = 32;

struct Step : Attention {
  int pieces, head_blocks;     // of a sequence; of the heads that share a key head
  float *m_l, *o;              // [sequences, q_heads, pieces]: m and l; elements
};

constexpr float kNoScore = -FLT_MAX / 2;             // (half of a product is no less)
__device__ __forceinline__ float twice_factor(float scale) { return fminf(2.0f * exponent_factor(scale), FLT_MAX); }

// The tiles of a sequence: `sinks` of them, then the window's.
struct StepTiles {
  int keys, low, sink_keys, sinks, count;
  __device__ __forceinline__ StepTiles(const Attention& a, int keys_of) {
    keys = keys_of;
    low = window_begin(a, keys - 1);
    sink_keys = min(a.sinks, low);
    sinks = (sink_keys + kKeys - 1) / kKeys;
    count = keys == 0 ? 0 : sinks + (keys - low + kKeys - 1) / kKeys;
  }
  __device__ __forceinline__ int each(int pieces) const { return (count + pieces - 1) / pieces; }        // tiles of a piece
  __device__ __forceinline__ int row(int t) const { return t < sinks ? t * kKeys : low + (t - sinks) * kKeys; }
  __device__ __forceinline__ int end(int t) const { return t < sinks ? sink_keys : keys; }
};

template <int DT, int DP>
__global__ __launch_bounds__(kWave, 2) void k_attention_step(const Step a) {
  using S = TileShape<DP>;
  constexpr int kTile = tile_bytes<DP>(kKeys), kStage = 2 * kTile;
  __shared__ __attribute__((aligned(16))) char lds[2 * kStage];
  const unsigned unit = blockIdx.x / (unsigned)a.pieces;
  const int piece = (int)(blockIdx.x % (unsigned)a.pieces);
  const int block = (int)(unit % (unsigned)a.head_blocks), kv_head = (int)(unit / (unsigned)a.head_blocks % (unsigned)a.kv_heads);
  const int b = (int)(unit / (unsigned)a.head_blocks / (unsigned)a.kv_heads);
  const int k_begin = uniform(within(a.k_starts[b], 0, a.k_rows));
  const StepTiles tiles(a, uniform(within(a.k_lengths[b], 0, a.k_rows - k_begin)));
  const int each = tiles.each(a.pieces), first = piece * each, last = min(first + each, tiles.count);
  if (first >= last && piece > 0) return;

  const int li = threadIdx.x & 31, lg = threadIdx.x >> 5;
  const bool mine = block * kHeads + li < a.group;
  const int head = kv_head * a.group + min(block * kHeads + li, a.group - 1);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char*)lds;
  TileFeed<DP, kKeys, 1> k_feed, v_feed;
  k_feed.begin(a.k, k_begin, kv_head, a.dim);
  v_feed.begin(a.v, k_begin, kv_head, a.dim);
  auto fetch = [&](int t, int stage) {
    k_feed.fetch(lds0 + stage * kStage, tiles.row(t), tiles.end(t));
    v_feed.fetch(lds0 + stage * kStage + kTile, tiles.row(t), tiles.end(t));
  };
  u32x4 q[S::kSteps];
  load_columns<DP>(a.q.at + b * a.q.token + head * a.q.head, a.dim, a.scale < 0.0f, q);
  if (first < last) fetch(first, 0);
  const float twice_c = twice_factor(a.scale);
  const ReadAlong<kKeys> k_read((lds_char*)lds);
  const ReadAcross<kKeys> v_read((lds_char*)lds + kTile);
  f32x16 o[S::kBlocks];
#pragma unroll
  for (int d = 0; d < S::kBlocks; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  float m = kNoScore, l = 0.0f;

  auto turn_tile = [&](int t, auto stage_constant) {
    constexpr int kAt = decltype(stage_constant)::value * kStage;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                   // the next tile's place has been read
    if (t + 1 < last) {
      fetch(t + 1, 1 - decltype(stage_constant)::value);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * TileFeed<DP, kKeys, 1>::kLoads) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    f32x16 p;
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < S::kSteps; ++x) p = mfma16<DT>(k_read.read(kAt, 0, x), q[x], p);
    const int there = tiles.end(t) - tiles.row(t);
    if (there < kKeys) {
      const int rows = there - first_row();
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = row_of_register(r) < rows ? p[r] : -INFINITY;
    }
    float top = p[0];
#pragma unroll
    for (int r = 1; r < 15; r += 2) top = largest(largest(top, p[r]), p[r + 1]);
    top = largest(top, p[15]);
    top = largest(top, from_other_half(top)) * 0.5f;
    if (__any(top > m)) {
      const float to = fmaxf(m, top), shrink = __builtin_amdgcn_exp2f((m - to) * twice_c);
      m = to;
      l *= shrink;
#pragma unroll
      for (int d = 0; d < S::kBlocks; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= shrink;
    }
    u32x4 w[2];
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int x = 0; x < 16; x += 2) {
      float e[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        e[y] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[x + y], 0.5f, -m) * twice_c);
        sum[y] += e[y];
      }
      w[x >> 3][(x & 7) >> 1] = narrow_pair<DT>(e[0], e[1]);
    }
    l += sum[0] + sum[1];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int d = 0; d < S::kBlocks; ++d) o[d] = mfma16<DT>(v_read.read(kAt, d, x), w[x], o[d]);
  };
  for (int t = first; t < last; t += 2) {
    turn_tile(t, std::integral_constant<int, 0>{});
    if (t + 1 < last) turn_tile(t + 1, std::integral_constant<int, 1>{});
  }
  l += from_other_half(l);

  if (a.pieces == 1) {
    const bool any = tiles.count > 0;
    char* const out = a.out.at + b * a.out.token + head * a.out.head;
#pragma unroll
    for (int d = 0; d < S::kBlocks; ++d) store_column_block<DT>(out, d, a.dim, mine, o[d], any ? 1.0f / l : 0.0f);
    return;
  }
  if (!mine) return;
  const int64_t at = ((int64_t)b * a.q_heads + head) * a.pieces + piece;
  if (lg == 0) {
    a.m_l[2 * at] = m;
    a.m_l[2 * at + 1] = l;
  }
#pragma unroll
  for (int d = 0; d < S::kBlocks; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int e = 32 * d + 8 * g + 4 * lg;
      if (e < a.dim) *reinterpret_cast<f32x4*>(a.o + at * a.dim + e) = f32x4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    }
}

// A workgroup to a head of a sequence: a thread to a piece for the weights, then four elements to a thread and every eighth piece, eight on their way.
constexpr int kJoinThreads = 256, kSlices = kJoinThreads / (kAttentionMaxDim / 4);
template <int DT>
__global__ __launch_bounds__(kJoinThreads) void k_attention_join(const Step a) {
  __shared__ float weights[kJoinThreads], waves[2][kJoinThreads / kWave];
  __shared__ f32x4 sums[kSlices][kAttentionMaxDim / 4];
  const int b = blockIdx.x, head = blockIdx.y, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int k_begin = uniform(within(a.k_starts[b], 0, a.k_rows));
  const StepTiles tiles(a, uniform(within(a.k_lengths[b], 0, a.k_rows - k_begin)));
  const int each = tiles.each(a.pieces), pieces = each == 0 ? 0 : (tiles.count + each - 1) / each;
  const int64_t first = ((int64_t)b * a.q_heads + head) * a.pieces;
  const int group = threadIdx.x % (kAttentionMaxDim / 4), slice = threadIdx.x / (kAttentionMaxDim / 4);
  float m = kNoScore, l = 0.0f;
  if ((int)threadIdx.x < pieces) {                                       // (at most kMostPieces)
    m = a.m_l[2 * (first + threadIdx.x)];
    l = a.m_l[2 * (first + threadIdx.x) + 1];
  }
  float high = m;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) high = largest(high, __shfl_xor(high, d, kWave));
  if (lane == 0) waves[0][wave] = high;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinThreads / kWave; ++w) high = largest(high, waves[0][w]);
  const float weight = __builtin_amdgcn_exp2f((m - high) * twice_factor(a.scale));
  weights[threadIdx.x] = weight;
  const float part = wave_sum(weight * l);
  if (lane == 0) waves[1][wave] = part;
  __syncthreads();
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  if (4 * group < a.dim) {
    const float* const from = a.o + first * a.dim + 4 * group;
#pragma unroll 8
    for (int i = slice; i < pieces; i += kSlices) {
      const f32x4 o = *reinterpret_cast<const f32x4*>(from + (int64_t)i * a.dim);
#pragma unroll
      for (int r = 0; r < 4; ++r) sum[r] = __builtin_fmaf(weights[i], o[r], sum[r]);
    }
  }
  sums[slice][group] = sum;
  __syncthreads();
  if (slice != 0 || 4 * group >= a.dim) return;
  float total = 0.0f;
#pragma unroll
  for (int w = 0; w < kJoinThreads / kWave; ++w) total += waves[1][w];
#pragma unroll
  for (int i = 1; i < kSlices; ++i) sum += sums[i][group];
  const float by = tiles.count > 0 ? 1.0f / total : 0.0f;
  u32x2 out;
  out.x = narrow_pair<DT>(sum[0] * by, sum[1] * by);
  out.y = narrow_pair<DT>(sum[2] * by, sum[3] * by);
  *reinterpret_cast<u32x2*>(a.out.at + b * a.out.token + head * a.out.head + group * 8) = out;
}

constexpr int kMostPieces = kJoinThreads;
// Into how many pieces sequences are cut: enough for two waves to a compute unit, of two tiles at least, and, where sequences may be of very different lengths,
// pieces of ten tiles as long as there are not more than 8192 of them; none where a sequence has so few tiles that the join costs more.  Measured, 32 on 8 heads,
// a window of 160 keys (5 tiles), one piece and pieces of two tiles: 1 sequence, heads of 128 7.8 and 8.6 us, 64 sequences 9.7 and 16.8; of 256 keys, one piece and
// pieces: 1 sequence 10.1 and 8.5, 16 sequences 10.5 and 9.4, 64 sequences (one piece each by this rule) 12.8 and 22.
constexpr int64_t kFill = 512, kEven = 8192, kOnePiece = 6;              // waves; waves; tiles
int64_t tiles_of(int64_t k_rows, int64_t window, int64_t sinks) {
  const int64_t most = window > 0 && window < k_rows && sinks < k_rows ? std::min(window + sinks, k_rows) : k_rows;
  return (most + kKeys - 1) / kKeys;
}
int64_t units_of(int q_heads, int kv_heads) { return kv_heads * (int64_t)((q_heads / kv_heads + kHeads - 1) / kHeads); }      // of a sequence
int pieces_of(int64_t sequences, int q_heads, int kv_heads, int64_t k_rows, int64_t window, int64_t sinks) {
  const int64_t units = sequences * units_of(q_heads, kv_heads), tiles = tiles_of(k_rows, window, sinks);
  if (tiles <= kOnePiece) return 1;
  const int64_t fill = std::min((kFill + units - 1) / units, (tiles + 1) / 2), even = std::min((kEven + units - 1) / units, tiles / 10);
  return (int)std::min<int64_t>(kMostPieces, std::max<int64_t>({1, fill, even}));
}
int64_t bytes_of(int64_t pieces, int q_heads, int head_dim) { return pieces * q_heads * (int64_t)sizeof(float) * (head_dim + 2); }

}  // namespace

int64_t daf_window_attention_step_workspace_size(int64_t sequences, int q_heads, int kv_heads, int head_dim, int64_t k_rows, int64_t window, int64_t sinks) {
  const int pieces = pieces_of(sequences, q_heads, kv_heads, k_rows, window, sinks);
  return pieces == 1 ? 0 : bytes_of(sequences * pieces, q_heads, head_dim);
}
// No less than that for these sequences and rows of the cache, nor for fewer: fewer sequences are cut into more pieces.
int64_t daf_window_attention_step_workspace_bound(int64_t sequences, int q_heads, int kv_heads, int head_dim, int64_t k_rows, int64_t window, int64_t sinks) {
  const int64_t units = units_of(q_heads, kv_heads), tiles = tiles_of(k_rows, window, sinks);
  // pieces of s sequences: s ceil(slots / (s units)) <= (slots - 1) / units + s, and none once there are `slots` units
  auto all = [&](int64_t slots, int64_t most) {
    const int64_t s = std::min(sequences, (slots - 1) / units);
    return most < 2 ? 0 : std::min((slots - 1) / units + s, s * std::min<int64_t>(most, kMostPieces));
  };
  return tiles <= kOnePiece ? 0 : bytes_of(std::max(all(kFill, (tiles + 1) / 2), all(kEven, tiles / 10)), q_heads, head_dim);
}

hipError_t daf_launch_window_attention_step(const daf_window_attention_t& p, const AttentionTensors& t, char* workspace, hipStream_t stream) {
  if (p.q_rows == 0) return hipSuccess;
  Step a = {};
  static_cast<Attention&>(a) = attention_of(p, t);
  a.pieces = pieces_of(p.sequences, p.q_heads, p.kv_heads, p.k_rows, p.window, p.sinks);
  a.head_blocks = (a.group + kHeads - 1) / kHeads;
  a.o = reinterpret_cast<float*>(workspace);                            // (first: its rows are 16 bytes, 8 elements at least)
  a.m_l = a.o + p.sequences * p.q_heads * a.pieces * (int64_t)p.head_dim;
  const unsigned blocks = (unsigned)(p.sequences * p.kv_heads * a.head_blocks * a.pieces);
  with_padded_dim(p, [&](auto dt, auto dp) {
    k_attention_step<dt.value, dp.value><<<blocks, kWave, 0, stream>>>(a);
    if (a.pieces > 1) k_attention_join<dt.value><<<dim3((unsigned)p.sequences, (unsigned)p.q_heads), kJoinThreads, 0, stream>>>(a);
  });
  return hipGetLastError();
}

// The products of the gated feed-forward block and the slopes of kept pre-activations, launched; built once for each 16-bit format (DAF_DT).
#include "gated_product.h"
#include "gated_product_large.h"
#include "gated_few_rows.h"

namespace {

constexpr int DT = DAF_DT;
using Tile128x256 = Tile<128, 256, 2, 2, 3>;
using Tile128x128 = Tile<128, 128, 2, 2, 4>;
using Tile64x128 = Tile<64, 128, 2, 2, 6>;

// da and du from what the forward pass kept.  A thread takes eight columns; the columns that pad [da du] become zero.  Bound by memory: 32768 x 2048
// float16 110 us for 671 MB, 6.1 TB/s.
template <int ACT>
__global__ __launch_bounds__(kEachThreads) void k_gated_slopes(const char* __restrict__ gate, const char* __restrict__ up,
                                                               const char* __restrict__ grad_h, char* __restrict__ out, int64_t m, int64_t n,
                                                               int64_t padded) {
  const int64_t units = padded / 8, i = element_of_thread();
  if (i >= m * units) return;
  const int64_t row = i / units, col = i % units * 8, at = (row * n + col) * 2;
  const int count = (int)(n - col);
  float a[8], u[8], g[8], da[8], du[8];
  widen_unit<DT>(load_unit_of<DT>(gate + at, count), a);
  widen_unit<DT>(load_unit_of<DT>(up + at, count), u);
  widen_unit<DT>(load_unit_of<DT>(grad_h + at, count), g);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float slope;
    const float f = activate<ACT, true>(a[e], slope);
    da[e] = g[e] * u[e] * slope;
    du[e] = g[e] * f;
  }
  char* const to = out + (row * 2 * padded + col) * 2;
  store_unit<DT>(to, narrow_unit<DT>(da));
  store_unit<DT>(to + padded * 2, narrow_unit<DT>(du));
}

// p with the tiles of the cut.
template <class S>
Product with_tiles(Product p, const GatedCut& cut, int64_t rows, int64_t cols) {
  const int64_t tile_rows = cut.whole > 0 ? 256 : S::kRows, tile_cols = cut.whole > 0 ? 256 : S::kCols;
  p.tiles_m = (int32_t)((rows + tile_rows - 1) / tile_rows);
  p.tiles_n = (int32_t)((cols + tile_cols - 1) / tile_cols);
  p.sub_m = (int32_t)(tile_rows / S::kRows);
  p.sub_n = (int32_t)(tile_cols / S::kCols);
  p.first = (int32_t)cut.whole;
  p.tiles = (int32_t)cut.tiles;
  p.slices = (int32_t)cut.slices;
  return p;
}

template <int KIND, class S>
hipError_t launch_tiles(const Product& product, const GatedCut& cut, int64_t rows, int64_t cols, hipStream_t stream) {
  const Product p = with_tiles<S>(product, cut, rows, cols);
  const dim3 blocks((unsigned)(cut.tiles * cut.slices)), threads(S::kThreads);
  if constexpr (std::is_same<S, TileLarge>::value) hipLaunchKernelGGL((k_gated_product_large<DT, KIND>), blocks, threads, 0, stream, p);
  else hipLaunchKernelGGL((k_gated_product<DT, KIND, S>), blocks, threads, 0, stream, p);
  if (const hipError_t error = hipGetLastError(); error != hipSuccess || cut.slices == 1) return error;
  hipLaunchKernelGGL((k_gated_join<DT, KIND, S>), dim3((unsigned)cut.tiles * JoinPart<KIND, S>::kBlocks), threads, 0, stream, p);
  return hipGetLastError();
}

template <int KIND>
hipError_t launch_kind(const Product& p, const GatedCut& cut, int64_t rows, int64_t cols, hipStream_t stream) {
  if (cut.whole > 0) {
    const hipError_t error = launch_tiles<KIND, TileLarge>(p, {0, 0, cut.whole, 1, 0}, rows, cols, stream);
    if (error != hipSuccess) return error;
  }
  if constexpr (is_gated(KIND)) {
    if (cut.form >= kGatedFewRows) {
      const dim3 blocks((unsigned)cut.tiles), threads(kFewThreads);
      const int few = cut.form - kGatedFewRows;
      auto kernel = few == 0 ? k_gated_few_rows<DT, KIND, 1, 16> : few == 1 ? k_gated_few_rows<DT, KIND, 2, 16> : few == 2 ? k_gated_few_rows<DT, KIND, 1, 8> : k_gated_few_rows<DT, KIND, 2, 8>;
      hipLaunchKernelGGL(kernel, blocks, threads, 0, stream, p);
      return hipGetLastError();
    }
  }
  switch (cut.form) {
    case 0: return launch_tiles<KIND, TileLarge>(p, cut, rows, cols, stream);
    case 1: return launch_tiles<KIND, Tile128x256>(p, cut, rows, cols, stream);
    case 2: return launch_tiles<KIND, Tile128x128>(p, cut, rows, cols, stream);
    default: return launch_tiles<KIND, Tile64x128>(p, cut, rows, cols, stream);
  }
}

template <class S>
hipError_t launch_gradients(const GatedProduct& input, const GatedCut& input_cut, const GatedProduct& weight, const GatedCut& weight_cut, hipStream_t stream) {
  const Product i = with_tiles<S>(input, input_cut, input.rows, input.k), w = with_tiles<S>(weight, weight_cut, weight.rows, weight.k);
  const dim3 threads(S::kThreads);
  const dim3 blocks((unsigned)(input_cut.tiles * input_cut.slices + weight_cut.tiles * weight_cut.slices));
  const int weights_first = w.steps / w.slices > i.steps / i.slices;
  if constexpr (std::is_same<S, TileLarge>::value) hipLaunchKernelGGL((k_gated_gradients_large<DT>), blocks, threads, 0, stream, i, w, weights_first);
  else hipLaunchKernelGGL((k_gated_gradients<DT, S>), blocks, threads, 0, stream, i, w, weights_first);
  if (const hipError_t error = hipGetLastError(); error != hipSuccess) return error;
  if (i.slices == 1 && w.slices == 1) return hipSuccess;
  if (i.slices == 1) hipLaunchKernelGGL((k_gated_join<DT, kWeight, S>), dim3((unsigned)w.tiles * JoinPart<kWeight, S>::kBlocks), threads, 0, stream, w);
  else if (w.slices == 1) hipLaunchKernelGGL((k_gated_join<DT, kInput, S>), dim3((unsigned)i.tiles * JoinPart<kInput, S>::kBlocks), threads, 0, stream, i);
  else hipLaunchKernelGGL((k_gated_join_gradients<DT, S>), dim3((unsigned)(i.tiles + w.tiles) * JoinPart<kInput, S>::kBlocks), threads, 0, stream, i, w);
  return hipGetLastError();
}

}  // namespace

#if DAF_DT == 1
#define DAF_OF_FORMAT(NAME) NAME##_f16
#else
#define DAF_OF_FORMAT(NAME) NAME##_bf16
#endif

hipError_t DAF_OF_FORMAT(daf_launch_gated_product)(GatedKind kind, const GatedProduct& p, const GatedCut& cut, int64_t rows, int64_t cols, hipStream_t stream) {
  switch (kind) {
    case kGated: return launch_kind<kGated>(p, cut, rows, cols, stream);
    case kGatedGrad: return launch_kind<kGatedGrad>(p, cut, rows, cols, stream);
    case kInput: return launch_kind<kInput>(p, cut, rows, cols, stream);
    default: return launch_kind<kWeight>(p, cut, rows, cols, stream);
  }
}

hipError_t DAF_OF_FORMAT(daf_launch_gated_gradients)(const GatedProduct& input, const GatedCut& input_cut, const GatedProduct& weight,
                                                     const GatedCut& weight_cut, hipStream_t stream) {
  switch (input_cut.form) {
    case 0: return launch_gradients<TileLarge>(input, input_cut, weight, weight_cut, stream);
    case 1: return launch_gradients<Tile128x256>(input, input_cut, weight, weight_cut, stream);
    case 2: return launch_gradients<Tile128x128>(input, input_cut, weight, weight_cut, stream);
    default: return launch_gradients<Tile64x128>(input, input_cut, weight, weight_cut, stream);
  }
}

hipError_t DAF_OF_FORMAT(daf_launch_gated_slopes)(int act, const void* gate, const void* up, const void* grad_h, char* out, int64_t m, int64_t n, int64_t padded,
                                                  hipStream_t stream) {
  auto kernel = act == DAF_ACT_SILU        ? k_gated_slopes<DAF_ACT_SILU>
                : act == DAF_ACT_GELU      ? k_gated_slopes<DAF_ACT_GELU>
                : act == DAF_ACT_GELU_TANH ? k_gated_slopes<DAF_ACT_GELU_TANH>
                                           : k_gated_slopes<DAF_ACT_RELU>;
  hipLaunchKernelGGL(kernel, blocks_for_each(m * (padded / 8)), dim3(kEachThreads), 0, stream, static_cast<const char*>(gate),
                     static_cast<const char*>(up), static_cast<const char*>(grad_h), out, m, n, padded);
  return hipGetLastError();
}

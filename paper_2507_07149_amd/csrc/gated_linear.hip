// The gated feed-forward product and its backward pass (daf_gated_linear, daf_gated_linear_backward): the products of gated_product.h, and what
// goes before and between them.
//
//   forward    a = x Wg^T, u = x Wu^T, h = f(a) u: one product whose epilogue has a and u of an output in the same lane
//   backward   da = grad_h u f'(a), du = grad_h f(a), from the kept a and u (bound by memory), or in the epilogue of the same product again;
//              both rounded to the format once, as the operands of
//              grad_x = da Wg + du Wu (one product over both) and grad_Wg = da^T x, grad_Wu = du^T x (one product for both)
#include "gated_linear.h"
#include "gated_product.h"
#include "gated_product_large.h"

namespace {

using Tile128x256 = Tile<128, 256, 2, 2, 3>;
using Tile128x128 = Tile<128, 128, 2, 2, 4>;
using Tile64x128 = Tile<64, 128, 2, 2, 6>;

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

// da and du from what the forward pass kept.  A thread takes eight columns; the columns that pad [da du] become zero.
template <int DT, int ACT>
__global__ __launch_bounds__(256) void k_gated_slopes(const char* __restrict__ gate, const char* __restrict__ up, const char* __restrict__ grad_h,
                                                      char* __restrict__ out, int64_t m, int64_t n, int64_t padded) {
  const int64_t units = padded / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
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

// Rows of k elements to rows of `padded`, a multiple of 8, with zeros behind them: rows then begin where a 16-byte load can.
__global__ __launch_bounds__(256) void k_pad_rows(const char* __restrict__ in, char* __restrict__ out, int64_t rows, int64_t k, int64_t padded) {
  const int64_t units = padded / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= rows * units) return;
  const int64_t row = i / units, col = i % units * 8;
  store_unit<kBF16>(out + (row * padded + col) * 2, load_unit_of<kBF16>(in + (row * k + col) * 2, (int)(k - col)));
}

__global__ __launch_bounds__(256) void k_clear_elements(uint16_t* out, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) out[i] = 0;
}

unsigned blocks_of(int64_t threads) { return (unsigned)((threads + 255) / 256); }

// ---- which tiles, and how many slices of l ----
// A round of 256 workgroups (one to a compute unit) takes `fixed` and `step` per 64 values of l, which lies between its value for a lone workgroup and for a
// full chip; the slices' sums go out and come back.  Microseconds.
constexpr struct Form {
  int rows, cols;
  float fixed, step_lone, step_full;
} kForms[] = {{256, 256, 12.6f, 0.82f, 1.38f}, {128, 256, 9.2f, 0.41f, 0.78f}, {128, 128, 4.9f, 0.26f, 0.48f}, {64, 128, 3.3f, 0.21f, 0.29f}};
constexpr int kFormCount = 4, kMostSlices = 16;

// An output's tiles: `whole` of 256 x 256, whole rounds of workgroups, and the others (all: whole == 0) in a form of its own, each sum in `slices`.
struct Cut {
  int64_t whole;
  int form;                       // of kForms
  int64_t tiles, slices;          // of the others
  int64_t partial_bytes;
};
float time_of(const Form& f, int64_t tiles, int64_t slices, int64_t steps) {
  const int64_t work = tiles * slices, rounds = work / 256, rest = work % 256, each = (steps + slices - 1) / slices;
  const float busy = (float)rest / 256.0f;
  float time = (float)rounds * (f.fixed + (float)each * f.step_full);
  if (rest > 0) time += f.fixed + (float)each * (f.step_lone + busy * (f.step_full - f.step_lone));
  return slices > 1 ? time + 8.0f + (float)(work * f.rows * f.cols) * 8.0f / 4e6f : time;
}
Cut cut_of(int64_t rows, int64_t cols, int64_t steps) {
  constexpr float kSecondLaunch = 4.0f;
  const int64_t large = ((rows + 255) / 256) * ((cols + 255) / 256), rounds = large / 256 * 256;
  Cut best = {};
  float best_time = 0.0f;
  for (const int64_t whole : {(int64_t)0, rounds}) {
    if (whole == large || (whole == 0 && rounds > 512)) continue;
    for (int form = 0; form < kFormCount; ++form) {
      const Form& f = kForms[form];
      const int64_t tiles = whole > 0 ? (large - whole) * (256 / f.rows) * (256 / f.cols) : (rows + f.rows - 1) / f.rows * ((cols + f.cols - 1) / f.cols);
      for (int64_t slices = 1; slices <= kMostSlices && (slices == 1 || (steps >= 4 * slices && tiles * slices <= 1024)); ++slices) {
        const float time = time_of(f, tiles, slices, steps) + (whole > 0 ? time_of(kForms[0], whole, 1, steps) + kSecondLaunch : 0.0f);
        if (best.slices == 0 || time < best_time) {
          best = {whole, form, tiles, slices, slices > 1 ? tiles * slices * f.rows * f.cols * 4 : 0};
          best_time = time;
        }
      }
    }
  }
  if (rounds == large && (best.slices == 0 || time_of(kForms[0], large, 1, steps) <= best_time)) best = {0, 0, large, 1, 0};
  return best;
}

struct Extent {
  int64_t rows, cols, steps;
};
Extent extent_of(int kind, const GatedSizes& s) {
  const int64_t k = round_up(s.k, 64) / 64, n = round_up(s.n, 64), m = round_up(s.m, 64) / 64;
  if (is_gated(kind)) return {s.m, 2 * n, k};
  if (kind == kInput) return {s.m, s.k, 2 * n / 64};
  return {2 * n, s.k, m};
}
Cut cut_of_product(int kind, const GatedSizes& s) {
  const Extent e = extent_of(kind, s);
  return cut_of(e.rows, e.cols, e.steps);
}

template <int DT, int KIND, class S>
hipError_t launch_tiles(Product p, const Extent& e, const Cut& cut, hipStream_t stream) {
  constexpr bool kLarge = std::is_same<S, TileLarge>::value;
  if (cut.whole > 0) {
    p.tiles_m = (int32_t)((e.rows + 255) / 256);
    p.tiles_n = (int32_t)((e.cols + 255) / 256);
    p.sub_m = 256 / S::kRows;
    p.sub_n = 256 / S::kCols;
  } else {
    p.tiles_m = (int32_t)((e.rows + S::kRows - 1) / S::kRows);
    p.tiles_n = (int32_t)((e.cols + S::kCols - 1) / S::kCols);
    p.sub_m = p.sub_n = 1;
  }
  p.first = (int32_t)cut.whole;
  p.tiles = (int32_t)cut.tiles;
  p.slices = (int32_t)cut.slices;
  const dim3 blocks((unsigned)(cut.tiles * cut.slices)), threads(S::kThreads);
  if (cut.slices == 1) {
    if constexpr (kLarge) hipLaunchKernelGGL((k_gated_product_large<DT, KIND, false>), blocks, threads, 0, stream, p);
    else hipLaunchKernelGGL((k_gated_product<DT, KIND, S, false>), blocks, threads, 0, stream, p);
    return hipGetLastError();
  }
  if constexpr (kLarge) hipLaunchKernelGGL((k_gated_product_large<DT, KIND, true>), blocks, threads, 0, stream, p);
  else hipLaunchKernelGGL((k_gated_product<DT, KIND, S, true>), blocks, threads, 0, stream, p);
  if (const hipError_t error = hipGetLastError(); error != hipSuccess) return error;
  hipLaunchKernelGGL((k_gated_join<DT, KIND, S>), dim3((unsigned)cut.tiles), threads, 0, stream, p);
  return hipGetLastError();
}

template <int DT, int KIND>
hipError_t launch_product(Product p, const GatedSizes& sizes, float* partial, hipStream_t stream) {
  const Extent e = extent_of(KIND, sizes);
  const Cut cut = cut_of(e.rows, e.cols, e.steps);
  p.partial = partial;
  if (cut.whole > 0) {
    const hipError_t error = launch_tiles<DT, KIND, TileLarge>(p, e, {0, 0, cut.whole, 1, 0}, stream);
    if (error != hipSuccess) return error;
  }
  switch (cut.form) {
    case 0: return launch_tiles<DT, KIND, TileLarge>(p, e, cut, stream);
    case 1: return launch_tiles<DT, KIND, Tile128x256>(p, e, cut, stream);
    case 2: return launch_tiles<DT, KIND, Tile128x128>(p, e, cut, stream);
    default: return launch_tiles<DT, KIND, Tile64x128>(p, e, cut, stream);
  }
}

// ---- the workspace ----
struct Workspace {
  int64_t pitch;                  // elements of a row of x, Wg and Wu as the products read them: k, or k made a multiple of 8 in copies
  int64_t padded;                 // columns of da
  int64_t x, w_gate, w_up, slopes, partial, bytes;   // where: the copies, [da du], the slices' sums
};
Workspace workspace_of(const GatedSizes& s, bool backward) {
  Workspace w = {};
  w.pitch = round_up(s.k, 8);
  w.padded = round_up(s.n, 64);
  auto take = [&](int64_t bytes) {
    const int64_t at = w.bytes;
    w.bytes += round_up(bytes, 256);
    return at;
  };
  if (w.pitch != s.k) {
    w.x = take(s.m * w.pitch * 2);
    w.w_gate = take(s.n * w.pitch * 2);
    w.w_up = take(s.n * w.pitch * 2);
  }
  int64_t partial = cut_of_product(kGated, s).partial_bytes;
  if (backward) {
    w.slopes = take(s.m * 2 * w.padded * 2);
    for (const int kind : {kInput, kWeight}) {
      const int64_t more = cut_of_product(kind, s).partial_bytes;
      if (more > partial) partial = more;
    }
  }
  w.partial = take(partial);
  return w;
}

// x, Wg and Wu with rows that begin at multiples of 16 bytes.
struct Operands {
  const char *x, *w_gate, *w_up;
};
hipError_t operands_of(const GatedLinear& g, const Workspace& w, Operands* out, hipStream_t stream) {
  *out = {static_cast<const char*>(g.x), static_cast<const char*>(g.w_gate), static_cast<const char*>(g.w_up)};
  if (w.pitch == g.sizes.k) return hipSuccess;
  auto pad = [&](const char*& t, int64_t rows, int64_t at) {
    hipLaunchKernelGGL(k_pad_rows, dim3(blocks_of(rows * (w.pitch / 8))), dim3(256), 0, stream, t, g.workspace + at, rows, g.sizes.k, w.pitch);
    t = g.workspace + at;
    return hipGetLastError();
  };
  hipError_t e = pad(out->x, g.sizes.m, w.x);
  if (e == hipSuccess) e = pad(out->w_gate, g.sizes.n, w.w_gate);
  if (e == hipSuccess) e = pad(out->w_up, g.sizes.n, w.w_up);
  return e;
}

Product gated_of(const GatedLinear& g, const Workspace& w, const Operands& o) {
  Product p = {};
  p.r = o.x;
  p.c[0] = o.w_gate;
  p.c[1] = o.w_up;
  p.r_pitch = p.c_pitch = w.pitch * 2;
  p.rows = (int32_t)g.sizes.m;
  p.cols = (int32_t)g.sizes.n;
  p.length = (int32_t)g.sizes.k;
  p.steps = (int32_t)(round_up(g.sizes.k, 64) / 64);
  p.n = g.sizes.n;
  p.k = g.sizes.k;
  p.padded = w.padded;
  p.act = g.act;
  return p;
}

template <int DT>
hipError_t forward(const GatedLinear& g, void* out_h, void* out_gate, void* out_up, hipStream_t stream) {
  const Workspace w = workspace_of(g.sizes, false);
  Operands o;
  if (const hipError_t e = operands_of(g, w, &o, stream); e != hipSuccess) return e;
  Product p = gated_of(g, w, o);
  p.out[0] = static_cast<char*>(out_h);
  p.out[1] = static_cast<char*>(out_gate);
  p.out[2] = static_cast<char*>(out_up);
  return launch_product<DT, kGated>(p, g.sizes, reinterpret_cast<float*>(g.workspace + w.partial), stream);
}

template <int DT>
hipError_t backward(const GatedLinear& g, const void* grad_h, const void* gate, const void* up, void* out_grad_x, void* out_grad_w_gate,
                    void* out_grad_w_up, void* out_h, hipStream_t stream) {
  const Workspace w = workspace_of(g.sizes, true);
  const GatedSizes& s = g.sizes;
  Operands o;
  if (const hipError_t e = operands_of(g, w, &o, stream); e != hipSuccess) return e;
  char* const slopes = g.workspace + w.slopes;
  float* const partial = reinterpret_cast<float*>(g.workspace + w.partial);
  hipError_t e;
  if (gate != nullptr) {
    auto kernel = g.act == DAF_ACT_SILU        ? k_gated_slopes<DT, DAF_ACT_SILU>
                  : g.act == DAF_ACT_GELU      ? k_gated_slopes<DT, DAF_ACT_GELU>
                  : g.act == DAF_ACT_GELU_TANH ? k_gated_slopes<DT, DAF_ACT_GELU_TANH>
                                               : k_gated_slopes<DT, DAF_ACT_RELU>;
    hipLaunchKernelGGL(kernel, dim3(blocks_of(s.m * (w.padded / 8))), dim3(256), 0, stream, static_cast<const char*>(gate),
                       static_cast<const char*>(up), static_cast<const char*>(grad_h), slopes, s.m, s.n, w.padded);
    e = hipGetLastError();
  } else {
    Product p = gated_of(g, w, o);
    p.out[0] = static_cast<char*>(out_h);
    p.out[1] = slopes;
    p.grad_h = static_cast<const char*>(grad_h);
    e = launch_product<DT, kGatedGrad>(p, s, partial, stream);
  }
  if (e == hipSuccess && out_grad_x != nullptr) {
    Product p = gated_of(g, w, o);
    p.r = slopes;
    p.r_pitch = 2 * w.padded * 2;
    p.cols = (int32_t)w.pitch;
    p.length = (int32_t)s.n;
    p.half = (int32_t)(w.padded / 64);
    p.steps = 2 * p.half;
    p.out[0] = static_cast<char*>(out_grad_x);
    e = launch_product<DT, kInput>(p, s, partial, stream);
  }
  if (e == hipSuccess && out_grad_w_gate != nullptr) {
    Product p = gated_of(g, w, o);
    p.r = slopes;
    p.r_pitch = 2 * w.padded * 2;
    p.c[0] = o.x;
    p.rows = (int32_t)(2 * w.padded);
    p.cols = (int32_t)w.pitch;
    p.length = (int32_t)s.m;
    p.steps = (int32_t)(round_up(s.m, 64) / 64);
    p.out[0] = static_cast<char*>(out_grad_w_gate);
    p.out[1] = static_cast<char*>(out_grad_w_up);
    e = launch_product<DT, kWeight>(p, s, partial, stream);
  }
  return e;
}

}  // namespace

void daf_gated_schedule(const GatedSizes& sizes, int product, daf_gated_schedule_t* out) {
  const int kind = product == DAF_GATED_FORWARD ? kGated : product == DAF_GATED_GRAD_INPUT ? kInput : kWeight;
  const Cut cut = cut_of_product(kind, sizes);
  *out = {kForms[cut.form].rows, kForms[cut.form].cols, (int32_t)cut.slices, cut.tiles, cut.whole};
}

int64_t daf_gated_workspace_size(const GatedSizes& sizes, bool backward) { return workspace_of(sizes, backward).bytes; }

hipError_t daf_launch_gated_linear(const GatedLinear& g, void* out_h, void* out_gate, void* out_up, hipStream_t stream) {
  return g.dtype == DAF_BF16 ? forward<kBF16>(g, out_h, out_gate, out_up, stream) : forward<kF16>(g, out_h, out_gate, out_up, stream);
}

hipError_t daf_launch_gated_linear_backward(const GatedLinear& g, const void* grad_h, const void* gate, const void* up, void* out_grad_x,
                                            void* out_grad_w_gate, void* out_grad_w_up, void* out_h, hipStream_t stream) {
  return g.dtype == DAF_BF16 ? backward<kBF16>(g, grad_h, gate, up, out_grad_x, out_grad_w_gate, out_grad_w_up, out_h, stream)
                             : backward<kF16>(g, grad_h, gate, up, out_grad_x, out_grad_w_gate, out_grad_w_up, out_h, stream);
}

hipError_t daf_launch_clear(void* out, int64_t bytes, hipStream_t stream) {
  hipLaunchKernelGGL(k_clear_elements, dim3(blocks_of(bytes / 2)), dim3(256), 0, stream, static_cast<uint16_t*>(out), bytes / 2);
  return hipGetLastError();
}

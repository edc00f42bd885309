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
template <int DT>
__global__ __launch_bounds__(256) void k_gated_slopes(const char* __restrict__ gate, const char* __restrict__ up, const char* __restrict__ grad_h,
                                                      char* __restrict__ out, int64_t m, int64_t n, int64_t padded, int act) {
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
    const float f = activate<true>(a[e], act, slope);
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
struct Cut {
  int form;                       // of kForms
  int64_t tiles_m, tiles_n, slices, partial_bytes;
};
Cut cut_of(int64_t rows, int64_t cols, int64_t steps) {
  Cut best = {};
  float best_time = 0.0f;
  for (int form = 0; form < 4; ++form) {
    const Form& f = kForms[form];
    const int64_t tm = (rows + f.rows - 1) / f.rows, tn = (cols + f.cols - 1) / f.cols, most = form == 0 ? 1 : 16;
    for (int64_t slices = 1; slices <= most && (slices == 1 || (steps >= 4 * slices && tm * tn * slices <= 512)); ++slices) {
      const int64_t work = tm * tn * slices, rounds = (work + 255) / 256, bytes = slices > 1 ? work * f.rows * f.cols * 4 : 0;
      const float busy = work >= 256 ? 1.0f : (float)work / 256.0f;
      const float time = (float)rounds * (f.fixed + (float)((steps + slices - 1) / slices) * (f.step_lone + busy * (f.step_full - f.step_lone))) +
                         (slices > 1 ? 5.0f + 2.0f * (float)bytes / 4e6f : 0.0f);
      if (best.slices == 0 || time < best_time) {
        best = {form, tm, tn, slices, bytes};
        best_time = time;
      }
    }
  }
  return best;
}

Cut cut_of_product(int kind, const GatedSizes& s) {
  const int64_t k = round_up(s.k, 64) / 64, n = round_up(s.n, 64), m = round_up(s.m, 64) / 64;
  if (is_gated(kind)) return cut_of(s.m, 2 * n, k);
  if (kind == kInput) return cut_of(s.m, s.k, 2 * n / 64);
  return cut_of(2 * n, s.k, m);
}

template <int DT, int KIND, class S>
hipError_t launch_tiles(const Product& p, hipStream_t stream) {
  const unsigned tiles = (unsigned)(p.tiles_m * p.tiles_n);
  if (p.slices == 1) {
    hipLaunchKernelGGL((k_gated_product<DT, KIND, S, false>), dim3(tiles), dim3(S::kThreads), 0, stream, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((k_gated_product<DT, KIND, S, true>), dim3(tiles * (unsigned)p.slices), dim3(S::kThreads), 0, stream, p);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  hipLaunchKernelGGL((k_gated_join<DT, KIND, S>), dim3(tiles), dim3(S::kThreads), 0, stream, p);
  return hipGetLastError();
}

template <int DT, int KIND>
hipError_t launch_product(Product p, const GatedSizes& sizes, float* partial, hipStream_t stream) {
  const Cut cut = cut_of_product(KIND, sizes);
  p.tiles_m = (int32_t)cut.tiles_m;
  p.tiles_n = (int32_t)cut.tiles_n;
  p.slices = (int32_t)cut.slices;
  p.partial = partial;
  switch (cut.form) {
    case 0:
      hipLaunchKernelGGL((k_gated_product_large<DT, KIND>), dim3((unsigned)(p.tiles_m * p.tiles_n)), dim3(TileLarge::kThreads), 0, stream, p);
      return hipGetLastError();
    case 1: return launch_tiles<DT, KIND, Tile128x256>(p, stream);
    case 2: return launch_tiles<DT, KIND, Tile128x128>(p, stream);
    default: return launch_tiles<DT, KIND, Tile64x128>(p, stream);
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
    hipLaunchKernelGGL(k_gated_slopes<DT>, dim3(blocks_of(s.m * (w.padded / 8))), dim3(256), 0, stream, static_cast<const char*>(gate),
                       static_cast<const char*>(up), static_cast<const char*>(grad_h), slopes, s.m, s.n, w.padded, g.act);
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
  *out = {kForms[cut.form].rows, kForms[cut.form].cols, (int32_t)cut.slices, cut.tiles_m * cut.tiles_n};
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

// The gated feed-forward product and its backward pass (daf_gated_linear, daf_gated_linear_backward): how their products are cut into tiles, the
// workspace, and what goes before and between the products of gated_product.h.
//
//   forward    a = x Wg^T, u = x Wu^T, h = f(a) u: one product whose epilogue has a and u of an output in the same lane
//   backward   da = grad_h u f'(a), du = grad_h f(a), from the kept a and u (bound by memory), or in the epilogue of the same product again;
//              both rounded to the format once, as the operands of
//              grad_x = da Wg + du Wu (one product over both) and grad_Wg = da^T x, grad_Wu = du^T x (one product for both)
#include "block_common.h"
#include "gated_linear.h"

namespace {

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

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
struct Cost {
  int rows, cols;
  float fixed, step_lone, step_full;
};
constexpr Cost kForms[] = {{256, 256, 12.6f, 0.82f, 1.38f}, {128, 256, 9.2f, 0.41f, 0.78f}, {128, 128, 4.9f, 0.26f, 0.48f}, {64, 128, 3.3f, 0.21f, 0.29f}};
constexpr int kFormCount = 4, kMostSlices = 16;
using Cut = GatedCut;
float time_of(const Cost& f, int64_t tiles, int64_t slices, int64_t steps) {
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
      const Cost& f = kForms[form];
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

bool is_gated(GatedKind kind) { return kind == kGated || kind == kGatedGrad; }

struct Extent {
  int64_t rows, cols, steps;
};
Extent extent_of(GatedKind kind, const GatedSizes& s) {
  const int64_t k = round_up(s.k, 64) / 64, n = round_up(s.n, 64), m = round_up(s.m, 64) / 64;
  if (is_gated(kind)) return {s.m, 2 * n, k};
  if (kind == kInput) return {s.m, s.k, 2 * n / 64};
  return {2 * n, s.k, m};
}
hipError_t launch_product(const GatedPlan& plan, const GatedLinear& g, GatedKind kind, GatedProduct p, hipStream_t stream) {
  const Extent e = extent_of(kind, plan.sizes);
  p.partial = reinterpret_cast<float*>(g.workspace + plan.partial);
  const GatedCut& cut = plan.cut[is_gated(kind) ? DAF_GATED_FORWARD : kind == kInput ? DAF_GATED_GRAD_INPUT : DAF_GATED_GRAD_WEIGHT];
  return g.dtype == DAF_BF16 ? daf_launch_gated_product_bf16(kind, p, cut, e.rows, e.cols, stream)
                             : daf_launch_gated_product_f16(kind, p, cut, e.rows, e.cols, stream);
}

// x, Wg and Wu with rows that begin at multiples of 16 bytes.
struct Operands {
  const char *x, *w_gate, *w_up;
};
hipError_t operands_of(const GatedPlan& plan, const GatedLinear& g, Operands* out, hipStream_t stream) {
  *out = {static_cast<const char*>(g.x), static_cast<const char*>(g.w_gate), static_cast<const char*>(g.w_up)};
  if (plan.pitch == plan.sizes.k) return hipSuccess;
  auto pad = [&](const char*& t, int64_t rows, int64_t at) {
    hipLaunchKernelGGL(k_pad_rows, dim3(blocks_of(rows * (plan.pitch / 8))), dim3(256), 0, stream, t, g.workspace + at, rows, plan.sizes.k, plan.pitch);
    t = g.workspace + at;
    return hipGetLastError();
  };
  hipError_t e = pad(out->x, plan.sizes.m, plan.x);
  if (e == hipSuccess) e = pad(out->w_gate, plan.sizes.n, plan.w_gate);
  if (e == hipSuccess) e = pad(out->w_up, plan.sizes.n, plan.w_up);
  return e;
}

GatedProduct product_of(const GatedPlan& plan, const GatedLinear& g, const Operands& o) {
  GatedProduct p = {};
  p.r = o.x;
  p.c[0] = o.w_gate;
  p.c[1] = o.w_up;
  p.r_pitch = p.c_pitch = plan.pitch * 2;
  p.rows = (int32_t)plan.sizes.m;
  p.cols = (int32_t)plan.sizes.n;
  p.length = (int32_t)plan.sizes.k;
  p.steps = (int32_t)(round_up(plan.sizes.k, 64) / 64);
  p.n = plan.sizes.n;
  p.k = plan.sizes.k;
  p.padded = plan.padded;
  p.act = g.act;
  return p;
}

}  // namespace

GatedPlan daf_gated_plan(const GatedSizes& s, bool backward) {
  GatedPlan w = {};
  w.sizes = s;
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
  int64_t partial = 0;
  for (const GatedKind kind : {kGated, kInput, kWeight}) {
    if (kind != kGated && !backward) continue;
    const Extent e = extent_of(kind, s);
    GatedCut& cut = w.cut[kind == kGated ? DAF_GATED_FORWARD : kind == kInput ? DAF_GATED_GRAD_INPUT : DAF_GATED_GRAD_WEIGHT];
    cut = cut_of(e.rows, e.cols, e.steps);
    if (cut.partial_bytes > partial) partial = cut.partial_bytes;
  }
  if (backward) w.slopes = take(s.m * 2 * w.padded * 2);
  w.partial = take(partial);
  return w;
}

hipError_t daf_launch_gated_linear(const GatedPlan& plan, const GatedLinear& g, void* out_h, void* out_gate, void* out_up, hipStream_t stream) {
  Operands o;
  if (const hipError_t e = operands_of(plan, g, &o, stream); e != hipSuccess) return e;
  GatedProduct p = product_of(plan, g, o);
  p.out[0] = static_cast<char*>(out_h);
  p.out[1] = static_cast<char*>(out_gate);
  p.out[2] = static_cast<char*>(out_up);
  return launch_product(plan, g, kGated, p, stream);
}

hipError_t daf_launch_gated_linear_backward(const GatedPlan& plan, const GatedLinear& g, const void* grad_h, const void* gate, const void* up,
                                            void* out_grad_x, void* out_grad_w_gate, void* out_grad_w_up, void* out_h, hipStream_t stream) {
  const GatedSizes& s = plan.sizes;
  Operands o;
  if (const hipError_t e = operands_of(plan, g, &o, stream); e != hipSuccess) return e;
  char* const slopes = g.workspace + plan.slopes;
  hipError_t e;
  if (gate != nullptr) {
    auto launch = g.dtype == DAF_BF16 ? daf_launch_gated_slopes_bf16 : daf_launch_gated_slopes_f16;
    e = launch(g.act, gate, up, grad_h, slopes, s.m, s.n, plan.padded, stream);
  } else {
    GatedProduct p = product_of(plan, g, o);
    p.out[0] = static_cast<char*>(out_h);
    p.out[1] = slopes;
    p.grad_h = static_cast<const char*>(grad_h);
    e = launch_product(plan, g, kGatedGrad, p, stream);
  }
  if (e == hipSuccess && out_grad_x != nullptr) {
    GatedProduct p = product_of(plan, g, o);
    p.r = slopes;
    p.r_pitch = 2 * plan.padded * 2;
    p.cols = (int32_t)plan.pitch;
    p.length = (int32_t)s.n;
    p.half = (int32_t)(plan.padded / 64);
    p.steps = 2 * p.half;
    p.out[0] = static_cast<char*>(out_grad_x);
    e = launch_product(plan, g, kInput, p, stream);
  }
  if (e == hipSuccess && out_grad_w_gate != nullptr) {
    GatedProduct p = product_of(plan, g, o);
    p.r = slopes;
    p.r_pitch = 2 * plan.padded * 2;
    p.c[0] = o.x;
    p.rows = (int32_t)(2 * plan.padded);
    p.cols = (int32_t)plan.pitch;
    p.length = (int32_t)s.m;
    p.steps = (int32_t)(round_up(s.m, 64) / 64);
    p.out[0] = static_cast<char*>(out_grad_w_gate);
    p.out[1] = static_cast<char*>(out_grad_w_up);
    e = launch_product(plan, g, kWeight, p, stream);
  }
  return e;
}

hipError_t daf_launch_clear(void* out, int64_t bytes, hipStream_t stream) {
  hipLaunchKernelGGL(k_clear_elements, dim3(blocks_of(bytes / 2)), dim3(256), 0, stream, static_cast<uint16_t*>(out), bytes / 2);
  return hipGetLastError();
}

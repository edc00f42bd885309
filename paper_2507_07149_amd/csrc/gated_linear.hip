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

// Rows of k elements to rows of `padded`, a multiple of 8, with zeros behind them: rows then begin where a 16-byte load can.  x, Wg and Wu in turn.
struct Pads {
  const char* in[3];
  char* out[3];
  int64_t rows[3];
};
__global__ __launch_bounds__(kEachThreads) void k_pad_rows(const Pads p, int64_t k, int64_t padded) {
  const int64_t units = padded / 8;
  int64_t i = element_of_thread();
#pragma unroll
  for (int t = 0; t < 3; ++t) {
    if (i < p.rows[t] * units) {
      const int64_t row = i / units, col = i % units * 8;
      store_unit<kBF16>(p.out[t] + (row * padded + col) * 2, load_unit_of<kBF16>(p.in[t] + (row * k + col) * 2, (int)(k - col)));
      return;
    }
    i -= p.rows[t] * units;
  }
}

__global__ __launch_bounds__(kEachThreads) void k_clear_elements(uint16_t* out, int64_t n) {
  const int64_t i = element_of_thread();
  if (i < n) out[i] = 0;
}

// ---- which tiles, and how many slices of l ----
// A round of 256 workgroups (one to a compute unit) takes `fixed` and `step` per 64 values of l, each between its value for a lone workgroup and for a full
// chip; slices have their sums go out and come back.  Microseconds, fitted to 2200 measurements: 29 shapes of 1 to 32768 rows, 64 to 11008 columns and
// 64 to 4096 inside, all four products, every form, 1 to 16 slices, with and without whole rounds in front; the sums' way to 1100 more of 13 shapes, the
// largest tiles to 470 of 9. The
// form picked was 0.8 % (of the 13: 0.6 %) behind the best of them on average, 17 % at most (60.6 against 51.8 us), before kHandOut and last_end, which only
// choose between both gradients side by side and apart.  kGatedGrad goes by kGated's cost, though its end reads grad_h and stores three tensors.
struct Cost {
  int rows, cols;
  float fixed_lone, fixed_full, step_lone, step_full;
};
constexpr Cost kForms[] = {{256, 256, 7.4f, 8.0f, 1.10f, 1.56f}, {128, 256, 4.1f, 4.3f, 0.61f, 0.97f}, {128, 128, 1.1f, 2.3f, 0.36f, 0.61f}, {64, 128, 0.6f, 1.9f, 0.29f, 0.43f}};
constexpr float kHandOut = 0.5f;                   // side by side, from one round to the next: from one shape, 127 x 6242 x 2952, 67 us in 2448 workgroups, 61 in 1272
constexpr float kSecondLaunch = 8.2f, kJoin = 2.4f, kJoinSlice = 0.18f, kJoinMegabyte = 0.2f;
constexpr float kAcrossStep = 0.84f;               // of a step where an operand runs across the output (whole rows of a tile to a load)
constexpr int kFormCount = 4, kMostSlices = 16;
using Cut = GatedCut;
float join_time(int64_t slices, int64_t bytes) { return slices > 1 ? kJoin + kJoinSlice * (float)slices + kJoinMegabyte * 1e-6f * (float)bytes : 0.0f; }
float time_of(const Cost& f, int64_t tiles, int64_t slices, int64_t steps, float scale) {
  const int64_t work = tiles * slices, rounds = work / 256, rest = work % 256, each = (steps + slices - 1) / slices;
  const float busy = (float)rest / 256.0f, all = scale * (float)each;
  float time = (float)rounds * (f.fixed_full + all * f.step_full);
  if (rest > 0) time += f.fixed_lone + busy * (f.fixed_full - f.fixed_lone) + all * (f.step_lone + busy * (f.step_full - f.step_lone));
  return time + join_time(slices, work * f.rows * f.cols * 4);
}
Cut cut_of(int64_t rows, int64_t cols, int64_t steps, float scale, float* its_time) {
  const int64_t large = ((rows + 255) / 256) * ((cols + 255) / 256), rounds = large / 256 * 256;
  Cut best = {};
  float best_time = 0.0f;
  for (const int64_t whole : {(int64_t)0, rounds}) {
    if (whole == large || (whole == 0 && rounds > 512)) continue;
    for (int form = 0; form < kFormCount; ++form) {
      const Cost& f = kForms[form];
      const int64_t tiles = whole > 0 ? (large - whole) * (256 / f.rows) * (256 / f.cols) : (rows + f.rows - 1) / f.rows * ((cols + f.cols - 1) / f.cols);
      for (int64_t slices = 1; slices <= kMostSlices && (slices == 1 || (steps >= 4 * slices && tiles * slices <= 1024)); ++slices) {
        const bool one = form == 0 && slices == 1;    // (the rest as the whole rounds: one launch)
        const float time = time_of(f, tiles, slices, steps, scale) + (whole > 0 ? time_of(kForms[0], whole, 1, steps, scale) + (one ? 0.0f : kSecondLaunch) : 0.0f);
        if (best.slices == 0 || time < best_time) {
          best = one ? Cut{0, 0, large, 1, 0} : Cut{whole, form, tiles, slices, slices > 1 ? tiles * slices * f.rows * f.cols * 4 : 0};
          best_time = time;
        }
      }
    }
  }
  if (rounds == large && (best.slices == 0 || time_of(kForms[0], large, 1, steps, scale) <= best_time)) best = {0, 0, large, 1, 0};
  *its_time = best_time;
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
// Few rows (gated_few_rows.h): 16 columns of h to a workgroup, 8 where these would be fewer than compute units, if that is faster than tiles.  Its time
// is that of W's bytes and of x for every workgroup out of the caches, a lone workgroup's own at least; tiles have rows that loads cannot begin
// at copied first.  Microseconds at 1 / 8 / 16 / 32 rows, beside the tiles': bfloat16, 11008 x 4096 35.9 / 39.6 / 44.3 / 55.8 and 38 to 41;
// 5592 x 614 5.2 / 5.5 / 5.9 / 7.2 and 14.3; 120 x 3584 6.8 / 8.1 / 9.3 / 11.5 and 12.8.
constexpr int kFewRows = 32;
Cut forward_cut(const GatedSizes& s, int64_t padded) {
  const Extent e = extent_of(kGated, s);
  float tiles_time;
  const Cut tiles = cut_of(e.rows, e.cols, e.steps, 1.0f, &tiles_time);
  if (s.m > kFewRows) return tiles;
  const bool narrow = padded / 16 < 256;
  const int64_t cols = narrow ? 8 : 16, blocks = padded / cols;
  const float w = (float)(4 * cols * s.k) * 1e-6f, x = (float)(2 * s.m * s.k) * 1e-6f;        // megabytes of a workgroup
  const float all = (float)blocks * (0.18f * w + 0.1f * x), lone = 25.0f * (w + x);
  const float time = 3.5f + (all > lone ? all : lone);
  if (tiles_time < 0.21f * (float)blocks * w) tiles_time = 0.21f * (float)blocks * w;
  if (s.k % 8 != 0) tiles_time += 4.0f + 0.4f * (float)blocks * w;
  if (time > 3.2f + tiles_time) return tiles;
  return {0, kGatedFewRows + (s.m > 16 ? 1 : 0) + (narrow ? 2 : 0), blocks, 1, 0};
}

// When the last of `n` long and then `m` short workgroups ends, each handed to the compute unit that is free first.
float last_end(int64_t n, float d, int64_t m, float e) {
  const int64_t late = n % 256, early = 256 - late;                // units that take one long workgroup more than the others
  const float begin = (float)(n / 256) * d, later = begin + d;
  const float least = (begin * (float)early + later * (float)late + (float)m * e) / 256.0f;
  auto done = [&](float t) {                                       // short ones ended by then
    auto of = [&](float from) { return t > from ? (int64_t)((t - from) / e + 0.001f) : 0; };
    return of(begin) * early + of(later) * late;
  };
  if (m == 0) return late > 0 ? later : begin;
  float end = 0.0f;
  for (const float from : {begin, later}) {                        // an end is a whole number of short ones behind either
    if (from == later && late == 0) continue;
    int64_t k = least > from ? (int64_t)((least - from) / e) : 0;
    while (done(from + (float)k * e) < m) ++k;
    const float t = from + (float)k * e;
    if (end == 0.0f || t < end) end = t;
  }
  return late > 0 && end < later ? later : end;
}
// Whether the two gradients take one launch, and how they are cut then.  The workgroups of a launch are handed out as they end, those that take longer
// first.
bool side_by_side(GatedPlan& w, const Extent& input, const Extent& weight) {
  auto alone = [](const GatedCut& cut, const Extent& e) {
    return time_of(kForms[cut.form], cut.tiles, cut.slices, e.steps, kAcrossStep) + (cut.whole > 0 ? time_of(kForms[0], cut.whole, 1, e.steps, kAcrossStep) + kSecondLaunch : 0.0f);
  };
  const float apart = alone(w.cut[DAF_GATED_GRAD_INPUT], input) + alone(w.cut[DAF_GATED_GRAD_WEIGHT], weight) + kSecondLaunch;
  float best = apart;
  for (int form = 0; form < kFormCount; ++form) {
    const Cost& f = kForms[form];
    auto tiles_of = [&](const Extent& e) { return (e.rows + f.rows - 1) / f.rows * ((e.cols + f.cols - 1) / f.cols); };
    const int64_t ti = tiles_of(input), tw = tiles_of(weight);
    auto may = [](const Extent& e, int64_t tiles, int64_t slices) { return slices == 1 || (slices <= kMostSlices && e.steps >= 4 * slices && tiles * slices <= 512); };
    for (int64_t si = 1; may(input, ti, si); si *= 2)
      for (int64_t sw = 1; may(weight, tw, sw); sw = sw < 4 ? sw + 1 : sw + sw / 4) {
        const int64_t ni = ti * si, nw = tw * sw;
        if (ni + nw >= kGatedMostTiles) continue;      // (cut_of has no so many: beyond 768 large tiles, whole rounds of them go first)
        const float busy = (float)(ni + nw) / 256.0f, full = busy < 1.0f ? busy : 1.0f;
        const float step = kAcrossStep * (f.step_lone + full * (f.step_full - f.step_lone)), fixed = f.fixed_lone + full * (f.fixed_full - f.fixed_lone);
        const float di = fixed + (float)((input.steps + si - 1) / si) * step, dw = fixed + (float)((weight.steps + sw - 1) / sw) * step;
        const float all = di > dw ? last_end(ni, di, nw, dw) : last_end(nw, dw, ni, di);
        const int64_t bi = si > 1 ? ni * f.rows * f.cols * 4 : 0, bw = sw > 1 ? nw * f.rows * f.cols * 4 : 0;
        const float time = all + kHandOut * busy + join_time(si > sw ? si : sw, bi + bw);
        if (time < best) {
          best = time;
          w.side[0] = {0, form, ti, si, bi};
          w.side[1] = {0, form, tw, sw, bw};
        }
      }
  }
  return best < apart;
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
  const Pads p = {{out->x, out->w_gate, out->w_up},
                  {g.workspace + plan.x, g.workspace + plan.w_gate, g.workspace + plan.w_up},
                  {plan.sizes.m, plan.sizes.n, plan.sizes.n}};
  *out = {p.out[0], p.out[1], p.out[2]};
  hipLaunchKernelGGL(k_pad_rows, blocks_for_each((plan.sizes.m + 2 * plan.sizes.n) * (plan.pitch / 8)), dim3(kEachThreads), 0, stream, p, plan.sizes.k, plan.pitch);
  return hipGetLastError();
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
  w.padded = round_up(s.n, 64);
  auto take = [&](int64_t bytes) {
    const int64_t at = w.bytes;
    w.bytes += round_up(bytes, 256);
    return at;
  };
  w.cut[DAF_GATED_FORWARD] = forward_cut(s, w.padded);
  w.pitch = w.cut[DAF_GATED_FORWARD].form >= kGatedFewRows && !backward ? s.k : round_up(s.k, 8);
  if (w.pitch != s.k) {
    w.x = take(s.m * w.pitch * 2);
    w.w_gate = take(s.n * w.pitch * 2);
    w.w_up = take(s.n * w.pitch * 2);
  }
  int64_t partial = w.cut[DAF_GATED_FORWARD].partial_bytes;
  if (backward) {
    for (const GatedKind kind : {kInput, kWeight}) {
      const Extent e = extent_of(kind, s);
      GatedCut& cut = w.cut[kind == kInput ? DAF_GATED_GRAD_INPUT : DAF_GATED_GRAD_WEIGHT];
      float time;
      cut = cut_of(e.rows, e.cols, e.steps, kAcrossStep, &time);
      if (cut.partial_bytes > partial) partial = cut.partial_bytes;
    }
    w.slopes = take(s.m * 2 * w.padded * 2);
    w.together = side_by_side(w, extent_of(kInput, s), extent_of(kWeight, s));
    if (w.together) {                                 // (the sums of the two lie behind each other, in the place of those of one after the other)
      const int64_t first = round_up(w.side[0].partial_bytes, 256), both = first + w.side[1].partial_bytes;
      if (both > partial) partial = both;
      w.side_partial = w.bytes + first;
    }
  }
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
  if (e != hipSuccess) return e;
  GatedProduct input = product_of(plan, g, o), weight = input;
  input.r = weight.r = slopes;
  input.r_pitch = weight.r_pitch = 2 * plan.padded * 2;
  input.cols = weight.cols = (int32_t)plan.pitch;
  input.length = (int32_t)s.n;
  input.half = (int32_t)(plan.padded / 64);
  input.steps = 2 * input.half;
  input.out[0] = static_cast<char*>(out_grad_x);
  weight.c[0] = o.x;
  weight.rows = (int32_t)(2 * plan.padded);
  weight.length = (int32_t)s.m;
  weight.steps = (int32_t)(round_up(s.m, 64) / 64);
  weight.out[0] = static_cast<char*>(out_grad_w_gate);
  weight.out[1] = static_cast<char*>(out_grad_w_up);
  if (plan.together && out_grad_x != nullptr && out_grad_w_gate != nullptr) {
    input.partial = reinterpret_cast<float*>(g.workspace + plan.partial);
    weight.partial = reinterpret_cast<float*>(g.workspace + plan.side_partial);
    auto launch = g.dtype == DAF_BF16 ? daf_launch_gated_gradients_bf16 : daf_launch_gated_gradients_f16;
    return launch(input, plan.side[0], weight, plan.side[1], stream);
  }
  if (out_grad_x != nullptr) e = launch_product(plan, g, kInput, input, stream);
  if (e == hipSuccess && out_grad_w_gate != nullptr) e = launch_product(plan, g, kWeight, weight, stream);
  return e;
}

hipError_t daf_launch_clear(void* out, int64_t bytes, hipStream_t stream) {
  hipLaunchKernelGGL(k_clear_elements, blocks_for_each(bytes / 2), dim3(kEachThreads), 0, stream, static_cast<uint16_t*>(out), bytes / 2);
  return hipGetLastError();
}

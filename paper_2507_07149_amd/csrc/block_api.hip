// C ABI of daf_block.h: argument checks and dispatch to the launchers.  Every check comes before the first HIP call.
#include "daf_block.h"
#include "gated_linear.h"
#include "grad_norm.h"
#include "residual_norm.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool known(int dtype) { return dtype == DAF_F32 || dtype == DAF_F16 || dtype == DAF_BF16; }
int64_t elem_bytes(int dtype) { return dtype == DAF_F32 ? 4 : 2; }
int status(hipError_t e) { return e == hipSuccess ? DAF_OK : DAF_EDEVICE; }

bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)b_bytes && y < x + (uintptr_t)a_bytes;
}

struct Range {
  const void* at;
  int64_t bytes;
};
// Whether one of `outs` reaches into another or into one of `ins`.
template <int OUTS, int INS>
bool any_overlap(const Range (&outs)[OUTS], const Range (&ins)[INS]) {
  auto meet = [](const Range& a, const Range& b) {
    return a.at != nullptr && b.at != nullptr && a.bytes > 0 && b.bytes > 0 && overlap(a.at, a.bytes, b.at, b.bytes);
  };
  for (int i = 0; i < OUTS; ++i) {
    for (int j = i + 1; j < OUTS; ++j)
      if (meet(outs[i], outs[j])) return true;
    for (const Range& in : ins)
      if (meet(outs[i], in)) return true;
  }
  return false;
}

constexpr int64_t kMostGradients = (int64_t)1 << 45;

int grad_norm(const daf_grad_item_t* items, int32_t n_items, bool clip, float max_norm, float* out_norm, void* workspace, void* stream) {
  if (items == nullptr || n_items < 1 || out_norm == nullptr || workspace == nullptr) return DAF_EINVAL;
  if (!aligned(out_norm, 4) || !aligned(workspace, 16)) return DAF_EINVAL;
  if (clip && !(max_norm >= 0.0f)) return DAF_EINVAL;
  int64_t all = 0;
  for (int32_t i = 0; i < n_items; ++i) {
    const daf_grad_item_t& x = items[i];
    if (!known(x.dtype)) return DAF_EUNSUPPORTED;
    if (x.n < 0) return DAF_EINVAL;
    if (x.n == 0) continue;
    if (x.n > kMostGradients || (all += x.n) > kMostGradients) return DAF_EUNSUPPORTED;
    const int64_t es = elem_bytes(x.dtype);
    if (x.grad == nullptr || !aligned(x.grad, (uintptr_t)es)) return DAF_EINVAL;
    if (!clip) continue;
    if (x.out == nullptr || !aligned(x.out, (uintptr_t)es)) return DAF_EINVAL;
    if (x.out != x.grad && overlap(x.out, x.n * es, x.grad, x.n * es)) return DAF_EINVAL;
  }
  return status(daf_launch_grad_norm(items, n_items, clip, max_norm, out_norm, static_cast<double*>(workspace), static_cast<hipStream_t>(stream)));
}

// An output that reaches into an input it is not.  `same`: it may be that input.
bool clashes(const void* out, const void* in, int64_t bytes, bool same) {
  if (out == nullptr || in == nullptr || bytes == 0) return false;
  return out == in ? !same : overlap(out, bytes, in, bytes);
}

int norm_sizes(int64_t rows, int64_t cols, int64_t gate_groups) {
  if (rows < 0 || cols < 1 || gate_groups < 1 || rows % gate_groups != 0) return DAF_EINVAL;
  if (rows > ((int64_t)1 << 31) - 65536 || cols > kResidualNormMaxCols || gate_groups > (1 << 20)) return DAF_EUNSUPPORTED;
  return DAF_OK;
}

int norm_parameters(const daf_residual_norm_t* p, const void* z) {
  if (p == nullptr) return DAF_EINVAL;
  if (!known(p->dtype) || (p->kind != DAF_NORM_RMS && p->kind != DAF_NORM_LAYER)) return DAF_EUNSUPPORTED;
  if (const int bad = norm_sizes(p->rows, p->cols, p->gate_groups)) return bad;
  if (p->post != 0 && p->post != 1) return DAF_EINVAL;
  if (!(p->eps >= 0.0f)) return DAF_EINVAL;
  if (p->gate == nullptr && p->gate_groups != 1) return DAF_EINVAL;
  if (z == nullptr && p->rows > 0 && (p->post || p->gate != nullptr)) return DAF_EINVAL;
  for (const void* v : {p->pre_weight, p->pre_bias, p->post_weight, p->post_bias, p->gate})
    if (!aligned(v, 16)) return DAF_EINVAL;
  return DAF_OK;
}

int gated_sizes(int64_t M, int64_t N, int64_t K, int dtype) {
  if (dtype != DAF_F16 && dtype != DAF_BF16) return DAF_EUNSUPPORTED;
  if (M < 0 || N < 1 || K < 1) return DAF_EINVAL;
  if (M >= (1 << 24) || N >= (1 << 20) || K >= (1 << 21)) return DAF_EUNSUPPORTED;   // (256 rows of an operand are then below 2^31 bytes)
  const int64_t both = 2 * ((N + 63) / 64 * 64);
  auto too_many = [](int64_t rows, int64_t cols) { return (rows + 255) / 256 * ((cols + 255) / 256) >= kGatedMostTiles; };
  if (too_many(M, both) || too_many(M, K) || too_many(both, K)) return DAF_EUNSUPPORTED;
  if (M * (N / 8 + 8) >= (int64_t)1 << 39 || M * (K / 8 + 1) >= (int64_t)1 << 39 || N * (K / 8 + 1) >= (int64_t)1 << 39) return DAF_EUNSUPPORTED;
  return DAF_OK;
}

}  // namespace

extern "C" {

int64_t daf_grad_norm_workspace_bytes(void) { return kGradNormBlocks * (int64_t)sizeof(double); }

int daf_grad_norm(const daf_grad_item_t* items, int32_t n_items, float* out_norm, void* workspace, void* stream) {
  return grad_norm(items, n_items, false, 0.0f, out_norm, workspace, stream);
}

int daf_clip_grad_norm(const daf_grad_item_t* items, int32_t n_items, float max_norm, float* out_norm, void* workspace, void* stream) {
  return grad_norm(items, n_items, true, max_norm, out_norm, workspace, stream);
}

int daf_residual_norm(const daf_residual_norm_t* parameters, const void* residual, const void* z, void* out_residual, void* out_y,
                      float* out_stats, void* stream) {
  if (const int bad = norm_parameters(parameters, z)) return bad;
  const daf_residual_norm_t& p = *parameters;
  if (p.rows > 0 && residual == nullptr) return DAF_EINVAL;
  if (p.rows > 0 && out_residual == nullptr && out_y == nullptr) return DAF_EINVAL;
  if (!aligned(residual, 16) || !aligned(z, 16) || !aligned(out_residual, 16) || !aligned(out_y, 16) || !aligned(out_stats, 16)) return DAF_EINVAL;
  const int64_t es = elem_bytes(p.dtype), bytes = p.rows * p.cols * es, vector = p.rows > 0 ? p.cols * es : 0;   // (no rows: nothing is written)
  for (void* out : {out_residual, out_y})
    if (clashes(out, residual, bytes, true) || clashes(out, z, bytes, true)) return DAF_EINVAL;
  const Range outs[] = {{out_residual, bytes}, {out_y, bytes}, {out_stats, p.rows * 16}}, stats[] = {outs[2]}, tensors[] = {{residual, bytes}, {z, bytes}};
  const Range vectors[] = {{p.pre_weight, vector}, {p.pre_bias, vector}, {p.post_weight, vector}, {p.post_bias, vector}, {p.gate, p.gate_groups * vector}};
  if (any_overlap(outs, vectors) || any_overlap(stats, tensors)) return DAF_EINVAL;
  return status(daf_launch_residual_norm(p, residual, z, out_residual, out_y, out_stats, static_cast<hipStream_t>(stream)));
}

int64_t daf_residual_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_groups) {
  return norm_sizes(rows, cols, gate_groups) == DAF_OK ? daf_residual_norm_workspace_size(rows, cols, gate_groups) : -1;
}

int daf_residual_norm_backward(const daf_residual_norm_t* parameters, const void* sum, const void* z, const float* stats, const void* grad_y,
                               const void* grad_sum, void* out_grad_residual, void* out_grad_z, const daf_residual_norm_grads_t* grads,
                               void* workspace, void* stream) {
  if (const int bad = norm_parameters(parameters, z)) return bad;
  const daf_residual_norm_t& p = *parameters;
  if (grads == nullptr) return DAF_EINVAL;
  if (p.rows > 0) {
    if (grad_y == nullptr && grad_sum == nullptr) return DAF_EINVAL;
    if ((grad_y != nullptr && sum == nullptr) || stats == nullptr || out_grad_residual == nullptr) return DAF_EINVAL;
    if ((z == nullptr) != (out_grad_z == nullptr)) return DAF_EINVAL;
    if ((grads->pre_weight != nullptr || grads->pre_bias != nullptr) && grad_y == nullptr) return DAF_EINVAL;
    if (grads->gate != nullptr && z == nullptr) return DAF_EINVAL;
  }
  if ((grads->post_weight != nullptr || grads->post_bias != nullptr) && !p.post) return DAF_EINVAL;
  for (const void* t : {sum, z, static_cast<const void*>(stats), grad_y, grad_sum, static_cast<const void*>(out_grad_residual),
                        static_cast<const void*>(out_grad_z), static_cast<const void*>(workspace)})
    if (!aligned(t, 16)) return DAF_EINVAL;
  bool vectors = false;
  for (const float* v : {grads->pre_weight, grads->pre_bias, grads->post_weight, grads->post_bias, grads->gate}) {
    if (!aligned(v, 4)) return DAF_EINVAL;
    vectors |= v != nullptr;
  }
  const int64_t need = vectors ? daf_residual_norm_workspace_size(p.rows, p.cols, p.gate_groups) : 0;
  if (need > 0 && workspace == nullptr) return DAF_EINVAL;
  const int64_t es = elem_bytes(p.dtype), bytes = p.rows * p.cols * es, vector = p.cols * es;
  if (clashes(out_grad_residual, grad_y, bytes, true) || clashes(out_grad_residual, grad_sum, bytes, true) ||
      clashes(out_grad_residual, sum, bytes, false) || clashes(out_grad_residual, z, bytes, false) ||
      clashes(out_grad_residual, out_grad_z, bytes, false) || clashes(out_grad_z, grad_y, bytes, true) ||
      clashes(out_grad_z, grad_sum, bytes, true) || clashes(out_grad_z, z, bytes, true) || clashes(out_grad_z, sum, bytes, false))
    return DAF_EINVAL;
  const Range own[] = {{grads->pre_weight, p.cols * 4}, {grads->pre_bias, p.cols * 4}, {grads->post_weight, p.cols * 4}, {grads->post_bias, p.cols * 4},
                       {grads->gate, p.gate_groups * p.cols * 4}, {workspace, need}};
  const Range tensors[] = {{sum, bytes}, {z, bytes}, {grad_y, bytes}, {grad_sum, bytes}, {out_grad_residual, bytes}, {out_grad_z, bytes}};
  const Range outs[] = {{out_grad_residual, bytes}, {out_grad_z, bytes}}, rows_of[] = {{stats, p.rows * 16}};
  const Range parameters_of[] = {{p.pre_weight, vector}, {p.post_weight, vector}, {p.post_bias, vector}, {p.gate, p.gate_groups * vector}};
  if (any_overlap(own, tensors) || any_overlap(own, rows_of) || any_overlap(own, parameters_of) || any_overlap(outs, rows_of) ||
      any_overlap(outs, parameters_of))
    return DAF_EINVAL;
  return status(daf_launch_residual_norm_backward(p, sum, z, stats, grad_y, grad_sum, out_grad_residual, out_grad_z, *grads,
                                                  static_cast<float*>(workspace), static_cast<hipStream_t>(stream)));
}

int64_t daf_gated_linear_workspace_bytes(int64_t M, int64_t N, int64_t K, daf_dtype_t dtype) {
  if (gated_sizes(M, N, K, dtype) != DAF_OK) return -1;
  return M == 0 ? 0 : daf_gated_plan({M, N, K}, false).bytes;
}

int daf_gated_linear(const void* x, const void* w_gate, const void* w_up, int64_t M, int64_t N, int64_t K, daf_dtype_t dtype, int activation,
                     void* out_h, void* out_gate, void* out_up, void* workspace, void* stream) {
  if (const int bad = gated_sizes(M, N, K, dtype)) return bad;
  if (activation < DAF_ACT_SILU || activation > DAF_ACT_RELU) return DAF_EUNSUPPORTED;
  if (M == 0) return DAF_OK;
  if (x == nullptr || w_gate == nullptr || w_up == nullptr || out_h == nullptr || (out_gate == nullptr) != (out_up == nullptr)) return DAF_EINVAL;
  for (const void* t : {x, w_gate, w_up, static_cast<const void*>(out_h), static_cast<const void*>(out_gate), static_cast<const void*>(out_up),
                        static_cast<const void*>(workspace)})
    if (!aligned(t, 16)) return DAF_EINVAL;
  const GatedPlan plan = daf_gated_plan({M, N, K}, false);
  const int64_t need = plan.bytes;
  if (need > 0 && workspace == nullptr) return DAF_EINVAL;
  const Range outs[] = {{out_h, M * N * 2}, {out_gate, M * N * 2}, {out_up, M * N * 2}, {need > 0 ? workspace : nullptr, need}};
  const Range ins[] = {{x, M * K * 2}, {w_gate, N * K * 2}, {w_up, N * K * 2}};
  if (any_overlap(outs, ins)) return DAF_EINVAL;
  const GatedLinear g = {(int)dtype, activation, x, w_gate, w_up, static_cast<char*>(workspace)};
  return status(daf_launch_gated_linear(plan, g, out_h, out_gate, out_up, static_cast<hipStream_t>(stream)));
}

int daf_gated_linear_schedule(int64_t M, int64_t N, int64_t K, int product, daf_gated_schedule_t* out) {
  if (out == nullptr || product < DAF_GATED_FORWARD || product > DAF_GATED_GRAD_WEIGHT_OF_BOTH) return DAF_EINVAL;
  if (const int bad = gated_sizes(M, N, K, DAF_BF16)) return bad;
  if (M == 0) return DAF_EINVAL;
  const GatedPlan plan = daf_gated_plan({M, N, K}, true);
  const int of_both = product - DAF_GATED_GRAD_INPUT_OF_BOTH;
  const GatedCut& cut = of_both < 0 ? plan.cut[product] : plan.together ? plan.side[of_both] : plan.cut[DAF_GATED_GRAD_INPUT + of_both];
  *out = {kGatedForms[cut.form].rows, kGatedForms[cut.form].cols, (int32_t)cut.slices, cut.tiles, cut.whole};
  return DAF_OK;
}

int64_t daf_gated_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, daf_dtype_t dtype) {
  if (gated_sizes(M, N, K, dtype) != DAF_OK) return -1;
  return M == 0 ? 0 : daf_gated_plan({M, N, K}, true).bytes;
}

int daf_gated_linear_backward(const void* x, const void* w_gate, const void* w_up, const void* gate, const void* up, const void* grad_h, int64_t M,
                              int64_t N, int64_t K, daf_dtype_t dtype, int activation, void* out_grad_x, void* out_grad_w_gate, void* out_grad_w_up,
                              void* out_h, void* workspace, void* stream) {
  if (const int bad = gated_sizes(M, N, K, dtype)) return bad;
  if (activation < DAF_ACT_SILU || activation > DAF_ACT_RELU) return DAF_EUNSUPPORTED;
  if ((out_grad_w_gate == nullptr) != (out_grad_w_up == nullptr)) return DAF_EINVAL;
  for (const void* t : {x, w_gate, w_up, gate, up, grad_h, static_cast<const void*>(out_grad_x), static_cast<const void*>(out_grad_w_gate),
                        static_cast<const void*>(out_grad_w_up), static_cast<const void*>(out_h), static_cast<const void*>(workspace)})
    if (!aligned(t, 16)) return DAF_EINVAL;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (M == 0) {
    if (out_grad_w_gate == nullptr) return DAF_OK;
    if (overlap(out_grad_w_gate, N * K * 2, out_grad_w_up, N * K * 2)) return DAF_EINVAL;
    const hipError_t e = daf_launch_clear(out_grad_w_gate, N * K * 2, s);
    return status(e == hipSuccess ? daf_launch_clear(out_grad_w_up, N * K * 2, s) : e);
  }
  if (x == nullptr || w_gate == nullptr || w_up == nullptr || grad_h == nullptr || workspace == nullptr || (gate == nullptr) != (up == nullptr))
    return DAF_EINVAL;
  if (gate != nullptr && out_h != nullptr) return DAF_EINVAL;
  if (out_grad_x == nullptr && out_grad_w_gate == nullptr && out_h == nullptr) return DAF_EINVAL;
  const GatedPlan plan = daf_gated_plan({M, N, K}, true);
  const Range outs[] = {{out_grad_x, M * K * 2}, {out_grad_w_gate, N * K * 2}, {out_grad_w_up, N * K * 2}, {out_h, M * N * 2},
                        {workspace, plan.bytes}};
  const Range ins[] = {{x, M * K * 2}, {w_gate, N * K * 2}, {w_up, N * K * 2}, {gate, M * N * 2}, {up, M * N * 2}, {grad_h, M * N * 2}};
  if (any_overlap(outs, ins)) return DAF_EINVAL;
  const GatedLinear g = {(int)dtype, activation, x, w_gate, w_up, static_cast<char*>(workspace)};
  return status(daf_launch_gated_linear_backward(plan, g, grad_h, gate, up, out_grad_x, out_grad_w_gate, out_grad_w_up, out_h, s));
}

}  // extern "C"

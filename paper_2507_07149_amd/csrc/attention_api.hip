// C ABI of daf_attention.h: argument checks and dispatch to the launchers.  Every check comes before the first HIP call.
#include <cmath>

#include "daf_attention.h"
#include "head_rotation.h"
#include "window_attention.h"

namespace {

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int status(hipError_t e) { return e == hipSuccess ? DAF_OK : DAF_EDEVICE; }

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 65536, kMostHeads = 4096, kMostStride = (int64_t)1 << 40,
                  kMostExtent = (int64_t)1 << 56;                       // (of elements: products of sizes stay below 2^63)

// Memory that a call reads or writes, in bytes: rows x heads pieces of `width`; plain memory is one piece.
struct Region {
  uintptr_t at;
  int64_t rows, heads, token, head, width;
  int64_t across() const { return head * (heads - 1) + width; }        // of one token's heads
  int64_t down() const { return token * (rows - 1) + width; }          // of one head's tokens
  int64_t extent() const { return token * (rows - 1) + across(); }
  bool empty() const { return at == 0 || rows <= 0 || heads <= 0 || width <= 0; }
  bool same(const Region& b) const { return at == b.at && rows == b.rows && heads == b.heads && token == b.token && head == b.head && width == b.width; }
  bool overlaps_itself() const { return !empty() && rows > 1 && heads > 1 && across() > token && down() > head; }
};
Region memory(const void* p, int64_t bytes) { return {reinterpret_cast<uintptr_t>(p), 1, 1, 0, 0, bytes}; }
Region region(const daf_heads_t* h, int64_t rows, int64_t heads, int64_t dim, int64_t es) {
  if (h == nullptr) return memory(nullptr, 0);
  return {reinterpret_cast<uintptr_t>(h->at), rows, heads, rows > 1 ? h->token_stride * es : 0, heads > 1 ? h->head_stride * es : 0, dim * es};
}
// Beside each other within a stride that they have in common.
bool beside(uintptr_t a, int64_t a_width, uintptr_t b, int64_t b_width, int64_t stride) {
  if (a_width > stride || b_width > stride) return false;
  const int64_t far = (int64_t)((b - a) % (uintptr_t)stride);
  const int64_t apart = b >= a ? far : (stride - (int64_t)((a - b) % (uintptr_t)stride)) % stride;
  return apart >= a_width && apart + b_width <= stride;
}
bool overlap(const Region& a, const Region& b) {
  if (a.empty() || b.empty()) return false;
  if (a.at + (uintptr_t)a.extent() <= b.at || b.at + (uintptr_t)b.extent() <= a.at) return false;
  if (a.rows > 1 && b.rows > 1 && a.token == b.token && beside(a.at, a.across(), b.at, b.across(), a.token)) return false;
  if (a.heads > 1 && b.heads > 1 && a.head == b.head && beside(a.at, a.down(), b.at, b.down(), a.head)) return false;
  return true;
}
// Whether one of `outs` reaches into itself, into another or into one of `ins`.
template <int OUTS, int INS>
bool any_overlap(const Region (&outs)[OUTS], const Region (&ins)[INS]) {
  for (int i = 0; i < OUTS; ++i) {
    if (outs[i].overlaps_itself()) return true;
    for (int j = i + 1; j < OUTS; ++j)
      if (overlap(outs[i], outs[j])) return true;
    for (const Region& in : ins)
      if (overlap(outs[i], in)) return true;
  }
  return false;
}

bool good_heads(const daf_heads_t* h, int64_t rows, int64_t heads, int64_t dim, int64_t es) {
  if (h == nullptr) return false;
  if (rows == 0) return true;
  if (h->at == nullptr || !aligned(h->at, 16)) return false;
  auto stride = [&](int64_t count, int64_t s) { return count <= 1 || (s >= dim && s <= kMostStride && s <= kMostExtent / count && s * es % 16 == 0); };
  return stride(rows, h->token_stride) && stride(heads, h->head_stride);
}

int rotation_sizes(int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t dim) {
  if (tokens < 0 || q_heads < 1 || kv_heads < 1 || dim < 1) return DAF_EINVAL;
  if (tokens > kMostRows || q_heads > kMostHeads || kv_heads > kMostHeads || dim > kRotationMaxDim || dim % 8 != 0) return DAF_EUNSUPPORTED;
  return DAF_OK;
}
int rotation_parameters(const daf_head_rotation_t* p) {
  if (p == nullptr) return DAF_EINVAL;
  if (p->dtype != DAF_F32 && p->dtype != DAF_F16 && p->dtype != DAF_BF16) return DAF_EUNSUPPORTED;
  if (p->pairing != DAF_ROTATE_HALVES && p->pairing != DAF_ROTATE_PAIRS) return DAF_EUNSUPPORTED;
  if (const int bad = rotation_sizes(p->tokens, p->q_heads, p->kv_heads, p->head_dim)) return bad;
  if (p->rotary_dim < 0 || p->positions < 0) return DAF_EINVAL;
  if (p->rotary_dim > p->head_dim || p->rotary_dim % 16 != 0 || p->positions > kMostRows) return DAF_EUNSUPPORTED;
  if (p->norm != 0 && p->norm != 1) return DAF_EINVAL;
  if (!(p->eps >= 0.0f)) return DAF_EINVAL;
  if (!p->norm && (p->q_weight != nullptr || p->k_weight != nullptr)) return DAF_EINVAL;
  for (const void* v : {p->q_weight, p->k_weight, static_cast<const void*>(p->cos), static_cast<const void*>(p->sin)})
    if (!aligned(v, 16)) return DAF_EINVAL;
  if (!aligned(p->position, 4)) return DAF_EINVAL;
  if (p->tokens > 0 && p->position == nullptr) return DAF_EINVAL;
  if (p->tokens > 0 && p->rotary_dim > 0 && p->positions > 0 && (p->cos == nullptr || p->sin == nullptr)) return DAF_EINVAL;
  return DAF_OK;
}

int attention_sizes(int64_t q_rows, int64_t k_rows, int64_t q_heads, int64_t kv_heads, int64_t dim, int64_t sequences, int64_t window, int64_t sinks,
                    int64_t most_sequences) {
  if (q_rows < 0 || k_rows < 0 || q_heads < 1 || kv_heads < 1 || dim < 1 || sequences < 1 || window < 0 || sinks < 0) return DAF_EINVAL;
  if (q_heads % kv_heads != 0) return DAF_EINVAL;
  if (q_rows >= kAttentionMostRows || k_rows >= kAttentionMostRows || q_heads > kMostHeads || dim > kAttentionMaxDim || dim % 8 != 0) return DAF_EUNSUPPORTED;
  if (sequences > most_sequences || q_heads * (q_rows / 32 + sequences) >= (int64_t)1 << 22) return DAF_EUNSUPPORTED;
  return DAF_OK;
}
int attention_parameters(const daf_window_attention_t* p, int64_t most_sequences = kAttentionMaxSequences) {
  if (p == nullptr) return DAF_EINVAL;
  if (p->dtype != DAF_F16 && p->dtype != DAF_BF16) return DAF_EUNSUPPORTED;
  if (const int bad = attention_sizes(p->q_rows, p->k_rows, p->q_heads, p->kv_heads, p->head_dim, p->sequences, p->window, p->sinks,
                                      most_sequences))
    return bad;
  if (!std::isfinite(p->scale)) return DAF_EINVAL;
  if (!aligned(p->q_starts, 4) || !aligned(p->k_starts, 4) || !aligned(p->k_lengths, 4)) return DAF_EINVAL;
  if ((p->k_starts == nullptr) != (p->k_lengths == nullptr)) return DAF_EINVAL;
  return DAF_OK;
}
constexpr int64_t kMostTokenStride = (int64_t)1 << 23;                  // (64 rows of heads are then below 2^31 bytes)
bool far_rows(const daf_heads_t* h, int64_t rows) { return rows > 1 && h->token_stride >= kMostTokenStride; }

}  // namespace

extern "C" {

int daf_head_rotation(const daf_head_rotation_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* v, const daf_heads_t* out_q,
                      const daf_heads_t* out_k, const daf_heads_t* out_v, const int32_t* rows, int64_t out_rows, void* stream) {
  if (const int bad = rotation_parameters(parameters)) return bad;
  const daf_head_rotation_t& p = *parameters;
  const int64_t n = p.tokens, d = p.head_dim, es = p.dtype == DAF_F32 ? 4 : 2;
  if (out_rows < 0 || !aligned(rows, 4) || (rows == nullptr && out_rows != n) || (v == nullptr) != (out_v == nullptr)) return DAF_EINVAL;
  if (out_rows > kMostRows) return DAF_EUNSUPPORTED;
  if (!good_heads(q, n, p.q_heads, d, es) || !good_heads(k, n, p.kv_heads, d, es) || !good_heads(out_q, n, p.q_heads, d, es)) return DAF_EINVAL;
  if (!good_heads(out_k, out_rows, p.kv_heads, d, es)) return DAF_EINVAL;
  if (v != nullptr && (!good_heads(v, n, p.kv_heads, d, es) || !good_heads(out_v, out_rows, p.kv_heads, d, es))) return DAF_EINVAL;
  const Region none = memory(nullptr, 0);
  const Region outs[] = {region(out_q, n, p.q_heads, d, es), region(out_k, out_rows, p.kv_heads, d, es), region(out_v, out_rows, p.kv_heads, d, es)};
  Region ins[] = {region(q, n, p.q_heads, d, es), region(k, n, p.kv_heads, d, es), region(v, n, p.kv_heads, d, es)};
  for (int i = 0; i < 3; ++i) {                                        // in place: against the others
    if (outs[i].same(ins[i]) && (i == 0 || rows == nullptr)) {
      for (int j = 0; j < 3; ++j)
        if (j != i && overlap(outs[j], ins[i])) return DAF_EINVAL;
      ins[i] = none;
    }
  }
  const Region beside[] = {memory(p.q_weight, d * es), memory(p.k_weight, d * es), memory(p.cos, p.positions * p.rotary_dim * 2),
                           memory(p.sin, p.positions * p.rotary_dim * 2), memory(p.position, n * 4), memory(rows, n * 4)};
  if (n > 0 && (any_overlap(outs, ins) || any_overlap(outs, beside))) return DAF_EINVAL;
  return status(daf_launch_head_rotation(p, *q, *k, v, *out_q, *out_k, out_v, rows, out_rows, static_cast<hipStream_t>(stream)));
}

int64_t daf_head_rotation_backward_workspace_bytes(int64_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim) {
  return rotation_sizes(tokens, q_heads, kv_heads, head_dim) == DAF_OK ? daf_head_rotation_workspace_size(tokens, head_dim) : -1;
}

int daf_head_rotation_backward(const daf_head_rotation_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* grad_q,
                               const daf_heads_t* grad_k, const daf_heads_t* out_grad_q, const daf_heads_t* out_grad_k, float* out_grad_q_weight,
                               float* out_grad_k_weight, void* workspace, void* stream) {
  if (const int bad = rotation_parameters(parameters)) return bad;
  const daf_head_rotation_t& p = *parameters;
  const int64_t n = p.tokens, d = p.head_dim, es = p.dtype == DAF_F32 ? 4 : 2;
  const bool weights = out_grad_q_weight != nullptr || out_grad_k_weight != nullptr;
  if (weights && !p.norm) return DAF_EINVAL;
  if (!aligned(out_grad_q_weight, 4) || !aligned(out_grad_k_weight, 4) || !aligned(workspace, 16)) return DAF_EINVAL;
  if (p.norm && (!good_heads(q, n, p.q_heads, d, es) || !good_heads(k, n, p.kv_heads, d, es))) return DAF_EINVAL;
  if (!good_heads(grad_q, n, p.q_heads, d, es) || !good_heads(grad_k, n, p.kv_heads, d, es)) return DAF_EINVAL;
  if (!good_heads(out_grad_q, n, p.q_heads, d, es) || !good_heads(out_grad_k, n, p.kv_heads, d, es)) return DAF_EINVAL;
  const int64_t need = weights ? daf_head_rotation_workspace_size(n, (int)d) : 0;
  if (need > 0 && workspace == nullptr) return DAF_EINVAL;
  const Region none = memory(nullptr, 0);
  const Region outs[] = {region(out_grad_q, n, p.q_heads, d, es), region(out_grad_k, n, p.kv_heads, d, es), memory(out_grad_q_weight, d * 4),
                         memory(out_grad_k_weight, d * 4), memory(need > 0 ? workspace : nullptr, need)};
  Region grads[] = {region(grad_q, n, p.q_heads, d, es), region(grad_k, n, p.kv_heads, d, es)};
  for (int i = 0; i < 2; ++i) {                                        // in place: against the others
    if (!outs[i].same(grads[i])) continue;
    for (int j = 0; j < 5; ++j)
      if (j != i && overlap(outs[j], grads[i])) return DAF_EINVAL;
    grads[i] = none;
  }
  const Region ins[] = {p.norm ? region(q, n, p.q_heads, d, es) : none, p.norm ? region(k, n, p.kv_heads, d, es) : none, memory(p.q_weight, d * es),
                        memory(p.k_weight, d * es), memory(p.cos, p.positions * p.rotary_dim * 2), memory(p.sin, p.positions * p.rotary_dim * 2),
                        memory(p.position, n * 4)};
  if (any_overlap(outs, grads) || any_overlap(outs, ins)) return DAF_EINVAL;
  const daf_heads_t unread = {nullptr, 0, 0};
  return status(daf_launch_head_rotation_backward(p, p.norm ? *q : unread, p.norm ? *k : unread, *grad_q, *grad_k, *out_grad_q, *out_grad_k,
                                                  out_grad_q_weight, out_grad_k_weight, static_cast<float*>(workspace), static_cast<hipStream_t>(stream)));
}

int daf_window_attention(const daf_window_attention_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* v,
                         const daf_heads_t* out, float* out_lse, void* stream) {
  if (const int bad = attention_parameters(parameters)) return bad;
  const daf_window_attention_t& p = *parameters;
  if ((p.q_starts == nullptr && p.sequences != 1) || (p.k_starts == nullptr && p.k_rows != p.q_rows)) return DAF_EINVAL;
  if (!aligned(out_lse, 4)) return DAF_EINVAL;
  const int64_t d = p.head_dim;
  if (!good_heads(q, p.q_rows, p.q_heads, d, 2) || !good_heads(out, p.q_rows, p.q_heads, d, 2) || !good_heads(k, p.k_rows, p.kv_heads, d, 2) ||
      !good_heads(v, p.k_rows, p.kv_heads, d, 2))
    return DAF_EINVAL;
  if (far_rows(q, p.q_rows) || far_rows(out, p.q_rows) || far_rows(k, p.k_rows) || far_rows(v, p.k_rows)) return DAF_EUNSUPPORTED;
  const Region outs[] = {region(out, p.q_rows, p.q_heads, d, 2), memory(out_lse, p.q_rows * p.q_heads * 4)};
  const Region ins[] = {region(q, p.q_rows, p.q_heads, d, 2), region(k, p.k_rows, p.kv_heads, d, 2), region(v, p.k_rows, p.kv_heads, d, 2),
                        memory(p.q_starts, (p.sequences + 1) * 4), memory(p.k_starts, p.sequences * 4), memory(p.k_lengths, p.sequences * 4)};
  if (any_overlap(outs, ins)) return DAF_EINVAL;
  return status(daf_launch_window_attention(p, {*q, *k, *v, *out, out_lse}, static_cast<hipStream_t>(stream)));
}

int64_t daf_window_attention_backward_workspace_bytes(int64_t rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t sequences, int64_t window,
                                                      int64_t sinks) {
  if (attention_sizes(rows, rows, q_heads, kv_heads, head_dim, sequences, window, sinks, kAttentionMaxSequences) != DAF_OK) return -1;
  return daf_window_attention_backward_workspace_bound(rows, q_heads, kv_heads, head_dim, sequences, window, sinks);
}

int daf_window_attention_backward(const daf_window_attention_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* v,
                                  const daf_heads_t* out, const float* lse, const daf_heads_t* grad_out, const daf_heads_t* out_grad_q,
                                  const daf_heads_t* out_grad_k, const daf_heads_t* out_grad_v, void* workspace, void* stream) {
  if (const int bad = attention_parameters(parameters)) return bad;
  const daf_window_attention_t& p = *parameters;
  if (p.k_starts != nullptr || p.k_rows != p.q_rows || (p.q_starts == nullptr && p.sequences != 1)) return DAF_EINVAL;
  const int64_t n = p.q_rows, d = p.head_dim;
  for (const daf_heads_t* h : {q, out, grad_out, out_grad_q})
    if (!good_heads(h, n, p.q_heads, d, 2)) return DAF_EINVAL;
  for (const daf_heads_t* h : {k, v, out_grad_k, out_grad_v})
    if (!good_heads(h, n, p.kv_heads, d, 2)) return DAF_EINVAL;
  for (const daf_heads_t* h : {q, k, v, out, grad_out, out_grad_q, out_grad_k, out_grad_v})
    if (far_rows(h, n)) return DAF_EUNSUPPORTED;
  if (!aligned(lse, 4) || !aligned(workspace, 16) || (n > 0 && (lse == nullptr || workspace == nullptr))) return DAF_EINVAL;
  const int64_t need = daf_window_attention_backward_workspace_size(n, p.q_heads, p.kv_heads, p.head_dim, p.sequences, p.window, p.sinks);
  const Region outs[] = {region(out_grad_q, n, p.q_heads, d, 2), region(out_grad_k, n, p.kv_heads, d, 2), region(out_grad_v, n, p.kv_heads, d, 2),
                         memory(workspace, need)};
  const Region ins[] = {region(q, n, p.q_heads, d, 2),   region(k, n, p.kv_heads, d, 2), region(v, n, p.kv_heads, d, 2),
                        region(out, n, p.q_heads, d, 2), region(grad_out, n, p.q_heads, d, 2), memory(lse, n * p.q_heads * 4),
                        memory(p.q_starts, (p.sequences + 1) * 4)};
  if (any_overlap(outs, ins)) return DAF_EINVAL;
  return status(daf_launch_window_attention_backward(p, {*q, *k, *v, *out, const_cast<float*>(lse)}, {*grad_out, *out_grad_q, *out_grad_k, *out_grad_v},
                                                     static_cast<char*>(workspace), static_cast<hipStream_t>(stream)));
}

int64_t daf_window_attention_step_workspace_bytes(int64_t sequences, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t k_rows, int64_t window,
                                                  int64_t sinks) {
  if (sequences == 0) return attention_sizes(0, k_rows, q_heads, kv_heads, head_dim, 1, window, sinks, 1) == DAF_OK ? 0 : -1;
  if (attention_sizes(sequences, k_rows, q_heads, kv_heads, head_dim, sequences, window, sinks, kAttentionMaxSteps) != DAF_OK) return -1;
  return daf_window_attention_step_workspace_bound(sequences, q_heads, kv_heads, head_dim, k_rows, window, sinks);
}

int daf_window_attention_step(const daf_window_attention_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* v,
                              const daf_heads_t* out, void* workspace, void* stream) {
  if (parameters != nullptr && parameters->q_rows == 0 && parameters->sequences == 0) return DAF_OK;
  if (const int bad = attention_parameters(parameters, kAttentionMaxSteps)) return bad;
  const daf_window_attention_t& p = *parameters;
  if (p.q_starts != nullptr || p.q_rows != p.sequences || p.k_starts == nullptr) return DAF_EINVAL;
  const int64_t d = p.head_dim;
  if (!good_heads(q, p.q_rows, p.q_heads, d, 2) || !good_heads(out, p.q_rows, p.q_heads, d, 2) || !good_heads(k, p.k_rows, p.kv_heads, d, 2) ||
      !good_heads(v, p.k_rows, p.kv_heads, d, 2))
    return DAF_EINVAL;
  if (far_rows(q, p.q_rows) || far_rows(out, p.q_rows) || far_rows(k, p.k_rows) || far_rows(v, p.k_rows)) return DAF_EUNSUPPORTED;
  const int64_t need = daf_window_attention_step_workspace_size(p.sequences, p.q_heads, p.kv_heads, p.head_dim, p.k_rows, p.window, p.sinks);
  if (!aligned(workspace, 16) || (need > 0 && workspace == nullptr)) return DAF_EINVAL;
  const Region outs[] = {region(out, p.q_rows, p.q_heads, d, 2), memory(need > 0 ? workspace : nullptr, need)};
  const Region ins[] = {region(q, p.q_rows, p.q_heads, d, 2), region(k, p.k_rows, p.kv_heads, d, 2), region(v, p.k_rows, p.kv_heads, d, 2),
                        memory(p.k_starts, p.sequences * 4), memory(p.k_lengths, p.sequences * 4)};
  if (any_overlap(outs, ins)) return DAF_EINVAL;
  return status(daf_launch_window_attention_step(p, {*q, *k, *v, *out, nullptr}, static_cast<char*>(workspace), static_cast<hipStream_t>(stream)));
}

}  // extern "C"

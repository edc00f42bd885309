/* daf_attention.h -- C ABI of the operators of a transformer block's attention half: the norms of every head and the rotation by position,
 * and causal attention with a window and first tokens that stay visible, for training (with their gradients) and for serving (prompts, pieces
 * of prompts over a cache, one token of each of many sequences).
 *
 * Conventions as in daf_block.h: DEVICE and HOST pointers, `stream` a hipStream_t as void*, status codes, no exceptions, no allocation, no
 * synchronization, argument checks before any HIP call.  Work runs on the current HIP device.  Calls may be captured into a HIP graph.  Results are
 * deterministic: the same call gives the same bits.  NaN and infinities in the inputs go through to the outputs as the formulas have them;
 * elements that a formula does not name (keys that a query does not see, rows of no sequence) have no influence, whatever they hold.
 */
#ifndef DAF_ATTENTION_H_
#define DAF_ATTENTION_H_

#include "daf_block.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Heads of tokens: element i of head h of row t is at[t * token_stride + h * head_stride + i] (strides in elements), on the DEVICE.  The first
 * element is at a multiple of 16 bytes; a stride by which more than one row (head) goes is a multiple of 16 bytes and at least head_dim.  A view of a projection's result [tokens, all heads x head_dim] is such heads, and so is [heads, tokens, head_dim].  Heads that are written
 * must not overlap one another: not themselves, nor anything else that the call reads or writes, where it is not named as the same.  Views of one
 * buffer that have a stride in common and lie beside each other within it do not overlap. */
typedef struct {
  void* at;
  int64_t token_stride, head_stride;
} daf_heads_t;

/* ---- norms of heads and rotation by position --------------------------------------------------
 *
 * daf_head_rotation -- for every head x of a token of queries and of keys, in one pass:
 *     n = x * rstd * weight, rstd = 1 / sqrt(mean(x^2) + eps)      (norm != 0; else n = x)
 *     a' = a cos - b sin,  b' = a sin + b cos                       for every pair (a, b) of the first rotary_dim elements of n
 * in binary32, rounded once.  The rest of n stays as it is.  With v its heads are copied as they are.
 *
 *   parameters    the struct below, on the HOST.
 *   pairing       DAF_ROTATE_HALVES: pair i is elements i and i + rotary_dim / 2; DAF_ROTATE_PAIRS: elements 2i and 2i + 1.
 *   q_weight, k_weight   DEVICE, head_dim elements of dtype, 16-byte aligned; NULL: 1.
 *   cos, sin      DEVICE, floats [positions, rotary_dim / 2], 16-byte aligned; may be NULL if positions or rotary_dim is 0.
 *   position      DEVICE, int32, one for each token: its row of cos and sin.  A token whose position is not one of 0 ... positions - 1 gets zeros
 *                 in queries and keys (and zero gradients), whatever it holds: rows that pad a batch.
 *   out_q, out_k, out_v  where the heads go; out_q may be q itself, with its strides, out_k k and out_v v (without `rows`).
 *   v, out_v      both or neither (NULL).
 *   rows          DEVICE, int32, one for each token: the row of out_k and out_v that it goes to (a cache), of out_rows that there are.  A token with
 *                 another number is not written there; a row that is named twice holds elements of either token.  NULL: row t, and out_rows is tokens.
 *
 * daf_head_rotation_backward -- from the gradients of the rotated heads (grad_q, grad_k): the gradients of q and k, which are read as the forward
 * pass read them, and of both weights, summed over tokens and heads in binary32 in a fixed order.
 *
 *   q, k          read only where norm != 0 (may be NULL otherwise).
 *   out_grad_q    may be grad_q itself, with its strides; out_grad_k likewise.
 *   out_grad_q_weight, out_grad_k_weight  DEVICE, head_dim floats, or NULL: not wanted.  Only with norm.
 *   workspace     DEVICE, daf_head_rotation_backward_workspace_bytes(...) bytes (enough for fewer tokens too), 16-byte aligned, needs no preparation; calls that share one
 *                 must not overlap in time.  May be NULL if no weight's gradient is wanted.
 *
 * tokens may be 0 (the weights' gradients are then zero).  head_dim: multiples of 8 up to 256; rotary_dim: multiples of 16 up to head_dim, or 0.
 * Errors: DAF_EINVAL (null or misaligned pointer, a size below its least, strides as they must not be, overlaps, eps negative or NaN),
 * DAF_EUNSUPPORTED (dtype, pairing, head_dim, rotary_dim, 2^31 - 2^16 or more tokens, rows or positions, more than 4096 heads of a kind), DAF_EDEVICE. */
typedef enum { DAF_ROTATE_HALVES = 0, DAF_ROTATE_PAIRS = 1 } daf_rotation_pairing_t;

typedef struct {
  int64_t tokens;
  int64_t positions;           /* rows of cos and sin */
  int32_t q_heads, kv_heads, head_dim, rotary_dim;
  int32_t dtype;               /* a daf_dtype_t */
  int32_t pairing;             /* a daf_rotation_pairing_t */
  int32_t norm;                /* 1: heads are normalized */
  float eps;
  const void *q_weight, *k_weight;
  const float *cos, *sin;
  const int32_t* position;
} daf_head_rotation_t;

int daf_head_rotation(const daf_head_rotation_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* v, const daf_heads_t* out_q,
                      const daf_heads_t* out_k, const daf_heads_t* out_v, const int32_t* rows, int64_t out_rows, void* stream);
int64_t daf_head_rotation_backward_workspace_bytes(int64_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim);
int daf_head_rotation_backward(const daf_head_rotation_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* grad_q,
                               const daf_heads_t* grad_k, const daf_heads_t* out_grad_q, const daf_heads_t* out_grad_k, float* out_grad_q_weight,
                               float* out_grad_k_weight, void* workspace, void* stream);

/* ---- attention with a window and sinks ---------------------------------------------------------
 *
 * daf_window_attention -- causal attention within each of `sequences` sequences.  Sequence b has queries q_starts[b] ... q_starts[b + 1] - 1 and
 * keys k_starts[b] ... k_starts[b] + k_lengths[b] - 1, at positions 0, 1, ...; its last query stands at its last key.  The query at position p
 * sees the keys j <= p for which p - j < window or j < sinks (window 0: all j <= p):
 *     s_j = scale * q . k_j,  lse = log(sum over seen j of exp(s_j)),  out = sum over seen j of exp(s_j - lse) v_j
 * Query head h reads key head h / (q_heads / kv_heads).  Scores, lse and sums are binary32; exp(s_j - max) is rounded to dtype for the product with v (on
 * the matrix cores), not for its own sum; out is rounded once.  A query that sees nothing (it stands in front of its first key) gets
 * out = 0 and lse = -infinity.
 *
 *   parameters  the struct below, on the HOST.
 *   q_starts    DEVICE, sequences + 1 int32 that do not decrease, within 0 ... q_rows; NULL: one sequence of all rows (sequences 1).  Rows
 *               in front of the first and behind the last are left as they were, in all outputs.
 *   k_starts, k_lengths   DEVICE, int32 for each sequence, within the k_rows rows; sequences may share rows.  NULL (both): each sequence's keys are its
 *               queries' rows (k_rows is q_rows).
 *               Starts and lengths that go out of the rows are cut to them.
 *   out_lse     floats [q_heads, q_rows], or NULL: not wanted (it is what the backward pass needs).
 *
 * daf_window_attention_backward -- for keys that are the queries' rows (k_starts and k_lengths NULL), from out and lse as the forward pass wrote them:
 *     P = exp(s - lse),  dP = grad_out . v,  dS = P (dP - sum(grad_out * out)) * scale
 *     grad_q = sum over keys of dS k,  grad_k = sum over queries, and heads that share the key, of dS q,  grad_v = the same sum of P grad_out
 * P and dS are rounded to dtype for their products; sums are binary32, in a fixed order, rounded once.
 *
 *   workspace   DEVICE, daf_window_attention_backward_workspace_bytes(...) bytes, as above.  As many are enough for fewer rows or sequences too.
 *
 * daf_window_attention_step -- one query for each sequence (q_rows is sequences, q_starts NULL), standing at its last key; k_starts and k_lengths as above
 * (not NULL).  For caches that many workgroups read at once: a sequence's keys are cut into pieces that are joined afterwards.
 * A q . k_j out of binary32's range is infinite here, whatever scale is.
 *
 *   workspace   DEVICE, daf_window_attention_step_workspace_bytes(...) bytes, as above, enough for fewer sequences or rows too; may be NULL if 0 are needed, also
 *               where the call itself, of so many sequences that none is cut, needs none (else it is refused).
 *
 * q_rows may be 0.  head_dim: multiples of 8 up to 128.  q_heads is a multiple of kv_heads.
 * Errors: DAF_EINVAL (null or misaligned pointer, a size below its least, heads that do not divide, window or sinks below 0, a scale that is no finite number,
 * strides as they must not be, outputs that overlap each other or an input), DAF_EUNSUPPORTED (binary32; head_dim; 2^30 or more rows; token strides of 2^23 elements or more;
 * more than 4096 heads of a kind; more than 2^16 sequences, in a step 2^20; q_heads * (q_rows / 32 + sequences) of 2^22 or more), DAF_EDEVICE.  The workspace queries return -1 for such sizes. */
typedef struct {
  int64_t q_rows, k_rows, sequences;
  int64_t window, sinks;
  int32_t q_heads, kv_heads, head_dim;
  int32_t dtype;               /* a daf_dtype_t */
  float scale;
  const int32_t *q_starts, *k_starts, *k_lengths;
} daf_window_attention_t;

int daf_window_attention(const daf_window_attention_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* v,
                         const daf_heads_t* out, float* out_lse, void* stream);
int64_t daf_window_attention_backward_workspace_bytes(int64_t rows, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t sequences, int64_t window,
                                                      int64_t sinks);
int daf_window_attention_backward(const daf_window_attention_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* v,
                                  const daf_heads_t* out, const float* lse, const daf_heads_t* grad_out, const daf_heads_t* out_grad_q,
                                  const daf_heads_t* out_grad_k, const daf_heads_t* out_grad_v, void* workspace, void* stream);
int64_t daf_window_attention_step_workspace_bytes(int64_t sequences, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t k_rows, int64_t window,
                                                  int64_t sinks);
int daf_window_attention_step(const daf_window_attention_t* parameters, const daf_heads_t* q, const daf_heads_t* k, const daf_heads_t* v,
                              const daf_heads_t* out, void* workspace, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* DAF_ATTENTION_H_ */

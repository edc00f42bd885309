/* daf_block.h -- C ABI of the operators that a transformer block's training step runs around the activations that daf.h keeps
 * packed: the norms, gate and residual sum between two blocks, the gated feed-forward product, and the clipping of the
 * gradients, each with its backward pass where it has one.
 *
 * Conventions as in daf.h: DEVICE and HOST pointers, `stream` a hipStream_t as void*, status codes, no exceptions, no
 * allocation, no synchronization, argument checks before any HIP call.  All tensors are row-major contiguous.  Work runs on the
 * current HIP device.  Calls may be captured into a HIP graph.  Results are deterministic: the same call gives the same bits.
 * NaN and infinities in the inputs go through to the outputs as the formulas have them.
 */
#ifndef DAF_BLOCK_H_
#define DAF_BLOCK_H_

#include "daf.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- clipping of gradients by their global norm -------------------------------------------
 *
 * daf_grad_norm -- norm = sqrt(sum over all tensors and elements of g^2).  Squares and sums are taken in 64 bits, in an order that
 * depends on the list alone; the result is rounded to binary32 once.
 *
 * daf_clip_grad_norm -- the same norm, and out = round_to_dtype(g * factor) for every element, with
 *     factor = min(1, max_norm / (norm + 1e-6))     (binary32, from the rounded norm; NaN if the norm is NaN)
 * computed on the device: no host round trip.  A factor of exactly 1 leaves gradients that are clipped in place unwritten.  An
 * infinite norm makes the factor 0 and the finite gradients with it, unless max_norm is infinite too: the factor is then 1.
 *
 *   items      HOST array; read during the call only.  A tensor of n elements (0 allowed) at `grad` (DEVICE, aligned to
 *              its element), in the format `dtype` (each item its own).  `out` (DEVICE, aligned to its element): where the
 *              clipped tensor goes, in the same format; `grad` itself, or memory that overlaps no tensor of the list
 *              (checked against the item's own grad).  daf_grad_norm does not read `out`.
 *   n_items    >= 1.  A launch carries up to 200 tensors, up to 144 in a call that does not clip all in place; longer lists take more.
 *   max_norm   >= 0; infinity clips nothing, whatever the norm (NaN apart).
 *   out_norm   DEVICE, one float.
 *   workspace  DEVICE, daf_grad_norm_workspace_bytes() bytes, 16-byte aligned; needs no preparation; calls that share
 *              one must not overlap in time.
 *
 * Errors: DAF_EINVAL (null or misaligned pointer, n < 0, n_items < 1, max_norm negative or NaN, out overlapping grad in part),
 * DAF_EUNSUPPORTED (dtype; more than 2^45 elements in the list), DAF_EDEVICE. */
typedef struct {
  const void* grad;
  void* out;
  int64_t n;
  int32_t dtype;       /* a daf_dtype_t */
} daf_grad_item_t;

int64_t daf_grad_norm_workspace_bytes(void);
int daf_grad_norm(const daf_grad_item_t* items, int32_t n_items, float* out_norm, void* workspace, void* stream);
int daf_clip_grad_norm(const daf_grad_item_t* items, int32_t n_items, float max_norm, float* out_norm, void* workspace, void* stream);

/* ---- the norms, gate and residual sum between two blocks -------------------------------------
 *
 * daf_residual_norm -- in one pass over a block's output z and the residual stream r, rows of `cols` elements:
 *     p = post(z)                        the norm behind the block (post != 0), else p = z
 *     s = r + scale * gate * p           residual sum; gate one value per column, per run of rows, or 1
 *     y = pre(s)                         the norm in front of the next block
 * A norm is n(v) = (v - mean) * rstd * weight + bias with rstd = 1 / sqrt(mean((v - mean)^2) + eps) over the row
 * (DAF_NORM_LAYER), or with mean = 0 (DAF_NORM_RMS).  Everything is computed in binary32 and rounded once where it is written; y
 * is the norm of s before its rounding.
 *
 *   parameters  the struct below, on the HOST; the vectors in it DEVICE, `cols` elements of dtype, 16-byte aligned, or NULL:
 *               a weight of 1, a bias of 0, no gate (gate_groups is then 1).  `post` and a gate need z.
 *   residual    DEVICE, rows * cols elements of dtype, aligned to 16 bytes as all tensors here.
 *   z           the block's output, or NULL: s = r (the norm alone).
 *   out_residual  s, or NULL: not wanted.  May be residual or z itself.
 *   out_y       y, or NULL: no norm behind the sum.  May be residual or z itself, not out_residual.
 *   out_stats   rows * 4 floats, what the backward pass needs: mean and rstd of the norm of z, then of s (0 where there is no such norm, and
 *               for the mean of DAF_NORM_RMS); or NULL.
 *
 * daf_residual_norm_backward -- with grad_y and grad_sum the gradients of y and of s (as the blocks behind left it):
 *     grad_s = grad_sum + gradient through pre;  grad_residual = grad_s;  grad_z = gradient of scale * gate * post(z)
 * and the gradients of the vectors, summed over rows (the gate's over its run of rows) in binary32, in a fixed order.
 *
 *   sum         s as the forward pass wrote it (read where grad_y is given); stats: as the forward pass wrote them.
 *   grad_y, grad_sum     either may be NULL: that part is zero.  Not both.
 *   out_grad_residual    may be grad_y or grad_sum itself.
 *   z, out_grad_z        both or neither.  out_grad_z may be z or any input gradient itself, not out_grad_residual.
 *   grads       the struct below, on the HOST: where the vectors' gradients go (floats, DEVICE), NULL: not wanted.  Those
 *               of the pre norm need grad_y, the others z.
 *   workspace   DEVICE, daf_residual_norm_backward_workspace_bytes(rows, cols, gate_groups or 1) bytes, 16-byte aligned; may be NULL if
 *               no gradient of a vector is wanted.
 *
 * rows may be 0: the gradients of the vectors are then zero.  cols: 1 ... 16384.
 * Errors: DAF_EINVAL (null or misaligned pointer, a size below its least, gate_groups not dividing rows, outputs (statistics, vectors'
 * gradients and the workspace too) that overlap each other or anything that is read, where they are not named above as the same, an eps
 * that is negative or NaN), DAF_EUNSUPPORTED (dtype, kind, cols above 16384, rows above 2^31 - 2^16, gate_groups above 2^20), DAF_EDEVICE.
 * daf_residual_norm_backward_workspace_bytes returns -1 for such sizes. */
typedef enum { DAF_NORM_RMS = 0, DAF_NORM_LAYER = 1 } daf_norm_kind_t;

typedef struct {
  int64_t rows, cols;
  int64_t gate_groups;         /* rows of the gate: row i of the tensors uses row i / (rows / gate_groups) of it; 1 for one value per column */
  int32_t dtype;               /* a daf_dtype_t */
  int32_t kind;                /* a daf_norm_kind_t, of both norms */
  int32_t post;                /* 1: z is normalized */
  float eps, scale;
  const void *pre_weight, *pre_bias, *post_weight, *post_bias;
  const void* gate;            /* gate_groups * cols elements */
} daf_residual_norm_t;

typedef struct {
  float *pre_weight, *pre_bias, *post_weight, *post_bias;
  float* gate;                 /* gate_groups * cols floats */
} daf_residual_norm_grads_t;

int daf_residual_norm(const daf_residual_norm_t* parameters, const void* residual, const void* z, void* out_residual, void* out_y,
                      float* out_stats, void* stream);
int64_t daf_residual_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t gate_groups);
int daf_residual_norm_backward(const daf_residual_norm_t* parameters, const void* sum, const void* z, const float* stats, const void* grad_y,
                               const void* grad_sum, void* out_grad_residual, void* out_grad_z, const daf_residual_norm_grads_t* grads,
                               void* workspace, void* stream);

/* ---- the gated feed-forward product ------------------------------------------------------------
 *
 * daf_gated_linear -- both projections of a gated feed-forward block, its activation and their product in one kernel:
 *     a = x Wg^T, u = x Wu^T, h = f(a) * u         x [M, K], Wg and Wu [N, K], a, u, h [M, N]
 * Products are accumulated in binary32 on the matrix cores; f and the product with u take the binary32 sums, and h is rounded to
 * dtype once (nearest even).  a and u are written (rounded) only where they are wanted for the backward pass.
 *
 *   f            DAF_ACT_SILU a / (1 + exp(-a)), DAF_ACT_GELU a (1 + erf(a / sqrt(2))) / 2, DAF_ACT_GELU_TANH its form with tanh,
 *                a (1 + tanh(sqrt(2 / pi) (a + 0.044715 a^3))) / 2, DAF_ACT_RELU max(a, 0).
 *   x, w_gate, w_up        DEVICE, dtype, row-major, 16-byte aligned.
 *   out_h                  DEVICE, dtype, 16-byte aligned.
 *   out_gate, out_up       a and u, DEVICE, dtype, 16-byte aligned; both or neither (NULL).
 *   workspace              DEVICE, daf_gated_linear_workspace_bytes(M, N, K, dtype) bytes, 16-byte aligned; needs no
 *                          preparation; calls that share one must not overlap in time.  May be NULL if 0 are needed.
 *
 * daf_gated_linear_backward -- with grad_h the gradient of h:
 *     da = grad_h * u * f'(a), du = grad_h * f(a)       (in binary32, rounded to dtype once)
 *     grad_x = da Wg + du Wu, grad_Wg = da^T x, grad_Wu = du^T x     (binary32 sums, rounded to dtype once)
 * f' of DAF_ACT_RELU at 0 is 0.
 *
 *   gate, up     a and u as the forward pass wrote them, or both NULL: they are computed again from x, Wg and Wu (and stay in
 *                binary32), so that a program keeps nothing but x, e.g. as daf_quantize_pack leaves it.
 *   out_h        h once more, for the gradient of the projection behind it (NULL: not wanted); only without gate and up.
 *   out_grad_x   NULL: not wanted.   out_grad_w_gate, out_grad_w_up  both or neither.  All DEVICE, dtype, 16-byte aligned.
 *   workspace    DEVICE, daf_gated_linear_backward_workspace_bytes(M, N, K, dtype) bytes, as above.
 *
 * M may be 0 (the weights' gradients are then zero); N, K >= 1.  Any sizes and none a multiple of anything; rows of x and W that do not begin at
 * multiples of 16 bytes (K no multiple of 8) are copied into the workspace first, except in a forward pass of few rows.  Outputs must not overlap anything else (checked).
 * Errors: DAF_EINVAL (null or misaligned pointer, a size below its least, no output wanted, an output that overlaps an input or another
 * output), DAF_EUNSUPPORTED (binary32; unknown activation; M of 2^24, N of 2^20, K of 2^21 or more; an output
 * of 2^24 or more tiles of 256 x 256), DAF_EDEVICE.  The workspace queries
 * return -1 for such sizes. */
typedef enum { DAF_ACT_SILU = 0, DAF_ACT_GELU = 1, DAF_ACT_GELU_TANH = 2, DAF_ACT_RELU = 3 } daf_activation_t;

int64_t daf_gated_linear_workspace_bytes(int64_t M, int64_t N, int64_t K, daf_dtype_t dtype);
int daf_gated_linear(const void* x, const void* w_gate, const void* w_up, int64_t M, int64_t N, int64_t K, daf_dtype_t dtype, int activation,
                     void* out_h, void* out_gate, void* out_up, void* workspace, void* stream);
int64_t daf_gated_linear_backward_workspace_bytes(int64_t M, int64_t N, int64_t K, daf_dtype_t dtype);
int daf_gated_linear_backward(const void* x, const void* w_gate, const void* w_up, const void* gate, const void* up, const void* grad_h, int64_t M,
                              int64_t N, int64_t K, daf_dtype_t dtype, int activation, void* out_grad_x, void* out_grad_w_gate, void* out_grad_w_up,
                              void* out_h, void* workspace, void* stream);

/* How a product of these calls runs: a host computation, for tuning and tests.  `whole_tiles` tiles of 256 x 256 come first (0: none), the rest
 * of the output is `tiles` tiles of tile_rows x tile_cols, each sum cut into `slices` that are added afterwards.  DAF_GATED_FORWARD is also the
 * product that computes a and u again; its tile_cols counts columns of a and of u.  Tiles of 16 and 32 rows are those of the kernel of few rows.
 * DAF_GATED_GRAD_INPUT and _WEIGHT are those gradients in a call that wants nothing of the other, the two _OF_BOTH in a call that wants both, where
 * they may share a launch and are then cut for it, in tiles of one size.
 * Errors: DAF_EINVAL (M < 1 too), DAF_EUNSUPPORTED as the calls for the same sizes. */
typedef enum {
  DAF_GATED_FORWARD = 0,
  DAF_GATED_GRAD_INPUT = 1,
  DAF_GATED_GRAD_WEIGHT = 2,
  DAF_GATED_GRAD_INPUT_OF_BOTH = 3,
  DAF_GATED_GRAD_WEIGHT_OF_BOTH = 4
} daf_gated_product_t;
typedef struct {
  int32_t tile_rows, tile_cols, slices;
  int64_t tiles, whole_tiles;
} daf_gated_schedule_t;
int daf_gated_linear_schedule(int64_t M, int64_t N, int64_t K, int product, daf_gated_schedule_t* out);

#ifdef __cplusplus
}
#endif
#endif /* DAF_BLOCK_H_ */

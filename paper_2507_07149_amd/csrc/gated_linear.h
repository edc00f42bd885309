// The gated feed-forward product between its translation units: sizes, how a product is cut, its arguments, launchers.
#pragma once
#include <hip/hip_runtime.h>

#include "daf_block.h"

struct GatedSizes {
  int64_t m, n, k;
};

enum GatedKind { kGated, kGatedGrad, kInput, kWeight };   // gated_product.h

// An output's tiles: `whole` of 256 x 256, whole rounds of workgroups, and the others (all: whole == 0) in a form of its own, each sum in `slices`.
struct GatedCut {
  int64_t whole;
  int form;                       // of kGatedForms
  int64_t tiles, slices;          // of the others
  int64_t partial_bytes;
};
constexpr struct GatedForm {
  int rows, cols;
} kGatedForms[] = {{256, 256}, {128, 256}, {128, 128}, {64, 128}, {16, 32}, {32, 32}, {16, 16}, {32, 16}};
constexpr int64_t kGatedMostTiles = (int64_t)1 << 24;   // that many tiles have 2^32 threads, more than a launch may
constexpr int kGatedFewRows = 4;     // the first of those of gated_few_rows.h

// What a call of these sizes does and needs: pure functions of the sizes.
struct GatedPlan {
  GatedSizes sizes;
  GatedCut cut[3];                // by daf_gated_product_t, each product in a launch of its own
  bool together;                  // both gradients in one launch, where both are wanted, cut as
  GatedCut side[2];               // grad_x, the weights'
  int64_t pitch;                  // elements of a row of x, Wg and Wu as the products read them: k, or k made a multiple of 8 in copies
  int64_t padded;                 // columns of da: n made a multiple of 64
  int64_t x, w_gate, w_up, slopes, partial, side_partial, bytes;   // the workspace: the copies, [da du], the slices' sums; all of it
};
GatedPlan daf_gated_plan(const GatedSizes& sizes, bool backward);

struct GatedProduct {
  const char *r, *c[2];          // c[1]: Wu where c[0] is Wg
  int64_t r_pitch, c_pitch;      // bytes of a row in memory
  int32_t rows, cols;            // of R and C that exist (kGated, kGatedGrad: of each of the two)
  int32_t length;                // of l: K; kInput: N, of each of the two halves; kWeight: M
  int32_t steps, half;           // of 64 values of l; kInput: in each of the two halves
  int32_t tiles_m, tiles_n;      // the places of tiles, in the order of tile_of_position
  int32_t first, sub_m, sub_n;   // of this launch: the places from `first` on, each cut into sub_m x sub_n tiles
  int32_t tiles, slices;         // its tiles, and into how many parts the sum of each is cut
  float* partial;                // slices > 1: the tiles of every slice as the lanes have them
  // what becomes of the sums
  char* out[3];                  // kGated: h, a, u; kGatedGrad: h, [da du]; kInput: grad_x; kWeight: grad_Wg, grad_Wu.  h of kGatedGrad, a and u: may be null
  const char* grad_h;
  int64_t n;                     // columns of h
  int64_t padded;                // of da, a multiple of 64: [da du] is [rows, 2 padded], zero where da and du have no column
  int64_t k;                     // columns of grad_x and the weights
  int32_t act;
};
// `rows` x `cols`: what the tiles cover.  tiles_m ... slices are filled in here.
hipError_t daf_launch_gated_product_f16(GatedKind kind, const GatedProduct& p, const GatedCut& cut, int64_t rows, int64_t cols, hipStream_t stream);
hipError_t daf_launch_gated_product_bf16(GatedKind kind, const GatedProduct& p, const GatedCut& cut, int64_t rows, int64_t cols, hipStream_t stream);
// kInput and kWeight in one launch; both cuts of one form, whole == 0.
hipError_t daf_launch_gated_gradients_f16(const GatedProduct& input, const GatedCut& input_cut, const GatedProduct& weight, const GatedCut& weight_cut,
                                          hipStream_t stream);
hipError_t daf_launch_gated_gradients_bf16(const GatedProduct& input, const GatedCut& input_cut, const GatedProduct& weight, const GatedCut& weight_cut,
                                           hipStream_t stream);
// da and du from a and u that the forward pass kept.
hipError_t daf_launch_gated_slopes_f16(int act, const void* gate, const void* up, const void* grad_h, char* out, int64_t m, int64_t n, int64_t padded,
                                       hipStream_t stream);
hipError_t daf_launch_gated_slopes_bf16(int act, const void* gate, const void* up, const void* grad_h, char* out, int64_t m, int64_t n, int64_t padded,
                                        hipStream_t stream);

// The calls: arguments checked, sizes of 1 and more.
struct GatedLinear {
  int dtype, act;
  const void *x, *w_gate, *w_up;
  char* workspace;
};
hipError_t daf_launch_gated_linear(const GatedPlan& plan, const GatedLinear& g, void* out_h, void* out_gate, void* out_up, hipStream_t stream);
hipError_t daf_launch_gated_linear_backward(const GatedPlan& plan, const GatedLinear& g, const void* grad_h, const void* gate, const void* up,
                                            void* out_grad_x, void* out_grad_w_gate, void* out_grad_w_up, void* out_h, hipStream_t stream);
hipError_t daf_launch_clear(void* out, int64_t bytes, hipStream_t stream);     // a multiple of 2

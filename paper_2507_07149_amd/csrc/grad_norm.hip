// The global norm of a model's gradients and their clipping (daf_grad_norm, daf_clip_grad_norm).
//
//   norm = sqrt(sum g^2),  out = g * min(1, max_norm / (norm + 1e-6))
//
// Two launches for up to 200 tensors that are clipped in place (144 with places of their own for the results): sums of squares, then the scaling,
// whose workgroups each add up the partial sums themselves (at most 2048 numbers out of a cache: cheaper than a launch in between).  Both
// are bound by memory: the gradients are read twice and written once, 541 MB of bfloat16 in 267 to 274 us (6.0 TB/s).  The second pass takes them
// from the end, so that what the first has just read comes out of the caches, and stores past these, which keeps it there (308 us without).  The list goes in the kernel's arguments: nothing has to be
// copied to the device first.  Short lists are launches and little else: 48 tensors of 6144 9.4 us.
#include "block_common.h"
#include "grad_norm.h"

namespace {

constexpr int kThreads = 256;
constexpr int kChunkBytes = 32768;                 // of one tensor, to a workgroup at a time: eight loads of 16 bytes a thread
constexpr int kLoads = kChunkBytes / 16 / kThreads;
constexpr int kMaxBlocks = kGradNormBlocks;

// The tensors of a launch, in its arguments.  OUT: with places of their own for the results; without, as where they are clipped in place, more
// of them fit.
template <bool OUT>
struct Tensors {
  static constexpr int kMost = OUT ? 144 : 200;
  const char* grad[kMost];
  char* out[OUT ? kMost : 1];
  uint64_t size[kMost];                            // elements, times 4, and the format
  uint32_t first[kMost];                           // number of its first chunk in the launch
  int32_t count;
  uint32_t chunks;
};
static_assert(sizeof(Tensors<false>) <= 4096 && sizeof(Tensors<true>) <= 4096, "kernel arguments");

struct Tensor {
  const char* grad;
  char* out;
  int64_t n;
  uint32_t first;
  int dtype;
};
template <bool OUT>
__device__ __forceinline__ Tensor tensor_at(const Tensors<OUT>& list, int i) {
  const char* const grad = list.grad[i];
  return {grad, OUT ? list.out[OUT ? i : 0] : const_cast<char*>(grad), (int64_t)(list.size[i] >> 2), list.first[i], (int)(list.size[i] & 3)};
}

// The tensor that has chunk `c`: the last whose first chunk is not behind it (tensors of no elements share theirs with the next).
template <bool OUT>
__device__ __forceinline__ int tensor_of(const Tensors<OUT>& list, uint32_t c) {
  int lo = 0, hi = list.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (list.first[mid] <= c) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Squares in 64 bits: the square of a binary32 number is exact there and can neither overflow nor vanish.
template <int DT>
__device__ __forceinline__ void add_squares(const u32x4& v, double (&sum)[2]) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (DT == kF32) {
      const double a = (double)u2f(v[w]);
      sum[w & 1] = __builtin_fma(a, a, sum[w & 1]);
    } else {
      const double a = (double)widen16<DT>(v[w] & 0xFFFFu);
      const double b = (double)(DT == kBF16 ? u2f(v[w] & 0xFFFF0000u) : widen16<DT>(v[w] >> 16));
      sum[0] = __builtin_fma(a, a, sum[0]);
      sum[1] = __builtin_fma(b, b, sum[1]);
    }
  }
}

template <int DT>
__device__ __forceinline__ void chunk_squares(const char* p, int64_t bytes, double (&sum)[2]) {
  constexpr int kBytes = ElemTraits<DT>::kBytes;
  const int t = threadIdx.x;
  if (bytes >= kChunkBytes) {
    u32x4 v[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) v[i] = load_any(p + (i * kThreads + t) * 16);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) add_squares<DT>(v[i], sum);
    return;
  }
  const int whole = (int)bytes / 16 * 16;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int at = (i * kThreads + t) * 16;
    if (at < whole) add_squares<DT>(load_any(p + at), sum);
  }
  const int last = whole + t * kBytes;             // fewer than 16 bytes are left
  if (last < (int)bytes) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if constexpr (DT == kF32) v[0] = *reinterpret_cast<const uint32_t*>(p + last);
    else v[0] = *reinterpret_cast<const uint16_t*>(p + last);
    add_squares<DT>(v, sum);
  }
}

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double part[kThreads / kWave];
#pragma unroll
  for (int d = kWave / 2; d > 0; d >>= 1) v += __shfl_xor(v, d);
  if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
  __syncthreads();
  double sum = part[0];
#pragma unroll
  for (int w = 1; w < kThreads / kWave; ++w) sum += part[w];
  return sum;
}

// Sum of squares of the workgroup's chunks: every gridDim.x-th.  With `add`: on top of those of the launch before.
__global__ __launch_bounds__(kThreads, 4) void k_grad_squares(const Tensors<false> list, double* __restrict__ partial, int add) {
  double sum[2] = {0.0, 0.0};
  uint32_t c = blockIdx.x;
  if (c < list.chunks) {
    int i = tensor_of(list, c);
    for (; c < list.chunks; c += gridDim.x) {
      while (i + 1 < list.count && list.first[i + 1] <= c) ++i;
      const Tensor x = tensor_at(list, i);
      const int64_t at = (int64_t)(c - x.first) * kChunkBytes;
      if (x.dtype == DAF_F32) chunk_squares<kF32>(x.grad + at, x.n * 4 - at, sum);
      else if (x.dtype == DAF_F16) chunk_squares<kF16>(x.grad + at, x.n * 2 - at, sum);
      else chunk_squares<kBF16>(x.grad + at, x.n * 2 - at, sum);
    }
  }
  const double all = block_sum(sum[0] + sum[1]);
  if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + all : all;
}

// The norm from the partial sums, the same in every workgroup.
__device__ __forceinline__ float norm_of(const double* __restrict__ partial, int blocks) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < blocks; i += kThreads) sum += partial[i];
  return (float)__builtin_sqrt(block_sum(sum));
}

template <int DT>
__device__ __forceinline__ u32x4 scaled(const u32x4& v, float factor) {
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (DT == kF32) {
      r[w] = f2u(u2f(v[w]) * factor);
    } else {
      const float lo = widen16<DT>(v[w] & 0xFFFFu), hi = DT == kBF16 ? u2f(v[w] & 0xFFFF0000u) : widen16<DT>(v[w] >> 16);
      r[w] = narrow_pair<DT>(lo * factor, hi * factor);
    }
  }
  return r;
}

template <int DT>
__device__ __forceinline__ void scale_chunk(const char* p, char* out, int64_t bytes, float factor) {
  constexpr int kBytes = ElemTraits<DT>::kBytes;
  const int t = threadIdx.x;
  if (bytes >= kChunkBytes) {
    u32x4 v[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) v[i] = load_any(p + (i * kThreads + t) * 16);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) stream_any(out + (i * kThreads + t) * 16, scaled<DT>(v[i], factor));
    return;
  }
  const int whole = (int)bytes / 16 * 16;
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int at = (i * kThreads + t) * 16;
    if (at < whole) stream_any(out + at, scaled<DT>(load_any(p + at), factor));
  }
  const int last = whole + t * kBytes;
  if (last < (int)bytes) {
    u32x4 v = {0u, 0u, 0u, 0u};
    if constexpr (DT == kF32) {
      v[0] = *reinterpret_cast<const uint32_t*>(p + last);
      *reinterpret_cast<uint32_t*>(out + last) = scaled<DT>(v, factor)[0];
    } else {
      v[0] = *reinterpret_cast<const uint16_t*>(p + last);
      *reinterpret_cast<uint16_t*>(out + last) = (uint16_t)scaled<DT>(v, factor)[0];
    }
  }
}

// Chunks from the last one on.
template <bool OUT>
__global__ __launch_bounds__(kThreads, 4) void k_grad_scale(const Tensors<OUT> list, const double* __restrict__ partial, int blocks, float max_norm,
                                                            float* __restrict__ out_norm) {
  const float norm = norm_of(partial, blocks);
  if (out_norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *out_norm = norm;
  const float ratio = max_norm / (norm + 1e-6f);
  const bool no_limit = max_norm == __builtin_inff() && norm == norm;   // (an infinite norm over it is no number)
  const float factor = ratio >= 1.0f || no_limit ? 1.0f : ratio;       // (NaN stays)
  if (blockIdx.x >= list.chunks) return;
  int64_t c = (int64_t)list.chunks - 1 - blockIdx.x;
  int i = tensor_of(list, (uint32_t)c);
  for (; c >= 0; c -= gridDim.x) {
    while (list.first[i] > (uint32_t)c) --i;
    const Tensor x = tensor_at(list, i);
    if (factor == 1.0f && x.out == x.grad) continue;
    const int64_t at = ((uint32_t)c - x.first) * (int64_t)kChunkBytes;
    if (x.dtype == DAF_F32) scale_chunk<kF32>(x.grad + at, x.out + at, x.n * 4 - at, factor);
    else if (x.dtype == DAF_F16) scale_chunk<kF16>(x.grad + at, x.out + at, x.n * 2 - at, factor);
    else scale_chunk<kBF16>(x.grad + at, x.out + at, x.n * 2 - at, factor);
  }
}

__global__ __launch_bounds__(kThreads) void k_grad_norm(const double* __restrict__ partial, int blocks, float* __restrict__ out_norm) {
  const float norm = norm_of(partial, blocks);
  if (threadIdx.x == 0) *out_norm = norm;
}

// Tensors from `first` on that fit a launch: as many as the table holds and as chunks can be counted in 31 bits.  Returns the next one.
constexpr int64_t kMostChunks = (int64_t)1 << 30;
template <bool OUT>
int32_t fill(const daf_grad_item_t* items, int32_t n_items, int32_t first, Tensors<OUT>* list) {
  list->count = 0;
  int64_t chunks = 0;
  int32_t i = first;
  for (; i < n_items && list->count < Tensors<OUT>::kMost; ++i) {
    const int64_t more = (items[i].n * (items[i].dtype == DAF_F32 ? 4 : 2) + kChunkBytes - 1) / kChunkBytes;
    if (list->count > 0 && chunks + more > kMostChunks) break;
    const int at = list->count++;
    list->grad[at] = static_cast<const char*>(items[i].grad);
    if constexpr (OUT) list->out[at] = static_cast<char*>(items[i].out);
    list->size[at] = (uint64_t)items[i].n << 2 | (uint64_t)items[i].dtype;
    list->first[at] = (uint32_t)chunks;
    chunks += more;
  }
  list->chunks = (uint32_t)chunks;
  return i;
}

// A call's launches: `launch` for each run of tensors that fits one.  As many workgroups as the longest has chunks, for all of them: each partial sum
// has one owner.
template <bool OUT, class F>
hipError_t for_each_launch(const daf_grad_item_t* items, int32_t n_items, F&& launch) {
  Tensors<OUT> list;
  int32_t next = fill(items, n_items, 0, &list);
  int64_t most = list.chunks;
  for (int32_t i = next; i < n_items;) {
    i = fill(items, n_items, i, &list);
    if ((int64_t)list.chunks > most) most = list.chunks;
  }
  const int blocks = (int)(most < 1 ? 1 : most < kMaxBlocks ? most : kMaxBlocks);
  if (next < n_items) next = fill(items, n_items, 0, &list);
  for (bool first = true;; first = false) {
    launch(list, blocks, first);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess || next == n_items) return e;
    next = fill(items, n_items, next, &list);
  }
}

template <bool OUT>
hipError_t launch_scale(const daf_grad_item_t* items, int32_t n_items, float max_norm, float* out_norm, const double* partial, int sums, hipStream_t stream) {
  return for_each_launch<OUT>(items, n_items, [&](const Tensors<OUT>& list, int blocks, bool first) {
    hipLaunchKernelGGL((k_grad_scale<OUT>), dim3(blocks), dim3(kThreads), 0, stream, list, partial, sums, max_norm, first ? out_norm : nullptr);
  });
}

}  // namespace

hipError_t daf_launch_grad_norm(const daf_grad_item_t* items, int32_t n_items, bool clip, float max_norm, float* out_norm, double* partial,
                                hipStream_t stream) {
  int sums = 0;
  const hipError_t e = for_each_launch<false>(items, n_items, [&](const Tensors<false>& list, int blocks, bool first) {
    sums = blocks;
    hipLaunchKernelGGL(k_grad_squares, dim3(blocks), dim3(kThreads), 0, stream, list, partial, first ? 0 : 1);
  });
  if (e != hipSuccess) return e;
  if (!clip) {
    hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(kThreads), 0, stream, partial, sums, out_norm);
    return hipGetLastError();
  }
  bool in_place = true;
  for (int32_t i = 0; i < n_items; ++i) in_place = in_place && (items[i].n == 0 || items[i].out == items[i].grad);
  return in_place ? launch_scale<false>(items, n_items, max_norm, out_norm, partial, sums, stream)
                  : launch_scale<true>(items, n_items, max_norm, out_norm, partial, sums, stream);
}

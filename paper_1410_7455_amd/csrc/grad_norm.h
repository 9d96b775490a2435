// The norm of many tensors as one vector, and clipping (gfx950, 64-lane wavefronts).
//   norm = sqrt(sum g^2);  factor = max_norm / norm where norm > max_norm, else 1;  clipped: g factor
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elements.h"

namespace ngsgd {

constexpr int kNormThreads = 256;
constexpr int kNormTensors = 128;       // whose addresses and sizes one launch carries (of 4 KB of arguments)
constexpr int kNormPieces = 2048;       // a launch's tensors are cut into about so many pieces of work
constexpr int kNormLeast = 4096;        // elements of a piece, but for a tensor's last

struct NormTensors {
  const void* g[kNormTensors];
  void* out[kNormTensors];
  int64_t n[kNormTensors];
  int first[kNormTensors];              // piece at which each begins
  int count;                            // tensors
  int64_t piece;                        // elements of one
};

struct NormResult {
  double norm, factor;
};

// The piece of work of this workgroup: a tensor and where it starts in it.
__device__ __forceinline__ int tensor_of(const NormTensors& a, const int piece) {
  int low = 0, high = a.count;          // first[low] <= piece < first[high]
  while (high - low > 1) {
    const int mid = (low + high) / 2;
    if (a.first[mid] <= piece) low = mid; else high = mid;
  }
  return low;
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int k = 1; k < 64; k *= 2) v += __shfl_xor(v, k);
  return v;
}
// To all threads.
__device__ __forceinline__ double block_sum_f64(double v) {
  __shared__ double part[kMaxWaves];
  v = wave_sum_f64(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  double sum = 0.0;
  for (int k = 0; k < (int)(blockDim.x >> 6); ++k) sum += part[k];
  return sum;
}

template <typename T>
__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(const NormTensors a, double* parts) {
  const int t = tensor_of(a, blockIdx.x);
  const int64_t from = (blockIdx.x - a.first[t]) * a.piece, to = min(from + a.piece, a.n[t]);
  const T* g = static_cast<const T*>(a.g[t]);
  double sum = 0.0;
  for (int64_t i = from + threadIdx.x; i < to; i += kNormThreads) {
    const double x = (double)to_float(g[i]);
    sum = fma(x, x, sum);
  }
  sum = block_sum_f64(sum);
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void grad_norm_finish_kernel(const double* parts, const int n_parts, const double max_norm, NormResult* result,
                                                                float* norm_out, float* factor_out) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < n_parts; i += 1024) sum += parts[i];
  sum = block_sum_f64(sum);
  if (threadIdx.x != 0) return;
  const double norm = sqrt(sum), factor = norm > max_norm ? max_norm / norm : norm == norm ? 1.0 : norm;
  *result = NormResult{norm, factor};
  if (norm_out != nullptr) *norm_out = (float)norm;
  if (factor_out != nullptr) *factor_out = (float)factor;
}

template <typename T>
__global__ __launch_bounds__(kNormThreads) void grad_clip_kernel(const NormTensors a, const NormResult* result) {
  const int t = tensor_of(a, blockIdx.x);
  const float factor = (float)result->factor;
  if (factor == 1.f && a.out[t] == a.g[t]) return;
  const int64_t from = (blockIdx.x - a.first[t]) * a.piece, to = min(from + a.piece, a.n[t]);
  const T* g = static_cast<const T*>(a.g[t]);
  T* out = static_cast<T*>(a.out[t]);
  for (int64_t i = from + threadIdx.x; i < to; i += kNormThreads) out[i] = from_float<T>(factor * to_float(g[i]));
}

}  // namespace ngsgd

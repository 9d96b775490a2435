// Cross-entropy of logits and its gradient (gfx950, 64-lane wavefronts).
//   m = max_j x_j;  e_j = exp(x_j - m);  S = sum_{j != y} e_j
//   loss = log(S + e_y) - (x_y - m);  d_j = scale e_j / (S + e_y),  d_y = -scale S / (S + e_y)
// The label's term is kept out of the sum: where it is almost all of it, S is what the loss and the label's gradient are made of.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elements.h"

namespace ngsgd {

constexpr int kLossThreads = 256;

struct CrossEntropy {
  const void* logits;
  int64_t ld;
  const void* labels;
  int64_t N;
  int V;
  float* loss;          // optional
  float scale;
  const float* dev_scale;   // optional
  void* dlogits;        // optional
  int64_t ldd;
};

__device__ __forceinline__ float wave_max_f32(float v) {
#pragma unroll
  for (int k = 1; k < 64; k *= 2) {
    const float o = __shfl_xor(v, k);
    v = v != v || v > o ? v : o;   // (a NaN stays)
  }
  return v;
}

// log(S + e) - (x_y - m)
__device__ __forceinline__ float loss_of(const float S, const float e, const float label, const float m) {
  // the label's is the largest logit: e = 1, and S may be far below it
  return label == m ? log1pf(S) : logf(S + e) - (label - m);
}

// A workgroup per row: three passes over it.
template <typename T, typename I>
__global__ __launch_bounds__(kLossThreads) void cross_entropy_kernel(const CrossEntropy a) {
  __shared__ BlockScratch red;
  __shared__ float top[kLossThreads / 64];
  const int64_t row = blockIdx.x;
  const int64_t label = static_cast<const I*>(a.labels)[row];
  const T* x = static_cast<const T*>(a.logits) + row * a.ld;
  T* d = static_cast<T*>(a.dlogits) + row * a.ldd;
  if (label < 0 || label >= a.V) {
    if (a.loss != nullptr && threadIdx.x == 0) a.loss[row] = 0.f;
    if (a.dlogits != nullptr)
      for (int j = threadIdx.x; j < a.V; j += kLossThreads) d[j] = from_float<T>(0.f);
    return;
  }
  float m = -INFINITY;
  for (int j = threadIdx.x; j < a.V; j += kLossThreads) {
    const float v = to_float(x[j]);
    m = m != m || m > v ? m : v;
  }
  m = wave_max_f32(m);
  if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kLossThreads / 64; ++k) {
    const float o = top[k];
    m = m != m || m > o ? m : o;
  }
  float S = 0.f;
  for (int j = threadIdx.x; j < a.V; j += kLossThreads) S += j == label ? 0.f : expf(to_float(x[j]) - m);
  S = block_sum_f32(S, red, 0);
  if (!(fabsf(m) < INFINITY)) S = NAN;   // a largest logit that is the label's and infinite would leave zeros
  const float xl = to_float(x[label]), e = expf(xl - m);
  if (a.loss != nullptr && threadIdx.x == 0) a.loss[row] = loss_of(S, e, xl, m);
  if (a.dlogits == nullptr) return;
  __syncthreads();   // the label's logit has been read: dlogits may be logits
  const float f = (a.dev_scale != nullptr ? a.scale * *a.dev_scale : a.scale) / (S + e);
  for (int j = threadIdx.x; j < a.V; j += kLossThreads) d[j] = from_float<T>(j == label ? -S * f : f * expf(to_float(x[j]) - m));
}

}  // namespace ngsgd

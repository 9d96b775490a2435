// Layer norm and its gradients (gfx950, 64-lane wavefronts).
//   forward:   y = xhat w + b,  xhat = (x - mean) rstd,  mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^(-1/2)
//   backward:  g = dy w,  dx = rstd (g - sum g / D - xhat sum(g xhat) / D),  dw = sum over rows dy xhat,  db = sum over rows dy
// Statistics, sums and gradients are held in fp32; the variance is summed from the differences to the mean, so that
// a mean far from zero costs no digits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elements.h"

namespace ngsgd {

struct LayerNormForward {
  const void* x;
  int64_t ldx;
  const void* w;     // nullptr: ones
  const void* b;     // nullptr: zeros
  void* y;
  int64_t ldy;
  float* mean;       // optional
  float* rstd;       // optional
  int64_t N;
  int D;
  float eps;
};

struct LayerNormBackward {
  const void* dy;
  int64_t lddy;
  const void* x;
  int64_t ldx;
  const void* w;     // nullptr: ones
  const float* mean;
  const float* rstd;
  void* dx;          // optional
  int64_t lddx;
  void* dw;          // optional
  void* db;          // optional
  int64_t N;
  int D;
  float* part;       // [groups][2][D] sums over a group of rows
  int groups;
};

// ---- rows of any width, read from memory in every pass ---------------------------------------------
constexpr int kNormThreads = 256;

template <typename T, typename W>
__global__ __launch_bounds__(kNormThreads) void layernorm_forward_wide_kernel(const LayerNormForward a) {
  __shared__ float red[2][2][kNormThreads / 64];
  const W* const w = static_cast<const W*>(a.w);
  const W* const b = static_cast<const W*>(a.b);
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    T* const y = static_cast<T*>(a.y) + row * a.ldy;
    float s = 0.f;
    for (int c = threadIdx.x; c < a.D; c += kNormThreads) s += to_float(x[c]);
    const float mean = block_sum_f32<kNormThreads / 64>(s, red, 0) / (float)a.D;
    float q = 0.f;
    for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
      const float d = to_float(x[c]) - mean;
      q += d * d;
    }
    const float rstd = 1.f / sqrtf(block_sum_f32<kNormThreads / 64>(q, red, 1) / (float)a.D + a.eps);
    for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
      float v = (to_float(x[c]) - mean) * rstd;
      if (w != nullptr) v *= to_float(w[c]);
      if (b != nullptr) v += to_float(b[c]);
      y[c] = from_float<T>(v);
    }
    if (threadIdx.x == 0) {
      if (a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
  }
}

template <typename T, typename W>
__global__ __launch_bounds__(kNormThreads) void layernorm_backward_rows_kernel(const LayerNormBackward a) {
  __shared__ float red[2][2][kNormThreads / 64];
  const W* const w = static_cast<const W*>(a.w);
  int parity = 0;
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x, parity ^= 1) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* const dy = static_cast<const T*>(a.dy) + row * a.lddy;
    T* const dx = static_cast<T*>(a.dx) + row * a.lddx;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float c1 = 0.f, c2 = 0.f;
    for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
      float g = to_float(dy[c]);
      if (w != nullptr) g *= to_float(w[c]);
      c1 += g;
      c2 += g * ((to_float(x[c]) - mean) * rstd);
    }
    block_sum_pair_f32<kNormThreads / 64>(c1, c2, red, parity);
    c1 /= (float)a.D;
    c2 /= (float)a.D;
    for (int c = threadIdx.x; c < a.D; c += kNormThreads) {
      float g = to_float(dy[c]);
      if (w != nullptr) g *= to_float(w[c]);
      const float xhat = (to_float(x[c]) - mean) * rstd;
      dx[c] = from_float<T>(rstd * (g - c1 - xhat * c2));
    }
  }
}

// Sums over the rows of a group: grid (columns / 256, groups), a thread per column.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void layernorm_backward_columns_kernel(const LayerNormBackward a) {
  const int64_t c = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
  if (c >= a.D) return;
  const int64_t first = a.N * blockIdx.y / a.groups, end = a.N * (blockIdx.y + 1) / a.groups;
  float dw = 0.f, db = 0.f;
  for (int64_t row = first; row < end; ++row) {
    const float dy = to_float(static_cast<const T*>(a.dy)[row * a.lddy + c]);
    dw += dy * ((to_float(static_cast<const T*>(a.x)[row * a.ldx + c]) - a.mean[row]) * a.rstd[row]);
    db += dy;
  }
  float* const part = a.part + (size_t)blockIdx.y * 2 * a.D;
  part[c] = dw;
  part[(size_t)a.D + c] = db;
}

// The groups' sums in a fixed order: grid (columns / 256, 2), dw and db.
template <typename W>
__global__ __launch_bounds__(kNormThreads) void layernorm_backward_sum_kernel(const LayerNormBackward a) {
  const int64_t c = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
  W* const out = static_cast<W*>(blockIdx.y == 0 ? a.dw : a.db);
  if (c >= a.D || out == nullptr) return;
  float s = 0.f;
  for (int g = 0; g < a.groups; ++g) s += a.part[((size_t)g * 2 + blockIdx.y) * a.D + c];
  out[c] = from_float<W>(s);
}

}  // namespace ngsgd

// Layer norm and its gradients (gfx950, 64-lane wavefronts).
//   forward:   y = xhat w + b,  xhat = (x - mean) rstd,  mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^(-1/2)
//   backward:  g = dy w,  dx = rstd (g - sum g / D - xhat sum(g xhat) / D),  dw = sum over rows dy xhat,  db = sum over rows dy
// Statistics, sums and gradients are held in fp32; the variance is summed from the differences to the mean, so that
// a mean far from zero costs no digits.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// ---- rows that a group of threads holds in registers ------------------------------------------------
// TPR threads share a row and E of its columns each, as E / VEC pieces of VEC neighbours; a workgroup of NT threads walks over the rows,
// NT / TPR at a time.  A thread keeps its columns of the weight, the bias and (backward) of the sums over the rows in registers,
// and requests its next row before it works on the one that it has.
template <typename T, int VEC_, int E_, int TPR_, int NT_>
struct RowShape {
  static constexpr int VEC = VEC_, E = E_, TPR = TPR_, NT = NT_, K = E / VEC, ROWS = NT / TPR;
  static_assert(E % VEC == 0 && NT % TPR == 0 && (TPR == NT || TPR <= 64), "a row belongs to a workgroup or within a wavefront");
  __device__ static int member() { return threadIdx.x % TPR; }
  __device__ static int row() { return threadIdx.x / TPR; }
  __device__ static int column(const int k) { return (k * TPR + member()) * VEC; }
};

// A thread's columns of a row as they lie in memory, two 16-bit elements to a register where pieces are loaded whole.
template <typename S, typename T>
struct RowPart {
  static constexpr bool kWords = S::VEC > 1 && sizeof(T) == 2;
  using Word = std::conditional_t<kWords, uint32_t, T>;
  static constexpr int PER = kWords ? 2 : 1;   // elements in a word
  Word v[S::E / PER];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < S::E / PER; ++i) v[i] = Word(0);
  }
  // Zeros behind column D.
  __device__ __forceinline__ void load(const T* p, const int D) {
#pragma unroll
    for (int k = 0; k < S::K; ++k) {
      const int c = S::column(k);
      if constexpr (S::VEC > 1) {
        constexpr int WORDS = S::VEC / PER;
        if (c + S::VEC <= D) {
          const Pack<Word, WORDS> q = *reinterpret_cast<const Pack<Word, WORDS>*>(p + c);
#pragma unroll
          for (int j = 0; j < WORDS; ++j) v[k * WORDS + j] = q.v[j];
        } else {
          Pack<T, S::VEC> q;
#pragma unroll
          for (int j = 0; j < S::VEC; ++j) q.v[j] = c + j < D ? p[c + j] : T(0.f);
          const Pack<Word, WORDS> w = __builtin_bit_cast(Pack<Word, WORDS>, q);
#pragma unroll
          for (int j = 0; j < WORDS; ++j) v[k * WORDS + j] = w.v[j];
        }
      } else {
        v[k] = c < D ? p[c] : T(0.f);
      }
    }
  }
  __device__ __forceinline__ float get(const int e) const {
    if constexpr (kWords)
      return to_float(__builtin_bit_cast(T, (uint16_t)(e & 1 ? v[e / 2] >> 16 : v[e / 2])));
    else
      return to_float(v[e]);
  }
};
template <typename S, typename T>
__device__ __forceinline__ void store_row(const float (&v)[S::E], T* p, const int D) {
#pragma unroll
  for (int k = 0; k < S::K; ++k) {
    const int c = S::column(k);
    if (S::VEC > 1 && c + S::VEC <= D) {
      Pack<T, S::VEC> o;
#pragma unroll
      for (int j = 0; j < S::VEC; ++j) o.v[j] = from_float<T>(v[k * S::VEC + j]);
      *reinterpret_cast<Pack<T, S::VEC>*>(p + c) = o;
    } else {
#pragma unroll
      for (int j = 0; j < S::VEC; ++j)
        if (c + j < D) p[c + j] = from_float<T>(v[k * S::VEC + j]);
    }
  }
}
template <typename S>
using RowScratch = float[2][2][S::TPR <= 64 ? 1 : S::TPR / 64];

// Sums over the threads of a row.
template <typename S>
__device__ __forceinline__ float row_sum(float v, RowScratch<S>& red, const int parity) {
  if constexpr (S::TPR == 16)
    return row16_sum_f32(v);
  else
    return block_sum_f32<S::TPR / 64>(v, red, parity);
}
template <typename S>
__device__ __forceinline__ void row_sum_pair(float& a, float& b, RowScratch<S>& red, const int parity) {
  if constexpr (S::TPR == 16) {
    a = row16_sum_f32(a);
    b = row16_sum_f32(b);
  } else {
    block_sum_pair_f32<S::TPR / 64>(a, b, red, parity);
  }
}

template <typename T, typename W, typename S>
__global__ __launch_bounds__(S::NT) void layernorm_forward_kernel(const LayerNormForward a) {
  __shared__ RowScratch<S> red;
  constexpr int E = S::E;
  RowPart<S, W> w, b;
  if (a.w != nullptr) w.load(static_cast<const W*>(a.w), a.D);
  if (a.b != nullptr) b.load(static_cast<const W*>(a.b), a.D);
  const int64_t step = (int64_t)gridDim.x * S::ROWS;
  int64_t row = (int64_t)blockIdx.x * S::ROWS + S::row();
  RowPart<S, T> next;
  next.clear();
  if (row < a.N) next.load(static_cast<const T*>(a.x) + row * a.ldx, a.D);
  for (int64_t first = (int64_t)blockIdx.x * S::ROWS; first < a.N; first += step, row += step) {   // (uniform in the workgroup)
    float x[E];
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] = next.get(e);
      s += x[e];
    }
    if (row + step < a.N) next.load(static_cast<const T*>(a.x) + (row + step) * a.ldx, a.D);
    const float mean = row_sum<S>(s, red, 0) / (float)a.D;
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] = S::column(e / S::VEC) + e % S::VEC < a.D ? x[e] - mean : 0.f;
      q += x[e] * x[e];
    }
    const float rstd = 1.f / sqrtf(row_sum<S>(q, red, 1) / (float)a.D + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] *= rstd;
      if (a.w != nullptr) x[e] *= w.get(e);
      if (a.b != nullptr) x[e] += b.get(e);
    }
    if (row < a.N) {
      store_row<S>(x, static_cast<T*>(a.y) + row * a.ldy, a.D);
      if (S::member() == 0) {
        if (a.mean != nullptr) a.mean[row] = mean;
        if (a.rstd != nullptr) a.rstd[row] = rstd;
      }
    }
  }
}

// What a thread needs of a row; zeros behind the last one.
template <typename S, typename T>
struct BackwardRow {
  RowPart<S, T> x, dy;
  float mean, rstd;
  __device__ __forceinline__ void load(const LayerNormBackward& a, const int64_t r) {
    if (r < a.N) {
      x.load(static_cast<const T*>(a.x) + r * a.ldx, a.D);
      dy.load(static_cast<const T*>(a.dy) + r * a.lddy, a.D);
      mean = a.mean[r];
      rstd = a.rstd[r];
    } else {
      x.clear();
      dy.clear();
      mean = rstd = 0.f;
    }
  }
};

// Sums of a workgroup's rows go to part[workgroup][dw, db][D].
template <typename T, typename W, typename S>
__global__ __launch_bounds__(S::NT) void layernorm_backward_kernel(const LayerNormBackward a) {
  __shared__ RowScratch<S> red;
  __shared__ float sums[S::ROWS > 1 ? S::NT * S::E : 1];
  constexpr int E = S::E;
  RowPart<S, W> w;
  if (a.w != nullptr) w.load(static_cast<const W*>(a.w), a.D);
  float dw[E], db[E];
#pragma unroll
  for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.f;
  const int64_t step = (int64_t)gridDim.x * S::ROWS;
  int64_t row = (int64_t)blockIdx.x * S::ROWS + S::row();
  BackwardRow<S, T> next;
  next.load(a, row);
  int parity = 0;
  for (int64_t first = (int64_t)blockIdx.x * S::ROWS; first < a.N; first += step, row += step, parity ^= 1) {   // (uniform in the workgroup)
    float xhat[E], g[E];
    const float rstd = next.rstd;
    float c1 = 0.f, c2 = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      xhat[e] = (next.x.get(e) - next.mean) * rstd;
      g[e] = next.dy.get(e);
      dw[e] += g[e] * xhat[e];
      db[e] += g[e];
      if (a.w != nullptr) g[e] *= w.get(e);
      c1 += g[e];
      c2 += g[e] * xhat[e];
    }
    next.load(a, row + step);
    if (a.dx != nullptr) {
      row_sum_pair<S>(c1, c2, red, parity);
      c1 /= (float)a.D;
      c2 /= (float)a.D;
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = rstd * (g[e] - c1 - xhat[e] * c2);
      if (row < a.N) store_row<S>(g, static_cast<T*>(a.dx) + row * a.lddx, a.D);
    }
  }
  if (a.part == nullptr) return;
  float* const part = a.part + (size_t)blockIdx.x * 2 * a.D;
  if (S::ROWS == 1) {
    store_row<S>(dw, part, a.D);
    store_row<S>(db, part + a.D, a.D);
    return;
  }
  // the rows that the workgroup worked on side by side, in order
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) sums[(S::row() * S::TPR + S::member()) * E + e] = which == 0 ? dw[e] : db[e];
    __syncthreads();
    for (int i = threadIdx.x; i < S::TPR * E; i += S::NT) {
      float v = 0.f;
#pragma unroll
      for (int r = 0; r < S::ROWS; ++r) v += sums[r * S::TPR * E + i];
      const int e = i % E, c = ((e / S::VEC) * S::TPR + i / E) * S::VEC + e % S::VEC;
      if (c < a.D) part[(size_t)which * a.D + c] = v;
    }
  }
}

// ---- rows of any width, read from memory in every pass ---------------------------------------------
constexpr int kNormThreads = 256;
constexpr int kRegisterColumns = 16384;   // the widest rows of the kernels above

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

// The groups' sums in a fixed order.  A workgroup takes 32 of the 2 D columns (a cache line of each group), every 32nd group in a thread, whose
// loads are requested sixteen at a time: their latency is what bounds it.  (A thread to a column: 130 us for 512 groups.)
constexpr int kSumColumns = 32, kSumThreads = 1024, kSumSlices = kSumThreads / kSumColumns;

template <typename W>
__global__ __launch_bounds__(kSumThreads) void layernorm_backward_sum_kernel(const LayerNormBackward a) {
  __shared__ float slices[kSumSlices][kSumColumns + 1];
  constexpr int AHEAD = 16;
  const int column = threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns;
  const size_t columns = 2 * (size_t)a.D, c = (size_t)blockIdx.x * kSumColumns + column;
  float s = 0.f;
  for (int g0 = slice; g0 < a.groups; g0 += AHEAD * kSumSlices) {
    float v[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int g = g0 + u * kSumSlices;
      v[u] = g < a.groups && c < columns ? a.part[g * columns + c] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) s += v[u];
  }
  slices[slice][column] = s;
  __syncthreads();
  if (slice != 0 || c >= columns) return;
  s = slices[0][column];
#pragma unroll
  for (int k = 1; k < kSumSlices; ++k) s += slices[k][column];
  const bool bias = c >= (size_t)a.D;
  W* const out = static_cast<W*>(bias ? a.db : a.dw);
  if (out != nullptr) out[bias ? c - a.D : c] = from_float<W>(s);
}

}  // namespace ngsgd

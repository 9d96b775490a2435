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
constexpr int kNormParts = kNormPieces + kNormTensors;   // pieces of a launch at most
constexpr int kNormAhead = 4;           // loads of 16 bytes that a thread has in flight

struct NormTensors {
  const void* g[kNormTensors];
  void* out[kNormTensors];
  int64_t n[kNormTensors];
  int first[kNormTensors];              // piece at which each begins; behind the last, a number that no piece reaches
  int64_t piece;                        // elements of one
  int pieces;
};
struct NormResult {
  double norm, factor;
};
struct NormOut {
  float *norm, *factor;                 // optional
};

__device__ __forceinline__ int tensor_of(const NormTensors& a, const int piece) {
  static_assert(kNormTensors == 128);
  const int lane = threadIdx.x & 63;
  return __builtin_popcountll(__builtin_amdgcn_ballot_w64(a.first[lane] <= piece)) +
         __builtin_popcountll(__builtin_amdgcn_ballot_w64(a.first[64 + lane] <= piece)) - 1;
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

// The squares of n elements, by threads 0, 1, ... of `threads`.  (fp64 costs the vector ALU what unpacked fp32 does, and the conversion four times that: half of
// the time that 16-bit elements take to arrive.)
template <typename T>
__device__ __forceinline__ double sum_of_squares(const T* g, const int64_t n, const int thread, const int threads) {
  constexpr int E = 16 / sizeof(T);
  const int64_t full = n / E;
  double sum[2] = {0.0, 0.0};
  const auto add = [&](const Pack<T, E>& v) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const double x = (double)to_float(v.v[j]);
      sum[j & 1] = fma(x, x, sum[j & 1]);
    }
  };
  int64_t p = thread;
  for (; p + (kNormAhead - 1) * threads < full; p += kNormAhead * threads) {
    Pack<T, E> v[kNormAhead];
#pragma unroll
    for (int k = 0; k < kNormAhead; ++k) v[k] = *reinterpret_cast<const Pack<T, E>*>(g + (p + k * threads) * E);
#pragma unroll
    for (int k = 0; k < kNormAhead; ++k) add(v[k]);
  }
  for (; p < full; p += threads) add(*reinterpret_cast<const Pack<T, E>*>(g + p * E));
  if (full * E + thread < n) {
    const double x = (double)to_float(g[full * E + thread]);
    sum[0] = fma(x, x, sum[0]);
  }
  return sum[0] + sum[1];
}

// From the last element to the first: what was read last may still be in the cache.
template <typename T>
__device__ __forceinline__ void clip_elements(const T* g, T* out, const int64_t n, const float factor, const int thread, const int threads) {
  constexpr int E = 16 / sizeof(T);
  const int64_t full = n / E;
  const auto clip = [&](const Pack<T, E>& v, T* to) {
    Pack<T, E> o;
#pragma unroll
    for (int j = 0; j < E; ++j) o.v[j] = from_float<T>(as_f32(factor * to_float(v.v[j])));
    store_pack(to, o);
  };
  if (full * E + thread < n) out[full * E + thread] = from_float<T>(as_f32(factor * to_float(g[full * E + thread])));
  int64_t p = full - 1 - thread;
  for (; p - (kNormAhead - 1) * threads >= 0; p -= kNormAhead * threads) {
    Pack<T, E> v[kNormAhead];
#pragma unroll
    for (int k = 0; k < kNormAhead; ++k) v[k] = *reinterpret_cast<const Pack<T, E>*>(g + (p - k * threads) * E);
#pragma unroll
    for (int k = 0; k < kNormAhead; ++k) clip(v[k], out + (p - k * threads) * E);
  }
  for (; p >= 0; p -= threads) clip(*reinterpret_cast<const Pack<T, E>*>(g + p * E), out + p * E);
}

__device__ __forceinline__ NormResult result_of(const double squares, const double max_norm) {
  const double norm = sqrt(squares);
  return NormResult{norm, norm > max_norm ? max_norm / norm : norm == norm ? 1.0 : norm};
}
__device__ __forceinline__ void write_result(const NormResult& r, const NormOut& out) {
  if (out.norm != nullptr) *out.norm = (float)r.norm;
  if (out.factor != nullptr) *out.factor = (float)r.factor;
}
// The sum of all pieces, in the same order for every workgroup that forms it.
__device__ __forceinline__ NormResult join_parts(const double* parts, const int n, const double max_norm) {
  double sum = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += blockDim.x) sum += parts[i];
  return result_of(block_sum_f64(sum), max_norm);
}

// A workgroup per piece; 2048 of them are what the chip holds at once.  Bound by memory: 1 G bf16 elements 386 us, 5.2 TB/s.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void grad_norm_kernel(const NormTensors a, double* parts) {
  const int t = tensor_of(a, blockIdx.x);
  const int64_t from = (blockIdx.x - a.first[t]) * a.piece;
  const double sum = block_sum_f64(sum_of_squares(static_cast<const T*>(a.g[t]) + from, min(a.piece, a.n[t] - from), threadIdx.x, kNormThreads));
  if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

__global__ __launch_bounds__(1024) void grad_norm_finish_kernel(const double* parts, const int n_parts, const double max_norm, NormResult* result,
                                                                const NormOut out) {
  const NormResult r = join_parts(parts, n_parts, max_norm);
  if (threadIdx.x != 0) return;
  *result = r;
  write_result(r, out);
}

// n_parts: of the sums that every workgroup joins for itself; 0: the result is there.  Bound by memory: 1 G bf16 elements 795 us, 5.1 TB/s.
template <typename T>
__global__ __launch_bounds__(kNormThreads) void grad_clip_kernel(const NormTensors a, const double* parts, const int n_parts, const double max_norm,
                                                                 const NormResult* result, const NormOut out) {
  const int t = tensor_of(a, blockIdx.x);
  const NormResult r = n_parts > 0 ? join_parts(parts, n_parts, max_norm) : *result;
  if (n_parts > 0 && blockIdx.x == 0 && threadIdx.x == 0) write_result(r, out);
  const float factor = (float)r.factor;
  if (factor == 1.f && a.out[t] == a.g[t]) return;
  const int64_t from = (blockIdx.x - a.first[t]) * a.piece;
  clip_elements(static_cast<const T*>(a.g[t]) + from, static_cast<T*>(a.out[t]) + from, min(a.piece, a.n[t] - from), factor, threadIdx.x, kNormThreads);
}

// Few pieces: one workgroup, a wavefront for every 16th piece, without a second launch.  29 k fp32 elements in seven tensors
// 3.8 us (in two launches 7); clipping 32 pieces 7.0 (3.6 + 4.5, and a launch more).
constexpr int kNormSmallThreads = 1024, kNormSmallPieces = 32;
template <typename T>
__global__ __launch_bounds__(kNormSmallThreads) void grad_small_kernel(const NormTensors a, const bool clip, const double max_norm, const NormOut out) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double sum = 0.0;
  for (int p = wave; p < a.pieces; p += kNormSmallThreads / 64) {
    const int t = __builtin_amdgcn_readfirstlane(tensor_of(a, p));
    const int64_t from = (p - a.first[t]) * a.piece;
    sum += sum_of_squares(static_cast<const T*>(a.g[t]) + from, min(a.piece, a.n[t] - from), lane, 64);
  }
  const NormResult r = result_of(block_sum_f64(sum), max_norm);
  if (threadIdx.x == 0) write_result(r, out);
  const float factor = (float)r.factor;
  for (int p = wave; clip && p < a.pieces; p += kNormSmallThreads / 64) {
    const int t = __builtin_amdgcn_readfirstlane(tensor_of(a, p));
    const int64_t from = (p - a.first[t]) * a.piece;
    if (factor != 1.f || a.out[t] != a.g[t])
      clip_elements(static_cast<const T*>(a.g[t]) + from, static_cast<T*>(a.out[t]) + from, min(a.piece, a.n[t] - from), factor, lane, 64);
  }
}

}  // namespace ngsgd

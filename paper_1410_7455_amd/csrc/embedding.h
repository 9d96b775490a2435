// Rows of a table by tokens, and the table's gradient (gfx950, 64-lane wavefronts).
//   y_i = scale W[t_i];   dW[v] = scale sum_{i: t_i = v} dy_i
// Tokens outside [0, V) are padding: zeros, and no gradient.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elements.h"

namespace ngsgd {

constexpr int kLookupThreads = 256;
constexpr int kLookupRows = 4;          // rows that a thread has in flight

struct EmbeddingForward {
  const void* tokens;
  int64_t N;
  const void* table;
  int64_t ldt;
  int64_t V;
  int D;
  float scale;
  void* y;
  int64_t ldy;
  int lanes;         // threads that share a row, a power of two
};

struct EmbeddingBackward {
  const void* dy;
  int64_t lddy;
  const void* tokens;
  int64_t N, V;
  int D;
  float scale;
  void* dtable;
  int64_t lddt;
  int accumulate;
};

// -1 for padding
template <typename I>
__device__ __forceinline__ int64_t token_of(const I* tokens, const int64_t i, const int64_t V) {
  const int64_t t = tokens[i];
  return t >= 0 && t < V ? t : -1;
}

// A thread has pieces of E elements of kLookupRows rows in flight: their tokens first, then the table's rows.  The last piece of a row is
// moved back to end with it (its first elements are written twice, with the same values).
template <typename W, typename T, typename I, int E>
__global__ __launch_bounds__(kLookupThreads) void embedding_forward_kernel(const EmbeddingForward a) {
  const int lane = threadIdx.x & (a.lanes - 1), per_round = kLookupThreads / a.lanes;
  const int64_t first = (int64_t)blockIdx.x * per_round * kLookupRows + threadIdx.x / a.lanes;
  int64_t token[kLookupRows];
#pragma unroll
  for (int k = 0; k < kLookupRows; ++k) {
    const int64_t row = first + k * per_round;
    token[k] = row < a.N ? token_of(static_cast<const I*>(a.tokens), row, a.V) : -2;
  }
  const int pieces = (a.D + E - 1) / E;
  for (int p = lane; p < pieces; p += a.lanes) {
    const int at = min(p * E, a.D - E);
    Pack<W, E> w[kLookupRows];
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k)
      if (token[k] >= 0) w[k] = *reinterpret_cast<const Pack<W, E>*>(static_cast<const W*>(a.table) + token[k] * a.ldt + at);
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k) {
      if (token[k] == -2) continue;
      Pack<T, E> y;
#pragma unroll
      for (int j = 0; j < E; ++j) y.v[j] = from_float<T>(token[k] >= 0 ? a.scale * to_float(w[k].v[j]) : 0.f);
      *reinterpret_cast<Pack<T, E>*>(static_cast<T*>(a.y) + (first + k * per_round) * a.ldy + at) = y;
    }
  }
}

// A wavefront per row of the table and 64 columns: it looks through all tokens and adds the rows that name it.
template <typename T, typename W, typename I>
__global__ __launch_bounds__(256) void embedding_backward_kernel(const EmbeddingBackward a) {
  const int lane = threadIdx.x & 63;
  const int64_t v = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (v >= a.V) return;
  for (int64_t c = (int64_t)blockIdx.y * 64 + lane; c - lane < a.D; c += (int64_t)gridDim.y * 64) {
    float sum = 0.f;
    bool named = false;
    for (int64_t base = 0; base < a.N; base += 64) {
      const bool here = base + lane < a.N && token_of(static_cast<const I*>(a.tokens), base + lane, a.V) == v;
      uint64_t mask = __builtin_amdgcn_ballot_w64(here);
      named |= mask != 0;
      for (; mask != 0; mask &= mask - 1) {
        const int64_t i = base + __builtin_ctzll(mask);
        if (c < a.D) sum += to_float(static_cast<const T*>(a.dy)[i * a.lddy + c]);
      }
    }
    if (c >= a.D || (a.accumulate && !named)) continue;
    W* out = static_cast<W*>(a.dtable) + v * a.lddt + c;
    *out = from_float<W>((a.accumulate ? to_float(*out) : 0.f) + a.scale * sum);
  }
}

}  // namespace ngsgd

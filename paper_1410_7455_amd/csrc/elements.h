// Element types of the operators that take 16-bit data: loads and stores of several elements, sums over a workgroup.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ngsgd {

using bf16 = __bf16;
using fp16 = _Float16;

template <typename T, int V>
struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Pack {
  T v[V];
};

// Arithmetic is in fp32.  A result is rounded once, to the nearest value of its type (ties to even), as it is stored.
template <typename T>
__device__ __forceinline__ float to_float(const T x) { return static_cast<float>(x); }
template <typename T>
__device__ __forceinline__ T from_float(const float x) { return static_cast<T>(x); }

// Sum over the 64 lanes, to all of them: through the vector ALU's cross-lane path within rows of 16 lanes, then across them.
template <int CTRL>
__device__ __forceinline__ float dpp_add_f32(const float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float row16_sum_f32(float v) {
  v = dpp_add_f32<0xB1>(v);    // quad_perm [1,0,3,2]
  v = dpp_add_f32<0x4E>(v);    // quad_perm [2,3,0,1]
  v = dpp_add_f32<0x141>(v);   // row_half_mirror
  return dpp_add_f32<0x140>(v);   // row_mirror
}
__device__ __forceinline__ float wave_sum_f32(float v) {
  v = row16_sum_f32(v);
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// Two sums over a workgroup of WAVES wavefronts at the price of one barrier: `red` is used in turn by parity, so that a wavefront that is
// ahead writes into the other half.
template <int WAVES>
__device__ __forceinline__ void block_sum_pair_f32(float& a, float& b, float (*red)[2][WAVES], const int parity) {
  a = wave_sum_f32(a);
  b = wave_sum_f32(b);
  if (WAVES == 1) return;
  if ((threadIdx.x & 63) == 0) {
    red[parity][0][threadIdx.x >> 6] = a;
    red[parity][1][threadIdx.x >> 6] = b;
  }
  __syncthreads();
  a = red[parity][0][0];
  b = red[parity][1][0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) {
    a += red[parity][0][w];
    b += red[parity][1][w];
  }
}
template <int WAVES>
__device__ __forceinline__ float block_sum_f32(float a, float (*red)[2][WAVES], const int parity) {
  a = wave_sum_f32(a);
  if (WAVES == 1) return a;
  if ((threadIdx.x & 63) == 0) red[parity][0][threadIdx.x >> 6] = a;
  __syncthreads();
  a = red[parity][0][0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) a += red[parity][0][w];
  return a;
}

}  // namespace ngsgd

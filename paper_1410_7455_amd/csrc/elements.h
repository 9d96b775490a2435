// Element types of the operators that take 16-bit data: loads and stores of several elements, sums over a workgroup.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ngsgd {

using bf16 = __bf16;
using fp16 = _Float16;

// V neighbours in memory, on any element's boundary: the target's vector loads and stores take addresses that are multiples of
// nothing, so one path serves every leading dimension and every start of a matrix.
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
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
// The two halves of 32 lanes, or of each half the two of 16, with their lanes exchanged: one instruction gives both addends.
__device__ __forceinline__ float half16_add_f32(const float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float half32_add_f32(const float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float wave_sum_f32(const float v) { return half32_add_f32(half16_add_f32(row16_sum_f32(v))); }

__device__ __forceinline__ bool any_lane(const bool b) { return __builtin_amdgcn_ballot_w64(b) != 0; }

// Sums over a workgroup of up to 16 wavefronts at the price of one barrier: `red` is used in turn by parity, so that a wavefront that is
// ahead writes into the other half.  A lane reads one wavefront's sums, and the 16 lanes of a row add them.
constexpr int kMaxWaves = 16;
using BlockScratch = Pack<float, 2>[2][kMaxWaves];

__device__ __forceinline__ void block_sum_pair_f32(float& a, float& b, BlockScratch& red, const int parity) {
  a = wave_sum_f32(a);
  b = wave_sum_f32(b);
  if ((threadIdx.x & 63) == 0) red[parity][threadIdx.x >> 6] = Pack<float, 2>{{a, b}};
  __syncthreads();
  const int wave = threadIdx.x & 15;
  const Pack<float, 2> of = red[parity][wave];
  const bool here = wave < (int)(blockDim.x >> 6);
  a = row16_sum_f32(here ? of.v[0] : 0.f);
  b = row16_sum_f32(here ? of.v[1] : 0.f);
}
__device__ __forceinline__ float block_sum_f32(float a, BlockScratch& red, const int parity) {
  float none = 0.f;
  block_sum_pair_f32(a, none, red, parity);
  return a;
}

}  // namespace ngsgd

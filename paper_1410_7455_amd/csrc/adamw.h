// AdamW over many tensors in one launch, with moments in fp32 or in 8 bits (gfx950, 64-lane wavefronts).
//   g' = scale g;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
//   p  = p (1 - lr decay) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// The moments of all tensors lie in one flat array, each tensor's on a multiple of 256 elements.
//
// In 8 bits the 256 elements of a block share an exponent E per moment, the least with 1.875 2^E >= the block's largest finite
// magnitude; a wavefront holds a block, four elements in a lane.  With E's bits as in fp32 and three bits behind the point, a code is a
// difference of the upper 12 bits of two fp32 numbers:
//   m: sign and 7 bits, 0: zero, 1 .. 127: (1 + 1/8) 2^(E-15) .. 1.875 2^E; the sign alone (0x80): NaN
//   v: held by its root (v spans twice the binades), 0: zero, 1 .. 254: 1.25 2^(E-31) .. 1.875 2^E; 255: NaN
// Scales are powers of two, so a code stands for exactly one value of at most 8 significant bits, and coding a value again gives its
// code.  Below the least code m is rounded to zero or to that code, and v, a divisor, up.
// Rounding: a step changes v by about (1 - b2) of itself, a thousandth, and half a step of the code is a sixteenth: rounded to nearest it
// would stay where it is for ever.  So `dither` (of a step, 20 bits) is added before the code is cut off.  For an element it is
// frac(i phi + t sqrt 2) in 32-bit integers, a sequence that visits [0, 1) evenly over the steps t: an element is
// rounded up as often as its fraction says, and no random numbers are read.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elements.h"

namespace ngsgd {

constexpr int kAdamBlock = 256;         // elements that share an exponent
constexpr int kAdamChunk = 4096;        // elements of a piece of work: a workgroup's four wavefronts take four blocks each
constexpr int kAdamThreads = 256;
constexpr int kAdamGrads = 448;         // gradients whose addresses one launch carries (of 4 KB of arguments)
constexpr uint32_t kDitherIndex = 0x9E3779B1u, kDitherStep = 0x6A09E667u;   // 2^32 times the fractions of phi (odd) and sqrt 2
constexpr uint32_t kDitherHalf = 1u << 19;                                  // to nearest

struct AdamTensor {
  void* p;
  int64_t n;
  int64_t offset;    // of its moments, a multiple of kAdamBlock
  float rate;        // factor on the learning rate
  float decay;
};
struct AdamChunk {
  int tensor;
  int index;         // elements [index kAdamChunk, ...) of the tensor
};
// On the device, so that a captured step counts on when it is replayed.
struct AdamScalars {
  int64_t t;                 // steps so far
  double b1_power, b2_power; // b1^t, b2^t
  unsigned done;             // workgroups of the step that have read these
};

struct AdamState {
  const AdamTensor* tensors;
  const AdamChunk* chunks;
  AdamScalars* scalars;
  float* master;             // fp32 copies of the parameters, flat as the moments
  float *m32, *v32;
  uint8_t *m8, *v8, *m_exp, *v_exp;   // codes, and exponents by block
};

struct AdamStep {
  AdamState s;
  int first_tensor, first_chunk, n_chunks;
  unsigned last;             // the workgroup that is the step's last one to be done
  float lr, scale, eps;
  double beta1, beta2;       // (in fp32, 1 - 0.999 would be off by 1e-5 of itself)
  const float* dev_lr;       // optional factors on lr and scale
  const float* dev_scale;
  const void* grads[kAdamGrads];
};

// ---- codes -------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t dither_of(const int64_t i, const int64_t t) {
  return ((uint32_t)i * kDitherIndex + (uint32_t)t * kDitherStep) >> 12;
}
__device__ __forceinline__ bool finite_bits(const uint32_t magnitude) { return magnitude < 0x7f800000u; }
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, off));
  return v;
}
// E (biased as in fp32) of a block with this largest finite magnitude; not below what the least code can be written with.
__device__ __forceinline__ uint32_t exponent_of(const uint32_t top, const uint32_t lowest) { return max((top + 0xFFFFFu) >> 23, lowest); }
constexpr uint32_t kLowestM = 16, kLowestV = 32;

__device__ __forceinline__ int base_m(const uint32_t e) { return (int)(e + 1) * 8 - 128; }
__device__ __forceinline__ int base_v(const uint32_t e) { return (int)(e + 1) * 8 - 255; }

__device__ __forceinline__ uint8_t code_m(const float m, const uint32_t e, const uint32_t dither) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, m), a = bits & 0x7fffffffu;
  if (!finite_bits(a)) return 0x80;
  const int base = base_m(e);
  const float magnitude = __builtin_bit_cast(float, a), least = __builtin_bit_cast(float, (uint32_t)(base + 1) << 20);
  int code = min(max((int)((a + dither) >> 20) - base, 1), 127);
  if (magnitude < least) code = magnitude > least * ((float)dither * 0x1p-20f) ? 1 : 0;
  return (uint8_t)(code == 0 ? 0 : code | (bits >> 31 << 7));
}
__device__ __forceinline__ float value_m(const uint32_t code, const uint32_t e) {
  if (code == 0x80u) return __builtin_nanf("");
  const uint32_t magnitude = (code & 0x7fu) == 0 ? 0u : ((code & 0x7fu) + base_m(e)) << 20;
  return __builtin_bit_cast(float, magnitude | (code >> 7 << 31));
}
__device__ __forceinline__ uint8_t code_root(const float r, const uint32_t e, const uint32_t dither) {
  const uint32_t bits = __builtin_bit_cast(uint32_t, r);
  if (!finite_bits(bits)) return 255;   // (a root is not negative; that of a negative number is NaN)
  return (uint8_t)(bits == 0 ? 0 : min(max((int)((bits + dither) >> 20) - base_v(e), 1), 254));
}
__device__ __forceinline__ float value_v(const uint32_t code, const uint32_t e) {
  if (code == 255u) return __builtin_nanf("");
  const float r = code == 0 ? 0.f : __builtin_bit_cast(float, (uint32_t)((int)code + base_v(e)) << 20);
  return r * r;
}

// Four consecutive elements of a lane; `here` of them exist.
template <typename T>
__device__ __forceinline__ void load4(float (&out)[4], const T* p, const int here, const bool aligned) {
  if (here >= 4 && aligned) {
    const Pack<T, 4> v = *reinterpret_cast<const Pack<T, 4>*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = to_float(v.v[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = k < here ? to_float(p[k]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store4(const float (&v)[4], T* p, const int here, const bool aligned) {
  if (here >= 4 && aligned) {
    Pack<T, 4> o;
#pragma unroll
    for (int k = 0; k < 4; ++k) o.v[k] = from_float<T>(v[k]);
    *reinterpret_cast<Pack<T, 4>*>(p) = o;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < here) p[k] = from_float<T>(v[k]);
  }
}

// The moments of a lane's four elements of block `block` (both numbered over the flat arrays).
template <int BITS>
__device__ __forceinline__ void load_moments(const AdamState& s, const int64_t block, float (&m)[4], float (&v)[4]) {
  const int64_t at = block * kAdamBlock + 4 * (threadIdx.x & 63);
  if (BITS == 32) {
    load4(m, s.m32 + at, 4, true);
    load4(v, s.v32 + at, 4, true);
  } else {
    const uint32_t mc = *reinterpret_cast<const uint32_t*>(s.m8 + at), vc = *reinterpret_cast<const uint32_t*>(s.v8 + at);
    const uint32_t me = s.m_exp[block], ve = s.v_exp[block];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = value_m(mc >> (8 * k) & 0xffu, me);
      v[k] = value_v(vc >> (8 * k) & 0xffu, ve);
    }
  }
}
template <int BITS>
__device__ __forceinline__ void store_moments(const AdamState& s, const int64_t block, const float (&m)[4], const float (&v)[4], const bool nearest,
                                              const int64_t t) {
  const int lane = threadIdx.x & 63;
  const int64_t at = block * kAdamBlock + 4 * lane;
  if (BITS == 32) {
    store4(m, s.m32 + at, 4, true);
    store4(v, s.v32 + at, 4, true);
  } else {
    float r[4];
    uint32_t mt = 0, rt = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      r[k] = sqrtf(v[k]);
      const uint32_t a = __builtin_bit_cast(uint32_t, m[k]) & 0x7fffffffu, b = __builtin_bit_cast(uint32_t, r[k]) & 0x7fffffffu;
      mt = max(mt, finite_bits(a) ? a : 0u);
      rt = max(rt, finite_bits(b) ? b : 0u);
    }
    const uint32_t me = exponent_of(wave_max_u32(mt), kLowestM), ve = exponent_of(wave_max_u32(rt), kLowestV);
    uint32_t mc = 0, vc = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t dither = nearest ? kDitherHalf : dither_of(at + k, t);
      mc |= (uint32_t)code_m(m[k], me, dither) << (8 * k);
      vc |= (uint32_t)code_root(r[k], ve, dither) << (8 * k);
    }
    *reinterpret_cast<uint32_t*>(s.m8 + at) = mc;
    *reinterpret_cast<uint32_t*>(s.v8 + at) = vc;
    if (lane == 0) {
      s.m_exp[block] = (uint8_t)me;
      s.v_exp[block] = (uint8_t)ve;
    }
  }
}

// ---- the step ------------------------------------------------------------------------------------------
// Workgroups walk over the chunks.  P: parameters, G: gradients.
template <typename P, typename G, int BITS, bool MASTER>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamStep a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  AdamScalars* const st = a.s.scalars;
  const int64_t t = st->t + 1;
  const double b1_power = st->b1_power * a.beta1, b2_power = st->b2_power * a.beta2;
  const float lr = a.dev_lr != nullptr ? a.lr * *a.dev_lr : a.lr;
  const float scale = a.dev_scale != nullptr ? a.scale * *a.dev_scale : a.scale;
  const float beta1 = (float)a.beta1, m_part = (float)(1.0 - a.beta1), beta2 = (float)a.beta2, v_part = (float)(1.0 - a.beta2);
  const float m_unbias = (float)(1.0 / (1.0 - b1_power)), v_unbias = (float)(1.0 / (1.0 - b2_power));
  for (int c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
    const AdamChunk chunk = a.s.chunks[a.first_chunk + c];
    const AdamTensor tensor = a.s.tensors[chunk.tensor];
    const G* const grad = static_cast<const G*>(a.grads[chunk.tensor - a.first_tensor]);
    if (grad == nullptr) continue;
    P* const param = static_cast<P*>(tensor.p);
    const float rate = lr * tensor.rate, keep = 1.f - rate * tensor.decay, step = rate * m_unbias;
    const bool aligned_g = (reinterpret_cast<uintptr_t>(grad) & (4 * sizeof(G) - 1)) == 0;
    const bool aligned_p = (reinterpret_cast<uintptr_t>(param) & (4 * sizeof(P) - 1)) == 0;
    for (int k = wave; k < kAdamChunk / kAdamBlock; k += kAdamThreads / 64) {
      const int64_t i = (int64_t)chunk.index * kAdamChunk + k * kAdamBlock + 4 * lane;
      if (i - 4 * lane >= tensor.n) break;   // (uniform in a wavefront)
      const int here = (int)min((int64_t)4, max((int64_t)0, tensor.n - i));
      const int64_t block = (tensor.offset + i) / kAdamBlock;
      float g[4], p[4], m[4], v[4];
      load4(g, grad + i, here, aligned_g);
      if (MASTER)
        load4(p, a.s.master + tensor.offset + i, 4, true);
      else
        load4(p, param + i, here, aligned_p);
      load_moments<BITS>(a.s, block, m, v);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float gs = g[u] * scale;
        m[u] = beta1 * m[u] + m_part * gs;
        v[u] = beta2 * v[u] + v_part * (gs * gs);
        p[u] = p[u] * keep - step * m[u] / (sqrtf(v[u] * v_unbias) + a.eps);
      }
      store_moments<BITS>(a.s, block, m, v, false, t);
      if (MASTER) store4(p, a.s.master + tensor.offset + i, 4, true);
      store4(p, param + i, here, aligned_p);
    }
  }
  // the last workgroup to be done counts the step: everybody has read the scalars
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    if (__hip_atomic_fetch_add(&st->done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == a.last) {
      st->t = t;
      st->b1_power = b1_power;
      st->b2_power = b2_power;
      st->done = 0;
    }
  }
}

// ---- state in and out -------------------------------------------------------------------------------------
// A wavefront per block of the flat arrays.
template <typename T>
__global__ __launch_bounds__(kAdamThreads) void adamw_get_state_kernel(const AdamState s, const int bits, const int64_t blocks, T* m_out, T* v_out) {
  const int64_t step = (int64_t)gridDim.x * (kAdamThreads / 64);
  for (int64_t block = (int64_t)blockIdx.x * (kAdamThreads / 64) + (threadIdx.x >> 6); block < blocks; block += step) {
    float m[4], v[4];
    if (bits == 32)
      load_moments<32>(s, block, m, v);
    else
      load_moments<8>(s, block, m, v);
    const int64_t at = block * kAdamBlock + 4 * (threadIdx.x & 63);
    if (m_out != nullptr) store4(m, m_out + at, 4, true);
    if (v_out != nullptr) store4(v, v_out + at, 4, true);
  }
}

// Moments, rounded to nearest, and the step count.  nullptr: zeros.
__global__ __launch_bounds__(kAdamThreads) void adamw_set_state_kernel(const AdamState s, const int bits, const int64_t blocks, const float* m_in,
                                                                       const float* v_in, const AdamScalars scalars) {
  const int64_t step = (int64_t)gridDim.x * (kAdamThreads / 64);
  for (int64_t block = (int64_t)blockIdx.x * (kAdamThreads / 64) + (threadIdx.x >> 6); block < blocks; block += step) {
    float m[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
    const int64_t at = block * kAdamBlock + 4 * (threadIdx.x & 63);
    if (m_in != nullptr) load4(m, m_in + at, 4, true);
    if (v_in != nullptr) load4(v, v_in + at, 4, true);
    if (bits == 32)
      store_moments<32>(s, block, m, v, true, 0);
    else
      store_moments<8>(s, block, m, v, true, 0);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *s.scalars = scalars;
}

// The parameters' fp32 copies, from the parameters or from a flat array, from which the parameters are then written too.
template <typename P>
__global__ __launch_bounds__(kAdamThreads) void adamw_set_master_kernel(const AdamState s, const int n_chunks, const float* in) {
  for (int c = blockIdx.x; c < n_chunks; c += gridDim.x) {
    const AdamChunk chunk = s.chunks[c];
    const AdamTensor tensor = s.tensors[chunk.tensor];
    P* const param = static_cast<P*>(tensor.p);
    const int64_t first = (int64_t)chunk.index * kAdamChunk, end = min(first + kAdamChunk, tensor.n);
    for (int64_t i = first + threadIdx.x; i < end; i += kAdamThreads) {
      if (in != nullptr) {
        s.master[tensor.offset + i] = in[tensor.offset + i];
        param[i] = from_float<P>(in[tensor.offset + i]);
      } else {
        s.master[tensor.offset + i] = to_float(param[i]);
      }
    }
  }
}

}  // namespace ngsgd

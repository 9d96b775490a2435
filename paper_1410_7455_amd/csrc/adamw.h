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
constexpr float kLargest = 3.4028234663852886e38f;                          // what fp32 holds

// A piece of work: up to kAdamChunk elements of a tensor, with all that a workgroup has to know of it (one read from memory before the data's).
struct AdamChunk {
  void* p;           // its parameters
  int64_t offset;    // of its moments, a multiple of kAdamBlock
  int tensor, index; // elements [index kAdamChunk, ...) of the tensor
  int n;             // how many
  float rate;        // factor on the learning rate
  float decay;
  int unused;
};
// On the device, so that a captured step counts on when it is replayed.
struct AdamScalars {
  int64_t t;                   // steps so far
  double b1_power, b2_power;   // b1^t, b2^t
  float m_unbias, root_unbias; // 1 / (1 - b1^t), (1 - b2^t)^(-1/2)
  unsigned done, unused;       // workgroups of a counting step that have read these
};

struct AdamExponents {
  uint8_t m, v;   // E of the block's m and of its roots of v, biased as in fp32
  uint16_t nan;   // not 0: some code stands for NaN
};

struct AdamState {
  const AdamChunk* chunks;
  AdamScalars* scalars;
  float* master;             // fp32 copies of the parameters, flat as the moments
  float *m32, *v32;
  uint8_t *m8, *v8;          // codes
  AdamExponents* exps;       // by block
};

struct AdamStep {
  AdamState s;
  int first_tensor, first_chunk;
  int part_bits;             // 2^part_bits workgroups share a chunk: 1 or 4
  int counts;                // the step's only launch, of few workgroups: the last one of them to be done counts the step
  float lr, scale, eps;
  double beta1, beta2;
  const float* dev_lr;       // optional factors on lr and scale
  const float* dev_scale;
  const void* grads[kAdamGrads];
};

// ---- codes -------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t dither_start(const int64_t i, const int64_t t) { return (uint32_t)i * kDitherIndex + (uint32_t)t * kDitherStep; }
__device__ __forceinline__ uint32_t dither_of(const uint32_t start, const int k) { return (start + (uint32_t)k * kDitherIndex) >> 12; }   // of element i + k
__device__ __forceinline__ bool finite_bits(const uint32_t magnitude) { return magnitude < 0x7f800000u; }

// Largest of the 64 lanes, in a scalar register.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_u32(const uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = dpp_max_u32<0xB1>(v);    // quad_perm [1,0,3,2]
  v = dpp_max_u32<0x4E>(v);    // quad_perm [2,3,0,1]
  v = dpp_max_u32<0x141>(v);   // row_half_mirror
  v = dpp_max_u32<0x140>(v);   // row_mirror
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max((uint32_t)a[0], (uint32_t)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __builtin_amdgcn_readfirstlane(max((uint32_t)b[0], (uint32_t)b[1]));
}

// E (biased as in fp32) of a block with this largest finite magnitude; not below what the least code can be written with, and not above what keeps
// the largest code, or its square, a finite number of fp32: what is above 1.875 2^127 (v: (1.875 2^63)^2) is held as that.
__device__ __forceinline__ uint32_t exponent_of(const uint32_t top, const uint32_t lowest, const uint32_t highest) {
  return max(min(top + 0xFFFFFu, highest << 23) >> 23, lowest);
}
constexpr uint32_t kLowestM = 16, kLowestV = 32, kHighestM = 127 + 127, kHighestV = 63 + 127;

__device__ __forceinline__ int base_m(const uint32_t e) { return (int)(e + 1) * 8 - 128; }
__device__ __forceinline__ int base_v(const uint32_t e) { return (int)(e + 1) * 8 - 255; }

// What is coded is held in 64 bits: with m or the root rounded to 32 first, one code in some 10^6 would lie on the other side of a border.
// The upper 15 bits of such a number (sign apart) are its binade and eighth: code = those, minus the block's base in the same units.
constexpr int kBase64 = (1023 - 127) * 8;   // between the two formats' exponents
__device__ __forceinline__ uint64_t bits_of(const double x) { return __builtin_bit_cast(uint64_t, x); }
__device__ __forceinline__ uint32_t eighths(const uint64_t magnitude, const uint32_t dither) {
  return (uint32_t)((magnitude + ((uint64_t)dither << 29)) >> 49);
}
__device__ __forceinline__ double least_of(const int base) { return __builtin_bit_cast(double, (uint64_t)(base + 1 + kBase64) << 49); }

__device__ __forceinline__ uint32_t code_m(const double m, const int base, const uint32_t dither) {
  const uint64_t bits = bits_of(m), a = bits & ~(1ull << 63);
  if (!(fabs(m) <= 3.4028234663852886e38)) return 0x80;   // (what fp32 holds)
  const double least = least_of(base);
  int code = min(max((int)eighths(a, dither) - base - kBase64, 1), 127);
  if (fabs(m) < least) code = fabs(m) > least * ((double)dither * 0x1p-20) ? 1 : 0;
  return code == 0 ? 0u : (uint32_t)code | (uint32_t)(bits >> 63 << 7);
}
__device__ __forceinline__ uint32_t code_root(const double r, const int base, const uint32_t dither) {
  if (!(r <= 3.4028234663852886e38)) return 255u;   // (a root is not negative; that of a negative number is NaN)
  return r == 0.0 ? 0u : (uint32_t)min(max((int)eighths(bits_of(r), dither) - base - kBase64, 1), 254);
}

// Four consecutive elements of a lane; `here` of them exist.
template <typename T>
__device__ __forceinline__ void load4(float (&out)[4], const T* p, const int here) {
  if (here >= 4) {
    const Pack<T, 4> v = *reinterpret_cast<const Pack<T, 4>*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = to_float(v.v[k]);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) out[k] = k < here ? to_float(p[k]) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store4(const float (&v)[4], T* p, const int here) {
  if (here >= 4) {
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

// The moments of a lane's four elements of block `block` (both numbered over the flat arrays), as they lie in memory.
template <int BITS>
struct Moments {
  Pack<float, 4> m, v;
  __device__ __forceinline__ void load(const AdamState& s, const int64_t block) {
    const int64_t at = block * kAdamBlock + 4 * (threadIdx.x & 63);
    m = *reinterpret_cast<const Pack<float, 4>*>(s.m32 + at);
    v = *reinterpret_cast<const Pack<float, 4>*>(s.v32 + at);
  }
  __device__ __forceinline__ void get(float (&m_out)[4], float (&v_out)[4]) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m_out[k] = m.v[k];
      v_out[k] = v.v[k];
    }
  }
};
template <>
struct Moments<8> {
  uint32_t m, v;
  AdamExponents exps;
  __device__ __forceinline__ void load(const AdamState& s, const int64_t block) {
    const int64_t at = block * kAdamBlock + 4 * (threadIdx.x & 63);
    m = *reinterpret_cast<const uint32_t*>(s.m8 + at);
    v = *reinterpret_cast<const uint32_t*>(s.v8 + at);
    exps = s.exps[block];
  }
  __device__ __forceinline__ void get(float (&m_out)[4], float (&v_out)[4]) const {
    const uint32_t e = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(uint32_t, exps));
    const uint32_t mb = (uint32_t)base_m(e & 0xffu), vb = (uint32_t)base_v(e >> 8 & 0xffu);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t mc = m >> (8 * k) & 0x7fu, vc = v >> (8 * k) & 0xffu, sign = m << (24 - 8 * k) & 0x80000000u;
      m_out[k] = __builtin_bit_cast(float, (mc == 0 ? 0u : (mc + mb) << 20) | sign);
      const float r = __builtin_bit_cast(float, vc == 0 ? 0u : (vc + vb) << 20);
      v_out[k] = r * r;
    }
    if (e >> 16 != 0) {   // (uniform)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if ((m >> (8 * k) & 0xffu) == 0x80u) m_out[k] = __builtin_nanf("");
        if ((v >> (8 * k) & 0xffu) == 0xffu) v_out[k] = __builtin_nanf("");
      }
    }
  }
};

// Codes of a lane's four elements of block `block`, given m and the roots of v.  `plain`: all are finite.  `start`: see dither_start.
__device__ __forceinline__ void store_codes(const AdamState& s, const int64_t block, const double (&m)[4], const double (&r)[4], const bool plain,
                                            const bool nearest, const uint32_t start) {
  const int lane = threadIdx.x & 63;
  const int64_t at = block * kAdamBlock + 4 * lane;
  uint32_t a[4], b[4], dither[4];   // as fp32
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    a[k] = __builtin_bit_cast(uint32_t, (float)m[k]) & 0x7fffffffu;
    b[k] = __builtin_bit_cast(uint32_t, (float)r[k]) & 0x7fffffffu;
    dither[k] = nearest ? kDitherHalf : dither_of(start, k);
  }
  uint32_t mt = max(max(a[0], a[1]), max(a[2], a[3])), rt = max(max(b[0], b[1]), max(b[2], b[3])), nan = 0;
  if (!plain) {   // (uniform)
    bool odd = false;
    mt = rt = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      mt = max(mt, finite_bits(a[k]) ? a[k] : 0u);
      rt = max(rt, finite_bits(b[k]) ? b[k] : 0u);
      odd |= !finite_bits(a[k]) || !finite_bits(b[k]);
    }
    nan = any_lane(odd) ? 1u : 0u;
  }
  const uint32_t me = exponent_of(wave_max_u32(mt), kLowestM, kHighestM), ve = exponent_of(wave_max_u32(rt), kLowestV, kHighestV);
  const int mb = base_m(me), vb = base_v(ve);
  // (a code's first number and the one above it: what rounds to the first in fp32 is not below it by more than that)
  const uint32_t m_least = ((uint32_t)(mb + 1) << 20) + 1, r_least = ((uint32_t)(vb + 1) << 20) + 1;
  uint32_t mc = 0, vc = 0;
  if (plain && !any_lane(min(min(a[0], a[1]), min(a[2], a[3])) < m_least || min(min(b[0], b[1]), min(b[2], b[3])) < r_least)) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {   // what the general form comes to where nothing is below the least code
      const uint64_t bits = bits_of(m[k]);
      mc |= (min(eighths(bits & ~(1ull << 63), dither[k]) - (uint32_t)(mb + kBase64), 127u) | ((uint32_t)(bits >> 56) & 0x80u)) << (8 * k);
      vc |= min(eighths(bits_of(r[k]), dither[k]) - (uint32_t)(vb + kBase64), 254u) << (8 * k);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      mc |= code_m(m[k], mb, dither[k]) << (8 * k);
      vc |= code_root(r[k], vb, dither[k]) << (8 * k);
    }
  }
  *reinterpret_cast<uint32_t*>(s.m8 + at) = mc;
  *reinterpret_cast<uint32_t*>(s.v8 + at) = vc;
  if (lane == 0) s.exps[block] = AdamExponents{(uint8_t)me, (uint8_t)ve, (uint16_t)nan};
}

// Classes of fp32 numbers, as v_cmp_class takes them.
constexpr int kClassNotFinite = 0x207, kClassZeroOrNormal = 0x160;   // NaN, -inf, +inf; -0, +0, a positive normal number

// Root of zero or of a number that is normal in fp32, by one step of Newton's from the hardware's estimate of v^(-1/2) (a third of the
// instructions of the library's, which has to do with subnormal numbers too): rounded to nearest in fp32 but for a few cases in a thousand, and
// with the step in 64 bits off by 2^-45 of itself.
__device__ __forceinline__ float quick_root(const float v) {
  const float y = __builtin_amdgcn_rsqf(v), s = v * y, h = 0.5f * y;
  return v == 0.f ? 0.f : fmaf(fmaf(-s, s, v), h, s);
}
__device__ __forceinline__ double quick_root(const double v, const float v32) {
  const float y = __builtin_amdgcn_rsqf(v32);
  const double s = (double)(v32 * y);
  return v32 == 0.f ? 0.0 : fma(fma(-s, s, v), (double)(0.5f * y), s);
}

// ---- the step ------------------------------------------------------------------------------------------
// beta held + (1 - beta) new in fp32.  beta is the sum of two fp32 numbers: with the first alone, a moment would fade by 1 - beta rounded to
// a multiple of 2^-24 (0.99999: 0.14 % too fast, 0.9999999: a fifth).  What fades by the second is kept finite, so that an infinite moment stays.
struct Beta {
  float high, low, part;
  __device__ __forceinline__ explicit Beta(const double beta) : high((float)beta), low((float)(beta - (double)(float)beta)), part((float)(1.0 - beta)) {}
  __device__ __forceinline__ float mix(const float held, const float now) const {
    return fmaf(high, held, fmaf(low, __builtin_amdgcn_fmed3f(held, -kLargest, kLargest), part * now));
  }
};

__device__ __forceinline__ AdamScalars counted(AdamScalars st, const double beta1, const double beta2) {
  st.t += 1;
  st.b1_power *= beta1;
  st.b2_power *= beta2;
  st.m_unbias = (float)(1.0 / (1.0 - st.b1_power));
  st.root_unbias = (float)sqrt(1.0 / (1.0 - st.b2_power));
  return st;
}
// Counts the step in a launch of its own, about 1.5 us (and 2.5 us of the host's time).  A counter by which the step's last workgroup knows itself
// costs 30 to 60 ns for each workgroup, one after the other: 90 us for 1536 of them, so only steps of few workgroups count that way.
__global__ void adamw_count_kernel(AdamScalars* st, const double beta1, const double beta2) { *st = counted(*st, beta1, beta2); }

// What no thread of the launch writes: read through the scalar cache.
template <typename T>
__device__ __forceinline__ T constant(const T* p, const int i) {
  static_assert(sizeof(T) % 8 == 0, "whole words");
  const auto* const from = reinterpret_cast<const __attribute__((address_space(4))) uint64_t*>(reinterpret_cast<uintptr_t>(p + i));
  uint64_t words[sizeof(T) / 8];
#pragma unroll
  for (size_t k = 0; k < sizeof(T) / 8; ++k) words[k] = from[k];
  return __builtin_bit_cast(T, words);
}

// A workgroup per chunk, or per quarter of one where there are few; a wavefront takes a block at a time.  P: parameters, G: gradients.  Bound by
// memory: 252 M elements with fp32 parameters, 16-bit gradients and moments in 8 bits 695 us (5.1 TB/s; 45 more with 1536 workgroups that walk
// over the chunks), in 32 bits 1352 us (5.2 TB/s).  In 8 bits the vector ALU is busy for nearly as long (84 instructions an element: with
// the library's root and quotient and codes that allow for everything in every block it took 884 us), and parameters and gradients of 16
// bits leave it the bound (201 M elements 508 us, 4.0 TB/s).  Blocks with a zero, or a number below the least code, take the general codes: 7 %
// more where every block has one (16 bits: 10 %), 21 % (27) with a NaN in every block.
template <typename P, typename G, int BITS, bool MASTER>
__global__ __launch_bounds__(kAdamThreads) void adamw_kernel(const AdamStep a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const AdamChunk chunk = constant(a.s.chunks, a.first_chunk + ((int)blockIdx.x >> a.part_bits));
  AdamScalars scalars = *a.s.scalars;
  if (a.counts) scalars = counted(scalars, a.beta1, a.beta2);
  const G* grad = static_cast<const G*>(a.grads[chunk.tensor - a.first_tensor]);
  if (grad != nullptr) {
    const float lr = (a.dev_lr != nullptr ? a.lr * *a.dev_lr : a.lr) * chunk.rate;
    const float scale = a.dev_scale != nullptr ? a.scale * *a.dev_scale : a.scale;
    const Beta beta1(a.beta1), beta2(a.beta2);
    const float fade = lr * chunk.decay, step = lr * scalars.m_unbias;
    grad += (int64_t)chunk.index * kAdamChunk;
    P* const param = static_cast<P*>(chunk.p);
    float* const master = MASTER ? a.s.master + chunk.offset : nullptr;
    const int64_t first_block = chunk.offset / kAdamBlock;
    const int blocks = kAdamChunk / kAdamBlock / (kAdamThreads / 64) >> a.part_bits;   // of a wavefront in a row
    const int first = (((int)blockIdx.x & ((1 << a.part_bits) - 1)) * (kAdamThreads / 64) + wave) * (blocks * kAdamBlock);
    for (int k = 0; k < blocks; ++k) {
      const int i0 = first + k * kAdamBlock, i = i0 + 4 * lane;
      if (i0 >= chunk.n) break;   // (uniform in a wavefront)
      const int64_t block = first_block + i0 / kAdamBlock;
      const int here = min(4, chunk.n - i);
      float g[4], p[4], m[4], v[4], r[4];
      Moments<BITS> held;
      held.load(a.s, block);
      load4(g, grad + i, here);
      if constexpr (MASTER)
        load4(p, master + i, 4);   // (the flat arrays have whole blocks)
      else
        load4(p, param + i, here);
      held.get(m, v);
      bool odd = false;
      double m64[4], v64[4], r64[4];   // moments that will be coded
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BITS == 32) {
          const float gs = g[e] * scale;
          m[e] = beta1.mix(m[e], gs);
          v[e] = beta2.mix(v[e], gs * gs);
        } else {
          const double gs = (double)g[e] * (double)scale;
          m64[e] = a.beta1 * (double)m[e] + (1.0 - a.beta1) * gs;
          v64[e] = a.beta2 * (double)v[e] + (1.0 - a.beta2) * (gs * gs);
          m[e] = (float)m64[e];
          v[e] = (float)v64[e];
        }
      }
      if (i0 + kAdamBlock > chunk.n) {   // (uniform) behind the tensor's end the moments stay zero, also where the factors are not finite
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (e < here) continue;
          m[e] = v[e] = 0.f;
          if constexpr (BITS == 8) m64[e] = v64[e] = 0.0;
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) odd |= __builtin_amdgcn_classf(m[e], kClassNotFinite) || !__builtin_amdgcn_classf(v[e], kClassZeroOrNormal);
      const bool plain = !any_lane(odd);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BITS == 32) {
          r[e] = plain ? quick_root(v[e]) : sqrtf(v[e]);
        } else {
          r64[e] = plain ? quick_root(v64[e], v[e]) : sqrt(v64[e]);
          r[e] = (float)r64[e];
        }
        // (the divisor is 0, epsilon or a normal number: the hardware's reciprocal is within a unit in the last place)
        // What an element loses is formed before it is taken off, so that its rounding is the element's own: 1 - lr decay, rounded to fp32, would be off
        // by up to 2^-25 in every element alike (lr 2e-5 with a decay of 0.01 would fade by 11 % too little).  An infinite p stays.
        p[e] -= fmaf(fade, __builtin_amdgcn_fmed3f(p[e], -kLargest, kLargest), (step * m[e]) * __builtin_amdgcn_rcpf(r[e] * scalars.root_unbias + a.eps));
      }
      if constexpr (BITS == 32) {
        const int64_t at = block * kAdamBlock + 4 * lane;
        store4(m, a.s.m32 + at, 4);
        store4(v, a.s.v32 + at, 4);
      } else {
        store_codes(a.s, block, m64, r64, plain, false, dither_start(block * kAdamBlock + 4 * lane, scalars.t));
      }
      if constexpr (MASTER) store4(p, master + i, here);
      store4(p, param + i, here);
    }
  }
  if (!a.counts) return;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    if (__hip_atomic_fetch_add(&a.s.scalars->done, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1) {
      scalars.done = 0;
      *a.s.scalars = scalars;   // everybody has read them
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
    if (bits == 32) {
      Moments<32> held;
      held.load(s, block);
      held.get(m, v);
    } else {
      Moments<8> held;
      held.load(s, block);
      held.get(m, v);
    }
    const int64_t at = block * kAdamBlock + 4 * (threadIdx.x & 63);
    if (m_out != nullptr) store4(m, m_out + at, 4);
    if (v_out != nullptr) store4(v, v_out + at, 4);
  }
}

// Moments, rounded to nearest, and the step count.  nullptr: zeros.
__global__ __launch_bounds__(kAdamThreads) void adamw_set_state_kernel(const AdamState s, const int bits, const int64_t blocks, const float* m_in,
                                                                       const float* v_in, const AdamScalars scalars) {
  const int64_t step = (int64_t)gridDim.x * (kAdamThreads / 64);
  for (int64_t block = (int64_t)blockIdx.x * (kAdamThreads / 64) + (threadIdx.x >> 6); block < blocks; block += step) {
    float m[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
    const int64_t at = block * kAdamBlock + 4 * (threadIdx.x & 63);
    if (m_in != nullptr) load4(m, m_in + at, 4);
    if (v_in != nullptr) load4(v, v_in + at, 4);
    if (bits == 32) {
      store4(m, s.m32 + at, 4);
      store4(v, s.v32 + at, 4);
    } else {
      double m64[4], r64[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m64[k] = (double)m[k];
        r64[k] = sqrt((double)v[k]);
      }
      store_codes(s, block, m64, r64, false, true, 0);
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *s.scalars = scalars;
}

// A workgroup per chunk: the parameters' fp32 copies, from the parameters or from a flat array, from which the parameters are then written too.
template <typename P>
__global__ __launch_bounds__(kAdamThreads) void adamw_set_master_kernel(const AdamState s, const float* in) {
  const AdamChunk chunk = s.chunks[blockIdx.x];
  P* const param = static_cast<P*>(chunk.p);
  for (int i = threadIdx.x; i < chunk.n; i += kAdamThreads) {
    if (in != nullptr) {
      s.master[chunk.offset + i] = in[chunk.offset + i];
      param[i] = from_float<P>(in[chunk.offset + i]);
    } else {
      s.master[chunk.offset + i] = to_float(param[i]);
    }
  }
}

}  // namespace ngsgd

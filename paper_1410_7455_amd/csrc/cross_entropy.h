// Cross-entropy of logits and its gradient (gfx950, 64-lane wavefronts).
//   m = max_j x_j;  e_j = exp(x_j - m);  S = sum_{j != y} e_j
//   loss = log(S + e_y) - (x_y - m);  d_j = scale e_j / (S + e_y),  d_y = -scale S / (S + e_y)
// The label's term is kept out of the sum: where it is almost all of it, S is what the loss and the label's gradient are made of.
//
// Exponentials are powers of two of x L - M, L = log2(e) in fp32 and M = m L rounded: one multiply-add, which rounds once, and the hardware's power.  What
// M's rounding adds, r = m L - M, is the same for all of a row, and the quotients do not see it; the loss takes the m that M stands for.  That needs 2^r to be a
// number: half a step of M is at most 64 up to |m| = 2^30 (2^93 for a sum of 2^29 of them), and 2^128 beyond 2^31.  Farther out L = 1: M is m itself, m gives 1,
// and any other number of fp32 lies at least 128 below, where the power and the definition's exponential are both 0 in fp32.  (Beyond 2^27 r is felt at the other
// end: a term that is less than 2^-60 of the row's largest may count as 0.)
//
// Rows of up to 16384 pieces of 16 bytes are held in registers: read once, written once.  Wider ones are read a second time for the gradient.  Few wide
// rows are cut into parts, whose statistics a second kernel joins.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "elements.h"

namespace ngsgd {

struct CrossEntropy {
  const void* logits;
  int64_t ld;
  const void* labels;
  int index_bytes;          // of a label: 4 or 8
  int64_t N;
  int V;
  float* loss;              // optional
  float scale;
  const float* dev_scale;   // optional
  void* dlogits;            // optional
  int64_t ldd;
  struct LossStats* stats;  // [N][parts + 1], of rows in parts; the last one's m is the label's logit
  int parts;
};

__device__ __forceinline__ int64_t label_of(const CrossEntropy& a, const int64_t row) {
  return a.index_bytes == 4 ? static_cast<const int32_t*>(a.labels)[row] : static_cast<const int64_t*>(a.labels)[row];
}

constexpr float kLog2e = 1.44269504088896341f;
constexpr double kLog2eMore = 1.44269504088896341 / (double)kLog2e;   // what one power of L is short of
constexpr float kLowest = -3.4028234663852886e38f;

// S of some columns: the sum of their powers, in units that go with their largest logit.
struct LossStats {
  float m, S;
};
struct PowerBase {
  float m, L, M;
  __device__ __forceinline__ explicit PowerBase(const float m) : m(m) {
    L = far() ? 1.f : kLog2e;
    M = m * L;
  }
  __device__ __forceinline__ bool far() const { return fabsf(m) > 0x1p30f; }
  __device__ __forceinline__ float power(const float x) const { return __builtin_amdgcn_exp2f(fmaf(x, L, -M)); }
  // What a sum in the units of a lower base is in these; the bases may be far apart, and all of the sum sees the error of this.
  __device__ __forceinline__ float share(const PowerBase& other) const {
    if (other.m == m) return 1.f;
    if (far() || other.far()) return 0.f;
    const double t = fmax(((double)other.M - (double)M) * kLog2eMore, -1000.0);
    const float high = (float)t;
    return __builtin_amdgcn_exp2f(high) * fmaf((float)(t - (double)high), 0.693147180559945309f, 1.f);
  }
};

// What a row's statistics make of its loss and gradient.
struct LossRow {
  PowerBase base;
  float f, label_gradient, loss;
  __device__ __forceinline__ LossRow(const CrossEntropy& a, const LossStats& others, const float label) : base(fmaxf(others.m, label)) {
    const float S = others.S * base.share(PowerBase(others.m)), e = base.power(label), total = S + e;
    f = (a.dev_scale != nullptr ? a.scale * *a.dev_scale : a.scale) / total;
    label_gradient = -f * S;
    if (label >= others.m)
      loss = log1pf(S / e);
    else
      loss = (float)((double)logf(total) + ((double)base.M / (double)base.L - (double)label));
  }
};

// A row's columns in pieces of E; the last one is moved back to end with the row, and its first elements, which the piece before has too, do not count.
template <typename T, int E>
struct LossPieces {
  const T* x;
  int V, pieces, label_piece, label_at;
  __device__ __forceinline__ LossPieces(const T* row, const int V, const int label) : x(row), V(V), pieces((V - 1) / E + 1) {
    label_piece = label / E;
    label_at = label - start(label_piece);
  }
  __device__ __forceinline__ int start(const int piece) const { return min(piece * E, V - E); }   // (V is at most 2^30)
  __device__ __forceinline__ int skip(const int piece) const { return piece * E - start(piece); }
  // (offsets in bytes, without a sign and below 2^32, are added to a scalar address as they are)
  __device__ __forceinline__ uint32_t offset(const int at) const { return (uint32_t)at * (uint32_t)sizeof(T); }
  __device__ __forceinline__ Pack<T, E> load(const int piece) const {
    return *reinterpret_cast<const Pack<T, E>*>(reinterpret_cast<const char*>(x) + offset(start(piece)));
  }
  // -infinity in the place of the label and of what does not count
  __device__ __forceinline__ void mask(Pack<T, E>& v, const int piece) const {
    if (piece != label_piece && piece != pieces - 1) return;
#pragma unroll
    for (int j = 0; j < E; ++j)
      if (j < skip(piece) || (piece == label_piece && j == label_at)) v.v[j] = from_float<T>(-INFINITY);
  }
  __device__ __forceinline__ void store(T* d, const Pack<T, E>& v, const int piece, const LossRow& row) const {
    Pack<T, E> out;
#pragma unroll
    for (int j = 0; j < E; ++j) out.v[j] = from_float<T>(row.f * row.base.power(to_float(v.v[j])));
    if (piece != label_piece && piece != pieces - 1) {
      store_pack(reinterpret_cast<T*>(reinterpret_cast<char*>(d) + offset(start(piece))), out);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j)
        if (j >= skip(piece)) d[start(piece) + j] = piece == label_piece && j == label_at ? from_float<T>(row.label_gradient) : out.v[j];
    }
  }
};
// Keeps a piece as it was loaded: the compiler would hold the numbers that it has unpacked from it, twice the registers, for the next time that they are
// used.
template <typename T, int E>
__device__ __forceinline__ void keep_packed(Pack<T, E>& v) {
  if constexpr (sizeof(v) == 16) {
    U32x4 bits = __builtin_bit_cast(U32x4, v);
    asm("" : "+v"(bits));
    v = __builtin_bit_cast(Pack<T, E>, bits);
  }
}
template <typename T, int E>
__device__ __forceinline__ float largest_of(const Pack<T, E>& v) {
  float m = to_float(v.v[0]);
#pragma unroll
  for (int j = 1; j < E; ++j) m = fmaxf(m, to_float(v.v[j]));
  return m;
}

// Over G lanes, or with G > 64 over a workgroup of G threads.
template <int CTRL>
__device__ __forceinline__ float dpp_max_f32(const float v) {
  return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true)));
}
__device__ __forceinline__ float row16_max_f32(float v) {
  v = dpp_max_f32<0xB1>(v);    // quad_perm [1,0,3,2]
  v = dpp_max_f32<0x4E>(v);    // quad_perm [2,3,0,1]
  v = dpp_max_f32<0x141>(v);   // row_half_mirror
  return dpp_max_f32<0x140>(v);   // row_mirror
}
__device__ __forceinline__ float wave_max_f32(float v) {
  v = row16_max_f32(v);
  const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  v = fmaxf(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
template <int G>
__device__ __forceinline__ float group_max(float v, BlockScratch& red) {
  if constexpr (G == 16) {
    return row16_max_f32(v);
  } else if constexpr (G == 64) {
    return wave_max_f32(v);
  } else {
    v = wave_max_f32(v);
    if ((threadIdx.x & 63) == 0) red[0][threadIdx.x >> 6].v[0] = v;
    __syncthreads();
    return row16_max_f32(red[0][min((int)(threadIdx.x & 15), G / 64 - 1)].v[0]);
  }
}
template <int G>
__device__ __forceinline__ float group_sum(const float v, BlockScratch& red) {
  if constexpr (G == 16) return row16_sum_f32(v);
  else if constexpr (G == 64) return wave_sum_f32(v);
  else return block_sum_f32(v, red, 1);
}

template <typename T>
__device__ __forceinline__ void clear_row(T* d, const int V, const int thread, const int threads) {
  constexpr int E = 16 / sizeof(T);
  Pack<T, E> zeros;
#pragma unroll
  for (int j = 0; j < E; ++j) zeros.v[j] = from_float<T>(0.f);
  for (int p = thread; p < V / E; p += threads) store_pack(d + p * E, zeros);
  if (V / E * E + thread < V) d[V / E * E + thread] = from_float<T>(0.f);   // (there are at least E threads)
}

// G threads hold a row, P pieces each; a workgroup has THREADS / G rows.  Bound by memory where two workgroups of a row each are on a compute unit (up to 8
// pieces a thread, 56 registers): 8192 x 32000 bf16 185 us (5.7 TB/s), 8192 x 50257 365 (4.5).  With 16 pieces one is, and nothing loads while it forms
// exponentials: 12288 x 100277 bf16 987 us (4.9), 8192 x 128256 868 (4.8).  (Asking for the next row's pieces as a row's gradient leaves took 128 registers and
// 552 bytes of memory a thread: 2.3 ms.)
template <typename T, int E, int G, int P, int THREADS>
__global__ __launch_bounds__(THREADS, P <= 8 ? 8 : 4) void cross_entropy_kernel(const CrossEntropy a) {
  __shared__ BlockScratch red;
  int row_in_group = threadIdx.x / G;
  if constexpr (G >= 64) row_in_group = __builtin_amdgcn_readfirstlane(row_in_group);   // (so that addresses are a scalar and an offset)
  const int64_t row = (int64_t)blockIdx.x * (THREADS / G) + row_in_group;
  int thread = threadIdx.x % G;
  if (row >= a.N) return;
  const int64_t label = label_of(a, row);
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  T* const d = static_cast<T*>(a.dlogits) + row * a.ldd;
  if (label < 0 || label >= a.V) {
    if (a.loss != nullptr && thread == 0) a.loss[row] = 0.f;
    if (a.dlogits != nullptr) clear_row(d, a.V, thread, G);
    return;
  }
  const LossPieces<T, E> pieces(x, a.V, (int)label);
  Pack<T, E> v[P];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (p * G + thread < pieces.pieces) {
      v[p] = pieces.load(p * G + thread);
    } else {
#pragma unroll
      for (int j = 0; j < E; ++j) v[p].v[j] = from_float<T>(-INFINITY);
    }
  }
  const float own = to_float(x[label]);
  float m = kLowest;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (p * G < pieces.pieces) {   // (uniform)
      pieces.mask(v[p], p * G + thread);
      keep_packed(v[p]);
      m = fmaxf(m, largest_of(v[p]));
      keep_packed(v[p]);
    }
  }
  m = group_max<G>(m, red);
  const PowerBase base(m);
  float S = 0.f;
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (p * G < pieces.pieces) {
#pragma unroll
      for (int j = 0; j < E; ++j) S += base.power(to_float(v[p].v[j]));
      keep_packed(v[p]);
    }
  }
  S = group_sum<G>(S, red);
  const LossRow out(a, LossStats{m, S}, own);
  if (a.loss != nullptr && thread == 0) a.loss[row] = out.loss;
  if (a.dlogits == nullptr) return;
  asm("" : "+v"(thread));   // the offsets are formed anew: kept, they would take a register a piece
#pragma unroll
  for (int p = 0; p < P; ++p)
    if (p * G + thread < pieces.pieces) pieces.store(d, v[p], p * G + thread, out);
}

// ---- rows that are read twice --------------------------------------------------------------------------
constexpr int kWideThreads = 1024, kPartThreads = 256, kStreamAhead = 4;

// Adds K pieces to a thread's statistics: it has its own largest logit, and its sum in units of that.
template <typename T, int E, int K>
__device__ __forceinline__ void add_pieces(LossStats& mine, Pack<T, E> (&v)[K]) {
  float m = mine.m;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    keep_packed(v[k]);
    m = fmaxf(m, largest_of(v[k]));
    keep_packed(v[k]);
  }
  const PowerBase base(m);
  if (m != mine.m) mine = LossStats{m, mine.S * base.share(PowerBase(mine.m))};
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int j = 0; j < E; ++j) mine.S += base.power(to_float(v[k].v[j]));
    keep_packed(v[k]);
  }
}
// Statistics of pieces [from, to) of a thread of a workgroup, and of all of them.
template <typename T, int E, int THREADS>
__device__ __forceinline__ LossStats stream_stats(const LossPieces<T, E>& pieces, const int from, const int to) {
  LossStats mine{kLowest, 0.f};
  for (int p = from + threadIdx.x; p < to; p += THREADS * kStreamAhead) {
    Pack<T, E> v[kStreamAhead];
#pragma unroll
    for (int k = 0; k < kStreamAhead; ++k) v[k] = pieces.load(min(p + k * THREADS, to - 1));
#pragma unroll
    for (int k = 0; k < kStreamAhead; ++k) {
      if (p + k * THREADS >= to) {
#pragma unroll
        for (int j = 0; j < E; ++j) v[k].v[j] = from_float<T>(-INFINITY);
      }
      pieces.mask(v[k], p + k * THREADS);
    }
    add_pieces(mine, v);
  }
  return mine;
}
template <int THREADS>
__device__ __forceinline__ LossStats join_stats(const LossStats& mine, BlockScratch& red) {
  const float m = group_max<THREADS>(mine.m, red);
  return LossStats{m, group_sum<THREADS>(mine.S * PowerBase(m).share(PowerBase(mine.m)), red)};
}
template <typename T, int E, int THREADS>
__device__ __forceinline__ void stream_gradient(const LossPieces<T, E>& pieces, const int from, const int to, T* d, const LossRow& row) {
  for (int p = from + threadIdx.x; p < to; p += THREADS * kStreamAhead) {
    Pack<T, E> v[kStreamAhead];
#pragma unroll
    for (int k = 0; k < kStreamAhead; ++k) v[k] = pieces.load(min(p + k * THREADS, to - 1));
#pragma unroll
    for (int k = 0; k < kStreamAhead; ++k)
      if (p + k * THREADS < to) pieces.store(d, v[k], p + k * THREADS, row);
  }
}

// A workgroup per row, which holds the last kHeld pieces a thread (112 registers; with 16 some are kept in memory) and reads the others twice, the second time
// from a cache.  4096 x 200064 bf16 769 us (4.3 TB/s of what has to be read and written; 845 with none held), 4096 x 100277 fp32 691 (4.8; 873).
constexpr int kHeld = 12, kHeldPieces = kHeld * kWideThreads;
template <typename T>
__global__ __launch_bounds__(kWideThreads) void cross_entropy_wide_kernel(const CrossEntropy a) {
  constexpr int E = 16 / sizeof(T);
  __shared__ BlockScratch red;
  const int64_t row = blockIdx.x, label = label_of(a, row);
  const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
  T* const d = static_cast<T*>(a.dlogits) + row * a.ldd;
  int thread = threadIdx.x;
  if (label < 0 || label >= a.V) {
    if (a.loss != nullptr && thread == 0) a.loss[row] = 0.f;
    if (a.dlogits != nullptr) clear_row(d, a.V, thread, kWideThreads);
    return;
  }
  const LossPieces<T, E> pieces(x, a.V, (int)label);
  const float own = to_float(x[label]);
  const int first = pieces.pieces - kHeldPieces;   // (there are more than that)
  Pack<T, E> v[kHeld];
#pragma unroll
  for (int p = 0; p < kHeld; ++p) v[p] = pieces.load(first + p * kWideThreads + thread);
  LossStats mine = stream_stats<T, E, kWideThreads>(pieces, 0, first);
#pragma unroll
  for (int p = 0; p < kHeld; ++p) pieces.mask(v[p], first + p * kWideThreads + thread);
  add_pieces(mine, v);
  const LossRow out(a, join_stats<kWideThreads>(mine, red), own);
  if (a.loss != nullptr && thread == 0) a.loss[row] = out.loss;
  if (a.dlogits == nullptr) return;
  asm("" : "+v"(thread));
#pragma unroll
  for (int p = 0; p < kHeld; ++p) pieces.store(d, v[p], first + p * kWideThreads + thread, out);
  stream_gradient<T, E, kWideThreads>(pieces, 0, first, d, out);
}

// Few wide rows: a workgroup per part of a row, which leaves its statistics; then one that joins a row's and writes its part of the gradient.  (The label's
// logit comes from the first kernel too: the gradient may be written in its place.)  24 x 128256 bf16 in 31 parts: 5.2 and 4.6 us, most of it latency; by a
// workgroup per row 24.
constexpr int kMostParts = 64;   // a lane for each

template <typename T>
__global__ __launch_bounds__(kPartThreads) void cross_entropy_part_kernel(const CrossEntropy a) {
  constexpr int E = 16 / sizeof(T);
  __shared__ BlockScratch red;
  const int64_t row = blockIdx.x / a.parts, label = label_of(a, row);
  const int part = (int)(blockIdx.x % a.parts);
  if (label < 0 || label >= a.V) return;
  const LossPieces<T, E> pieces(static_cast<const T*>(a.logits) + row * a.ld, a.V, (int)label);
  const int share = (pieces.pieces + a.parts - 1) / a.parts, from = min(part * share, pieces.pieces), to = min(from + share, pieces.pieces);
  LossStats* const stats = a.stats + row * (a.parts + 1);
  const LossStats mine = join_stats<kPartThreads>(stream_stats<T, E, kPartThreads>(pieces, from, to), red);
  if (threadIdx.x != 0) return;
  stats[part] = mine;
  if (part == 0) stats[a.parts].m = to_float(pieces.x[label]);
}

template <typename T>
__global__ __launch_bounds__(kPartThreads) void cross_entropy_join_kernel(const CrossEntropy a) {
  constexpr int E = 16 / sizeof(T);
  const int64_t row = blockIdx.x / a.parts, label = label_of(a, row);
  const int part = (int)(blockIdx.x % a.parts), lane = threadIdx.x & 63;
  const bool counts = label >= 0 && label < a.V;
  const LossPieces<T, E> pieces(static_cast<const T*>(a.logits) + row * a.ld, a.V, counts ? (int)label : 0);
  const int share = (pieces.pieces + a.parts - 1) / a.parts, from = min(part * share, pieces.pieces), to = min(from + share, pieces.pieces);
  T* const d = static_cast<T*>(a.dlogits) + row * a.ldd;
  if (!counts) {
    if (part == 0 && threadIdx.x == 0 && a.loss != nullptr) a.loss[row] = 0.f;
    if (a.dlogits != nullptr && from < to) clear_row(d + pieces.start(from), (to == pieces.pieces ? a.V : to * E) - pieces.start(from), threadIdx.x, kPartThreads);
    return;
  }
  const LossStats* const stats = a.stats + row * (a.parts + 1);
  const LossStats mine = lane < a.parts ? stats[lane] : LossStats{kLowest, 0.f};
  const float m = wave_max_f32(mine.m);
  const LossRow out(a, LossStats{m, wave_sum_f32(mine.S * PowerBase(m).share(PowerBase(mine.m)))}, stats[a.parts].m);
  if (part == 0 && threadIdx.x == 0 && a.loss != nullptr) a.loss[row] = out.loss;
  if (a.dlogits != nullptr) stream_gradient<T, E, kPartThreads>(pieces, from, to, d, out);
}

}  // namespace ngsgd

// Layer norm and its gradients (gfx950, 64-lane wavefronts).
//   forward:   y = xhat w + b,  xhat = (x - mean) rstd,  mean = sum x / D,  rstd = (sum (x - mean)^2 / D + eps)^(-1/2)
//   backward:  g = dy w,  dx = rstd (g - sum g / D - xhat sum(g xhat) / D),  dw = sum over rows dy xhat,  db = sum over rows dy
// Statistics, sums and gradients are held in fp32.  The differences to the mean give the variance and, summed themselves where the mean is far from
// zero, what it is off by, which is taken off them: it costs no digits, and equal numbers give the bias (3000.1 1000 times: else 0.15 off).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "elements.h"
#include "layer_norm_args.h"

namespace ngsgd {

// ---- rows that a group of threads holds in registers ------------------------------------------------
// TPR threads share a row, a part of a wavefront (16, 32 or 64) or the whole workgroup (0), which then has as many
// wavefronts as the width asks for.  A thread holds E columns, as pieces of 16 bytes; the workgroup walks over the rows.  Its columns of
// the weight, the bias and (backward) of the sums over the rows stay in registers, and rows to come are requested before the one
// that is there is worked on: SLOTS rows are in flight or in hand.  Rows shorter than 16 bytes have pieces of an element.
template <int VEC_, int E_, int TPR_, int MAX_THREADS, int SLOTS_>
struct RowShape {
  static constexpr int VEC = VEC_, E = E_, K = E / VEC, TPR = TPR_, NT = MAX_THREADS, SLOTS = SLOTS_;
  static constexpr int ROWS = TPR == 0 ? 1 : NT / TPR;   // rows that a workgroup works on side by side
  static_assert(E % VEC == 0 && NT % 64 == 0 && NT <= 64 * kMaxWaves, "whole pieces, whole wavefronts");
  __device__ static int threads() { return TPR == 0 ? (int)blockDim.x : TPR; }
  __device__ static int member() { return TPR == 0 ? (int)threadIdx.x : (int)threadIdx.x % TPR; }
  __device__ static int row() { return TPR == 0 ? 0 : (int)threadIdx.x / TPR; }
  __device__ static int column(const int k) { return (k * threads() + member()) * VEC; }
};

// Where a thread's pieces lie.  A row's last piece is moved back to end at column D, so that it is loaded and stored whole like the others: its
// first columns are the end of the piece before it, which count there (loading it by elements, and waiting for them in one wavefront
// and so at the barrier in all, took 90 us for 8192 x 5000 bf16 backward where 8192 x 5120 took 51).  D >= VEC.
template <typename S>
struct RowColumns {
  int D, at[S::K];
  __device__ __forceinline__ explicit RowColumns(const int D_) : D(D_) {
#pragma unroll
    for (int k = 0; k < S::K; ++k) at[k] = min(S::column(k), D - S::VEC);
  }
  __device__ __forceinline__ bool here(const int k) const { return S::column(k) < D; }
  // element e of the thread counts: it is a column of the row, and of no other piece
  __device__ __forceinline__ bool counts(const int e) const {
    const int k = e / S::VEC, c = at[k] + e % S::VEC;
    return c >= S::column(k) && c < D;
  }
};

// A thread's columns of a row as they lie in memory (two 16-bit elements to a register).
template <typename S, typename T>
struct RowPart {
  static constexpr int PER = S::VEC > 1 ? 4 / sizeof(T) : 1, WORDS = S::VEC / PER;   // elements of a register, registers of a piece
  struct __attribute__((packed, aligned(sizeof(T)))) Words {
    uint32_t v[WORDS];
  };
  uint32_t v[S::E / PER];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < S::E / PER; ++i) v[i] = 0u;
  }
  // Keeps what is formed from these registers in a loop from being formed before it, in registers of its own.
  __device__ __forceinline__ void stay() {
#pragma unroll
    for (int i = 0; i < S::E / PER; ++i) asm("" : "+v"(v[i]));
  }
  // What is behind the row's end keeps its value (what else writes to v waits for the load).
  __device__ __forceinline__ void load(const T* p, const RowColumns<S>& cols) {
#pragma unroll
    for (int k = 0; k < S::K; ++k) {
      if (!cols.here(k)) continue;
      if constexpr (S::VEC * sizeof(T) < 4) {
        v[k] = __builtin_bit_cast(uint16_t, p[cols.at[k]]);
      } else {
        const Words q = *reinterpret_cast<const Words*>(p + cols.at[k]);
#pragma unroll
        for (int j = 0; j < WORDS; ++j) v[k * WORDS + j] = q.v[j];
      }
    }
  }
  __device__ __forceinline__ float get(const int e) const {
    if constexpr (sizeof(T) == 2)
      return to_float(__builtin_bit_cast(T, (uint16_t)(PER == 2 && e & 1 ? v[e / PER] >> 16 : v[e / PER])));
    else
      return __builtin_bit_cast(float, v[e]);
  }
};
// Both pieces that hold a column write the same number to it; with ONCE only the one where it counts.
template <typename S, bool ONCE, typename T>
__device__ __forceinline__ void store_row(const float (&v)[S::E], T* p, const RowColumns<S>& cols) {
#pragma unroll
  for (int k = 0; k < S::K; ++k) {
    if (!cols.here(k)) continue;
    if (!ONCE || cols.at[k] == S::column(k)) {
      Pack<T, S::VEC> o;
#pragma unroll
      for (int j = 0; j < S::VEC; ++j) o.v[j] = from_float<T>(v[k * S::VEC + j]);
      *reinterpret_cast<Pack<T, S::VEC>*>(p + cols.at[k]) = o;
    } else {
#pragma unroll
      for (int j = 0; j < S::VEC; ++j)
        if (cols.counts(k * S::VEC + j)) p[cols.at[k] + j] = from_float<T>(v[k * S::VEC + j]);
    }
  }
}

// Sums over the threads of a row.
template <typename S>
__device__ __forceinline__ void row_sum_pair(float& a, float& b, BlockScratch& red, const int parity) {
  if constexpr (S::TPR == 0) {
    block_sum_pair_f32(a, b, red, parity);
  } else {
    a = row16_sum_f32(a);
    b = row16_sum_f32(b);
    if constexpr (S::TPR >= 32) {
      a = half16_add_f32(a);
      b = half16_add_f32(b);
    }
    if constexpr (S::TPR == 64) {
      a = half32_add_f32(a);
      b = half32_add_f32(b);
    }
  }
}
template <typename S>
__device__ __forceinline__ float row_sum(float v, BlockScratch& red, const int parity) {
  float none = 0.f;
  row_sum_pair<S>(v, none, red, parity);
  return v;
}

// A mean so many deviations from zero is off by enough of its last bits to show in xhat: such rows take one more sum, of their differences to it, by which
// it is set right: 8192 x 5000 bf16 38 us if all rows are such, else 32.  (To ask costs up to 2 %, the sum in all rows up to 18 %.)
__device__ __forceinline__ bool far_from_zero(const float mean, const float var, const float eps) { return mean * mean > 256.f * (var + eps); }
// The variance about mean + shift, from that about mean.  (NaN stays.)
__device__ __forceinline__ float variance_about(const float var, const float shift) {
  const float v = fmaf(-shift, shift, var);
  return v < 0.f ? 0.f : v;
}

// Bound by memory.
template <typename T, typename W, typename S>
__global__ __launch_bounds__(S::NT) void layernorm_forward_kernel(const LayerNormForward a) {
  __shared__ BlockScratch red;
  constexpr int E = S::E;
  const RowColumns<S> cols(a.D);
  RowPart<S, W> w, b;
  w.clear();
  b.clear();
  if (a.w != nullptr) w.load(static_cast<const W*>(a.w), cols);
  if (a.b != nullptr) b.load(static_cast<const W*>(a.b), cols);
  const int64_t step = (int64_t)gridDim.x * S::ROWS;
  int64_t row = (int64_t)blockIdx.x * S::ROWS + S::row();
  RowPart<S, T> next;
  next.clear();
  if (row < a.N) next.load(static_cast<const T*>(a.x) + row * a.ldx, cols);
  for (int64_t first = (int64_t)blockIdx.x * S::ROWS; first < a.N; first += step, row += step) {   // (uniform in the workgroup)
    float x[E];
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] = next.get(e);
      s += cols.counts(e) ? x[e] : 0.f;
    }
    if (row + step < a.N) next.load(static_cast<const T*>(a.x) + (row + step) * a.ldx, cols);
    float mean = row_sum<S>(s, red, 0) / (float)a.D;
    float q = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] -= mean;
      q += cols.counts(e) ? x[e] * x[e] : 0.f;
    }
    float var = row_sum<S>(q, red, 1) / (float)a.D;
    const bool far = far_from_zero(mean, var, a.eps);
    if (any_lane(far)) {   // (all threads of a row have the same bits: uniform in the workgroup where it shares a row)
      float d = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) d += cols.counts(e) ? x[e] : 0.f;
      const float sum = row_sum<S>(d, red, 0), shift = far ? sum / (float)a.D : 0.f;   // (a row's result is its own, whoever shares the wavefront)
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] -= shift;
      mean += shift;
      var = variance_about(var, shift);
      if constexpr (S::TPR == 0) __syncthreads();   // the next row's first sum takes the same half of `red`
    }
    const float rstd = 1.f / sqrtf(var + a.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      x[e] *= rstd;
      if (a.w != nullptr) x[e] *= w.get(e);
      if (a.b != nullptr) x[e] += b.get(e);
    }
    if (row < a.N) {
      T* const y = static_cast<T*>(a.y) + row * a.ldy;
      store_row<S, false>(x, y, cols);
      for (int c = a.D + S::member(); c < a.pad_to; c += S::threads()) y[c] = from_float<T>(c == a.D ? 1.f : 0.f);
      if (S::member() == 0) {
        if (a.mean != nullptr) a.mean[row] = mean;
        if (a.rstd != nullptr) a.rstd[row] = rstd;
      }
    }
  }
}

// What a thread needs of a row; zeros behind the last one.
template <typename S, typename T, bool SLABS>
struct BackwardRow {
  RowPart<S, T> x, dy;
  float mean, rstd;
  __device__ __forceinline__ float xhat(const int e) const { return (x.get(e) - mean) * rstd; }
  __device__ __forceinline__ void load(const LayerNormBackward& a, const RowColumns<S>& cols, const int64_t r) {
    float m = 0.f, s = 0.f;
    if (r < a.N) {
      const T* const p = static_cast<const T*>(a.dy) + r * a.lddy;
      x.load(static_cast<const T*>(a.x) + r * a.ldx, cols);
      dy.load(p, cols);
      // (fp32) In a fixed order.  The sum waits for the slabs' loads here, before the row in hand is worked on: rows behind split products are not
      // in flight beside it, as others are.
      if constexpr (SLABS) {
        for (int k = 1; k < a.n_slabs; ++k) {
          RowPart<S, T> more;
          more.clear();
          more.load(p + k * a.slab_stride, cols);
#pragma unroll
          for (int e = 0; e < S::E; ++e) dy.v[e] = __builtin_bit_cast(uint32_t, dy.get(e) + more.get(e));
        }
      }
      m = a.mean[r];
      s = a.rstd[r];
    } else {
      x.clear();
      dy.clear();
    }
    mean = m;   // (assigned in the branches, one in another order than the other, the structure ends up in memory)
    rstd = s;
  }
};

// Sums over the rows that a workgroup worked on side by side, in order, to `to_w` and `to_b` (nullptr: not asked for).
template <typename S, typename T, int LDS>
__device__ __forceinline__ void store_sums(const float (&dw)[S::E], const float (&db)[S::E], T* to_w, T* to_b, float (&sums)[LDS],
                                           const RowColumns<S>& cols) {
  constexpr int E = S::E;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    T* const to = which == 0 ? to_w : to_b;
    if (to == nullptr) continue;   // (uniform)
    if constexpr (S::ROWS == 1) {
      store_row<S, true>(which == 0 ? dw : db, to, cols);
    } else {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) sums[threadIdx.x * E + e] = which == 0 ? dw[e] : db[e];
      __syncthreads();
      if (S::row() != 0) continue;
      float v[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[e] = 0.f;
#pragma unroll
        for (int r = 0; r < S::ROWS; ++r) v[e] += sums[(r * S::threads() + S::member()) * E + e];
      }
      store_row<S, true>(v, to, cols);
    }
  }
}

// Sums of a workgroup's rows go to part[workgroup][dw, db][D].  Bound by memory, as long as enough rows are in flight: 16384 x 8192 bf16 takes
// 168 us with one row to come and 151 with two (5.3 TB/s, the rate of a large copy); the gradient is formed from x and dy again behind the
// row's sums, so that registers hold rows to come instead of xhat and g.
template <typename T, typename W, typename S, bool SLABS>
__global__ __launch_bounds__(S::NT) void layernorm_backward_kernel(const LayerNormBackward a) {
  __shared__ BlockScratch red;
  __shared__ float sums[S::ROWS > 1 ? S::NT * S::E : 1];
  constexpr int E = S::E, SLOTS = S::SLOTS;
  // The widest rows in 16 bits just fit in a workgroup of 1024's 128 registers (8192 x 16384 bf16: 162 us; 235 with 17 of them in
  // memory).  In fp32 they do not, and it is the better for what is formed once (16384 x 16384: 746 us, else 865).
  constexpr bool TIGHT = SLOTS == 1 && sizeof(T) == 2;
  const RowColumns<S> cols(a.D);
  RowPart<S, W> w;
  w.clear();
  if (a.w != nullptr) w.load(static_cast<const W*>(a.w), cols);
  float dw[E], db[E];
#pragma unroll
  for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.f;
  const int64_t step = (int64_t)gridDim.x * S::ROWS;
  int64_t row = (int64_t)blockIdx.x * S::ROWS + S::row();
  BackwardRow<S, T, SLABS> rows[SLOTS];
#pragma unroll
  for (int k = 0; k < SLOTS; ++k) {
    rows[k].x.clear();
    rows[k].dy.clear();
    rows[k].load(a, cols, row + k * step);
  }
  int parity = 0;
  for (int64_t first = (int64_t)blockIdx.x * S::ROWS; first < a.N; first += SLOTS * step) {
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      if (first + k * step < a.N) {   // (uniform in the workgroup)
        BackwardRow<S, T, SLABS>& r = rows[k];
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float xhat = r.xhat(e), dy = cols.counts(e) ? r.dy.get(e) : 0.f, g = a.w != nullptr ? dy * w.get(e) : dy;
          dw[e] += dy * xhat;
          db[e] += dy;
          c1 += g;
          c2 += g * xhat;
        }
        if (a.dx != nullptr) {
          row_sum_pair<S>(c1, c2, red, parity);
          c1 /= (float)a.D;
          c2 /= (float)a.D;
          if constexpr (TIGHT) {   // nothing formed above is kept
            r.x.stay();
            r.dy.stay();
            w.stay();
          }
          float dx[E];
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float dy = r.dy.get(e), g = a.w != nullptr ? dy * w.get(e) : dy;
            dx[e] = r.rstd * (g - c1 - r.xhat(e) * c2);
          }
          if (row < a.N) store_row<S, false>(dx, static_cast<T*>(a.dx) + row * a.lddx, cols);
        }
        rows[k].load(a, cols, row + SLOTS * step);
        parity ^= 1;
        row += step;
      }
    }
  }
  if (a.part == nullptr) return;
  if (a.groups == 1) {   // these are the sums
    store_sums<S>(dw, db, static_cast<W*>(a.dw), static_cast<W*>(a.db), sums, cols);
  } else {
    float* const part = a.part + (size_t)blockIdx.x * 2 * a.D;
    store_sums<S>(dw, db, part, part + a.D, sums, cols);
  }
}

// ---- rows of any width, read from memory in every pass -------------------------------------------------
// Bound by the passes' latencies: with the pieces in flight a thread takes 78 to 121 registers, so that one workgroup is on a compute unit and its waits
// are not covered by another's work.  4096 x 20000 bf16 forward 143 us (2.3 TB/s), backward 267 us.
constexpr int kWideThreads = 1024;

// f(piece, its place, how many of its columns belong to the piece before) for a thread's pieces of a row, after `load` of AHEAD of them, which are
// requested together: no condition stands between the loads, the last piece is moved back to end with the row (D >= V).
template <typename PIECE, int V, typename LOAD, typename F>
__device__ __forceinline__ void for_pieces(const int D, LOAD load, F f) {
  constexpr int AHEAD = 4, STEP = kWideThreads * V;
  for (int c = (int)threadIdx.x * V; c < D; c += AHEAD * STEP) {
    PIECE piece[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(piece[u], min(c + u * STEP, D - V));
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int at = min(c + u * STEP, D - V);
      if (c + u * STEP < D) f(piece[u], at, c + u * STEP - at);
    }
  }
}
template <typename T, int V>
__device__ __forceinline__ void load_piece(Pack<T, V>& out, const T* p) { out = *reinterpret_cast<const Pack<T, V>*>(p); }
// Without the columns of the piece before, which its own thread writes (and may have read from the same place).
template <typename T, int V>
__device__ __forceinline__ void store_piece(const float (&v)[V], T* p, const int skip) {
  if (skip == 0) {
    Pack<T, V> q;
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = from_float<T>(v[j]);
    *reinterpret_cast<Pack<T, V>*>(p) = q;
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (j >= skip) p[j] = from_float<T>(v[j]);
  }
}

template <typename T, typename W>
__global__ __launch_bounds__(kWideThreads) void layernorm_forward_wide_kernel(const LayerNormForward a) {
  __shared__ BlockScratch red;
  constexpr int V = 16 / sizeof(T);
  const W* const w = static_cast<const W*>(a.w);
  const W* const b = static_cast<const W*>(a.b);
  struct Affine {
    Pack<T, V> x;
    Pack<W, V> w, b;
  };
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    T* const y = static_cast<T*>(a.y) + row * a.ldy;
    auto load_x = [&](Pack<T, V>& q, const int at) { load_piece(q, x + at); };
    float s = 0.f;
    for_pieces<Pack<T, V>, V>(a.D, load_x, [&](const Pack<T, V>& q, int, const int skip) {
#pragma unroll
      for (int j = 0; j < V; ++j) s += j >= skip ? to_float(q.v[j]) : 0.f;
    });
    const float mean = block_sum_f32(s, red, 0) / (float)a.D;
    float sq = 0.f;
    for_pieces<Pack<T, V>, V>(a.D, load_x, [&](const Pack<T, V>& q, int, const int skip) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = to_float(q.v[j]) - mean;
        sq += j >= skip ? d * d : 0.f;
      }
    });
    float var = block_sum_f32(sq, red, 1) / (float)a.D, shift = 0.f;
    if (any_lane(far_from_zero(mean, var, a.eps))) {   // (uniform in the workgroup)
      float sum = 0.f;
      for_pieces<Pack<T, V>, V>(a.D, load_x, [&](const Pack<T, V>& q, int, const int skip) {
#pragma unroll
        for (int j = 0; j < V; ++j) sum += j >= skip ? to_float(q.v[j]) - mean : 0.f;
      });
      shift = block_sum_f32(sum, red, 0) / (float)a.D;
      var = variance_about(var, shift);
      __syncthreads();   // the next row's first sum takes the same half of `red`
    }
    const float rstd = 1.f / sqrtf(var + a.eps);
    for_pieces<Affine, V>(
        a.D,
        [&](Affine& q, const int at) {
          load_piece(q.x, x + at);
          if (w != nullptr) load_piece(q.w, w + at);
          if (b != nullptr) load_piece(q.b, b + at);
        },
        [&](const Affine& q, const int at, const int skip) {
          float v[V];
#pragma unroll
          for (int j = 0; j < V; ++j) {
            v[j] = (to_float(q.x.v[j]) - mean - shift) * rstd;
            if (w != nullptr) v[j] *= to_float(q.w.v[j]);
            if (b != nullptr) v[j] += to_float(q.b.v[j]);
          }
          store_piece(v, y + at, skip);
        });
    for (int c = a.D + (int)threadIdx.x; c < a.pad_to; c += kWideThreads) y[c] = from_float<T>(c == a.D ? 1.f : 0.f);
    if (threadIdx.x == 0) {
      if (a.mean != nullptr) a.mean[row] = mean + shift;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
  }
}

template <typename T, typename W>
__global__ __launch_bounds__(kWideThreads) void layernorm_backward_rows_kernel(const LayerNormBackward a) {
  __shared__ BlockScratch red;
  constexpr int V = 16 / sizeof(T);
  const W* const w = static_cast<const W*>(a.w);
  struct Derivative {
    Pack<T, V> x, dy;
    Pack<W, V> w;
  };
  int parity = 0;
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x, parity ^= 1) {
    const T* const x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* const dy = static_cast<const T*>(a.dy) + row * a.lddy;
    T* const dx = static_cast<T*>(a.dx) + row * a.lddx;
    const float mean = a.mean[row], rstd = a.rstd[row];
    auto load = [&](Derivative& q, const int at) {
      load_piece(q.x, x + at);
      load_piece(q.dy, dy + at);
      if (w != nullptr) load_piece(q.w, w + at);
    };
    auto xhat_of = [&](const Derivative& q, const int j) { return (to_float(q.x.v[j]) - mean) * rstd; };
    auto g_of = [&](const Derivative& q, const int j) { return w != nullptr ? to_float(q.dy.v[j]) * to_float(q.w.v[j]) : to_float(q.dy.v[j]); };
    float c1 = 0.f, c2 = 0.f;
    for_pieces<Derivative, V>(a.D, load, [&](const Derivative& q, int, const int skip) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float g = j >= skip ? g_of(q, j) : 0.f;
        c1 += g;
        c2 += g * xhat_of(q, j);
      }
    });
    block_sum_pair_f32(c1, c2, red, parity);
    c1 /= (float)a.D;
    c2 /= (float)a.D;
    for_pieces<Derivative, V>(a.D, load, [&](const Derivative& q, const int at, const int skip) {
      float v[V];
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = rstd * (g_of(q, j) - c1 - xhat_of(q, j) * c2);
      store_piece(v, dx + at, skip);
    });
  }
}

// Sums over the rows of a group: grid (columns / 256, groups), a thread per column, four rows requested together.
constexpr int kColumnThreads = 256;
template <typename T>
__global__ __launch_bounds__(kColumnThreads) void layernorm_backward_columns_kernel(const LayerNormBackward a) {
  const int64_t c = (int64_t)blockIdx.x * kColumnThreads + threadIdx.x;
  if (c >= a.D) return;
  const int64_t first = a.N * blockIdx.y / a.groups, end = a.N * (blockIdx.y + 1) / a.groups;
  constexpr int AHEAD = 4;
  float dw = 0.f, db = 0.f;
  for (int64_t row = first; row < end; row += AHEAD) {
    float x[AHEAD], dy[AHEAD], mean[AHEAD], rstd[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int64_t r = min(row + u, end - 1);
      dy[u] = to_float(static_cast<const T*>(a.dy)[r * a.lddy + c]);
      x[u] = to_float(static_cast<const T*>(a.x)[r * a.ldx + c]);
      mean[u] = a.mean[r];
      rstd[u] = a.rstd[r];
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (row + u < end) {
        dw += dy[u] * ((x[u] - mean[u]) * rstd[u]);
        db += dy[u];
      }
    }
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

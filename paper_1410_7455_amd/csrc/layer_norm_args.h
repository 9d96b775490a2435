// Arguments of the layer-norm kernels.
#pragma once

#include <stdint.h>

namespace ngsgd {

constexpr int kRegisterColumns = 16384;   // wider rows are read from memory in every pass

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
  int pad_to;        // above D: y[D] = 1 and zeros up to this column (the bias input of a layer behind)
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
  float* part;       // [groups][2][D] sums over a group of rows; nullptr: none
  int groups;
  int n_slabs;       // dy is the sum of so many matrices (partial products), slab_stride elements apart; 1 above kRegisterColumns
  int64_t slab_stride;
};

}  // namespace ngsgd

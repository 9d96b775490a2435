// C ABI of layer norm: argument checks and launches.  Declarations and contracts are in include/ngsgd.h.
#include "layer_norm.h"

#include <algorithm>
#include <cmath>

#include "host.h"
#include "operators.h"

using namespace ngsgd;

namespace {

constexpr int kMostColumns = 1 << 25;   // (a launch has less than 2^32 threads)
// Rows wider than registers hold: workgroups that walk over them; groups of rows, with at most so many columns of sums in all where
// there are more than eight of them.
constexpr int kWideGrid = 2048, kWideGroups = 512, kWideSums = 1 << 23;

inline int64_t parts(const int64_t N, const int size) { return N / size + (N % size != 0); }   // (any N: N + size - 1 may not fit)

// The threads of a row by its width: as few wavefronts, or parts of one, as hold it with 8 columns a thread; 16 where that keeps it within a
// wavefront (no barriers) and where a workgroup cannot be larger, and for the forward pass, which has registers to spare, in wide rows
// (32768 x 8192 bf16 forward: 209 us, with 8 columns 285; 8192 x 5000 backward with 16 columns 71 us instead of 54).
struct RowPlan {
  int tpr, e, nt;   // tpr: 16, 32, 64 threads or (0) the workgroup; e 0: from memory
  int rows() const { return tpr == 0 ? 1 : nt / tpr; }
};
RowPlan row_plan(const int D, const bool backward) {
  if (D < 8) return {16, 1, 256};
  if (D <= 128) return {16, 8, 256};
  if (D <= 256) return {32, 8, 256};
  if (D <= 512) return {64, 8, 256};
  if (D <= 1024) return {64, 16, 256};
  if (D > kRegisterColumns) return {0, 0, kWideThreads};
  const int e = D <= (backward ? 8192 : 2048) ? 8 : 16;
  return {0, e, (D + 64 * e - 1) / (64 * e) * 64};
}
// Groups of rows whose sums are formed on their own: the workgroups of the backward pass, about ten wavefronts to a compute unit.  (Their
// sums are written and read once more: with 16 wavefronts to a unit 32768 x 4096 bf16 takes 165 us instead of 150, 16384 x 1024 29 instead of 25.)
int backward_grid(const int64_t N, const RowPlan& p) {
  return (int)std::min<int64_t>(256 * std::max(1, 640 / p.nt), std::max<int64_t>(1, parts(N, p.rows())));
}
int norm_groups(const int64_t N, const int D) {
  const RowPlan p = row_plan(D, true);
  if (p.e == 0) return (int)std::min<int64_t>({kWideGroups, std::max(8, kWideSums / D), std::max<int64_t>(1, parts(N, 8))});
  // Few rows: one workgroup takes them and has the sums, without a second launch.  Four rounds are no slower than it: 64 x 128 fp32 5.6 us
  // instead of 6.1, 16 x 512 bf16 4.6 instead of 5.4, 4 x 4096 5.8 instead of 5.9 (eight rounds: 8 x 4096 8.9 instead of 6.0), and the host
  // saves 3 of 14 us.  With one row in hand at a time only one is: 4 x 16384 29 instead of 16.
  if (N <= (p.e == 16 && p.tpr == 0 ? 1 : 4) * p.rows()) return 1;
  return backward_grid(N, p);
}
unsigned forward_grid(const int64_t N, const RowPlan& p) {
  return (unsigned)std::min<int64_t>(256 * std::max(1, 1536 / p.nt), parts(N, p.rows()));
}

// f(shape) for rows of this width
template <typename T, typename F>
void with_row_shape(const RowPlan& p, F f) {
  constexpr int VEC = 16 / sizeof(T);
  if (p.e == 1) return f(RowShape<1, 1, 16, 256, 2>());
  if (p.tpr == 16) return f(RowShape<VEC, 8, 16, 256, 2>());
  if (p.tpr == 32) return f(RowShape<VEC, 8, 32, 256, 2>());
  if (p.tpr == 64 && p.e == 8) return f(RowShape<VEC, 8, 64, 256, 2>());
  if (p.tpr == 64) return f(RowShape<VEC, 16, 64, 256, 2>());
  if (p.e == 8) return f(RowShape<VEC, 8, 0, 1024, 3>());
  f(RowShape<VEC, 16, 0, 1024, 1>());   // (two rows would not fit in the 128 registers of a workgroup of 1024)
}

// All arguments have been checked.  SLABS: dy is in partial products.
template <typename T, typename W, bool SLABS>
int launch_backward(const LayerNormBackward& a, hipStream_t s) {
  const RowPlan plan = row_plan(a.D, true);
  const int64_t columns = ((int64_t)a.D + kColumnThreads - 1) / kColumnThreads;
  if (a.N > 0 && plan.e != 0) {
    with_row_shape<T>(plan, [&](auto shape) {
      hipLaunchKernelGGL((layernorm_backward_kernel<T, W, decltype(shape), SLABS>), dim3(a.part != nullptr ? a.groups : backward_grid(a.N, plan)),
                         dim3(plan.nt), 0, s, a);
    });
    LAUNCH_CHECK();
  } else if (SLABS) {
    return NGSGD_EINVAL;
  } else if (a.N > 0) {
    if (a.part != nullptr) {   // the sums first: the gradient may overwrite dy
      hipLaunchKernelGGL(layernorm_backward_columns_kernel<T>, dim3((unsigned)columns, a.groups), dim3(kColumnThreads), 0, s, a);
      LAUNCH_CHECK();
    }
    if (a.dx != nullptr) {
      hipLaunchKernelGGL((layernorm_backward_rows_kernel<T, W>), dim3((unsigned)std::min<int64_t>(a.N, kWideGrid)), dim3(kWideThreads), 0, s, a);
      LAUNCH_CHECK();
    }
  }
  if (a.part != nullptr && (plan.e == 0 || a.groups != 1)) {
    hipLaunchKernelGGL(layernorm_backward_sum_kernel<W>, dim3((unsigned)((2 * (int64_t)a.D + kSumColumns - 1) / kSumColumns)), dim3(kSumThreads),
                       0, s, a);
    LAUNCH_CHECK();
  }
  return NGSGD_OK;
}
template <typename T, typename W>
int launch_forward(const LayerNormForward& a, hipStream_t s) {
  const RowPlan plan = row_plan(a.D, false);
  if (plan.e == 0) {
    hipLaunchKernelGGL((layernorm_forward_wide_kernel<T, W>), dim3((unsigned)std::min<int64_t>(a.N, kWideGrid)), dim3(kWideThreads), 0, s, a);
  } else {
    with_row_shape<T>(plan, [&](auto shape) {
      hipLaunchKernelGGL((layernorm_forward_kernel<T, W, decltype(shape)>), dim3(forward_grid(a.N, plan)), dim3(plan.nt), 0, s, a);
    });
  }
  LAUNCH_CHECK();
  return NGSGD_OK;
}

// f(element, weight element) for the types of a call
template <typename F>
int with_types(const int type, const int weight_type, F f) {
  if (type == NGSGD_FLOAT32) return f(float(), float());
  if (type == NGSGD_BFLOAT16) return weight_type == NGSGD_FLOAT32 ? f(bf16(), float()) : f(bf16(), bf16());
  return weight_type == NGSGD_FLOAT32 ? f(fp16(), float()) : f(fp16(), fp16());
}

int check_types(const int type, const int weight_type, const int64_t N, const int32_t D) {
  if (!known_type(type) || !known_type(weight_type) || (weight_type != type && weight_type != NGSGD_FLOAT32)) return NGSGD_EINVAL;
  return N < 0 || D < 1 || D > kMostColumns ? NGSGD_EINVAL : NGSGD_OK;
}

}  // namespace

namespace ngsgd {

int layernorm_forward_f32(const LayerNormForward& a, hipStream_t s) { return launch_forward<float, float>(a, s); }

int layernorm_backward_f32(LayerNormBackward a, hipStream_t s) {
  a.groups = norm_groups(a.N, a.D);
  return a.n_slabs > 1 ? launch_backward<float, float, true>(a, s) : launch_backward<float, float, false>(a, s);
}

size_t layernorm_part_floats(const int64_t max_rows, const int D) { return (size_t)norm_groups(max_rows, D) * 2 * D; }

}  // namespace ngsgd

extern "C" int ngsgd_layernorm_forward(const void* dev_x, int64_t ldx, int32_t type, const void* dev_weight, const void* dev_bias,
                                       int32_t weight_type, int64_t N, int32_t D, float epsilon, void* dev_y, int64_t ldy, float* dev_mean,
                                       float* dev_rstd, void* hip_stream) {
  NG_TRY(check_types(type, weight_type, N, D));
  if (!(epsilon >= 0.f) || !std::isfinite(epsilon)) return NGSGD_EINVAL;
  if (!good_matrix(dev_x, ldx, type, N, D) || !good_matrix(dev_y, ldy, type, N, D)) return NGSGD_EINVAL;
  if (!on_element(dev_weight, weight_type) || !on_element(dev_bias, weight_type)) return NGSGD_EINVAL;
  if (!on_element(dev_mean, NGSGD_FLOAT32) || !on_element(dev_rstd, NGSGD_FLOAT32)) return NGSGD_EINVAL;
  if (N == 0) return NGSGD_OK;
  const LayerNormForward a{dev_x, ldx, dev_weight, dev_bias, dev_y, ldy, dev_mean, dev_rstd, N, D, epsilon, 0};
  return with_types(type, weight_type, [&](auto t, auto w) { return launch_forward<decltype(t), decltype(w)>(a, static_cast<hipStream_t>(hip_stream)); });
}

extern "C" int ngsgd_layernorm_workspace_bytes(int64_t max_rows, int32_t D, size_t* out_bytes) {
  if (out_bytes == nullptr || max_rows < 0 || D < 1 || D > kMostColumns) return NGSGD_EINVAL;
  Carver c(nullptr);
  (void)c.take<float>(layernorm_part_floats(max_rows, D));
  *out_bytes = align_up(c.off, 256);
  return NGSGD_OK;
}

extern "C" int ngsgd_layernorm_backward(const void* dev_dy, int64_t lddy, const void* dev_x, int64_t ldx, int32_t type, const void* dev_weight,
                                        int32_t weight_type, const float* dev_mean, const float* dev_rstd, int64_t N, int32_t D, void* dev_dx,
                                        int64_t lddx, void* dev_dweight, void* dev_dbias, void* dev_workspace, size_t workspace_bytes,
                                        void* hip_stream) {
  NG_TRY(check_types(type, weight_type, N, D));
  const bool sums = dev_dweight != nullptr || dev_dbias != nullptr;
  if (!good_matrix(dev_dy, lddy, type, N, D) || !good_matrix(dev_x, ldx, type, N, D)) return NGSGD_EINVAL;
  if (dev_dx != nullptr && !good_matrix(dev_dx, lddx, type, N, D)) return NGSGD_EINVAL;
  if (dev_dx == nullptr && !sums) return NGSGD_EINVAL;
  if (N > 0 && (dev_mean == nullptr || dev_rstd == nullptr)) return NGSGD_EINVAL;
  if (!on_element(dev_mean, NGSGD_FLOAT32) || !on_element(dev_rstd, NGSGD_FLOAT32)) return NGSGD_EINVAL;
  if (!on_element(dev_weight, weight_type) || !on_element(dev_dweight, weight_type) || !on_element(dev_dbias, weight_type)) return NGSGD_EINVAL;
  if (sums) {
    if (dev_workspace == nullptr || (reinterpret_cast<uintptr_t>(dev_workspace) & 255u)) return NGSGD_EINVAL;
    size_t need = 0;
    NG_TRY(ngsgd_layernorm_workspace_bytes(N, D, &need));
    if (workspace_bytes < need) return NGSGD_ENOMEM;
  }
  const LayerNormBackward a{dev_dy, lddy, dev_x, ldx, dev_weight, dev_mean, dev_rstd, dev_dx, lddx, dev_dweight, dev_dbias, N, D,
                            sums ? static_cast<float*>(dev_workspace) : nullptr, N > 0 ? norm_groups(N, D) : 0, 1, 0};
  return with_types(type, weight_type,
                    [&](auto t, auto w) { return launch_backward<decltype(t), decltype(w), false>(a, static_cast<hipStream_t>(hip_stream)); });
}

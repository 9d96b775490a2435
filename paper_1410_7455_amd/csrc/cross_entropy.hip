// C ABI of the cross-entropy: argument checks, launches.  Declarations and contracts are in include/ngsgd.h.
#include "cross_entropy.h"

#include <algorithm>

#include "host.h"

using namespace ngsgd;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;
constexpr int32_t kMostClasses = 1 << 30;

template <typename F>
int with_types(const int type, const int index_type, F f) {
  const auto g = [&](auto t) { return index_type == NGSGD_INT32 ? f(t, int32_t()) : f(t, int64_t()); };
  return type == NGSGD_FLOAT32 ? g(float()) : type == NGSGD_BFLOAT16 ? g(bf16()) : g(fp16());
}

}  // namespace

extern "C" int ngsgd_cross_entropy_workspace_bytes(int64_t max_rows, int32_t V, size_t* out_bytes) {
  if (out_bytes == nullptr || max_rows < 0 || max_rows > kMostRows || V < 1 || V > kMostClasses) return NGSGD_EINVAL;
  *out_bytes = 256;
  return NGSGD_OK;
}

extern "C" int ngsgd_cross_entropy(const void* dev_logits, int64_t ld, int32_t type, const void* dev_labels, int32_t index_type, int64_t N, int32_t V,
                                   float* dev_loss, float scale, const float* dev_scale, void* dev_dlogits, int64_t ldd, void* dev_workspace,
                                   size_t workspace_bytes, void* hip_stream) {
  size_t need = 0;
  if (!known_type(type) || !known_index(index_type)) return NGSGD_EINVAL;
  NG_TRY(ngsgd_cross_entropy_workspace_bytes(N, V, &need));
  if (N == 0) return NGSGD_OK;
  if (dev_labels == nullptr || !on_index(dev_labels, index_type) || !good_matrix(dev_logits, ld, type, N, V)) return NGSGD_EINVAL;
  if (dev_loss == nullptr && dev_dlogits == nullptr) return NGSGD_EINVAL;
  if (!on_element(dev_loss, NGSGD_FLOAT32) || !on_element(dev_scale, NGSGD_FLOAT32)) return NGSGD_EINVAL;
  if (dev_dlogits != nullptr && !good_matrix(dev_dlogits, ldd, type, N, V)) return NGSGD_EINVAL;
  if (dev_dlogits == dev_logits && N > 1 && ldd != ld) return NGSGD_EINVAL;
  NG_TRY(check_workspace(dev_workspace, workspace_bytes, need));
  const CrossEntropy a{dev_logits, ld, dev_labels, N, V, dev_loss, scale, dev_scale, dev_dlogits, ldd};
  return with_types(type, index_type, [&](auto t, auto i) {
    hipLaunchKernelGGL((cross_entropy_kernel<decltype(t), decltype(i)>), dim3((unsigned)N), dim3(kLossThreads), 0, static_cast<hipStream_t>(hip_stream), a);
    LAUNCH_CHECK();
    return NGSGD_OK;
  });
}

// C ABI of the embedding: argument checks, launches.  Declarations and contracts are in include/ngsgd.h.
#include "embedding.h"

#include <algorithm>
#include <cmath>

#include "host.h"

using namespace ngsgd;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;
constexpr int32_t kMostColumns = 1 << 25;

int check_types(const int index_type, const int table_type, const int type, const int64_t N, const int64_t V, const int32_t D) {
  if (!known_index(index_type) || !known_type(type) || !known_type(table_type) || (table_type != type && table_type != NGSGD_FLOAT32)) return NGSGD_EINVAL;
  return N < 0 || N > kMostRows || V < 1 || V > kMostRows || D < 1 || D > kMostColumns ? NGSGD_EINVAL : NGSGD_OK;
}

// f(element, table's element, token) for the types of a call
template <typename F>
int with_types(const int type, const int table_type, const int index_type, F f) {
  const auto g = [&](auto t, auto w) { return index_type == NGSGD_INT32 ? f(t, w, int32_t()) : f(t, w, int64_t()); };
  if (type == NGSGD_FLOAT32) return g(float(), float());
  if (type == NGSGD_BFLOAT16) return table_type == NGSGD_FLOAT32 ? g(bf16(), float()) : g(bf16(), bf16());
  return table_type == NGSGD_FLOAT32 ? g(fp16(), float()) : g(fp16(), fp16());
}

template <typename W, typename T, typename I, int E>
int launch_forward(EmbeddingForward a, hipStream_t s) {
  const int pieces = (a.D + E - 1) / E;
  for (a.lanes = 1; a.lanes < pieces && a.lanes < kLookupThreads; a.lanes *= 2) {
  }
  const int64_t rows = (int64_t)kLookupThreads / a.lanes * kLookupRows;
  hipLaunchKernelGGL((embedding_forward_kernel<W, T, I, E>), dim3((unsigned)((a.N + rows - 1) / rows)), dim3(kLookupThreads), 0, s, a);
  LAUNCH_CHECK();
  return NGSGD_OK;
}

}  // namespace

extern "C" int ngsgd_embedding_forward(const void* dev_tokens, int32_t index_type, int64_t N, const void* dev_table, int64_t ldt, int32_t table_type,
                                       int64_t V, int32_t D, float scale, void* dev_y, int64_t ldy, int32_t type, void* hip_stream) {
  NG_TRY(check_types(index_type, table_type, type, N, V, D));
  if (!std::isfinite(scale)) return NGSGD_EINVAL;
  if (N == 0) return NGSGD_OK;
  if (dev_tokens == nullptr || !on_index(dev_tokens, index_type)) return NGSGD_EINVAL;
  if (!good_matrix(dev_table, ldt, table_type, V, D) || !good_matrix(dev_y, ldy, type, N, D)) return NGSGD_EINVAL;
  const EmbeddingForward a{dev_tokens, N, dev_table, ldt, V, D, scale, dev_y, ldy, 0};
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  return with_types(type, table_type, index_type, [&](auto t, auto w, auto i) {
    using T = decltype(t);
    constexpr int E = 16 / sizeof(T);
    return a.D >= E ? launch_forward<decltype(w), T, decltype(i), E>(a, s) : launch_forward<decltype(w), T, decltype(i), 1>(a, s);
  });
}

extern "C" int ngsgd_embedding_workspace_bytes(int64_t max_tokens, int64_t V, int32_t D, size_t* out_bytes) {
  if (out_bytes == nullptr || max_tokens < 0 || max_tokens > kMostRows || V < 1 || V > kMostRows || D < 1 || D > kMostColumns) return NGSGD_EINVAL;
  *out_bytes = 256;
  return NGSGD_OK;
}

extern "C" int ngsgd_embedding_backward(const void* dev_dy, int64_t lddy, int32_t type, const void* dev_tokens, int32_t index_type, int64_t N,
                                        int64_t V, int32_t D, float scale, void* dev_dtable, int64_t lddt, int32_t table_type, int32_t accumulate,
                                        void* dev_workspace, size_t workspace_bytes, void* hip_stream) {
  NG_TRY(check_types(index_type, table_type, type, N, V, D));
  if (!std::isfinite(scale) || (accumulate != 0 && accumulate != 1)) return NGSGD_EINVAL;
  if (N > 0 && (dev_tokens == nullptr || !on_index(dev_tokens, index_type))) return NGSGD_EINVAL;
  if (!good_matrix(dev_dy, lddy, type, N, D) || !good_matrix(dev_dtable, lddt, table_type, V, D)) return NGSGD_EINVAL;
  size_t need = 0;
  NG_TRY(ngsgd_embedding_workspace_bytes(N, V, D, &need));
  NG_TRY(check_workspace(dev_workspace, workspace_bytes, need));
  const EmbeddingBackward a{dev_dy, lddy, dev_tokens, N, V, D, scale, dev_dtable, lddt, accumulate};
  return with_types(type, table_type, index_type, [&](auto t, auto w, auto i) {
    const dim3 grid((unsigned)((V + 3) / 4), (unsigned)std::min(D / 64 + 1, 64));
    hipLaunchKernelGGL((embedding_backward_kernel<decltype(t), decltype(w), decltype(i)>), grid, dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    LAUNCH_CHECK();
    return NGSGD_OK;
  });
}

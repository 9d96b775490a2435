// C ABI of the cross-entropy: argument checks, launches.  Declarations and contracts are in include/ngsgd.h.
#include "cross_entropy.h"

#include <algorithm>

#include "host.h"

using namespace ngsgd;

namespace {

constexpr int64_t kMostRows = (int64_t)1 << 30;
constexpr int32_t kMostClasses = 1 << 29;   // (offsets in a row are 32 bits of bytes)
constexpr int64_t kLaunchRows = (int64_t)1 << 21;

constexpr int kRegisterPieces = 16384;     // of 16 bytes: of wider rows some are read twice
static_assert(kRegisterPieces >= kHeldPieces);
constexpr int kPartPieces = 4096;          // rows of more are cut into parts
// if there are fewer than so many.  127 rows in parts and 128 without, gradient, us: bf16 4100 pieces 11.5, 9.7; 8192 14.4, 14.4; 16384 26.2, 25.7; 25000 35.6, 39.7; 250000
// 345, 416; fp32 4100 10.4, 7.5; 8192 12.4, 9.8; 16384 23.6, 18.2; 25000 32.9, 31.1; 250000 332, 352: the border is right for rows that a workgroup does not hold, and too
// high for those that it does (64 rows in parts: 4100 pieces 10.5, 16384 13.6 bf16 and 12.0 fp32).
constexpr int kPartRows = 128;
constexpr int kPartGroups = 1024;          // into about so many workgroups' worth
constexpr int kPartLeast = 512;            // of at least so many pieces

int parts_of(const int64_t N, const int pieces) {
  if (N >= kPartRows || pieces <= kPartPieces) return 1;
  return (int)std::min<int64_t>({kMostParts, (kPartGroups + N - 1) / N, pieces / kPartLeast});
}
size_t stats_of(const int64_t max_rows, const int32_t V) {   // for so many rows or fewer, of any type
  if (V / 4 < kPartPieces) return 0;
  const int64_t rows = std::min<int64_t>(max_rows, kPartRows - 1);
  return (size_t)std::min<int64_t>(rows * (kMostParts + 1), kPartGroups + 2 * rows);
}

template <typename T, int E, int G, int P, int THREADS>
int launch_rows(const CrossEntropy& a, hipStream_t s) {
  constexpr int rows = THREADS / G;
  hipLaunchKernelGGL((cross_entropy_kernel<T, E, G, P, THREADS>), dim3((unsigned)((a.N + rows - 1) / rows)), dim3(THREADS), 0, s, a);
  LAUNCH_CHECK();
  return NGSGD_OK;
}

template <typename T>
int launch(CrossEntropy a, hipStream_t s) {
  constexpr int E = 16 / sizeof(T);
  if (a.V < E) return launch_rows<T, 1, 16, 1, 256>(a, s);
  const int pieces = (a.V - 1) / E + 1;
  a.parts = parts_of(a.N, pieces);
  if (a.parts > 1) {
    const dim3 grid((unsigned)(a.N * a.parts));
    hipLaunchKernelGGL((cross_entropy_part_kernel<T>), grid, dim3(kPartThreads), 0, s, a);
    LAUNCH_CHECK();
    hipLaunchKernelGGL((cross_entropy_join_kernel<T>), grid, dim3(kPartThreads), 0, s, a);
    LAUNCH_CHECK();
    return NGSGD_OK;
  }
  // The fewest threads that hold a row in up to 8 pieces each, while wavefronts of their own rows fill the chip.  bf16, this and the next larger or smaller group, us:
  // 65536 x 100 15 (16 lanes), 42 (64); 65536 x 256 21, 42; 32768 x 1000 34 (64 lanes), 77 (256 threads); 16384 x 2048 30, 61; 16384 x 4096 49, 62; 8192 x 8192 50
  // (256), 59 (512), 81 (1024); 8192 x 16384 95 (512), 99 (256), 117 (1024); 8192 x 32000 180 (1024), 195 (512).
  if (pieces <= 16) return launch_rows<T, E, 16, 1, 256>(a, s);
  if (pieces <= 32) return launch_rows<T, E, 16, 2, 256>(a, s);
  if (pieces <= 64) return launch_rows<T, E, 64, 1, 256>(a, s);
  if (pieces <= 128) return launch_rows<T, E, 64, 2, 256>(a, s);
  if (pieces <= 256) return launch_rows<T, E, 64, 4, 256>(a, s);
  if (pieces <= 512) return launch_rows<T, E, 64, 8, 256>(a, s);
  if (pieces <= 1024) return launch_rows<T, E, 256, 4, 256>(a, s);
  if (pieces <= 2048) return launch_rows<T, E, 512, 4, 512>(a, s);
  if (pieces <= 4096) return launch_rows<T, E, 1024, 4, 1024>(a, s);
  if (pieces <= 8192) return launch_rows<T, E, 1024, 8, 1024>(a, s);
  if (pieces <= kRegisterPieces) return launch_rows<T, E, 1024, 16, 1024>(a, s);
  hipLaunchKernelGGL((cross_entropy_wide_kernel<T>), dim3((unsigned)a.N), dim3(kWideThreads), 0, s, a);
  LAUNCH_CHECK();
  return NGSGD_OK;
}

}  // namespace

extern "C" int ngsgd_cross_entropy_workspace_bytes(int64_t max_rows, int32_t V, size_t* out_bytes) {
  if (out_bytes == nullptr || max_rows < 0 || max_rows > kMostRows || V < 1 || V > kMostClasses) return NGSGD_EINVAL;
  Carver c(nullptr);
  (void)c.take<LossStats>(stats_of(max_rows, V));
  *out_bytes = align_up(std::max<size_t>(c.off, 1), 256);
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
  hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const int index_bytes = index_type == NGSGD_INT32 ? 4 : 8;
  for (int64_t first = 0; first < N; first += kLaunchRows) {   // (a launch has less than 2^32 threads)
    const CrossEntropy a{static_cast<const char*>(dev_logits) + first * ld * type_bytes(type), ld,
                         static_cast<const char*>(dev_labels) + first * index_bytes, index_bytes, std::min(kLaunchRows, N - first), V,
                         dev_loss != nullptr ? dev_loss + first : nullptr, scale, dev_scale,
                         dev_dlogits != nullptr ? static_cast<char*>(dev_dlogits) + first * ldd * type_bytes(type) : nullptr, ldd,
                         static_cast<LossStats*>(dev_workspace), 1};
    NG_TRY(type == NGSGD_FLOAT32 ? launch<float>(a, s) : type == NGSGD_BFLOAT16 ? launch<bf16>(a, s) : launch<fp16>(a, s));
  }
  return NGSGD_OK;
}

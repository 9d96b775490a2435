// What the host code of all sources shares: error handling, sizes, element types, the workspace carver.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "ngsgd.h"

namespace ngsgd {

inline thread_local int g_last_hip_error = 0;

#define HIP_TRY(expr)                         \
  do {                                        \
    hipError_t e__ = (expr);                  \
    if (e__ != hipSuccess) {                  \
      g_last_hip_error = (int)e__;            \
      return NGSGD_EHIP;                      \
    }                                         \
  } while (0)
#define NG_TRY(expr)                \
  do {                              \
    int rc__ = (expr);              \
    if (rc__ != NGSGD_OK) return rc__; \
  } while (0)
#define LAUNCH_CHECK() HIP_TRY(hipGetLastError())

inline int pad32(int x) { return (x + 31) / 32 * 32; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool known_type(int type) { return type == NGSGD_FLOAT32 || type == NGSGD_BFLOAT16 || type == NGSGD_FLOAT16; }
inline int type_bytes(int type) { return type == NGSGD_FLOAT32 ? 4 : 2; }
inline bool on_element(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(type_bytes(type) - 1)) == 0; }
inline bool known_index(int type) { return type == NGSGD_INT32 || type == NGSGD_INT64; }
inline bool on_index(const void* p, int type) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(type == NGSGD_INT32 ? 3 : 7)) == 0; }
// A matrix argument of N rows of D elements: present, rows that do not overlap, whole elements.
inline bool good_matrix(const void* p, int64_t ld, int type, int64_t N, int64_t D) {
  if (N == 0) return true;
  return p != nullptr && on_element(p, type) && (ld >= D || N == 1) && ld >= 0 && ld <= INT64_MAX / 8 / N;
}
// A workspace argument.
inline int check_workspace(const void* p, size_t bytes, size_t need) {
  if (p == nullptr || (reinterpret_cast<uintptr_t>(p) & 255u)) return NGSGD_EINVAL;
  return bytes < need ? NGSGD_ENOMEM : NGSGD_OK;
}
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Carves typed arrays out of a caller-provided device workspace; with base == nullptr it only sizes.
struct Carver {
  char* base;
  size_t off = 0;
  explicit Carver(void* b) : base(static_cast<char*>(b)) {}
  template <typename T>
  T* take(size_t n) {
    off = align_up(off, 256);
    T* p = base ? reinterpret_cast<T*>(base + off) : nullptr;
    off += n * sizeof(T);
    return p;
  }
};

}  // namespace ngsgd

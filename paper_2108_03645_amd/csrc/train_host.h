// Host side of the training operators: argument checks, error texts, launches.
#pragma once

#include "ones.h"
#include "ones_train.h"

#include <hip/hip_runtime.h>

namespace ones {

// Keeps the failure's text for ones_strerror(ONES_E_HIP) on this thread (ones_api.hip).
int hip_fail(hipError_t e, const char *what);

namespace train {

constexpr int64_t kMaxElements = int64_t{1} << 46;      // of one array: products of sizes stay far inside 64 bits

inline bool is_type(int32_t t) { return t == ONES_F32 || t == ONES_F16 || t == ONES_BF16; }
inline int64_t type_bytes(int32_t t) { return t == ONES_F32 ? 4 : 2; }
inline bool aligned(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align_up(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

inline int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ONES_OK : hip_fail(e, what);
}

// The sizes of a two-dimensional array of `rows` rows of `cols` elements, rows `stride` elements apart.
inline int check_rows(int64_t rows, int64_t cols, int64_t stride) {
  if (rows < 0 || cols < 0 || stride < cols) return ONES_E_INVALID_ARG;
  if (rows && stride > kMaxElements / rows) return ONES_E_BOUNDS;
  return ONES_OK;
}

inline int check_workspace(const void *p, size_t bytes, size_t need) {
  if (need == 0) return ONES_OK;
  if (!p) return ONES_E_INVALID_ARG;
  return bytes < need || !aligned(p, 256) ? ONES_E_WORKSPACE_TOO_SMALL : ONES_OK;
}

}  // namespace train
}  // namespace ones

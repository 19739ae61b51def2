// Host side of the training operators: argument checks, error texts, launches.
#pragma once

#include "train_plan.h"

#include <hip/hip_runtime.h>

namespace ones {

// Keeps the failure's text for ones_strerror(ONES_E_HIP) on this thread (ones_api.hip).
int hip_fail(hipError_t e, const char *what);

namespace train {

inline bool aligned(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }

inline int launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? ONES_OK : hip_fail(e, what);
}

inline int check_workspace(const void *p, size_t bytes, size_t need) {
  if (need == 0) return ONES_OK;
  if (!p) return ONES_E_INVALID_ARG;
  return bytes < need || !aligned(p, 256) ? ONES_E_WORKSPACE_TOO_SMALL : ONES_OK;
}

}  // namespace train
}  // namespace ones

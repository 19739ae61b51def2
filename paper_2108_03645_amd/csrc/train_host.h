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

// The tiles of the matrix products (train_matmul.h), and how long a launch of them takes, by what was measured: so many
// microseconds for 64 k where every workgroup has a compute unit of its own, so many where `places` of them are at work, and so
// many for a workgroup's start and end.  From products of sides 256 to 4096 (k 4096, lower triangle of 4096 rows, us: large 92,
// middle 95, deep 109, small 106, tiny 160; of 3000 rows 93, 52, 67, 55, 90; of 2048, k 2048: 56, 30, 21, 26, 24; of 1024, k 4096:
// 90, 43, 29, 43, 16; eight of 256, k 256: 24, 16, 9, 9, 6; all tiles of 4096 x 4096, k 4096: 118, 146, 157, 141, 200).
enum Tiles : int { kLarge, kMiddle, kDeep, kSmall, kTiny };
struct TileCost {
  int64_t bm, bn, places;
  double alone, shared, fixed;
};
constexpr TileCost kTileCosts[] = {
    {256, 256, 256, 1.35, 1.45, 8.0}, {192, 128, 256, 0.72, 0.70, 6.0}, {128, 128, 256, 0.45, 0.47, 5.0}, {128, 128, 512, 0.62, 0.78, 5.0}, {64, 64, 512, 0.20, 0.38, 4.5}};

inline double item_time(const TileCost &c, int64_t items, int64_t k) { return ceil_div(k, 64) * (items <= 256 ? c.alone : c.shared) + c.fixed; }
inline double launch_time(const TileCost &c, int64_t items, int64_t k) { return ceil_div(items, c.places) * item_time(c, items, k); }

}  // namespace train
}  // namespace ones

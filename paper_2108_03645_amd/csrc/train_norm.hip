// Layer norm over the last dimension, forward and backward (ones_layer_norm_*).
//
//   mean = sum x / D, rstd = (sum (x - mean)^2 / D + eps)^-1/2, xh = (x - mean) rstd, y = xh w + b
//   g = dy w, dx = rstd (g - avg(g) - xh avg(g xh)), dw = sum over rows of dy xh, db = sum over rows of dy
//
// Both directions touch every element once: a row is held in registers by a wave (D up to 2048), four waves (up to 8192) or
// sixteen (up to 32768), so that the centred sum of squares (no cancellation, unlike the sum of squares less the square of the
// mean) and the results need no second read.  What bounds them is memory.  Workgroups take rows in turn, which keeps the
// weights in registers, and backward the sums of dw and db over a workgroup's rows as well: it leaves one row of partial sums a
// workgroup, which a second small launch adds up in a fixed order; few short rows are left to a single workgroup, which writes dw
// and db itself.  No atomics: the results are the same bits every time.
//
// Measured at 32768 x 2048 bf16, next to a copy of 4 GiB at 4.65 TB/s: forward 48 us (269 MB, 5.6 TB/s, part of them from the
// last-level cache), backward 88 us (403 MB and 17 MB of partial sums, 4.8 TB/s) and 8 us for the sums.  At 5003 x 1001 fp16, whose
// rows begin at any even address, 9 us (20 MB, 2.2 TB/s), 14.5 us and 4 us: as long as the calls take the host.
#include "train_device.h"
#include "train_host.h"

#include <algorithm>

namespace ones {
namespace train {
namespace {

constexpr int kBlock = 256;
// Backward, whether the next row is read ahead: not where 1024 threads share a row, as a workgroup of so many has 128 registers a
// thread; they read the weights for every row, too.  (Forward, waves enough for each other's gaps: reading ahead costs 5 to 15 %.)
template <int TPR>
constexpr bool kAhead = TPR < 1024;
// Backward, what a single workgroup of 16 waves takes: rows of a wave (PER is 8), up to four each.  It saves the launch that adds up
// the workgroups' sums: in a graph 16 x 512 takes 3.3 us against 5.3, 64 x 256 8.3 against 5.5 (1.5 us for a row of every wave, as all
// run on one compute unit); calls one after another, where the launches are what the host waits for, 12.4 us against 16.
constexpr int64_t kAloneCols = 512, kAloneRows = 64;
template <int TPR, int BLOCK>
constexpr bool kAlone = TPR < BLOCK && BLOCK > kBlock;

struct NormArgs {
  const void *x, *dy;
  void *out;                       // y forward, dx backward
  const void *weight, *bias;       // may be null (bias is used forward only)
  float *mean, *rstd;              // written forward, read backward
  float *partial;                  // backward: [workgroups][2][D]; null: one workgroup, which writes dweight and dbias (may be null)
  void *dweight, *dbias;
  int64_t rows, x_stride, dy_stride;
  int32_t cols, weight_type;
  float eps;
  bool past;                       // out goes past the caches
};

// A row as read: thread t holds elements (k * TPR + t) * VEC + 0..VEC-1, k < PER / VEC; zeros beyond the last column.
template <typename T, int PER, int VEC, int TPR>
struct Row {
  Pack<T, VEC> p[PER / VEC];
  __device__ __forceinline__ void load(const T *row, int t, int cols) {
#pragma unroll
    for (int k = 0; k < PER / VEC; ++k) {
      const int c = (k * TPR + t) * VEC;
      p[k] = load_some<T, VEC>(row + c, cols - c);
    }
  }
  __device__ __forceinline__ float operator[](int i) const { return static_cast<float>(p[i / VEC].v[i % VEC]); }
};
template <typename T, int PER, int VEC, int TPR>
__device__ __forceinline__ void store_row(T *row, int t, int cols, const float *v, bool past) {
#pragma unroll
  for (int k = 0; k < PER / VEC; ++k) {
    const int c = (k * TPR + t) * VEC;
    store_some<T, VEC>(row + c, v + k * VEC, cols - c, past);
  }
}
template <typename W, int PER, int VEC, int TPR>
__device__ __forceinline__ void load_weights_as(const W *p, int t, int cols, float *v) {
  Row<W, PER, VEC, TPR> row;
  row.load(p, t, cols);
#pragma unroll
  for (int i = 0; i < PER; ++i) v[i] = row[i];
}
template <int PER, int VEC, int TPR>
__device__ __forceinline__ void load_weights(const void *p, int type, float otherwise, int t, int cols, float *v) {
  if (!p) {
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = (i / VEC * TPR + t) * VEC + i % VEC < cols ? otherwise : 0.f;
  } else if (type == kF32) {
    load_weights_as<float, PER, VEC, TPR>(static_cast<const float *>(p), t, cols, v);
  } else if (type == kF16) {
    load_weights_as<f16, PER, VEC, TPR>(static_cast<const f16 *>(p), t, cols, v);
  } else {
    load_weights_as<bf16, PER, VEC, TPR>(static_cast<const bf16 *>(p), t, cols, v);
  }
}

template <typename T, int PER, int VEC, int TPR>
__global__ __launch_bounds__(TPR > kBlock ? TPR : kBlock) void norm_forward_kernel(NormArgs a) {
  constexpr int block = TPR > kBlock ? TPR : kBlock, rows_at_once = block / TPR;
  __shared__ float part[2][2 * (block / kWave)];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[PER], b[PER];
  load_weights<PER, VEC, TPR>(a.weight, a.weight_type, 1.f, t, a.cols, w);
  load_weights<PER, VEC, TPR>(a.bias, a.weight_type, 0.f, t, a.cols, b);
  const float n = static_cast<float>(a.cols);
  const int64_t step = static_cast<int64_t>(gridDim.x) * rows_at_once;
  int64_t row = static_cast<int64_t>(blockIdx.x) * rows_at_once + sub;
  const T *x = static_cast<const T *>(a.x);
  for (; row < a.rows; row += step) {
    Row<T, PER, VEC, TPR> now;
    now.load(x + row * a.x_stride, t, a.cols);
    float v[PER];
    float sum = 0.f, none = 0.f, square = 0.f, rest = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += v[i] = now[i];
    row_sum2<TPR>(sum, none, part[0]);
    float mean = sum / n;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool inside = (i / VEC * TPR + t) * VEC + i % VEC < a.cols;
      const float d = inside ? v[i] - mean : 0.f;
      v[i] = d;
      rest += d;
      square += d * d;
    }
    row_sum2<TPR>(square, rest, part[1]);
    // what the first mean was off by (its rounding, where the values lie far from zero) is the mean of the differences
    rest /= n;
    mean += rest;
    const float rstd = 1.f / sqrtf(fmaxf(square / n - rest * rest, 0.f) + a.eps);
#pragma unroll
    for (int i = 0; i < PER; ++i) v[i] = (v[i] - rest) * rstd * w[i] + b[i];
    store_row<T, PER, VEC, TPR>(static_cast<T *>(a.out) + row * a.cols, t, a.cols, v, a.past);
    if (t == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
  }
}

template <typename T, int PER, int VEC, int TPR, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_backward_kernel(NormArgs a) {
  constexpr int rows_at_once = BLOCK / TPR;
  __shared__ float part[2][2 * (BLOCK / kWave)];
  __shared__ __align__(16) float sums[rows_at_once > 1 ? rows_at_once : 1][2][rows_at_once > 1 ? PER * TPR : 1];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float w[PER], dw[PER], db[PER];
  if (kAhead<TPR>) load_weights<PER, VEC, TPR>(a.weight, a.weight_type, 1.f, t, a.cols, w);
#pragma unroll
  for (int i = 0; i < PER; ++i) dw[i] = db[i] = 0.f;
  const float n = static_cast<float>(a.cols);
  int turn = 0;
  const int64_t step = static_cast<int64_t>(gridDim.x) * rows_at_once;
  int64_t row = static_cast<int64_t>(blockIdx.x) * rows_at_once + sub;
  struct Read {
    Row<T, PER, VEC, TPR> x, dy;
    float mean, rstd;
  };
  auto load = [&](int64_t r, Read &to) {
    to.x.load(static_cast<const T *>(a.x) + r * a.x_stride, t, a.cols);
    to.dy.load(static_cast<const T *>(a.dy) + r * a.dy_stride, t, a.cols);
    to.mean = a.mean[r];
    to.rstd = a.rstd[r];
  };
  auto take = [&](int64_t r, const Read &from) {
    float x[PER], dy[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) { x[i] = from.x[i]; dy[i] = from.dy[i]; }
    float sg = 0.f, sgx = 0.f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {                 // past the last column dy and w are zero
      const float xh = (x[i] - from.mean) * from.rstd, g = dy[i] * w[i];
      x[i] = xh;
      dw[i] += dy[i] * xh;
      db[i] += dy[i];
      sg += g;
      sgx += g * xh;
    }
    row_sum2<TPR>(sg, sgx, part[turn]);
    turn ^= 1;
    sg /= n;
    sgx /= n;
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = from.rstd * (dy[i] * w[i] - sg - x[i] * sgx);
    store_row<T, PER, VEC, TPR>(static_cast<T *>(a.out) + r * a.cols, t, a.cols, x, a.past);
  };
  if constexpr (kAhead<TPR>) {
    Read now, next;
    if (row < a.rows) load(row, now);
    for (; row < a.rows; row += step) {
      if (row + step < a.rows) load(row + step, next);
      take(row, now);
      now = next;
    }
  } else {
    Read now;
    for (; row < a.rows; row += step) {
      load(row, now);
      load_weights<PER, VEC, TPR>(a.weight, a.weight_type, 1.f, t, a.cols, w);
      take(row, now);
    }
  }
  float *to = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * a.cols;
  if constexpr (rows_at_once > 1) {                 // the waves' sums, in order
#pragma unroll
    for (int k = 0; k < PER / VEC; ++k) {
      const int c = (k * TPR + t) * VEC;
      store_pack<float, VEC>(&sums[sub][0][c], dw + k * VEC);
      store_pack<float, VEC>(&sums[sub][1][c], db + k * VEC);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.cols; c += BLOCK) {
      const int which = c >= a.cols, at = which ? c - a.cols : c;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < rows_at_once; ++i) s += sums[i][which][at];
      if (!kAlone<TPR, BLOCK>) to[c] = s;
      else if (void *out = which ? a.dbias : a.dweight) store_as(out, a.weight_type, at, s);
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < PER / VEC; ++k) {
    const int c = (k * TPR + t) * VEC;
    store_some<float, VEC>(to + c, dw + k * VEC, a.cols - c);
    store_some<float, VEC>(to + a.cols + c, db + k * VEC, a.cols - c);
  }
}

// dw and db from n rows of partial sums: 16 threads share 64 of the 2 D columns.
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float *partial, int32_t n, int32_t cols, void *dweight, void *dbias, int32_t type) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x % 64, part = threadIdx.x / 64;
  const int c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < 2 * cols) {
#pragma unroll 4
    for (int i = part; i < n; i += 16) s += partial[static_cast<int64_t>(i) * 2 * cols + c];
  }
  sums[part][lane] = s;
  __syncthreads();
  if (part || c >= 2 * cols) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += sums[i][lane];
  void *to = c < cols ? dweight : dbias;
  if (to) store_as(to, type, c < cols ? c : c - cols, s);
}

// Threads of a row: up to 32 elements a thread forward; up to 16 backward, which keeps four of each in registers (beyond 16384
// columns 32).
int threads_per_row(int64_t cols, bool backward) {
  const int64_t most = backward ? 16 : 32;
  return cols <= 64 * most ? 64 : cols <= 256 * most ? 256 : 1024;
}
// Workgroups.  Forward as many as eight waves a SIMD.  Backward what the registers let run at once, since each leaves partial sums
// behind: with 8 elements a thread four waves a SIMD, with 16 two or three.
// (Backward, bf16, 32768 x 2048: 256 threads of 8 elements and 1024 workgroups 95 us, 64 of 32 and 512 125 us, 256 of 8 and 2048
// 114 us; 16384 x 4096: 256 of 16 and 768 110 us, 1024 of 8 148 us; 65536 x 512: 64 of 8 and 1024 43 us, 512 49 us.)
int64_t norm_blocks(int64_t rows, int64_t cols, bool backward) {
  const int64_t tpr = threads_per_row(cols, backward), at_once = tpr > kBlock ? 1 : kBlock / tpr;
  const bool few = cols <= tpr * 8;
  const int64_t most = !backward ? (tpr == 1024 ? 512 : 2048) : tpr == 1024 ? (few ? 512 : 256) : few ? 1024 : tpr == 256 ? 768 : 512;
  return std::min(ceil_div(rows, at_once), most);
}

// Whether a single workgroup takes the backward pass.
bool alone(int64_t rows, int64_t cols) { return rows && rows <= kAloneRows && cols <= kAloneCols; }

template <typename T, int PER, int VEC, int TPR>
void launch_norm(const NormArgs &a, bool backward, hipStream_t s) {
  constexpr int threads = TPR > kBlock ? TPR : kBlock;
  // what threads_per_row() leaves to each
  constexpr bool has_forward = TPR == 64 || PER > 8, has_backward = TPR == 1024 || PER <= 16;
  const dim3 grid(static_cast<uint32_t>(norm_blocks(a.rows, a.cols, backward))), block(threads);
  if constexpr (TPR == 64 && PER == 8)
    if (backward && !a.partial) {
      hipLaunchKernelGGL((norm_backward_kernel<T, PER, VEC, TPR, 1024>), dim3(1), dim3(1024), 0, s, a);
      return;
    }
  if constexpr (has_backward)
    if (backward) hipLaunchKernelGGL((norm_backward_kernel<T, PER, VEC, TPR, threads>), grid, block, 0, s, a);
  if constexpr (has_forward)
    if (!backward) hipLaunchKernelGGL((norm_forward_kernel<T, PER, VEC, TPR>), grid, block, 0, s, a);
}

template <typename T, int VEC, int TPR>
void launch_norm_per(const NormArgs &a, bool backward, hipStream_t s) {
  const int64_t per = ceil_div(a.cols, TPR);
  if (per <= 8) return launch_norm<T, 8, VEC, TPR>(a, backward, s);
  if (per <= 16) return launch_norm<T, 16, VEC, TPR>(a, backward, s);
  launch_norm<T, 32, VEC, TPR>(a, backward, s);
}

template <typename T>
void launch_norm(const NormArgs &a, bool backward, hipStream_t s) {
  constexpr int vec = 16 / sizeof(T);
  switch (threads_per_row(a.cols, backward)) {
    case 64: return launch_norm_per<T, vec, 64>(a, backward, s);
    case 256: return launch_norm_per<T, vec, 256>(a, backward, s);
    default: return launch_norm_per<T, vec, 1024>(a, backward, s);
  }
}

void launch_norm_type(const NormArgs &a, int32_t type, bool backward, hipStream_t s) {
  if (type == ONES_F32) launch_norm<float>(a, backward, s);
  else if (type == ONES_F16) launch_norm<f16>(a, backward, s);
  else launch_norm<bf16>(a, backward, s);
}

bool past(int64_t rows, int64_t cols, int32_t type) { return rows * cols * type_bytes(type) >= kPastBytes; }

int check_norm(int64_t rows, int64_t cols, int64_t stride, int32_t type, int32_t weight_type) {
  if (int rc = check_rows(rows, cols, stride)) return rc;
  if (cols < 1 || !is_type(type) || (weight_type != ONES_F32 && weight_type != type)) return ONES_E_INVALID_ARG;
  return cols > ONES_MAX_NORM_COLUMNS ? ONES_E_BOUNDS : ONES_OK;
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

int ones_layer_norm_forward(const void *x, int64_t x_stride, int64_t rows, int64_t cols, int32_t type, const void *weight, const void *bias,
                            int32_t weight_type, float eps, void *y, float *mean, float *rstd, void *hip_stream) {
  if (int rc = check_norm(rows, cols, x_stride, type, weight_type)) return rc;
  if (!(eps >= 0.f)) return ONES_E_INVALID_ARG;
  if (rows == 0) return ONES_OK;
  if (!x || !y || !mean || !rstd) return ONES_E_INVALID_ARG;
  const NormArgs a{x, nullptr, y, weight, bias, mean, rstd, nullptr, nullptr, nullptr, rows, x_stride, 0, static_cast<int32_t>(cols),
                   weight_type, eps, past(rows, cols, type)};
  launch_norm_type(a, type, false, static_cast<hipStream_t>(hip_stream));
  return launched("layer norm forward");
}

size_t ones_layer_norm_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || cols > ONES_MAX_NORM_COLUMNS || alone(rows, cols)) return 0;
  return align_up(static_cast<size_t>(std::max<int64_t>(1, norm_blocks(rows, cols, true))) * 2 * static_cast<size_t>(cols) * 4);
}

int ones_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int64_t rows, int64_t cols, int32_t type,
                             const void *weight, int32_t weight_type, const float *mean, const float *rstd, void *dx, void *dweight,
                             void *dbias, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_norm(rows, cols, x_stride, type, weight_type)) return rc;
  if (int rc = check_rows(rows, cols, dy_stride)) return rc;
  if (rows && (!dy || !x || !mean || !rstd || !dx)) return ONES_E_INVALID_ARG;
  if (int rc = check_workspace(d_workspace, workspace_bytes, ones_layer_norm_workspace_bytes(rows, cols))) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const bool single = alone(rows, cols);
  const NormArgs a{x, dy, dx, weight, nullptr, const_cast<float *>(mean), const_cast<float *>(rstd),
                   single ? nullptr : static_cast<float *>(d_workspace), dweight, dbias, rows, x_stride, dy_stride, static_cast<int32_t>(cols), weight_type, 0.f, past(rows, cols, type)};
  if (rows) launch_norm_type(a, type, true, s);
  if (!single && (dweight || dbias))
    hipLaunchKernelGGL(norm_reduce_kernel, dim3(static_cast<uint32_t>(ceil_div(2 * cols, 64))), dim3(1024), 0, s, a.partial,
                       static_cast<int32_t>(norm_blocks(rows, cols, true)), a.cols, dweight, dbias, weight_type);
  return launched("layer norm backward");
}

}  // extern "C"

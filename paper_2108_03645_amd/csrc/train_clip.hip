// Clipping of many gradients by their global norm (ones_clip_gradients): norm = (sum g^2)^1/2, g *= min(1, limit / (norm + eps)).
//
// One launch sums the squares, in 64 bits, so that finite gradients of any size have a norm; a second one scales.  The tensors' addresses are
// arguments of the launches, so nothing is copied to the device and a captured graph keeps them.  The sums of the workgroups have
// a place each; every workgroup of the second launch adds all of them up in the same order, and goes through its pieces from the last one on, which
// the caches have yet.
//
// What bounds it is memory: 148 bf16 tensors of 2^27 elements: squares 41 us (268 MB, 6.5 TB/s, half of it from the last-level cache when the
// gradients have just been written), scaling 87 us (6.2 TB/s, likewise).  12 small tensors: 4 and 2 us, less than the host takes.
#include "train_device.h"
#include "train_host.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

namespace ones {
namespace train {
namespace {

struct ClipArgs {
  void *p[kClipTable];
  int32_t first[kClipTable + 1];              // piece of a tensor's first element
  uint16_t last[kClipTable];                  // elements of its last piece less one, and its type above them
  int32_t tensors, part;                      // part: place of this launch's first sum
  int32_t parts;                              // of all launches
  float limit, eps;
  double *sums;
  float *norm;                                // written by the launch that has it
};
static_assert(sizeof(ClipArgs) <= 4096);

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double waves[4];
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) v += __shfl_xor(v, m);
  if (threadIdx.x % kWave == 0) waves[threadIdx.x / kWave] = v;
  __syncthreads();
  return (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

// The pieces of a workgroup lie next to each other: from piece begin on, below end.
__device__ __forceinline__ void pieces_of(const ClipArgs &a, int32_t &begin, int32_t &end) {
  const int64_t all = a.first[a.tensors];
  begin = static_cast<int32_t>(all * blockIdx.x / gridDim.x);
  end = static_cast<int32_t>(all * (blockIdx.x + 1) / gridDim.x);
}
__device__ __forceinline__ int tensor_of(const ClipArgs &a, int32_t piece) {
  int lo = 0, hi = a.tensors;                 // the last tensor that begins at or before it and has a piece
  while (hi - lo > 1) {
    const int m = (lo + hi) / 2;
    if (a.first[m] <= piece) lo = m;
    else hi = m;
  }
  return lo;
}

constexpr int kVec = 8, kRuns = static_cast<int>(kClipPiece / (256 * kVec));
static_assert(kRuns * 256 * kVec == kClipPiece && kClipPiece <= 1 << 13);

// A thread's elements of a piece: runs of eight, all of them loaded before the first is used.
template <typename T>
struct Runs {
  Pack<T, kVec> v[kRuns];
  __device__ __forceinline__ Runs(const T *p, int n) {
    const int i = static_cast<int>(threadIdx.x) * kVec;
    if (n == kClipPiece) {
#pragma unroll
      for (int r = 0; r < kRuns; ++r) v[r] = load_pack<T, kVec>(p + r * 256 * kVec + i);
    } else {
#pragma unroll
      for (int r = 0; r < kRuns; ++r) v[r] = load_some<T, kVec>(p + r * 256 * kVec + i, n - r * 256 * kVec - i);
    }
  }
};
template <typename T>
__device__ __forceinline__ double squares(const void *tensor, int64_t begin, int n) {
  const Runs<T> runs(static_cast<const T *>(tensor) + begin, n);
  double s = 0.;
#pragma unroll
  for (int r = 0; r < kRuns; ++r)
#pragma unroll
    for (int j = 0; j < kVec; ++j) { const double x = static_cast<double>(static_cast<float>(runs.v[r].v[j])); s = __builtin_fma(x, x, s); }
  return s;
}
template <typename T, typename F>
__device__ __forceinline__ void scale(void *tensor, int64_t begin, int n, F factor) {
  T *const p = static_cast<T *>(tensor) + begin;
  const Runs<T> runs(p, n);
#pragma unroll
  for (int r = 0; r < kRuns; ++r) {
    const int i = (r * 256 + static_cast<int>(threadIdx.x)) * kVec;
    float x[kVec];
#pragma unroll
    for (int j = 0; j < kVec; ++j) x[j] = static_cast<float>(static_cast<F>(static_cast<float>(runs.v[r].v[j])) * factor);
    store_some<T, kVec>(p + i, x, n - i);
  }
}
// A piece: its tensor, type, first element and elements.
struct Piece {
  void *p;
  int64_t begin;
  int type, n;
  __device__ __forceinline__ Piece(const ClipArgs &a, int32_t piece) {
    const int t = tensor_of(a, piece);
    p = a.p[t];
    begin = static_cast<int64_t>(piece - a.first[t]) * kClipPiece;
    n = piece + 1 == a.first[t + 1] ? (a.last[t] & (kClipPiece - 1)) + 1 : static_cast<int>(kClipPiece);
    type = a.last[t] >> 13;
  }
};

// The workgroup's pieces times factor, from the last one on, which the caches have yet.
template <typename F>
__device__ __forceinline__ void scale_pieces(const ClipArgs &a, F factor) {
  int32_t begin, piece;
  pieces_of(a, begin, piece);
  while (--piece >= begin) {
    const Piece at(a, piece);
    if (at.type == kF32) scale<float>(at.p, at.begin, at.n, factor);
    else if (at.type == kF16) scale<f16>(at.p, at.begin, at.n, factor);
    else scale<bf16>(at.p, at.begin, at.n, factor);
  }
}

__global__ __launch_bounds__(256) void squares_kernel(ClipArgs a) {
  int32_t piece, end;
  pieces_of(a, piece, end);
  double s = 0.;
  for (; piece < end; ++piece) {
    const Piece at(a, piece);
    if (at.type == kF32) s += squares<float>(at.p, at.begin, at.n);
    else if (at.type == kF16) s += squares<f16>(at.p, at.begin, at.n);
    else s += squares<bf16>(at.p, at.begin, at.n);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) a.sums[a.part + blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void clip_kernel(ClipArgs a) {
  double s = 0.;
  for (int i = threadIdx.x; i < a.parts; i += 256) s += a.sums[i];
  const double norm = sqrt(block_sum(s)), with = norm + a.eps;
  if (a.norm && blockIdx.x == 0 && threadIdx.x == 0) *a.norm = static_cast<float>(norm);
  if (!(with > a.limit) || !(norm < static_cast<double>(INFINITY))) return;
  // A factor that is no normal float, of a norm beyond 1e38 as it is with ordinary limits, would lose its bits in 32.
  const double factor = a.limit / with;
  if (factor < 0x1p-126) scale_pieces(a, factor);
  else scale_pieces(a, static_cast<float>(factor));
}

struct Span {
  uintptr_t begin, end;
};

// Whether no two of the tensors have an element in common.
int check_apart(void *const *gradients, const int64_t *counts, const int32_t *types, int64_t tensors) {
  Span *const spans = new (std::nothrow) Span[static_cast<size_t>(tensors)];
  if (!spans) return ONES_E_BOUNDS;
  int64_t n = 0;
  for (int64_t i = 0; i < tensors; ++i)
    if (counts[i]) {
      const uintptr_t at = reinterpret_cast<uintptr_t>(gradients[i]);
      spans[n++] = Span{at, at + static_cast<uintptr_t>(counts[i] * type_bytes(types[i]))};
    }
  std::sort(spans, spans + n, [](const Span &a, const Span &b) { return a.begin < b.begin; });
  bool apart = true;
  for (int64_t i = 1; i < n; ++i) apart = apart && spans[i - 1].end <= spans[i].begin;
  delete[] spans;
  return apart ? ONES_OK : ONES_E_INVALID_ARG;
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

size_t ones_clip_gradients_workspace_bytes(int64_t tensors) {
  return tensors < 0 || tensors > ONES_MAX_GRADIENTS ? 0 : clip_workspace(tensors);
}

int ones_clip_gradients(void *const *gradients, const int64_t *counts, const int32_t *types, int64_t tensors, float limit, float eps,
                        float *norm, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
  if (tensors < 0 || !norm || !(limit >= 0.f) || !(eps >= 0.f) || (tensors && (!gradients || !counts || !types))) return ONES_E_INVALID_ARG;
  if (tensors > ONES_MAX_GRADIENTS) return ONES_E_BOUNDS;
  int64_t pieces = 0;
  for (int64_t i = 0; i < tensors; ++i) {
    if (counts[i] < 0 || !is_type(types[i]) || (counts[i] && (!gradients[i] || !aligned(gradients[i], type_bytes(types[i]))))) return ONES_E_INVALID_ARG;
    if (counts[i] > kMaxElements) return ONES_E_BOUNDS;
    pieces += ceil_div(counts[i], kClipPiece);
    if (pieces >= (int64_t{1} << 31)) return ONES_E_BOUNDS;
  }
  if (int rc = check_workspace(d_workspace, workspace_bytes, clip_workspace(tensors))) return rc;
  if (tensors)
    if (int rc = check_apart(gradients, counts, types, tensors)) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  // of the workgroups every launch has its share, by its pieces, or enough for most compute units
  auto table = [&](int64_t from, ClipArgs &a) {
    a.tensors = static_cast<int32_t>(std::min(tensors - from, kClipTable));
    a.first[0] = 0;
    for (int32_t i = 0; i < a.tensors; ++i) {
      a.p[i] = gradients[from + i];
      a.last[i] = static_cast<uint16_t>(((counts[from + i] + kClipPiece - 1) % kClipPiece) | types[from + i] << 13);
      a.first[i + 1] = a.first[i] + static_cast<int32_t>(ceil_div(counts[from + i], kClipPiece));
    }
    const int64_t mine = a.first[a.tensors];
    return std::min(mine, std::max(kClipLeast, mine * kClipBlocks / std::max<int64_t>(pieces, 1)));
  };
  ClipArgs a{};
  a.limit = limit;
  a.eps = eps;
  a.sums = static_cast<double *>(d_workspace);
  for (int64_t from = 0; from < tensors; from += kClipTable)
    if (const int64_t blocks = table(from, a)) {
      hipLaunchKernelGGL(squares_kernel, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, s, a);
      a.part += static_cast<int32_t>(blocks);
    }
  a.parts = a.part;
  a.norm = norm;
  for (int64_t from = 0; from < tensors || from == 0; from += kClipTable) {
    const int64_t blocks = tensors ? table(from, a) : 0;
    if (!blocks && !(a.norm && from + kClipTable >= tensors)) continue;
    hipLaunchKernelGGL(clip_kernel, dim3(static_cast<uint32_t>(std::isinf(limit) ? 1 : std::max<int64_t>(blocks, 1))), dim3(256), 0, s, a);
    a.norm = nullptr;
    if (std::isinf(limit)) break;
  }
  return launched("clipping");
}

}  // extern "C"

// What the attention kernels over packed sequences share (train_attention.hip forward, train_attention_backward.hip): their arguments, and the sums
// of rows that products of matrices cannot give.
#pragma once

#include "train_attention.h"
#include "train_host.h"

#include <hip/hip_runtime.h>

#include <cmath>

namespace ones {
namespace train {
namespace {

struct AttentionArgs {
  const void *q, *k, *v, *dout;
  int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head, do_stride, do_head;      // elements
  void *o, *rest;
  float *lse;
  void *dq, *dk, *dv;
  float2 *terms;                              // of every row: lse in base 2, delta
  float *dout_norm, *v_norm;                  // |do| of every row; the largest |do| and |v| of every slot (fp16)
  float *partial;                             // dk and dv of parts of a group's heads, in 32 bits
  const int32_t *offsets;
  int32_t sequences, tokens, heads, kv_heads, dim, parts;
  float scale;
};

template <typename T>
__device__ __forceinline__ const T *at(const void *p, int64_t row, int64_t stride, int32_t head, int64_t head_stride) {
  return static_cast<const T *>(p) + row * stride + head * head_stride;
}

// How far, as a power of two, an exponential may exceed 1 before the largest score is taken over.  (0 costs 4 % forward; the largest exponential is rounded
// then as the others are, which a row of few large ones sees: bf16 o is off by 2.2e-3 of its norm instead of 1.9e-3.)
constexpr float kSlack = 6.f;

// A weight of 0 does not take a row out of a product where that row has infinities or NaN, so those of a token would reach the rows
// that it is masked for, as far as they share a step with it.  Each kernel looks for NaN in what it has summed.  Where there is some, the rows
// that may have it from there are summed once more without products of matrices, over what they do see, which is slow and right:
//   sums[e] = sum over y of weights(r, y)[e] * element d of row(e, y)
// for the rows 0 <= r < rows of the workgroup, elements d < dim, and 0 <= y < last(r).  has(r, d): what of element d of row r asks for it, 0 if nothing
// does; weights(r, y, w): whether row r sees y at all; write(r, d, sums, what asked).
template <int N, class Has, class Last, class Weights, class Row, class Write>
__device__ __forceinline__ void sum_by_rows(unsigned char *lds, int32_t rows, int32_t dim, Has has, Last last, Weights weights, Row row, Write write) {
  struct Held {
    float w[N];
    int32_t seen;
  };
  constexpr int kChunk = 256;
  Held *const held = reinterpret_cast<Held *>(lds);
  const int d = threadIdx.x;
  for (int32_t r = 0; r < rows; ++r) {
    const int asks = d < dim ? has(r, d) : 0;
    if (!__syncthreads_or(asks)) continue;
    const int32_t end = last(r);
    float sums[N] = {};
    for (int32_t y0 = 0; y0 < end; y0 += kChunk) {
      Held mine{};
      if (d < kChunk && y0 + d < end) mine.seen = weights(r, y0 + d, mine.w);
      __syncthreads();
      if (d < kChunk) held[d] = mine;
      __syncthreads();
      if (d >= dim) continue;
      for (int32_t y = y0; y < min(end, y0 + kChunk); ++y)
        if (held[y - y0].seen) {
#pragma unroll
          for (int e = 0; e < N; ++e) sums[e] += held[y - y0].w[e] * static_cast<float>(row(e, y)[d]);
        }
    }
    if (asks) write(r, d, sums, asks);
  }
}
// Whether of element d of rows first <= y < last, `stride` apart, one is not finite.
template <typename T>
__device__ __forceinline__ bool any_infinite(const T *rows, int64_t stride, int32_t first, int32_t last, int d) {
  bool found = false;
  for (int32_t y = first; y < last; ++y) {
    const float x = static_cast<float>(rows[y * stride + d]);
    found |= x - x != 0.f;
  }
  return found;
}
template <typename T>
__device__ __forceinline__ float dot(const T *a, const T *b, int32_t dim) {
  float s = 0.f;
  for (int i = 0; i < dim; ++i) s = __builtin_fmaf(static_cast<float>(a[i]), static_cast<float>(b[i]), s);
  return s;
}

constexpr int kQueries = kAttentionRows;
// Keys of a step, by the rows of 16 of a wave's part: of 32 where there is one, so that more workgroups fit into a compute unit.
template <int TN>
constexpr int kKeys = TN == 1 ? 32 : 64;

}  // namespace
}  // namespace train
}  // namespace ones

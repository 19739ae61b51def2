// Causal attention over packed sequences, query heads in groups that share a key head, with its gradients (ones_attention_*).
//
//   z_ij = scale q_i . k_j for j <= i, lse_i = log sum_j exp z_ij, p_ij = exp(z_ij - lse_i), o_i = sum_j p_ij v_j
//   delta_i = do_i . o_i, ds_ij = p_ij (do_i . v_j - delta_i)
//   dv_j = sum_i p_ij do_i, dk_j = scale sum_i ds_ij q_i (both over the heads of a group, too), dq_i = scale sum_j ds_ij k_j
#include "train_attention.h"
#include "train_host.h"

#include <hip/hip_runtime.h>

#include <cmath>

namespace ones {
namespace train {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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

// fp16 keeps 2^-24 and up: the exponentials below the row's largest are held in units of 2^-8.
template <typename T>
constexpr float kShift = __is_same(T, f16) ? 8.f : 0.f;

constexpr float kSlack = 6.f;                 // 2^(kShift + kSlack) is far from fp16's end

// A weight of 0 does not take a row out of a product where that row has infinities or NaN, so those of a token would reach the rows
// that it is masked for, as far as they share a step with it.  Each kernel looks for NaN in what it has summed.  Where there is some, the rows
// that have it are summed once more without products of matrices, over what they do see, which is slow and right:
//   sums[e] = sum over y of weights(r, y)[e] * element d of row(e, y)
// for the rows 0 <= r < rows of the workgroup, elements d < dim, and 0 <= y < last(r).  has(r, d): whether element d of row r asks for it;
// weights(r, y, w): whether row r sees y at all; write(r, d, sums).
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
    if (!__syncthreads_or(d < dim && has(r, d))) continue;
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
    if (d < dim) write(r, d, sums);
  }
}
template <typename T>
__device__ __forceinline__ float dot(const T *a, const T *b, int32_t dim) {
  float s = 0.f;
  for (int i = 0; i < dim; ++i) s = __builtin_fmaf(static_cast<float>(a[i]), static_cast<float>(b[i]), s);
  return s;
}

constexpr int kQueries = kAttentionRows, kKeys = 64;       // of a workgroup; of a step

template <typename T, int D, bool REST>
__global__ __launch_bounds__(256, 2) void attention_forward_kernel(AttentionArgs a) {
  constexpr int TN = 2, kThreads = 256, kMine = 16 * TN;
  using Tile = RowTile<D, kKeys, kThreads>;
  __shared__ __attribute__((aligned(256))) unsigned char lds[4 * Tile::bytes];
  const Turn turn = turn_of(blockIdx.x, a.heads, a.kv_heads);
  const int32_t last_slot = static_cast<int32_t>(slots_of(a.tokens, a.sequences, kQueries)) - 1;
  const Rows rows = rows_of<kQueries>(a.offsets, a.sequences, a.tokens, last_slot - turn.slot);      // the longest tiles first
  if (rows.at >= rows.length || rows.at < 0) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t out_stride = static_cast<int64_t>(a.heads) * a.dim;
  const int32_t here = rows.first + rows.at, count = min(rows.length - rows.at, kQueries);
  T *const o = const_cast<T *>(at<T>(a.o, here, out_stride, turn.head, a.dim)), *const rest = a.rest ? const_cast<T *>(at<T>(a.rest, here, out_stride, turn.head, a.dim)) : nullptr;
  float *const lse = a.lse + static_cast<int64_t>(turn.head) * a.tokens + here;
  if (!rows.real) {
    write_zeros(o, out_stride, count, a.dim);
    write_zeros(rest, out_stride, count, a.dim);
    for (int i = threadIdx.x; i < count; i += kThreads) lse[i] = -INFINITY;
    return;
  }
  Tile k, v;
  k.start(at<T>(a.k, rows.first, a.k_stride, turn.kv, a.k_head), a.k_stride, rows.length, a.dim);
  v.start(at<T>(a.v, rows.first, a.v_stride, turn.kv, a.v_head), a.v_stride, rows.length, a.dim);
  k.load(lds);
  v.load(lds + 2 * Tile::bytes);
  const int mine = wave * kMine;                 // the wave's first row in the tile
  s16x8 q[TN][D / 32];
#pragma unroll
  for (int n = 0; n < TN; ++n)
    read_rows<D>(at<T>(a.q, here + mine + n * 16, a.q_stride, turn.head, a.q_head), a.q_stride, count - mine - n * 16, a.dim, lane, q[n]);
  int along[D / 32], across[D / 16];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) along[s] = Tile::along(lane, s);
#pragma unroll
  for (int b = 0; b < D / 16; ++b) across[b] = Tile::across(lane, b);
  const float c = a.scale * kLog2e;
  f32x4 acc[D / 16][TN];
  float top[TN], sum[TN];
#pragma unroll
  for (int n = 0; n < TN; ++n) {
    top[n] = -INFINITY;
    sum[n] = 0.f;
#pragma unroll
    for (int b = 0; b < D / 16; ++b) acc[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int steps = (rows.at + count + kKeys - 1) / kKeys, first_row = rows.at + mine;
  for (int step = 0; step < steps; ++step) {
    meet<0>();
    const unsigned char *ks = lds + (step & 1) * Tile::bytes, *vs = ks + 2 * Tile::bytes;
    if (step + 1 < steps) {
      k.load(lds + (~step & 1) * Tile::bytes);
      v.load(lds + (2 + (~step & 1)) * Tile::bytes);
    }
    const int key = step * kKeys;
    if (key > first_row + kMine - 1) continue;       // keys behind all of the wave's rows
    f32x4 z[4][TN];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
#pragma unroll
      for (int n = 0; n < TN; ++n) z[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        const s16x8 f = Tile::read_along(ks, b * 16, along[s]);
#pragma unroll
        for (int n = 0; n < TN; ++n) z[b][n] = mfma<T>(f, q[n][s], z[b][n]);
      }
    }
    if (key + kKeys - 1 > first_row) {
#pragma unroll
      for (int n = 0; n < TN; ++n) {
        const int row = first_row + n * 16 + (lane & 15) - key;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (b * 16 + (lane >> 4) * 4 + r > row) z[b][n][r] = -INFINITY;
      }
    }
    // the largest score: taken over where it has grown by more than 2^kSlack, which exponentials may exceed 1 by
    float most[TN];
    bool grown = false;
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      float m[2] = {fmaxf(z[0][n][0], z[0][n][1]), fmaxf(z[1][n][0], z[1][n][1])};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        m[h] = fmaxf(fmaxf(m[h], z[h][n][2]), z[h][n][3]);
        m[h] = fmaxf(fmaxf(m[h], z[2 + h][n][0]), z[2 + h][n][1]);
        m[h] = fmaxf(fmaxf(m[h], z[2 + h][n][2]), z[2 + h][n][3]);
      }
      most[n] = across_max(fmaxf(m[0], m[1]));
      grown |= (most[n] - top[n]) * c > kSlack;
    }
    if (__any(grown)) {
#pragma unroll
      for (int n = 0; n < TN; ++n) {
        const float next = fmaxf(top[n], most[n]), factor = next == top[n] ? 1.f : __builtin_amdgcn_exp2f((top[n] - next) * c);
        sum[n] *= factor;
#pragma unroll
        for (int b = 0; b < D / 16; ++b) acc[b][n] *= factor;
        top[n] = next;
      }
    }
    s16x8 p[2][TN], lost[2][TN];              // lost: what the rounding takes from the exponentials
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      const float base = (top[n] == -INFINITY ? 0.f : top[n] * c) - kShift<T>;
      float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[b][n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][n][r], c, -base));
          sums[r] += z[b][n][r];
        }
      sum[n] += (sums[0] + sums[1]) + (sums[2] + sums[3]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        p[h][n] = rounded<T>(z[2 * h][n], z[2 * h + 1][n]);
        if constexpr (REST) lost[h][n] = remainder<T>(z[2 * h][n], z[2 * h + 1][n], p[h][n]);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int b = 0; b < D / 16; ++b) {
        const s16x8 f = Tile::read_across(vs, h * 32, across[b]);
#pragma unroll
        for (int n = 0; n < TN; ++n) {
          acc[b][n] = mfma<T>(f, p[h][n], acc[b][n]);
          if constexpr (REST) acc[b][n] = mfma<T>(f, lost[h][n], acc[b][n]);
        }
      }
    }
  }
  float factor[TN];
#pragma unroll
  for (int n = 0; n < TN; ++n) {
    const float s = across_sum(sum[n]);
    factor[n] = 1.f / s;
    const int r = mine + n * 16 + (lane & 15);
    if (lane < 16 && r < count) lse[r] = (top[n] * c - kShift<T> + __builtin_amdgcn_logf(s)) * kLn2;
  }
  write_rows<T, D, TN, REST>(acc, factor, o + mine * out_stride, rest ? rest + mine * out_stride : nullptr, out_stride, count - mine, a.dim, lane);
  if (__syncthreads_or(any_nan<D, TN>(acc))) {
    __syncthreads();
    const T *const q0 = at<T>(a.q, here, a.q_stride, turn.head, a.q_head), *const k0 = at<T>(a.k, rows.first, a.k_stride, turn.kv, a.k_head);
    const T *const v0 = at<T>(a.v, rows.first, a.v_stride, turn.kv, a.v_head);
    sum_by_rows<1>(
        lds, count, a.dim, [&](int32_t r, int d) { const float x = static_cast<float>(o[r * out_stride + d]); return x != x && lse[r] == lse[r]; },
        [&](int32_t r) { return rows.at + r + 1; },
        [&](int32_t r, int32_t y, float (&w)[1]) {
          w[0] = __builtin_amdgcn_exp2f(dot(q0 + r * a.q_stride, k0 + y * a.k_stride, a.dim) * c - lse[r] * kLog2e);
          return true;
        },
        [&](int, int32_t y) { return v0 + y * a.v_stride; },
        [&](int32_t r, int d, const float (&sums)[1]) {
          o[r * out_stride + d] = static_cast<T>(sums[0]);
          if (rest) rest[r * out_stride + d] = static_cast<T>(sums[0] - static_cast<float>(static_cast<T>(sums[0])));
        });
  }
}

// delta of every row of a slot and head, and its |do|; of a key head, the largest |v|.  (fp16 scales by the norms, see unit_of().)
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_delta_kernel(AttentionArgs a) {
  constexpr int lanes = D / 8, at_once = 256 / lanes;
  constexpr bool norms = __is_same(T, f16);
  __shared__ float part[4];
  const int32_t all = a.heads + (norms ? a.kv_heads : 0);
  const int32_t slot = blockIdx.x / all, head = blockIdx.x % all;
  const Rows rows = rows_of<kQueries>(a.offsets, a.sequences, a.tokens, slot);
  if (rows.at >= rows.length || rows.at < 0 || !rows.real) return;
  const int32_t here = rows.first + rows.at, count = min(rows.length - rows.at, kQueries);
  const int p = threadIdx.x % lanes, r0 = threadIdx.x / lanes;
  const bool inside = p * 8 < a.dim;
  float most = 0.f;
  if (head < a.heads) {
    const int64_t stride = static_cast<int64_t>(a.heads) * a.dim;
    const T *g = at<T>(a.dout, here, a.do_stride, head, a.do_head) + p * 8, *o = at<T>(a.o, here, stride, head, a.dim) + p * 8;
    const T *rest = a.rest ? at<T>(a.rest, here, stride, head, a.dim) + p * 8 : nullptr;
    for (int r = r0; r < (count + at_once - 1) / at_once * at_once; r += at_once) {
      float dot = 0.f, square = 0.f;
      if (inside && r < count) {
        const Pack<T, 8> x = *reinterpret_cast<const Pack<T, 8> *>(g + r * a.do_stride), y = *reinterpret_cast<const Pack<T, 8> *>(o + r * stride);
        Pack<T, 8> z{};
        if (rest) z = *reinterpret_cast<const Pack<T, 8> *>(rest + r * stride);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float d = static_cast<float>(x.v[i]);
          dot = __builtin_fmaf(d, static_cast<float>(y.v[i]) + static_cast<float>(z.v[i]), dot);
          square = __builtin_fmaf(d, d, square);
        }
      }
#pragma unroll
      for (int m = 1; m < lanes; m *= 2) { dot += __shfl_xor(dot, m); square += __shfl_xor(square, m); }
      if (p == 0 && r < count) {
        const int64_t i = static_cast<int64_t>(head) * a.tokens + here + r;
        a.terms[i] = make_float2(a.lse[i] * kLog2e, dot);
      }
      if (norms && square < INFINITY) most = fmaxf(most, square);
      if (norms && p == 0 && r < count) a.dout_norm[static_cast<int64_t>(head) * a.tokens + here + r] = square < INFINITY ? sqrtf(square) : 0.f;
    }
    if (!norms) return;
  } else {
    const T *v = at<T>(a.v, here, a.v_stride, head - a.heads, a.v_head) + p * 8;
    for (int r = r0; r < (count + at_once - 1) / at_once * at_once; r += at_once) {
      float square = 0.f;
      if (inside && r < count) {
        const Pack<T, 8> x = *reinterpret_cast<const Pack<T, 8> *>(v + r * a.v_stride);
#pragma unroll
        for (int i = 0; i < 8; ++i) { const float d = static_cast<float>(x.v[i]); square = __builtin_fmaf(d, d, square); }
      }
#pragma unroll
      for (int m = 1; m < lanes; m *= 2) square += __shfl_xor(square, m);
      if (square < INFINITY) most = fmaxf(most, square);
    }
  }
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    most = sqrtf(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    a.v_norm[static_cast<int64_t>(slot) * all + head] = most;      // of do's heads as well
  }
}

// The unit that ds is held in where it is rounded to fp16: a power of two that brings |ds| <= 2 |do| |v| to at most 2^14.  (bf16 has the
// exponents of 32 bits: 1.)
__device__ __forceinline__ float unit_of(float bound) {
  if (!(bound > 0.f) || !(bound < INFINITY)) return 1.f;
  int e;
  frexpf(bound, &e);                          // bound < 2^e
  return ldexpf(1.f, min(max(13 - e, -100), 100));
}
// The largest of the norms that the slots of a sequence have for `heads` heads from `head` on.
__device__ __forceinline__ float largest_norm(const float *norms, int32_t all, int32_t head, int32_t heads, int32_t slot, int32_t slots) {
  float most = 0.f;
  const int lane = threadIdx.x % kWave;
  for (int32_t i = lane; i < slots * heads; i += kWave) most = fmaxf(most, norms[static_cast<int64_t>(slot + i / heads) * all + head + i % heads]);
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
  return most;
}

template <typename T, int D>
__device__ __forceinline__ void gradient_of_queries(const AttentionArgs &a, uint32_t id, unsigned char *lds) {
  using Tile = RowTile<D, kKeys, 256>;
  const Turn turn = turn_of(id, a.heads, a.kv_heads);
  const int32_t slot = static_cast<int32_t>(slots_of(a.tokens, a.sequences, kQueries)) - 1 - turn.slot;
  const Rows rows = rows_of<kQueries>(a.offsets, a.sequences, a.tokens, slot);
  if (rows.at >= rows.length || rows.at < 0) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t out_stride = static_cast<int64_t>(a.heads) * a.dim;
  const int32_t here = rows.first + rows.at, count = min(rows.length - rows.at, kQueries);
  T *const dq = const_cast<T *>(at<T>(a.dq, here, out_stride, turn.head, a.dim));
  if (!rows.real) return write_zeros(dq, out_stride, count, a.dim);
  Tile k, v;
  k.start(at<T>(a.k, rows.first, a.k_stride, turn.kv, a.k_head), a.k_stride, rows.length, a.dim);
  v.start(at<T>(a.v, rows.first, a.v_stride, turn.kv, a.v_head), a.v_stride, rows.length, a.dim);
  k.load(lds);
  v.load(lds + 2 * Tile::bytes);
  const int mine = wave * 32;
  const float c = a.scale * kLog2e;
  float v_most = 0.f;
  if constexpr (__is_same(T, f16)) {
    const int32_t all = a.heads + a.kv_heads;
    v_most = largest_norm(a.v_norm, all, a.heads + turn.kv, 1, slot_of<kQueries>(rows.sequence, rows.first), (rows.length + kQueries - 1) / kQueries);
  }
  s16x8 q[2][D / 32], g[2][D / 32];
  float lse[2], delta[2], unit[2], factor[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int r = mine + n * 16;
    read_rows<D>(at<T>(a.q, here + r, a.q_stride, turn.head, a.q_head), a.q_stride, count - r, a.dim, lane, q[n]);
    read_rows<D>(at<T>(a.dout, here + r, a.do_stride, turn.head, a.do_head), a.do_stride, count - r, a.dim, lane, g[n]);
    const int64_t i = static_cast<int64_t>(turn.head) * a.tokens + here + min(r + (lane & 15), count - 1);
    const float2 terms = a.terms[i];
    lse[n] = terms.x;
    delta[n] = terms.y;
    unit[n] = 1.f;
    if constexpr (__is_same(T, f16)) unit[n] = unit_of(2.f * a.dout_norm[i] * v_most);
    factor[n] = a.scale / unit[n];
  }
  int along[D / 32], across[D / 16];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) along[s] = Tile::along(lane, s);
#pragma unroll
  for (int b = 0; b < D / 16; ++b) across[b] = Tile::across(lane, b);
  f32x4 acc[D / 16][2];
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int b = 0; b < D / 16; ++b) acc[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = (rows.at + count + kKeys - 1) / kKeys, first_row = rows.at + mine;
  for (int step = 0; step < steps; ++step) {
    meet<0>();
    const unsigned char *ks = lds + (step & 1) * Tile::bytes, *vs = ks + 2 * Tile::bytes;
    if (step + 1 < steps) {
      k.load(lds + (~step & 1) * Tile::bytes);
      v.load(lds + (2 + (~step & 1)) * Tile::bytes);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int key = step * kKeys + h * 32;
      if (key > first_row + 31) break;
      f32x4 z[2][2], d[2][2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int n = 0; n < 2; ++n) z[b][n] = d[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < D / 32; ++s) {
          const s16x8 f = Tile::read_along(ks, h * 32 + b * 16, along[s]), e = Tile::read_along(vs, h * 32 + b * 16, along[s]);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            z[b][n] = mfma<T>(f, q[n][s], z[b][n]);
            d[b][n] = mfma<T>(e, g[n][s], d[b][n]);
          }
        }
      }
      s16x8 ds[2];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int row = first_row + n * 16 + (lane & 15) - key;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][n][r], c, -lse[n]));
            const float s = p * (d[b][n][r] - delta[n]) * unit[n];
            z[b][n][r] = b * 16 + (lane >> 4) * 4 + r > row ? 0.f : s;
          }
        ds[n] = rounded<T>(z[0][n], z[1][n]);
      }
#pragma unroll
      for (int b = 0; b < D / 16; ++b) {
        const s16x8 f = Tile::read_across(ks, h * 32, across[b]);
#pragma unroll
        for (int n = 0; n < 2; ++n) acc[b][n] = mfma<T>(f, ds[n], acc[b][n]);
      }
    }
  }
  write_rows<T, D, 2>(acc, factor, dq + mine * out_stride, nullptr, out_stride, count - mine, a.dim, lane);
  if (__syncthreads_or(any_nan<D, 2>(acc))) {
    __syncthreads();
    const T *const q0 = at<T>(a.q, here, a.q_stride, turn.head, a.q_head), *const k0 = at<T>(a.k, rows.first, a.k_stride, turn.kv, a.k_head);
    const T *const g0 = at<T>(a.dout, here, a.do_stride, turn.head, a.do_head), *const v0 = at<T>(a.v, rows.first, a.v_stride, turn.kv, a.v_head);
    const float2 *const terms = a.terms + static_cast<int64_t>(turn.head) * a.tokens + here;
    sum_by_rows<1>(
        lds, count, a.dim,
        [&](int32_t r, int d) { const float x = static_cast<float>(dq[r * out_stride + d]), t = terms[r].x + terms[r].y; return x != x && t == t; },
        [&](int32_t r) { return rows.at + r + 1; },
        [&](int32_t r, int32_t y, float (&w)[1]) {
          const float p = __builtin_amdgcn_exp2f(dot(q0 + r * a.q_stride, k0 + y * a.k_stride, a.dim) * c - terms[r].x);
          w[0] = p * (dot(g0 + r * a.do_stride, v0 + y * a.v_stride, a.dim) - terms[r].y);
          return true;
        },
        [&](int, int32_t y) { return k0 + y * a.k_stride; },
        [&](int32_t r, int d, const float (&sums)[1]) { dq[r * out_stride + d] = static_cast<T>(sums[0] * a.scale); });
  }
}

constexpr int kStepRows = 32, kKeyRows = kAttentionKeys;        // of the keys' gradients: queries of a step; keys of a workgroup
#ifndef DKV_TN
#define DKV_TN 1
#define DKV_OCC 3
#endif

template <typename T, int D>
constexpr int kKeysLds = 4 * RowTile<D, kStepRows, 4 * kKeyRows / DKV_TN>::bytes + 2 * kStepRows * 8;

template <typename T, int D>
__device__ __forceinline__ void gradient_of_keys(const AttentionArgs &a, uint32_t id, unsigned char *lds) {
  constexpr int TN = DKV_TN, kMine = 16 * TN;
  using Tile = RowTile<D, kStepRows, 4 * kKeyRows / TN>;
  const int32_t kv = static_cast<int32_t>(id % a.kv_heads), group = a.heads / a.kv_heads;
  id /= a.kv_heads;
  const int32_t part = static_cast<int32_t>(id % a.parts), slot = static_cast<int32_t>(id / a.parts);
  const Rows rows = rows_of<kKeyRows>(a.offsets, a.sequences, a.tokens, slot);
  if (rows.at >= rows.length || rows.at < 0) return;
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const int64_t out_stride = static_cast<int64_t>(a.kv_heads) * a.dim;
  const int32_t here = rows.first + rows.at, count = min(rows.length - rows.at, kKeyRows);
  T *const dk = const_cast<T *>(at<T>(a.dk, here, out_stride, kv, a.dim)), *const dv = const_cast<T *>(at<T>(a.dv, here, out_stride, kv, a.dim));
  if (!rows.real) {
    if (part) return;
    write_zeros(dk, out_stride, count, a.dim);
    write_zeros(dv, out_stride, count, a.dim);
    return;
  }
  const int mine = wave * kMine;
  const float c = a.scale * kLog2e;
  float unit = 1.f;
  if constexpr (__is_same(T, f16)) {
    const int32_t all = a.heads + a.kv_heads, first = slot_of<kQueries>(rows.sequence, rows.first), slots = (rows.length + kQueries - 1) / kQueries;
    unit = unit_of(2.f * largest_norm(a.v_norm, all, kv * group, group, first, slots) * largest_norm(a.v_norm, all, a.heads + kv, 1, first, slots));
  }
  constexpr float kWeights = __is_same(T, f16) ? 16384.f : 1.f;       // the unit of p, at most 1 and a rounding
  s16x8 k[TN][D / 32], v[TN][D / 32];
#pragma unroll
  for (int n = 0; n < TN; ++n) {
    const int r = mine + n * 16;
    read_rows<D>(at<T>(a.k, here + r, a.k_stride, kv, a.k_head), a.k_stride, count - r, a.dim, lane, k[n]);
    read_rows<D>(at<T>(a.v, here + r, a.v_stride, kv, a.v_head), a.v_stride, count - r, a.dim, lane, v[n]);
  }
  int along0 = Tile::along(lane, 0), across0 = Tile::across(lane, 0);
  f32x4 of_k[D / 16][TN], of_v[D / 16][TN];
#pragma unroll
  for (int n = 0; n < TN; ++n)
#pragma unroll
    for (int b = 0; b < D / 16; ++b) of_k[b][n] = of_v[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
  // the queries from the tile's first key on, head after head
  const int32_t left = rows.length - rows.at;
  const int steps = (left + kStepRows - 1) / kStepRows, each = (group + a.parts - 1) / a.parts, head0 = kv * group + part * each;
  const int heads = min(each, group - part * each), all_steps = steps * max(heads, 0);
  Tile q, g;
  const unsigned char *terms;
  auto begin = [&](int head) {
    q.start(at<T>(a.q, here, a.q_stride, head0 + head, a.q_head), a.q_stride, left, a.dim);
    g.start(at<T>(a.dout, here, a.do_stride, head0 + head, a.do_head), a.do_stride, left, a.dim);
    terms = reinterpret_cast<const unsigned char *>(a.terms + static_cast<int64_t>(head0 + head) * a.tokens + here);
  };
  auto load = [&](int to) {
    if (wave == 0) {
      const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((LdsBytes *)(lds + 4 * Tile::bytes + to * kStepRows * 8)));
      load_words_to_lds(terms, static_cast<uint32_t>(max(min(q.left, kStepRows), 0)) * 8, lane * 4, at);
    }
    terms += kStepRows * 8;
    q.load(lds + to * Tile::bytes);
    g.load(lds + (2 + to) * Tile::bytes);
  };
  if (all_steps) {
    begin(0);
    load(0);
  }
  int head = 0, step = 0;
  for (int t = 0; t < all_steps; ++t) {
    meet<0>();
    const unsigned char *qs = lds + (t & 1) * Tile::bytes, *gs = qs + 2 * Tile::bytes;
    const float *ts = reinterpret_cast<const float *>(lds + 4 * Tile::bytes + (t & 1) * kStepRows * 8) + (lane >> 4) * 8;
    const int first = step * kStepRows;                                      // from the tile's first key on
    if (++step == steps) {
      step = 0;
      if (++head < heads) begin(head);
    }
    if (t + 1 < all_steps) load(~t & 1);
    if (first + kStepRows - 1 < mine) continue;                              // queries in front of all of the wave's keys
    const bool border = first < mine + kMine - 1;
    asm volatile("" : "+v"(along0), "+v"(across0));      // places are formed from these two where they are needed: registers are short
    Pack<T, 8> p[TN], ds[TN];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x4 z[TN], d[TN];
#pragma unroll
      for (int n = 0; n < TN; ++n) z[n] = d[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < D / 32; ++s) {
        const s16x8 f = Tile::read_along(qs, b * 16, along0 ^ (s << 6)), e = Tile::read_along(gs, b * 16, along0 ^ (s << 6));
#pragma unroll
        for (int n = 0; n < TN; ++n) {
          z[n] = mfma<T>(f, k[n][s], z[n]);
          d[n] = mfma<T>(e, v[n][s], d[n]);
        }
      }
      const f32x4 t0 = *reinterpret_cast<const f32x4 *>(ts + b * 32), t1 = *reinterpret_cast<const f32x4 *>(ts + b * 32 + 4);
      const float lse[4] = {t0[0], t0[2], t1[0], t1[2]}, delta[4] = {t0[1], t0[3], t1[1], t1[3]};
#pragma unroll
      for (int n = 0; n < TN; ++n) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[n][r], c, -lse[r]));
          d[n][r] = z[n][r] * (d[n][r] - delta[r]);
          if constexpr (__is_same(T, f16)) { z[n][r] *= kWeights; d[n][r] *= unit; }
        }
        if (border) {
          const int row = mine + n * 16 + (lane & 15) - first - b * 16 - (lane >> 4) * 4;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (r < row) z[n][r] = d[n][r] = 0.f;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          p[n].v[b * 4 + r] = static_cast<T>(z[n][r]);
          ds[n].v[b * 4 + r] = static_cast<T>(d[n][r]);
        }
      }
    }
#pragma unroll
    for (int b = 0; b < D / 16; ++b) {
      const s16x8 f = Tile::read_across(gs, 0, across0 ^ (b << 5)), e = Tile::read_across(qs, 0, across0 ^ (b << 5));
#pragma unroll
      for (int n = 0; n < TN; ++n) {
        of_v[b][n] = mfma<T>(f, __builtin_bit_cast(s16x8, p[n]), of_v[b][n]);
        of_k[b][n] = mfma<T>(e, __builtin_bit_cast(s16x8, ds[n]), of_k[b][n]);
      }
    }
  }
  float k_factor[TN], v_factor[TN];
#pragma unroll
  for (int n = 0; n < TN; ++n) {
    k_factor[n] = a.scale / unit;
    v_factor[n] = 1.f / kWeights;
  }
  if (a.parts == 1) {
    write_rows<T, D, TN>(of_k, k_factor, dk + mine * out_stride, nullptr, out_stride, count - mine, a.dim, lane);
    write_rows<T, D, TN>(of_v, v_factor, dv + mine * out_stride, nullptr, out_stride, count - mine, a.dim, lane);
  }
  float *const partial = a.partial + ((static_cast<int64_t>(part) * a.tokens + here) * a.kv_heads + kv) * 2 * a.dim;
  const int64_t partial_stride = static_cast<int64_t>(a.kv_heads) * 2 * a.dim;
#pragma unroll
  for (int n = 0; n < TN; ++n) {
    const int r = mine + n * 16 + (lane & 15);
    if (a.parts == 1 || r >= count) continue;
    float *to = partial + r * partial_stride;
#pragma unroll
    for (int b = 0; b < D / 16; ++b) {
      const int i = b * 16 + (lane >> 4) * 4;
      if (i >= a.dim) continue;
      *reinterpret_cast<f32x4 *>(to + i) = of_k[b][n] * k_factor[n];
      *reinterpret_cast<f32x4 *>(to + a.dim + i) = of_v[b][n] * v_factor[n];
    }
  }
  if (__syncthreads_or(any_nan<D, TN>(of_k) || any_nan<D, TN>(of_v))) {
    __syncthreads();
    const T *const k0 = at<T>(a.k, here, a.k_stride, kv, a.k_head), *const v0 = at<T>(a.v, here, a.v_stride, kv, a.v_head);
    // the queries of all heads in a row, from the tile's first key on
    sum_by_rows<2>(
        lds, count, a.dim,
        [&](int32_t r, int d) {
          const float x = a.parts == 1 ? static_cast<float>(dk[r * out_stride + d]) + static_cast<float>(dv[r * out_stride + d])
                                       : partial[r * partial_stride + d] + partial[r * partial_stride + a.dim + d];
          const float own = dot(k0 + r * a.k_stride, v0 + r * a.v_stride, a.dim);
          return x != x && own - own == 0.f;  // a key or value that is not finite has no other gradient
        },
        [&](int32_t) { return all_steps ? heads * left : 0; },
        [&](int32_t r, int32_t y, float (&w)[2]) {
          const int32_t h = head0 + y / left, i = y % left;
          if (i < r) return false;
          const float2 terms = a.terms[static_cast<int64_t>(h) * a.tokens + here + i];
          w[1] = __builtin_amdgcn_exp2f(dot(at<T>(a.q, here + i, a.q_stride, h, a.q_head), k0 + r * a.k_stride, a.dim) * c - terms.x);
          w[0] = w[1] * (dot(at<T>(a.dout, here + i, a.do_stride, h, a.do_head), v0 + r * a.v_stride, a.dim) - terms.y) * a.scale;
          return true;
        },
        [&](int e, int32_t y) {
          return e ? at<T>(a.dout, here + y % left, a.do_stride, head0 + y / left, a.do_head) : at<T>(a.q, here + y % left, a.q_stride, head0 + y / left, a.q_head);
        },
        [&](int32_t r, int d, const float (&sums)[2]) {
          if (a.parts > 1) {
            partial[r * partial_stride + d] = sums[0];
            partial[r * partial_stride + a.dim + d] = sums[1];
          } else {
            dk[r * out_stride + d] = static_cast<T>(sums[0]);
            dv[r * out_stride + d] = static_cast<T>(sums[1]);
          }
        });
  }
}

// The parts of dk and dv, in order.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionArgs a) {
  const int64_t n = static_cast<int64_t>(a.tokens) * a.kv_heads * a.dim / 4, step = static_cast<int64_t>(gridDim.x) * 256;
  const int32_t first = min(max(a.offsets[0], 0), a.tokens), end = min(max(a.offsets[a.sequences], 0), a.tokens);
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < 2 * n; i += step) {
    const int64_t row = i / (a.dim / 2), in = i % (a.dim / 2) * 4;       // of [tokens][kv_heads], 2 dim elements
    const int64_t token = row / a.kv_heads;
    if (token < first || token >= end) continue;
    f32x4 s{0.f, 0.f, 0.f, 0.f};
    for (int32_t p = 0; p < a.parts; ++p)
      s += *reinterpret_cast<const f32x4 *>(a.partial + ((static_cast<int64_t>(p) * a.tokens * a.kv_heads + row) * 2 * a.dim + in));
    T *to = in < a.dim ? static_cast<T *>(a.dk) + row * a.dim + in : static_cast<T *>(a.dv) + row * a.dim + in - a.dim;
    const float v[4] = {s[0], s[1], s[2], s[3]};
    store_pack<T, 4>(to, v);
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attention_dq_kernel(AttentionArgs a) {
  __shared__ __attribute__((aligned(256))) unsigned char lds[4 * RowTile<D, kKeys, 256>::bytes];
  gradient_of_queries<T, D>(a, blockIdx.x, lds);
}
template <typename T, int D>
__global__ __launch_bounds__(4 * kKeyRows / DKV_TN, DKV_OCC) void attention_dkv_kernel(AttentionArgs a) {
  __shared__ __attribute__((aligned(256))) unsigned char lds[kKeysLds<T, D>];
  gradient_of_keys<T, D>(a, blockIdx.x, lds);
}

template <typename T, int D>
void launch_forward(const AttentionArgs &a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(slots_of(a.tokens, a.sequences, kQueries) * a.heads)), block(256);
  if (a.rest) hipLaunchKernelGGL((attention_forward_kernel<T, D, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((attention_forward_kernel<T, D, false>), grid, block, 0, s, a);
}
template <typename T, int D>
void launch_backward(const AttentionArgs &a, hipStream_t s) {
  const int64_t slots = slots_of(a.tokens, a.sequences, kQueries), all = a.heads + (__is_same(T, f16) ? a.kv_heads : 0);
  hipLaunchKernelGGL((attention_delta_kernel<T, D>), dim3(static_cast<uint32_t>(slots * all)), dim3(256), 0, s, a);
  hipLaunchKernelGGL((attention_dkv_kernel<T, D>), dim3(static_cast<uint32_t>(slots_of(a.tokens, a.sequences, kKeyRows) * a.kv_heads * a.parts)), dim3(4 * kKeyRows / DKV_TN), 0, s, a);
  if (a.parts > 1) hipLaunchKernelGGL((attention_join_kernel<T>), dim3(2048), dim3(256), 0, s, a);
  hipLaunchKernelGGL((attention_dq_kernel<T, D>), dim3(static_cast<uint32_t>(slots * a.heads)), dim3(256), 0, s, a);
}
template <typename T>
void launch(const AttentionArgs &a, bool backward, hipStream_t s) {
  if (a.dim <= 64) backward ? launch_backward<T, 64>(a, s) : launch_forward<T, 64>(a, s);
  else backward ? launch_backward<T, 128>(a, s) : launch_forward<T, 128>(a, s);
}
void launch_type(const AttentionArgs &a, int32_t type, bool backward, hipStream_t s) {
  if (type == ONES_F16) launch<f16>(a, backward, s);
  else launch<bf16>(a, backward, s);
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

int ones_attention_forward(const void *q, int64_t q_stride, int64_t q_head_stride, const void *k, int64_t k_stride, int64_t k_head_stride,
                           const void *v, int64_t v_stride, int64_t v_head_stride, int64_t tokens, int64_t heads, int64_t kv_heads,
                           int64_t dim, int32_t type, const int32_t *offsets, int64_t sequences, float scale, void *o, void *rest,
                           float *lse, void *hip_stream) {
  if (int rc = check_attention(tokens, heads, kv_heads, dim, type, sequences, scale)) return rc;
  if (tokens == 0) return ONES_OK;
  if (int rc = check_head_rows(q, q_stride, q_head_stride, heads, dim)) return rc;
  if (int rc = check_head_rows(k, k_stride, k_head_stride, kv_heads, dim)) return rc;
  if (int rc = check_head_rows(v, v_stride, v_head_stride, kv_heads, dim)) return rc;
  if (!offsets || !o || !lse || !aligned(o, 16) || !aligned(rest, 16)) return ONES_E_INVALID_ARG;
  AttentionArgs a{};
  a.q = q; a.k = k; a.v = v;
  a.q_stride = q_stride; a.q_head = q_head_stride; a.k_stride = k_stride; a.k_head = k_head_stride; a.v_stride = v_stride; a.v_head = v_head_stride;
  a.o = o; a.rest = rest; a.lse = lse; a.offsets = offsets;
  a.sequences = static_cast<int32_t>(sequences); a.tokens = static_cast<int32_t>(tokens); a.heads = static_cast<int32_t>(heads);
  a.kv_heads = static_cast<int32_t>(kv_heads); a.dim = static_cast<int32_t>(dim); a.scale = scale;
  launch_type(a, type, false, static_cast<hipStream_t>(hip_stream));
  return launched("attention forward");
}

size_t ones_attention_workspace_bytes(int64_t tokens, int64_t sequences, int64_t heads, int64_t kv_heads, int64_t dim) {
  if (check_attention(tokens, heads, kv_heads, dim, ONES_F16, sequences, 1.f)) return 0;
  return attention_plan(tokens, sequences, heads, kv_heads, dim).bytes;
}

int ones_attention_backward(const void *dout, int64_t do_stride, int64_t do_head_stride, const void *q, int64_t q_stride, int64_t q_head_stride,
                            const void *k, int64_t k_stride, int64_t k_head_stride, const void *v, int64_t v_stride, int64_t v_head_stride,
                            int64_t tokens, int64_t heads, int64_t kv_heads, int64_t dim, int32_t type, const int32_t *offsets,
                            int64_t sequences, float scale, const void *o, const void *rest, const float *lse, void *dq, void *dk, void *dv,
                            void *d_workspace, size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_attention(tokens, heads, kv_heads, dim, type, sequences, scale)) return rc;
  if (tokens == 0) return ONES_OK;
  if (int rc = check_head_rows(dout, do_stride, do_head_stride, heads, dim)) return rc;
  if (int rc = check_head_rows(q, q_stride, q_head_stride, heads, dim)) return rc;
  if (int rc = check_head_rows(k, k_stride, k_head_stride, kv_heads, dim)) return rc;
  if (int rc = check_head_rows(v, v_stride, v_head_stride, kv_heads, dim)) return rc;
  if (!offsets || !o || !lse || !dq || !dk || !dv) return ONES_E_INVALID_ARG;
  if (!aligned(o, 16) || !aligned(rest, 16) || !aligned(dq, 16) || !aligned(dk, 16) || !aligned(dv, 16)) return ONES_E_INVALID_ARG;
  const AttentionPlan plan = attention_plan(tokens, sequences, heads, kv_heads, dim);
  if (int rc = check_workspace(d_workspace, workspace_bytes, plan.bytes)) return rc;
  AttentionArgs a{};
  a.dout = dout; a.q = q; a.k = k; a.v = v;
  a.do_stride = do_stride; a.do_head = do_head_stride;
  a.q_stride = q_stride; a.q_head = q_head_stride; a.k_stride = k_stride; a.k_head = k_head_stride; a.v_stride = v_stride; a.v_head = v_head_stride;
  a.o = const_cast<void *>(o); a.rest = const_cast<void *>(rest); a.lse = const_cast<float *>(lse); a.offsets = offsets;
  a.dq = dq; a.dk = dk; a.dv = dv;
  unsigned char *const w = static_cast<unsigned char *>(d_workspace);
  a.terms = reinterpret_cast<float2 *>(w + plan.terms);
  a.partial = reinterpret_cast<float *>(w + plan.partial);
  a.parts = static_cast<int32_t>(plan.parts);
  a.dout_norm = reinterpret_cast<float *>(w + plan.dout_norm);
  a.v_norm = reinterpret_cast<float *>(w + plan.slot_norms);
  a.sequences = static_cast<int32_t>(sequences); a.tokens = static_cast<int32_t>(tokens); a.heads = static_cast<int32_t>(heads);
  a.kv_heads = static_cast<int32_t>(kv_heads); a.dim = static_cast<int32_t>(dim); a.scale = scale;
  launch_type(a, type, true, static_cast<hipStream_t>(hip_stream));
  return launched("attention backward");
}

}  // extern "C"

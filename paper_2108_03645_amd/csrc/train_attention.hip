// Causal attention over packed sequences, query heads in groups that share a key head, with its gradients (ones_attention_*).
//
//   z_ij = scale q_i . k_j for j <= i, lse_i = log sum_j exp z_ij, p_ij = exp(z_ij - lse_i), o_i = sum_j p_ij v_j
//   delta_i = do_i . o_i, ds_ij = p_ij (do_i . v_j - delta_i)
//   dv_j = sum_i p_ij do_i, dk_j = scale sum_i ds_ij q_i (both over the heads of a group, too), dq_i = scale sum_j ds_ij k_j
//
// A workgroup takes 128 queries (64 where these would be too few workgroups) of one head and walks along the keys that they see, 64 (or 32) at a
// step: keys and values come to LDS by direct loads into two places in turn, a wave keeps its 32 (16) queries, the largest score so far, the sum
// of exponentials and o in registers.  Keys are the rows of the first product and the k of the second, so that exponentials go from one to the
// other where they are.  Queries that end late are begun first.
//
// Exponentials are rounded to the operands' type for the product with the values: o is off by about as much again as by its own rounding.
// For the gradients that is too much: delta_i = do_i . o_i is subtracted from numbers of its own size, and dq of short sequences would be off by
// three times its rounding.  With `rest` wanted, what the rounding takes from the exponentials goes through a second product, and
// what it takes from o is left behind.
//
// What bounds it: the matrix units, the exponentials, of which little hides behind them, and the power that both draw.  16384 tokens, 16 heads over 2 of 128, bf16: 1.01 to 1.09 ms, 1.0 to 1.1 PFLOP/s of the causal half (the same of zeros: 0.90 ms;
// a library product of 8192 cubed: 1.27 to 1.35 PFLOP/s, of zeros 1.75); the matrix units are busy half of the cycles, the vector units 60 %, LDS
// 25 %.  16 x 2048 tokens with `rest`: 0.47 ms.  Tried and not kept: four waves a SIMD with 16 queries each (1.17 ms), scores a run ahead
// of the exponentials (1.10), wave priorities (1.08), groups of instructions set by hand (1.10 to 1.19).
#include "train_attention_sequences.h"

namespace ones {
namespace train {
namespace {

template <typename T, int D, int TN, bool REST>
__global__ __launch_bounds__(256, 2) void attention_forward_kernel(AttentionArgs a) {
  constexpr int kThreads = 256, kMine = 16 * TN, kRows = 4 * kMine;
  constexpr int kStep = kKeys<TN>, kHalves = kStep / 32;                    // keys of a step, and runs of 32 of them
  using Tile = RowTile<D, kStep, kThreads>;
  __shared__ __attribute__((aligned(256))) unsigned char lds[4 * Tile::bytes];
  const Turn turn = turn_of(blockIdx.x, a.heads, a.kv_heads);
  const int32_t last_slot = static_cast<int32_t>(slots_of(a.tokens, a.sequences, kRows)) - 1;
  const Rows rows = rows_of<kRows>(a.offsets, a.sequences, a.tokens, last_slot - turn.slot);      // the longest tiles first
  if (rows.at >= rows.length || rows.at < 0) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t out_stride = static_cast<int64_t>(a.heads) * a.dim;
  const int32_t here = rows.first + rows.at, count = min(rows.length - rows.at, kRows);
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
  const int steps = (rows.at + count + kStep - 1) / kStep, first_row = rows.at + mine;
  for (int step = 0; step < steps; ++step) {
    meet<0>();
    const unsigned char *ks = lds + (step & 1) * Tile::bytes, *vs = ks + 2 * Tile::bytes;
    if (step + 1 < steps) {
      k.load(lds + (~step & 1) * Tile::bytes);
      v.load(lds + (2 + (~step & 1)) * Tile::bytes);
    }
    const int key = step * kStep;
    if (key > first_row + kMine - 1) continue;       // keys behind all of the wave's rows
    // LDS answers after some hundred cycles: every read is issued ahead of its product, eight of them before the first; those of the values
    // before the exponentials.
    constexpr int kSteps = D / 32, kBlocks = D / 16, kReads = 2 * kHalves * kSteps, kAhead = kReads < 8 ? kReads : 8;
    s16x8 f[kAhead], fs[kBlocks];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) f[i] = Tile::read_along(ks, i / kSteps * 16, along[i % kSteps]);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 z[2 * kHalves][TN];
#pragma unroll
    for (int b = 0; b < 2 * kHalves; ++b) {
#pragma unroll
      for (int n = 0; n < TN; ++n) z[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int i = b * kSteps + s, next = i + kAhead;
#pragma unroll
        for (int n = 0; n < TN; ++n) z[b][n] = mfma<T>(f[i % kAhead], q[n][s], z[b][n]);
        if (next < kReads) f[i % kAhead] = Tile::read_along(ks, next / kSteps * 16, along[next % kSteps]);
        else if (next - kReads < kBlocks) fs[next - kReads] = Tile::read_across(vs, 0, across[next - kReads]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (key + kStep - 1 > first_row) {
#pragma unroll
      for (int n = 0; n < TN; ++n) {
        const int row = first_row + n * 16 + (lane & 15) - key;
#pragma unroll
        for (int b = 0; b < 2 * kHalves; ++b)
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
      float m[kHalves];
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        m[h] = fmaxf(z[h][n][0], z[h][n][1]);
        m[h] = fmaxf(fmaxf(m[h], z[h][n][2]), z[h][n][3]);
        m[h] = fmaxf(fmaxf(m[h], z[kHalves + h][n][0]), z[kHalves + h][n][1]);
        m[h] = fmaxf(fmaxf(m[h], z[kHalves + h][n][2]), z[kHalves + h][n][3]);
      }
      most[n] = across_max(fmaxf(m[0], m[kHalves - 1]));
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
    s16x8 p[kHalves][TN], lost[kHalves][TN];              // lost: what the rounding takes from the exponentials
#pragma unroll
    for (int n = 0; n < TN; ++n) {
      const float base = (top[n] == -INFINITY ? 0.f : top[n] * c) - kShift<T>;
      float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int b = 0; b < 2 * kHalves; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[b][n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][n][r], c, -base));
          sums[r] += z[b][n][r];
        }
      sum[n] += (sums[0] + sums[1]) + (sums[2] + sums[3]);
#pragma unroll
      for (int h = 0; h < kHalves; ++h) {
        p[h][n] = rounded<T>(z[2 * h][n], z[2 * h + 1][n]);
        if constexpr (REST) lost[h][n] = remainder<T>(z[2 * h][n], z[2 * h + 1][n], p[h][n]);
      }
    }
#pragma unroll
    for (int i = 0; i < kHalves * kBlocks; ++i) {
      const int h = i / kBlocks, b = i % kBlocks;
#pragma unroll
      for (int n = 0; n < TN; ++n) {
        acc[b][n] = mfma<T>(fs[b], p[h][n], acc[b][n]);
        if constexpr (REST) acc[b][n] = mfma<T>(fs[b], lost[h][n], acc[b][n]);
      }
      if (h + 1 < kHalves) fs[b] = Tile::read_across(vs, 32, across[b]);
      __builtin_amdgcn_sched_barrier(0);
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
        lds, count, a.dim,
        [&, seen = Seen()](int32_t r, int d) mutable {
          const float x = static_cast<float>(o[r * out_stride + d]);
          if (x == x || lse[r] != lse[r]) return false;
          seen.through(v0, a.v_stride, rows.at + r, d);
          if (seen.no_number()) return false;         // NaN is right: every weight is above 0
          if (seen.finite()) return true;
          o[r * out_stride + d] = static_cast<T>(seen.up() ? __builtin_inff() : -__builtin_inff());
          if (rest) rest[r * out_stride + d] = static_cast<T>(0.f);
          return false;
        },
        [&](int32_t r) { return rows.at + r + 1; },
        [&](int32_t r, int32_t y, float (&w)[1]) {
          w[0] = __builtin_amdgcn_exp2f(dot(q0 + r * a.q_stride, k0 + y * a.k_stride, a.dim) * c - lse[r] * kLog2e);
          return true;
        },
        [&](int, int32_t y) { return v0 + y * a.v_stride; },
        [&](int32_t r, int d, const float (&sums)[1], int) {
          o[r * out_stride + d] = static_cast<T>(sums[0]);
          if (rest) rest[r * out_stride + d] = static_cast<T>(lost<T>(sums[0]));
        });
  }
}

template <typename T, int D, int TN>
void launch_rows(const AttentionArgs &a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(slots_of(a.tokens, a.sequences, 64 * TN) * a.heads)), block(256);
  if (a.rest) hipLaunchKernelGGL((attention_forward_kernel<T, D, TN, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((attention_forward_kernel<T, D, TN, false>), grid, block, 0, s, a);
}
template <typename T, int D>
void launch(const AttentionArgs &a, hipStream_t s) {
  attention_few(a.tokens, a.heads) ? launch_rows<T, D, 1>(a, s) : launch_rows<T, D, 2>(a, s);
}
template <typename T>
void launch(const AttentionArgs &a, hipStream_t s) {
  if (a.dim <= 32) return launch<T, 32>(a, s);
  if (a.dim <= 64) return launch<T, 64>(a, s);
  if (a.dim <= 96) return launch<T, 96>(a, s);
  launch<T, 128>(a, s);
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
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  type == ONES_F16 ? launch<f16>(a, s) : launch<bf16>(a, s);
  return launched("attention forward");
}

}  // extern "C"

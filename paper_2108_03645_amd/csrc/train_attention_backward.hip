// The gradients of causal attention over packed sequences (ones_attention_backward; the formulas stand in train_attention.hip).
//
// Scores and their gradients are formed twice, by workgroups that own 64 keys and walk along the queries and by others that own 64 queries and walk
// along the keys: seven products instead of five, but every sum has one owner and a fixed order.  Both are one launch.  dk and dv of a
// key head are sums over the query heads of its group, which follow each other in the same workgroup; where that leaves too few
// workgroups the group is parted and a last launch adds the parts up.  A first launch forms delta.
//
// A wave keeps the 16 rows that it owns, and their sums, in registers, and reads the other side from LDS along and across its rows.  Three waves a
// SIMD fit then; with 32 keys a wave it is two, whose registers spill (the keys' part alone, sizes as below: 754 us against 720).  In fp16 the
// scores' gradients are held in units that follow from the norms of do and v (unit_of()).
//
// What bounds it: the matrix units are busy 48 % of the cycles, LDS 51 % (every row of the other side is read for 16 of this one), the vector units 46 %; waits
// between them are the rest.  16 x 2048 tokens, 16 heads over 2 of 128, bf16: delta 74 us (402 MB, 5.5 TB/s), gradients 1.03 to 1.06 ms (0.91 to 0.94
// PFLOP/s of seven products), the parts' sums 30 us.
#include "train_attention_sequences.h"

namespace ones {
namespace train {
namespace {

// delta of every row of a slot and head, and its |do|; of a key head, the largest |v|.  (fp16 scales by the norms, see unit_of().)
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_delta_kernel(AttentionArgs a) {
  constexpr int lanes = kPieces<D>, at_once = 256 / lanes;
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

// The unit that ds is held in where it is rounded to fp16: a power of two that brings |ds| <= 2 |do| |v| to at most 2^14.  |do| is a query's own, for keys
// the largest of the queries from their slot on, |v| the largest up to a query's slot, for keys of the sequence; what is more than 2^27 below such
// a bound loses bits.  (bf16 has the exponents of 32 bits: 1.)
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
  constexpr int kMine = 16, kRows = 4 * kMine, kStep = kKeys<1>;
  static_assert(kStep == 32);
  using Tile = RowTile<D, kStep, 256>;
  const Turn turn = turn_of(id, a.heads, a.kv_heads);
  const int32_t slot = static_cast<int32_t>(slots_of(a.tokens, a.sequences, kRows)) - 1 - turn.slot;
  const Rows rows = rows_of<kRows>(a.offsets, a.sequences, a.tokens, slot);
  if (rows.at >= rows.length || rows.at < 0) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t out_stride = static_cast<int64_t>(a.heads) * a.dim;
  const int32_t here = rows.first + rows.at, count = min(rows.length - rows.at, kRows);
  T *const dq = const_cast<T *>(at<T>(a.dq, here, out_stride, turn.head, a.dim));
  if (!rows.real) return write_zeros(dq, out_stride, count, a.dim);
  Tile k, v;
  k.start(at<T>(a.k, rows.first, a.k_stride, turn.kv, a.k_head), a.k_stride, rows.length, a.dim);
  v.start(at<T>(a.v, rows.first, a.v_stride, turn.kv, a.v_head), a.v_stride, rows.length, a.dim);
  k.load(lds);
  v.load(lds + 2 * Tile::bytes);
  const int mine = wave * kMine;
  const float c = a.scale * kLog2e;
  float v_most = 0.f;
  if constexpr (__is_same(T, f16)) {
    const int32_t all = a.heads + a.kv_heads;
    v_most = largest_norm(a.v_norm, all, a.heads + turn.kv, 1, slot_of<kQueries>(rows.sequence, rows.first), (rows.at + count + kQueries - 1) / kQueries);
  }
  s16x8 q[D / 32], g[D / 32];
  read_rows<D>(at<T>(a.q, here + mine, a.q_stride, turn.head, a.q_head), a.q_stride, count - mine, a.dim, lane, q);
  read_rows<D>(at<T>(a.dout, here + mine, a.do_stride, turn.head, a.do_head), a.do_stride, count - mine, a.dim, lane, g);
  const int64_t term = static_cast<int64_t>(turn.head) * a.tokens + here + min(mine + (lane & 15), count - 1);
  const float lse = a.terms[term].x, delta = a.terms[term].y;
  float unit = 1.f;
  if constexpr (__is_same(T, f16)) unit = unit_of(2.f * a.dout_norm[term] * v_most);
  const float factor[1] = {a.scale / unit};
  int along[D / 32], across[D / 16];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) along[s] = Tile::along(lane, s);
#pragma unroll
  for (int b = 0; b < D / 16; ++b) across[b] = Tile::across(lane, b);
  f32x4 acc[D / 16][1];
#pragma unroll
  for (int b = 0; b < D / 16; ++b) acc[b][0] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = (rows.at + count + kStep - 1) / kStep, first_row = rows.at + mine;
  for (int step = 0; step < steps; ++step) {
    meet<0>();
    const unsigned char *ks = lds + (step & 1) * Tile::bytes, *vs = ks + 2 * Tile::bytes;
    if (step + 1 < steps) {
      k.load(lds + (~step & 1) * Tile::bytes);
      v.load(lds + (2 + (~step & 1)) * Tile::bytes);
    }
    // reads ahead of their products, as in gradient_of_keys
    constexpr int kSteps = D / 32, kBlocks = D / 16, kAhead = D == 96 ? 3 : D == 32 ? 2 : 4, kEach = (kAhead + kSteps - 1) / kSteps;
    s16x8 f[kSteps], e[kSteps], fs[kAhead];
    const auto rows_at = [&](int b, int s) {
      f[s] = Tile::read_along(ks, b * 16, along[s]);
      e[s] = Tile::read_along(vs, b * 16, along[s]);
    };
    const int key = step * kStep;
    if (key > first_row + kMine - 1) continue;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) rows_at(0, s);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 z[2], d[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      z[b] = d[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        z[b] = mfma<T>(f[s], q[s], z[b]);
        d[b] = mfma<T>(e[s], g[s], d[b]);
        if (b == 0) rows_at(1, s);
        else
#pragma unroll
          for (int i = s * kEach; i < min((s + 1) * kEach, kAhead); ++i) fs[i] = Tile::read_across(ks, 0, across[i]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][r], c, -lse));
        z[b][r] = p * (d[b][r] - delta);
        if constexpr (__is_same(T, f16)) z[b][r] *= unit;
      }
    if (key + kStep - 1 > first_row) {
      const int row = first_row + (lane & 15) - key;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (b * 16 + (lane >> 4) * 4 + r > row) z[b][r] = 0.f;
    }
    const s16x8 ds = rounded<T>(z[0], z[1]);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      acc[b][0] = mfma<T>(fs[b % kAhead], ds, acc[b][0]);
      if (b + kAhead < kBlocks) fs[b % kAhead] = Tile::read_across(ks, 0, across[b + kAhead]);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  write_rows<T, D, 1>(acc, factor, dq + mine * out_stride, nullptr, out_stride, count - mine, a.dim, lane);
  if (__syncthreads_or(any_nan<D, 1>(acc))) {
    __syncthreads();
    const T *const q0 = at<T>(a.q, here, a.q_stride, turn.head, a.q_head), *const k0 = at<T>(a.k, rows.first, a.k_stride, turn.kv, a.k_head);
    const T *const g0 = at<T>(a.dout, here, a.do_stride, turn.head, a.do_head), *const v0 = at<T>(a.v, rows.first, a.v_stride, turn.kv, a.v_head);
    const float2 *const terms = a.terms + static_cast<int64_t>(turn.head) * a.tokens + here;
    sum_by_rows<1>(
        lds, count, a.dim,
        [&, seen = Seen()](int32_t r, int d) mutable {
          const float x = static_cast<float>(dq[r * out_stride + d]), t = terms[r].x + terms[r].y;
          if (x == x || t - t != 0.f) return false;
          const int32_t i = rows.at + r, end = min(i / kStep * kStep + kStep, rows.length);
          if (!any_infinite(k0, a.k_stride, i + 1, end, d)) return false;
          // infinite or NaN in a key makes its score so, and this element NaN, for the rows that see it
          if (seen.finite()) seen.through(k0, a.k_stride, i, d);
          return seen.finite();
        },
        [&](int32_t r) { return rows.at + r + 1; },
        [&](int32_t r, int32_t y, float (&w)[1]) {
          const float p = __builtin_amdgcn_exp2f(dot(q0 + r * a.q_stride, k0 + y * a.k_stride, a.dim) * c - terms[r].x);
          w[0] = p * (dot(g0 + r * a.do_stride, v0 + y * a.v_stride, a.dim) - terms[r].y);
          return true;
        },
        [&](int, int32_t y) { return k0 + y * a.k_stride; },
        [&](int32_t r, int d, const float (&sums)[1], int) { dq[r * out_stride + d] = static_cast<T>(sums[0] * a.scale); });
  }
}

constexpr int kStepRows = 32, kKeyRows = kAttentionKeys;        // of the keys' gradients: queries of a step; keys of a workgroup

template <typename T, int D>
constexpr int kKeysLds = 4 * RowTile<D, kStepRows, 4 * kKeyRows>::bytes + 2 * kStepRows * 8;

template <typename T, int D>
__device__ __forceinline__ void gradient_of_keys(const AttentionArgs &a, uint32_t id, unsigned char *lds) {
  constexpr int kMine = 16;
  using Tile = RowTile<D, kStepRows, 4 * kKeyRows>;
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
    const int32_t front = rows.at / kQueries;        // slots whose queries do not see the tile's keys; the others' o has values of all
    unit = unit_of(2.f * largest_norm(a.v_norm, all, kv * group, group, first + front, slots - front) * largest_norm(a.v_norm, all, a.heads + kv, 1, first, slots));
  }
  constexpr float kWeights = __is_same(T, f16) ? 16384.f : 1.f;       // the unit of p, at most 1 and a rounding
  s16x8 k[D / 32], v[D / 32];
  read_rows<D>(at<T>(a.k, here + mine, a.k_stride, kv, a.k_head), a.k_stride, count - mine, a.dim, lane, k);
  read_rows<D>(at<T>(a.v, here + mine, a.v_stride, kv, a.v_head), a.v_stride, count - mine, a.dim, lane, v);
  int along0 = Tile::along(lane, 0), across0 = Tile::across(lane, 0);
  f32x4 of_k[D / 16][1], of_v[D / 16][1];
#pragma unroll
  for (int b = 0; b < D / 16; ++b) of_k[b][0] = of_v[b][0] = f32x4{0.f, 0.f, 0.f, 0.f};
  // The queries from the tile's first key on, the last ones first, of all heads before the next ones: the workgroups of a sequence end at different
  // queries but begin at the same ones, so that they read the same rows at the same time, which then come from L2 (head after head
  // from the first query on, 16 x 2048 x 16 over 2 x 128 read 4 GB from behind L2).
  const int32_t left = rows.length - rows.at;
  const int steps = (left + kStepRows - 1) / kStepRows, each = (group + a.parts - 1) / a.parts, head0 = kv * group + part * each;
  const int heads = min(each, group - part * each), all_steps = steps * max(heads, 0);
  Tile q, g;
  q.start(at<T>(a.q, here, a.q_stride, head0, a.q_head), a.q_stride, left, a.dim);
  g.start(at<T>(a.dout, here, a.do_stride, head0, a.do_head), a.do_stride, left, a.dim);
  const unsigned char *const q0 = q.base, *const g0 = g.base, *const terms0 = reinterpret_cast<const unsigned char *>(a.terms + static_cast<int64_t>(head0) * a.tokens + here);
  auto load = [&](int to, int step, int head) {
    const int64_t row = step * kStepRows;
    q.left = g.left = left - step * kStepRows;
    q.base = q0 + row * q.row_bytes + head * a.q_head * 2;
    g.base = g0 + row * g.row_bytes + head * a.do_head * 2;
    if (wave == 0) {
      const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((LdsBytes *)(lds + 4 * Tile::bytes + to * kStepRows * 8)));
      load_words_to_lds(terms0 + (row + static_cast<int64_t>(head) * a.tokens) * 8, static_cast<uint32_t>(min(q.left, kStepRows)) * 8, lane * 4, at);
    }
    q.load(lds + to * Tile::bytes);
    g.load(lds + (2 + to) * Tile::bytes);
  };
  int head = 0, step = steps - 1;
  if (all_steps) load(0, step, 0);
  for (int t = 0; t < all_steps; ++t) {
    meet<0>();
    const unsigned char *qs = lds + (t & 1) * Tile::bytes, *gs = qs + 2 * Tile::bytes;
    const float *ts = reinterpret_cast<const float *>(lds + 4 * Tile::bytes + (t & 1) * kStepRows * 8) + (lane >> 4) * 8;
    const int first = step * kStepRows;                                      // from the tile's first key on
    if (++head == heads) {
      head = 0;
      --step;
    }
    if (t + 1 < all_steps) load(~t & 1, step, head);
    if (first + kStepRows - 1 < mine) continue;                              // queries in front of all of the wave's keys
    const bool border = first < mine + kMine - 1;
    asm volatile("" : "+v"(along0), "+v"(across0));      // places are formed from these two where they are needed: registers are short
    // LDS answers after some hundred cycles, so every read is issued a phase ahead of its product, in this order: what the products of the
    // second 16 queries need between those of the first, what those across the rows need between those of the second.
    constexpr int kSteps = D / 32, kBlocks = D / 16, kAhead = D > 64 ? 3 : D == 32 ? 2 : 4, kEach = (kAhead + kSteps - 1) / kSteps;
    s16x8 f[kSteps], e[kSteps], fs[kAhead], es[kAhead];
    Pack<T, 8> p, ds;
    const auto rows_at = [&](int b, int s) {
      f[s] = Tile::read_along(qs, b * 16, along0 ^ (s << 6));
      e[s] = Tile::read_along(gs, b * 16, along0 ^ (s << 6));
    };
    const auto block_at = [&](int b) {
      fs[b % kAhead] = Tile::read_across(gs, 0, across0 ^ (b << 5));
      es[b % kAhead] = Tile::read_across(qs, 0, across0 ^ (b << 5));
    };
#pragma unroll
    for (int s = 0; s < kSteps; ++s) rows_at(0, s);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32x4 z{0.f, 0.f, 0.f, 0.f}, d = z;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        z = mfma<T>(f[s], k[s], z);
        d = mfma<T>(e[s], v[s], d);
        if (b == 0) rows_at(1, s);
        else
#pragma unroll
          for (int i = s * kEach; i < min((s + 1) * kEach, kAhead); ++i) block_at(i);
        __builtin_amdgcn_sched_barrier(0);
      }
      const f32x4 t0 = *reinterpret_cast<const f32x4 *>(ts + b * 32), t1 = *reinterpret_cast<const f32x4 *>(ts + b * 32 + 4);
      const float lse[4] = {t0[0], t0[2], t1[0], t1[2]}, delta[4] = {t0[1], t0[3], t1[1], t1[3]};
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        z[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[r], c, -lse[r]));
        d[r] = z[r] * (d[r] - delta[r]);
        if constexpr (__is_same(T, f16)) { z[r] *= kWeights; d[r] *= unit; }
      }
      if (border) {
        const int row = mine + (lane & 15) - first - b * 16 - (lane >> 4) * 4;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (r < row) z[r] = d[r] = 0.f;
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        p.v[b * 4 + r] = static_cast<T>(z[r]);
        ds.v[b * 4 + r] = static_cast<T>(d[r]);
      }
    }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      of_v[b][0] = mfma<T>(fs[b % kAhead], __builtin_bit_cast(s16x8, p), of_v[b][0]);
      of_k[b][0] = mfma<T>(es[b % kAhead], __builtin_bit_cast(s16x8, ds), of_k[b][0]);
      if (b + kAhead < kBlocks) block_at(b + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  const float k_factor[1] = {a.scale / unit}, v_factor[1] = {1.f / kWeights};
  if (a.parts == 1) {
    write_rows<T, D, 1>(of_k, k_factor, dk + mine * out_stride, nullptr, out_stride, count - mine, a.dim, lane);
    write_rows<T, D, 1>(of_v, v_factor, dv + mine * out_stride, nullptr, out_stride, count - mine, a.dim, lane);
  }
  float *const partial = a.partial + ((static_cast<int64_t>(part) * a.tokens + here) * a.kv_heads + kv) * 2 * a.dim;
  const int64_t partial_stride = static_cast<int64_t>(a.kv_heads) * 2 * a.dim;
  if (const int r = mine + (lane & 15); a.parts > 1 && r < count) {
    float *const to = partial + r * partial_stride;
#pragma unroll
    for (int b = 0; b < D / 16; ++b) {
      const int i = b * 16 + (lane >> 4) * 4;
      if (i >= a.dim) continue;
      *reinterpret_cast<f32x4 *>(to + i) = of_k[b][0] * k_factor[0];
      *reinterpret_cast<f32x4 *>(to + a.dim + i) = of_v[b][0] * v_factor[0];
    }
  }
  if (__syncthreads_or(any_nan<D, 1>(of_k) || any_nan<D, 1>(of_v))) {
    __syncthreads();
    const T *const k0 = at<T>(a.k, here, a.k_stride, kv, a.k_head), *const v0 = at<T>(a.v, here, a.v_stride, kv, a.v_head);
    const auto is_nan = [](auto x) { const float v = static_cast<float>(x); return v != v ? 1 : 0; };
    // What the queries from .. to - 1 of all heads hold: NaN in lse, which makes both results of a key that sees it NaN, and in delta, all of dk; and what is not
    // finite in element d of do, which goes into that element of dv.
    struct Held {
      uint32_t lse, delta;                    // as Seen::size
      Seen dout;
    };
    auto look = [&](int32_t from, int32_t to, int d, Held held) __attribute__((always_inline)) {
      for (int32_t h = head0; h < head0 + heads; ++h) {
        const float2 *const terms = a.terms + static_cast<int64_t>(h) * a.tokens + here;
        for (int32_t i = from; i < to && held.lse <= 0x7f800000; i += 4)
#pragma unroll
          for (int n = 0; n < 4; ++n) {
            const float2 t = terms[min(i + n, to - 1)];
            held.lse = max(held.lse, __float_as_uint(t.x) & 0x7fffffff);
            held.delta = max(held.delta, __float_as_uint(t.y) & 0x7fffffff);
          }
        held.dout.next = from;
        held.dout.through(at<T>(a.dout, here, a.do_stride, h, a.do_head), a.do_stride, to - 1, d);
      }
      return held;
    };
    // the queries of all heads in a row, from the tile's first key on
    sum_by_rows<2>(
        lds, count, a.dim,
        [&, behind = Held{}, looked = false](int32_t r, int d) mutable {
          // which of dk and dv are NaN
          const int nan = a.parts == 1 ? is_nan(dk[r * out_stride + d]) + 2 * is_nan(dv[r * out_stride + d])
                                       : is_nan(partial[r * partial_stride + d]) + 2 * is_nan(partial[r * partial_stride + a.dim + d]);
          if (!nan) return 0;
          // from queries and gradients that the key does not see, in the one step that it shares with them
          int asks = 0;
          const int32_t step = r / kStepRows * kStepRows;
          for (int32_t h = head0; h < head0 + heads; ++h) {
            if (nan & 1) asks |= any_infinite(at<T>(a.q, here, a.q_stride, h, a.q_head), a.q_stride, step, r, d) ? 1 : 0;
            if (nan & 2) asks |= any_infinite(at<T>(a.dout, here, a.do_stride, h, a.do_head), a.do_stride, step, r, d) ? 2 : 0;
          }
          const int32_t tile = min(kKeyRows, left);
          Held held = behind;                   // of the queries behind the tile, which all of its keys see; looked for once
#pragma unroll 1
          for (int turn = looked; turn < 2; ++turn) {
            held = look(turn ? r : tile, turn ? tile : left, d, held);
            if (turn == 0) behind = held;
          }
          looked = true;
          if ((nan & 2) && held.lse <= 0x7f800000 && held.dout.infinite()) {        // also where weights are 0 in 32 bits
            const float all = held.dout.up() ? __builtin_inff() : -__builtin_inff();
            if (a.parts == 1) dv[r * out_stride + d] = static_cast<T>(all);
            else partial[r * partial_stride + a.dim + d] = all;
          }
          // The rows behind the sequence that its last step has are zeros, but their scores with a key that has infinities NaN: where all that the key
          // sees is finite, its own scores were -infinity.
          if (left % kStepRows && max(held.lse, held.delta) < 0x7f800000) asks = nan;
          return held.lse > 0x7f800000 ? 0 : asks & ((held.delta <= 0x7f800000 ? 1 : 0) | (held.dout.finite() ? 2 : 0));
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
        [&](int32_t r, int d, const float (&sums)[2], int asks) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (!(asks >> e & 1)) continue;
            if (a.parts > 1) partial[r * partial_stride + e * a.dim + d] = sums[e];
            else (e ? dv : dk)[r * out_stride + d] = static_cast<T>(sums[e]);
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

// The gradients of keys and queries side by side, the first `keys` workgroups those of the keys: each fills what the other leaves idle.
template <typename T, int D>
__global__ __launch_bounds__(256, 3) void attention_gradients_kernel(AttentionArgs a, uint32_t keys) {
  constexpr int queries = 4 * RowTile<D, kKeys<1>, 256>::bytes, bytes = queries > kKeysLds<T, D> ? queries : kKeysLds<T, D>;
  __shared__ __attribute__((aligned(256))) unsigned char lds[bytes];
  if (blockIdx.x < keys) gradient_of_keys<T, D>(a, blockIdx.x, lds);
  else gradient_of_queries<T, D>(a, blockIdx.x - keys, lds);
}

template <typename T, int D>
void launch(const AttentionArgs &a, hipStream_t s) {
  const int64_t slots = slots_of(a.tokens, a.sequences, kQueries), half_slots = slots_of(a.tokens, a.sequences, 64);
  const int64_t all = a.heads + (__is_same(T, f16) ? a.kv_heads : 0);
  const uint32_t keys = static_cast<uint32_t>(half_slots * a.kv_heads * a.parts);
  static_assert(kKeyRows == 64);
  hipLaunchKernelGGL((attention_delta_kernel<T, D>), dim3(static_cast<uint32_t>(slots * all)), dim3(256), 0, s, a);
  hipLaunchKernelGGL((attention_gradients_kernel<T, D>), dim3(keys + static_cast<uint32_t>(half_slots * a.heads)), dim3(256), 0, s, a, keys);
  if (a.parts > 1) hipLaunchKernelGGL((attention_join_kernel<T>), dim3(2048), dim3(256), 0, s, a);
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
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  type == ONES_F16 ? launch<f16>(a, s) : launch<bf16>(a, s);
  return launched("attention backward");
}

}  // extern "C"

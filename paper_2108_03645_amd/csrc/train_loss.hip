// Softmax cross entropy of x W^T over a large vocabulary, with its gradient, without the logits (ones_cross_entropy_*).
//
//   z_iv = x_i . W_v, lse_i = log sum_v exp z_iv, loss_i = lse_i - z_i,target
//   G_iv = dloss_i (exp(z_iv - lse_i) - [v = target_i]), dx = G W, dW = G^T x
//
// What bounds it are the products: 2 N V D forward, and backward the logits' again (they are not kept: N V of them would be read and
// written at 32 bits) and the two of the gradients.  Forward, the epilogue of a tile of logits leaves for every row of x the
// largest logit of a wave's part of the vocabulary and the sum of exponentials below it; a small second launch joins them.
// Backward goes through the vocabulary in pieces: one launch forms G of a piece, rounded to 16 bits (the operands' type, as
// a product of that type needs), and one launch its dW and what it adds to dx, which is summed in 32 bits over the pieces.
// A piece's G has at most 128 MiB, with the sums of products whose k is split where that leaves more than 256 words: half of the
// last-level cache, so that the two products that read it mostly find it there.  More than 262144 rows, of which 256 words would be
// more, are taken in blocks within each piece, and dW is summed in 32 bits over them.
//
// Measured, where a large library product reaches 1.35 (8192 cubed) to 1.5 PFLOP/s: logits of 16384 x 32000, k 512, with their
// epilogue 455 us (1.18 PFLOP/s; a tile of 256 x 256 takes 1.4 us for 64 k and 5 us for its start and its exponentials), 8192 x
// 32000, k 1024, 437 us (1.23).  A piece of 8192 rows and words, k 1024: G 120 to 144 us (1.0), its two products 208 to 240 us (1.2
// to 1.3); joining the parts 4 to 11 us, packing x 3 to 9 us.
//
// G is held in units of the largest finite |dloss| over 2^14 and the products are scaled back in 32 bits.  fp16 would lose small
// probabilities times small dloss otherwise; and where all dloss are equal, as in a mean, the target's entry comes to
// 2^14 (p - 1), next to a power of two for small p, instead of a value whose rounding error is the same in every row (error of
// fp16 gradients against 64 bits, 1003 rows of 514, 10007 words: 4.1e-4 with a power of two as the unit; half a step's is 2.1e-4).
// A row whose |dloss| lies far below the largest would still lose its small probabilities to fp16's smallest step, and its dx with them
// (30000 words, a dloss 2^-24 of the largest: all of it).  So from 2^-14 of the largest on, G of the row is held 2^k times as large and x's
// copy 2^-k times, k up to 12: dW = G^T x stays as it is, the logits and dx are scaled back in 32 bits.
// (The unit has to be there before x is copied then, by a launch of its own: 1003 rows of 514, 10007 words, both calls 117 us before, 120 now.)
// Rows whose target is below 0 are copied as zeros first, so that whatever they hold (they are padding) meets the zeros of G
// as zeros.
#include "train_host.h"
#include "train_matmul.h"

#include <algorithm>

namespace ones {
namespace train {
namespace {

constexpr float kLog2E = 1.44269504f;

struct LossArgs {
  Operand w, x;
  int32_t v0, vocabulary;                     // the first word of w, words in all
  const int64_t *target;
  Part *parts;                                // [parts of the vocabulary][rows]
  float *at_target;
  const float *lse, *dloss, *scale;           // scale: of G, back, and the largest |dloss|
  void *g;                                    // [rows][g_ld]
  int64_t g_ld;
};

// k of a row, above.
constexpr int kKept = 14, kLift = 12;
__device__ __forceinline__ int lift_of(float dloss, float most) {
  const float d = fabsf(dloss);
  return d > 0.f && d < most ? max(min(ilogbf(most) - ilogbf(d) - kKept, kLift), 0) : 0;
}

// Tiles of logits.  GRADIENT: writes G; otherwise what the loss needs of it.  A workgroup takes tiles in turn and has the next one's
// first operands on their way while it deals with one's logits.
template <typename T, typename S, bool GRADIENT>
__global__ __launch_bounds__(S::threads, S::resident) void logits_kernel(LossArgs a) {
  __shared__ __align__(16) unsigned char lds[S::lds];
  const int32_t tm = (a.w.extent + S::BM - 1) / S::BM, tn = (a.x.extent + S::BN - 1) / S::BN, tiles = tm * tn;
  int32_t id = static_cast<int32_t>(blockIdx.x), m, n;
  Product<T, false, false, S> product;
  Sums<S> acc;
  tile_of(id, tiles, tm, tn, m, n);
  product.begin(a.w, a.x, m * S::BM, n * S::BN, 0, a.w.k, lds);
  const float unit = GRADIENT ? a.scale[0] : 0.f;
  for (;;) {
    const Place<S> at(m * S::BM, n * S::BN);
    const int part = m * S::WM + static_cast<int>(threadIdx.x) / kWave / S::WN;
    const bool ragged = (m + 1) * S::BM > a.w.extent;
    // read ahead of the products, looked at behind them
    int64_t target[S::TN];
    float lse[S::TN], weight[S::TN];
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int32_t row = at.n + j * 16;
      const bool inside = row < a.x.extent;
      target[j] = inside ? a.target[row] : -1;
      if (GRADIENT) {
        lse[j] = inside ? a.lse[row] : 0.f;
        weight[j] = inside ? a.dloss[row] : 0.f;
      }
    }
    product.run(lds, acc);
    id += static_cast<int32_t>(gridDim.x);
    if (id < tiles) {
      tile_of(id, tiles, tm, tn, m, n);
      product.begin(a.w, a.x, m * S::BM, n * S::BN, 0, a.w.k, lds);
    }
    // words beyond the last: no logits forward, no G backward.  (Blocks that most tiles skip, ahead of the others: as a condition at
    // every logit they would be a select at every logit.)
    if (!GRADIENT && ragged) {
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool beyond = at.m + i * 16 + r >= a.w.extent;
#pragma unroll
          for (int j = 0; j < S::TN; ++j) acc[i][j][r] = beyond ? -INFINITY : acc[i][j][r];
        }
    }
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int32_t row = at.n + j * 16;
      const bool inside = row < a.x.extent, ignored = target[j] < 0, unknown = target[j] >= a.vocabulary;
      // 16 i + r of the target, if that is in this lane's runs
      const int32_t in = ignored || unknown ? -1 : static_cast<int32_t>(target[j]) - a.v0 - at.m;
      const int32_t hit = in >= 0 && in < S::TM * 16 && in % 16 < 4 ? in : -1;
      const bool hits = __any(hit >= 0);                      // one of 16 rows, in a few tiles
      if constexpr (GRADIENT) {
        const float base = lse[j] * -kLog2E;                  // rounded by 2^-24 of lse, as the logits are by more
        const int lift = __is_same(T, f16) ? lift_of(weight[j], a.scale[2]) : 0;
        const float slope = __is_same(T, f16) ? ldexpf(kLog2E, lift) : kLog2E;
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][r], slope, base));
        if (hits) {
          asm volatile("");                                   // a block of its own, no selects
#pragma unroll
          for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] -= hit == i * 16 + r ? 1.f : 0.f;
        }
        const float factor = unknown ? __builtin_nanf("") : __is_same(T, f16) ? ldexpf(weight[j] * unit, lift) : weight[j] * unit;
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] *= factor;
        if (ragged || __any(ignored)) {                       // whatever came out there
#pragma unroll
          for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[i][j][r] = ignored || at.m + i * 16 + r >= a.w.extent ? 0.f : acc[i][j][r];
        }
        // a lane has runs of four words, its neighbours' runs of 16 lanes on are next to them: of every two runs one goes to the lane
        // 16 on or back, so that each writes eight words
        T *to = static_cast<T *>(a.g) + row * a.g_ld + swapped_m<S>(at.m);
#pragma unroll
        for (int i = 0; i < S::TM; i += 2) {
          const Pack<uint32_t, 4> eight = swapped<T>(acc[i][j], acc[i + 1][j]);
          if (inside) *reinterpret_cast<Pack<uint32_t, 4> *>(to + i * 16) = eight;
        }
      } else {
        if (hits) {
          float of_target = 0.f;
#pragma unroll
          for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) of_target = hit == i * 16 + r ? acc[i][j][r] : of_target;
          if (hit >= 0) a.at_target[row] = of_target;
        }
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, acc[i][j][r]);
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float base = top == -INFINITY ? 0.f : top * -kLog2E;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
          for (int r = 0; r < 4; ++r) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][r], kLog2E, base));
        // top in units of log 2 was rounded: by the same factor in every term
        sum *= __builtin_amdgcn_exp2f(-__builtin_fmaf(top == -INFINITY ? 0.f : top, kLog2E, base));
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (inside && threadIdx.x % kWave < 16) a.parts[static_cast<int64_t>(part) * a.x.extent + row] = Part{top, sum};
      }
    }
    if (id >= tiles) return;
  }
}

// The parts of every row joined: ROWS rows a workgroup, its 1024 threads' shares of them first within the waves, then across.  Eight
// rows where 64 would leave most compute units without any (us with 64 and 8: one row of 1000 parts 23 and 5.7, 128 of 2000 49 and 9.3,
// 512 of 392 12 and 5.0, 1000 of 314 10.1 and 4.5, 8192 of 250 9.3 and 10.8, 16000 of 250 9.9 and 18).
constexpr int kJoinThreads = 1024;
__device__ __forceinline__ void join(float &top, float &sum, const Part &one) {
  const float both = fmaxf(top, one.top);     // skips NaN; the sum has it then
  sum = both == -INFINITY ? sum + one.sum : sum * __expf(top - both) + one.sum * __expf(one.top - both);
  top = both;
}
template <int ROWS>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const Part *parts, int32_t n_parts, int32_t rows, int32_t vocabulary,
                                                            const int64_t *target, const float *at_target, float *loss, float *lse) {
  constexpr int waves = kJoinThreads / kWave;
  __shared__ Part shared[waves][ROWS];
  const int mine = threadIdx.x % ROWS, share = threadIdx.x / ROWS, wave = threadIdx.x / kWave;
  const int32_t row = blockIdx.x * ROWS + mine;
  float top = -INFINITY, sum = 0.f;
  if (row < rows) {
#pragma unroll 4
    for (int p = share; p < n_parts; p += kJoinThreads / ROWS) join(top, sum, parts[static_cast<int64_t>(p) * rows + row]);
  }
#pragma unroll
  for (int m = ROWS; m < kWave; m <<= 1) join(top, sum, Part{__shfl_xor(top, m), __shfl_xor(sum, m)});
  if (static_cast<int>(threadIdx.x) % kWave < ROWS) shared[wave][mine] = Part{top, sum};
  __syncthreads();
  if (threadIdx.x >= ROWS || row >= rows) return;
#pragma unroll
  for (int s = 1; s < waves; ++s) join(top, sum, shared[s][mine]);
  const float all = top + logf(sum);
  const int64_t t = target[row];
  lse[row] = all;
  loss[row] = t < 0 ? 0.f : t >= vocabulary ? __builtin_nanf("") : all - at_target[row];
}

// Rows of two arrays copied with their columns padded with zeros; x's rows of ignored targets as zeros.  The last workgroup
// finds G's unit instead, or, for fp16, whose rows are copied by it, a launch of its own.
struct PackArgs {
  const uint16_t *from[2];
  uint16_t *to[2];
  int64_t from_ld[2];
  int32_t rows[2], cols, to_ld;
  const int64_t *target;                      // of the rows of array 0, or null
  const float *dloss;
  float *scale;                               // null: not wanted
  int32_t lifts;                              // array 0 is fp16, scale is there already
};
__device__ __forceinline__ void find_unit(const PackArgs &a) {
  __shared__ float part[4];
  float most = 0.f;
#pragma unroll 8
  for (int32_t i = threadIdx.x; i < a.rows[0]; i += 256) {
    const int64_t t = a.target[i];
    const float d = fabsf(a.dloss[i]);
    // An infinite one takes no unit away from the others.  (Not with &&: as a branch that puts the loads one after another, 8192 rows
    // 21 us instead of 9.)
    const bool counts = (t >= 0) & (d < INFINITY);
    most = counts ? fmaxf(most, d) : most;
  }
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    most = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    const bool usable = most > 1e-30f;
    a.scale[0] = usable ? 16384.f / most : 1.f;
    a.scale[1] = usable ? most / 16384.f : 1.f;
    a.scale[2] = usable ? most : 0.f;
  }
}
__global__ __launch_bounds__(256) void unit_kernel(PackArgs a) { find_unit(a); }
__global__ __launch_bounds__(256) void pack_kernel(PackArgs a) {
  const bool finds = a.scale && !a.lifts;
  if (finds && blockIdx.x == gridDim.x - 1) return find_unit(a);
  const int64_t blocks = gridDim.x - (finds ? 1 : 0), pieces = a.to_ld / 8, total = (static_cast<int64_t>(a.rows[0]) + a.rows[1]) * pieces;
  for (int64_t i = blockIdx.x * 256ll + threadIdx.x; i < total; i += blocks * 256) {
    int64_t row = i / pieces;
    const int32_t c = static_cast<int32_t>(i - row * pieces) * 8;
    const int which = row >= a.rows[0];
    if (which) row -= a.rows[0];
    const uint16_t *from = a.from[which] + row * a.from_ld[which] + c;
    const bool skip = !which && a.target && a.target[row] < 0;
    Pack<uint16_t, 8> v;
    if (skip) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v.v[k] = 0;
    } else if (c + 8 <= a.cols && reinterpret_cast<uintptr_t>(from) % 16 == 0) {
      v = load_pack<uint16_t, 8>(from);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v.v[k] = c + k < a.cols ? from[k] : uint16_t{0};
    }
    const int lift = a.lifts && !which && !skip ? lift_of(a.dloss[row], a.scale[2]) : 0;
    if (lift) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v.v[k] = __builtin_bit_cast(uint16_t, static_cast<f16>(ldexpf(static_cast<float>(__builtin_bit_cast(f16, v.v[k])), -lift)));
    }
    *reinterpret_cast<Pack<uint16_t, 8> *>(a.to[which] + row * a.to_ld + c) = v;
  }
}

struct GradientArgs {
  Operand w_turned, g, x_turned, g_turned;
  Split of_dx, of_dw;
  const int64_t *target;
  const float *dloss, *scale;
  float *dx_sum, *dw_sum;                     // [splits][rows][cols], [splits][words][cols]
  void *dx, *dweight;                         // dweight: of the piece's first word
  int32_t cols, wide;                         // wide: runs of four of dx and dW can be written at once
  int32_t dx_first, dx_last, dw_first, dw_last;       // of the pieces that dx is summed over, of the blocks of rows that dW is
  int32_t dw_parts;                           // parts of dW to be added up behind the last block; 0: written here
};

// The tiles of dx of a block of rows first, then those of a piece's dW.  dx is added up over the pieces in 32 bits, dW over the blocks, in
// as many places as k is split; a product in one part that is complete is rounded and written.
template <typename T, typename S>
__global__ __launch_bounds__(S::threads, S::resident) void gradients_kernel(GradientArgs a) {
  __shared__ __align__(16) unsigned char lds[S::lds];
  const int32_t tm = (a.cols + S::BM - 1) / S::BM, dx_tiles = tm * ((a.g.extent + S::BN - 1) / S::BN);
  const int32_t dw_tiles = tm * ((a.g_turned.extent + S::BN - 1) / S::BN);
  const bool of_dx = static_cast<int32_t>(blockIdx.x) < dx_tiles * a.of_dx.splits;
  const int32_t id = static_cast<int32_t>(blockIdx.x) - (of_dx ? 0 : dx_tiles * a.of_dx.splits), tiles = of_dx ? dx_tiles : dw_tiles;
  const Split split = of_dx ? a.of_dx : a.of_dw;
  const int32_t part = id / tiles, k0 = part * split.k_each;
  Sums<S> acc;
  int32_t m, n;
  tile_of(id - part * tiles, tiles, tm, tiles / tm, m, n);
  if (of_dx) product<T, true, false, S>(a.w_turned, a.g, m * S::BM, n * S::BN, k0, min(a.g.k, k0 + split.k_each), lds, acc);
  else product<T, true, true, S>(a.x_turned, a.g_turned, m * S::BM, n * S::BN, k0, min(a.g_turned.k, k0 + split.k_each), lds, acc);
  const Place<S> at(m * S::BM, n * S::BN);
  const bool wide = a.wide, whole = of_dx ? split.splits == 1 && a.dx_last : !a.dw_parts, adds = !(of_dx ? a.dx_first : a.dw_first);
  const int32_t rows = of_dx ? a.g.extent : a.g_turned.extent;
  float *sum = (of_dx ? a.dx_sum : a.dw_sum) + static_cast<int64_t>(part) * rows * a.cols;
  T *to = static_cast<T *>(of_dx ? a.dx : a.dweight);
#pragma unroll
  for (int j = 0; j < S::TN; ++j) {
    const int32_t row = at.n + j * 16;
    if (row >= rows) continue;
    const bool ignored = whole && of_dx && a.target[row] < 0;
    const float back = !whole ? 1.f : __is_same(T, f16) && of_dx ? ldexpf(a.scale[1], -lift_of(a.dloss[row], a.scale[2])) : a.scale[1];
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int32_t c = at.m + i * 16;
      if (c >= a.cols) continue;
      const int64_t o = static_cast<int64_t>(row) * a.cols + c;
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r];
      if (adds) {
        if (wide) {
          const Pack<float, 4> old = load_pack<float, 4>(sum + o);
#pragma unroll
          for (int r = 0; r < 4; ++r) v[r] += old.v[r];
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r) if (c + r < a.cols) v[r] += sum[o + r];
        }
      }
      if (whole) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = ignored ? 0.f : v[r] * back;
        if (wide) store_pack<T, 4>(to + o, v);
        else
#pragma unroll
          for (int r = 0; r < 4; ++r) if (c + r < a.cols) to[o + r] = static_cast<T>(v[r]);
      } else {
        if (wide) store_pack<float, 4>(sum + o, v);
        else
#pragma unroll
          for (int r = 0; r < 4; ++r) if (c + r < a.cols) sum[o + r] = v[r];
      }
    }
  }
}

// The parts of products that were split, added up in order and rounded: dx of a block after the last piece, dW of a piece after the last block.
struct FinishArgs {
  const float *sum[2];
  void *to[2];
  int64_t size[2];                            // elements; 0: not split
  int32_t splits[2], cols, wide;
  const int64_t *target;                      // of the rows of dx
  const float *dloss, *scale;
};
template <typename T, int V>
__global__ __launch_bounds__(256) void finish_kernel(FinishArgs a) {
  int64_t i = (blockIdx.x * 256ll + threadIdx.x) * V;
  const int which = i >= a.size[0];
  if (which) i -= a.size[0];
  if (i >= a.size[which]) return;
  const float *sum = a.sum[which] + i;
  float v[V];
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = 0.f;
#pragma unroll 4
  for (int s = 0; s < a.splits[which]; ++s, sum += a.size[which]) {
    const Pack<float, V> one = load_pack<float, V>(sum);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] += one.v[k];
  }
  const int64_t row = which ? 0 : i / a.cols;
  const bool ignored = !which && a.target[row] < 0;
  const float back = __is_same(T, f16) && !which ? ldexpf(a.scale[1], -lift_of(a.dloss[row], a.scale[2])) : a.scale[1];
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = ignored ? 0.f : v[k] * back;
  store_pack<T, V>(static_cast<T *>(a.to[which]) + i, v);
}

// Rows that the products can load as they lie: 16 bytes at a time, the rows of a tile (256 at most) inside 2^31 bytes,
// below which the loads' offsets lie.
bool loadable(const void *p, int64_t stride, int64_t cols) {
  return cols % 8 == 0 && stride % 8 == 0 && stride <= kMaxLoadableStride && aligned(p, 16);
}

void launch_pack(const PackArgs &a, hipStream_t s) {
  const int64_t total = (static_cast<int64_t>(a.rows[0]) + a.rows[1]) * (a.to_ld / 8);
  const int64_t blocks = std::min<int64_t>(ceil_div(total, 256), 4096) + (a.scale && !a.lifts ? 1 : 0);
  if (a.lifts) hipLaunchKernelGGL(unit_kernel, dim3(1), dim3(256), 0, s, a);
  if (blocks) hipLaunchKernelGGL(pack_kernel, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, s, a);
}

template <typename T, typename S, bool GRADIENT>
void launch_logits(const LossArgs &a, hipStream_t s) {
  const int64_t tiles = ceil_div(a.w.extent, S::BM) * ceil_div(a.x.extent, S::BN), blocks = std::min<int64_t>(tiles, 256 * S::resident);
  hipLaunchKernelGGL((logits_kernel<T, S, GRADIENT>), dim3(static_cast<uint32_t>(blocks)), dim3(S::threads), 0, s, a);
}
template <typename T, bool GRADIENT>
void launch_logits(const LossArgs &a, Tiles tiles, hipStream_t s) {
  switch (tiles) {
    case kLarge: return launch_logits<T, Large, GRADIENT>(a, s);
    case kDeep: return launch_logits<T, Deep, GRADIENT>(a, s);
    case kSmall: return launch_logits<T, Small, GRADIENT>(a, s);
    default: return launch_logits<T, Tiny, GRADIENT>(a, s);
  }
}
template <typename T, typename S>
void launch_gradients(const GradientArgs &a, hipStream_t s) {
  const int64_t blocks = ceil_div(a.cols, S::BM) * (ceil_div(a.g.extent, S::BN) * a.of_dx.splits + ceil_div(a.g_turned.extent, S::BN) * a.of_dw.splits);
  hipLaunchKernelGGL((gradients_kernel<T, S>), dim3(static_cast<uint32_t>(blocks)), dim3(S::threads), 0, s, a);
}
template <typename T>
void launch_gradients(const GradientArgs &a, Tiles tiles, hipStream_t s) {
  switch (tiles) {
    case kLarge: return launch_gradients<T, Large>(a, s);
    case kDeep: return launch_gradients<T, Deep>(a, s);
    case kSmall: return launch_gradients<T, Small>(a, s);
    default: return launch_gradients<T, Tiny>(a, s);
  }
}
template <typename T>
void launch_finish(const FinishArgs &a, hipStream_t s) {
  const int64_t total = a.size[0] + a.size[1];
  if (total == 0) return;
  if (a.wide) hipLaunchKernelGGL((finish_kernel<T, 4>), dim3(static_cast<uint32_t>(ceil_div(total, 1024))), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((finish_kernel<T, 1>), dim3(static_cast<uint32_t>(ceil_div(total, 256))), dim3(256), 0, s, a);
}

// A piece of the vocabulary and a block of rows: its G, and what it adds to dW and dx.
template <typename T>
void launch_piece(const LossArgs &a, const GradientArgs &b, const LossPlan &p, hipStream_t s) {
  if (a.x.extent) launch_logits<T, true>(a, p.logits_piece, s);
  launch_gradients<T>(b, p.gradients.tiles, s);
  FinishArgs f{};
  f.sum[0] = b.dx_sum; f.sum[1] = b.dw_sum;
  f.to[0] = b.dx; f.to[1] = b.dweight;
  f.splits[0] = b.of_dx.splits; f.splits[1] = b.dw_parts;
  f.size[0] = b.of_dx.splits > 1 && b.dx_last ? static_cast<int64_t>(b.g.extent) * b.cols : 0;
  f.size[1] = b.dw_parts && b.dw_last ? static_cast<int64_t>(b.g_turned.extent) * b.cols : 0;
  f.cols = b.cols;
  f.wide = b.wide;
  f.target = b.target;
  f.dloss = b.dloss;
  f.scale = b.scale;
  launch_finish<T>(f, s);
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

size_t ones_cross_entropy_forward_workspace_bytes(int64_t rows, int64_t cols, int64_t vocabulary, int32_t wide) {
  if (check_loss(rows, cols, vocabulary, cols, cols, ONES_BF16) != ONES_OK) return 0;
  return loss_plan(rows, cols, vocabulary, !wide, !wide, false).forward;
}
size_t ones_cross_entropy_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t vocabulary, int32_t wide) {
  if (check_loss(rows, cols, vocabulary, cols, cols, ONES_BF16) != ONES_OK) return 0;
  return loss_plan(rows, cols, vocabulary, true, !wide, true).backward;
}

int ones_cross_entropy_forward(const void *x, int64_t x_stride, const void *weight, int64_t weight_stride, int64_t rows, int64_t cols,
                               int64_t vocabulary, int32_t type, const int64_t *target, float *loss, float *lse, void *d_workspace,
                               size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_loss(rows, cols, vocabulary, x_stride, weight_stride, type)) return rc;
  if (rows == 0) return ONES_OK;
  if (!x || !weight || !target || !loss || !lse) return ONES_E_INVALID_ARG;
  const bool copy_x = !loadable(x, x_stride, cols), copy_w = !loadable(weight, weight_stride, cols);
  const LossPlan p = loss_plan(rows, cols, vocabulary, copy_x, copy_w, false);
  if (int rc = check_workspace(d_workspace, workspace_bytes, p.forward)) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(d_workspace);
  const int32_t n = static_cast<int32_t>(rows), v = static_cast<int32_t>(vocabulary), d8 = static_cast<int32_t>(p.cols8);
  if (copy_x || copy_w) {
    PackArgs a{{static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(weight)},
               {reinterpret_cast<uint16_t *>(ws + p.x), reinterpret_cast<uint16_t *>(ws + p.w)}, {x_stride, weight_stride},
               {copy_x ? n : 0, copy_w ? v : 0}, static_cast<int32_t>(cols), d8, nullptr, nullptr, nullptr, 0};
    launch_pack(a, s);
  }
  LossArgs a{};
  a.w = copy_w ? Operand{ws + p.w, d8, v, d8} : Operand{weight, weight_stride, v, static_cast<int32_t>(cols)};
  a.x = copy_x ? Operand{ws + p.x, d8, n, d8} : Operand{x, x_stride, n, static_cast<int32_t>(cols)};
  a.vocabulary = v;
  a.target = target;
  a.parts = reinterpret_cast<Part *>(ws + p.part);
  a.at_target = reinterpret_cast<float *>(ws + p.at_target);
  if (type == ONES_F16) launch_logits<f16, false>(a, p.logits, s);
  else launch_logits<bf16, false>(a, p.logits, s);
  auto join = [&](auto kernel, int64_t each) {
    hipLaunchKernelGGL(kernel, dim3(static_cast<uint32_t>(ceil_div(rows, each))), dim3(kJoinThreads), 0, s, a.parts, static_cast<int32_t>(p.parts), n, v,
                       target, a.at_target, loss, lse);
  };
  if (rows < 4096) join(join_kernel<8>, 8);
  else join(join_kernel<64>, 64);
  return launched("cross entropy forward");
}

int ones_cross_entropy_backward(const float *dloss, const void *x, int64_t x_stride, const void *weight, int64_t weight_stride, int64_t rows,
                                int64_t cols, int64_t vocabulary, int32_t type, const int64_t *target, const float *lse, void *dx,
                                void *dweight, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_loss(rows, cols, vocabulary, x_stride, weight_stride, type)) return rc;
  if (!weight || !dweight || (rows && (!dloss || !x || !target || !lse || !dx))) return ONES_E_INVALID_ARG;
  const bool copy_w = !loadable(weight, weight_stride, cols);
  const LossPlan p = loss_plan(rows, cols, vocabulary, true, copy_w, true);
  if (int rc = check_workspace(d_workspace, workspace_bytes, p.backward)) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(d_workspace);
  const int32_t n = static_cast<int32_t>(rows), d8 = static_cast<int32_t>(p.cols8);
  float *scale = reinterpret_cast<float *>(ws + p.scale);
  PackArgs pack{{static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(weight)},
                {reinterpret_cast<uint16_t *>(ws + p.x), reinterpret_cast<uint16_t *>(ws + p.w)}, {x_stride, weight_stride},
                {n, copy_w ? static_cast<int32_t>(vocabulary) : 0}, static_cast<int32_t>(cols), d8, target, dloss, scale, type == ONES_F16};
  launch_pack(pack, s);
  const char *w = copy_w ? ws + p.w : static_cast<const char *>(weight);
  const int64_t w_ld = copy_w ? d8 : weight_stride;
  for (int64_t v0 = 0; v0 < vocabulary; v0 += p.piece) {
    const int32_t words = static_cast<int32_t>(std::min(p.piece, vocabulary - v0));
    const char *wp = w + v0 * w_ld * 2;
    int64_t r0 = 0;
    do {                                      // once for no rows: dW is zeros then
      const int32_t some = static_cast<int32_t>(std::min(p.block, rows - r0));
      const char *xp = ws + p.x + r0 * d8 * 2;
      LossArgs a{};
      a.w = Operand{wp, w_ld, words, d8};
      a.x = Operand{xp, d8, some, d8};
      a.v0 = static_cast<int32_t>(v0);
      a.vocabulary = static_cast<int32_t>(vocabulary);
      a.target = target + r0; a.lse = lse + r0; a.dloss = dloss + r0; a.scale = scale;
      a.g = ws + p.g;
      a.g_ld = p.piece;
      GradientArgs b{};
      b.w_turned = Operand{wp, w_ld, d8, words};
      b.g = Operand{ws + p.g, p.piece, some, words};          // the rest of the last eight words is zeros
      b.x_turned = Operand{xp, d8, d8, some};
      b.g_turned = Operand{ws + p.g, p.piece, words, some};
      b.target = target + r0; b.dloss = dloss + r0; b.scale = scale;
      b.of_dx = p.gradients.of_dx;
      b.of_dw = p.gradients.of_dw;
      b.dx_sum = reinterpret_cast<float *>(ws + p.dx_sum) + b.of_dx.splits * r0 * cols;
      b.dw_sum = reinterpret_cast<float *>(ws + p.dw_sum);
      b.dx = static_cast<char *>(dx) + r0 * cols * 2;
      b.dweight = static_cast<char *>(dweight) + v0 * cols * 2;
      b.cols = static_cast<int32_t>(cols);
      b.wide = cols % 4 == 0 && aligned(dx, 8) && aligned(dweight, 8);
      b.dx_first = v0 == 0;
      b.dx_last = v0 + p.piece >= vocabulary;
      b.dw_first = r0 == 0;
      b.dw_last = r0 + p.block >= rows;
      b.dw_parts = p.blocks > 1 || b.of_dw.splits > 1 ? b.of_dw.splits : 0;
      if (type == ONES_F16) launch_piece<f16>(a, b, p, s);
      else launch_piece<bf16>(a, b, p, s);
      r0 += p.block;
    } while (r0 < rows);
  }
  return launched("cross entropy backward");
}

}  // extern "C"

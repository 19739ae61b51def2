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
// A piece's G has at most 128 MiB, half of the last-level cache, so that the two products that read it mostly find it there.
//
// G is held in units of the largest |dloss| over 2^14 and the products are scaled back in 32 bits.  fp16 would lose small
// probabilities times small dloss otherwise; and where all dloss are equal, as in a mean, the target's entry comes to
// 2^14 (p - 1), next to a power of two for small p, instead of a value whose rounding error is the same in every row (error of
// fp16 gradients against 64 bits, 1003 rows of 514, 10007 words: 4.1e-4 with a power of two as the unit; half a step's is 2.1e-4).
// Rows whose target is below 0 are copied as zeros first, so that whatever they hold (they are padding) meets the zeros of G
// as zeros.
#include "train_host.h"
#include "train_matmul.h"

#include <algorithm>

namespace ones {
namespace train {
namespace {

constexpr int64_t kPieceBytes = 128 << 20;

struct Part { float top, sum; };              // of some logits of a row: the largest, and the sum of exp(z - top)

struct LossArgs {
  Operand w, x;
  int32_t v0, vocabulary;                     // the first word of w, words in all
  const int64_t *target;
  Part *parts;                                // [parts of the vocabulary][rows]
  float *at_target;
  const float *lse, *dloss, *scale;           // scale: of G, and back
  void *g;                                    // [rows][g_ld]
  int64_t g_ld;
};

// One tile of logits.  GRADIENT: writes G; otherwise what the loss needs of it.
template <typename T, typename S, bool GRADIENT>
__global__ __launch_bounds__(S::threads) void logits_kernel(LossArgs a) {
  __shared__ __align__(16) unsigned char lds[S::lds];
  const int32_t tm = (a.w.extent + S::BM - 1) / S::BM, tn = (a.x.extent + S::BN - 1) / S::BN;
  int32_t m, n;
  tile_of(static_cast<int32_t>(blockIdx.x), tm * tn, tm, tn, m, n);
  const int part = m * S::WM + static_cast<int>(threadIdx.x) / kWave / S::WN;
  Sums<S> acc;
  product<T, false, false, S>(a.w, a.x, m * S::BM, n * S::BN, lds, acc);
  const Place<S> at(m * S::BM, n * S::BN);
#pragma unroll
  for (int j = 0; j < S::TN; ++j) {
    const int32_t row = at.n + j * 16;
    const bool inside = row < a.x.extent;
    const int64_t target = inside ? a.target[row] : -1;
    const int32_t hit = target >= 0 && target < a.vocabulary ? static_cast<int32_t>(target) - a.v0 - at.m : -1;   // 16 i + r, if in this run
    if constexpr (GRADIENT) {
      if (!inside) continue;
      const float lse = a.lse[row];
      const float weight = target < 0 ? 0.f : target >= a.vocabulary ? __builtin_nanf("") : a.dloss[row] * a.scale[0];
#pragma unroll
      for (int i = 0; i < S::TM; ++i) {
        const int32_t v = at.m + i * 16;
        float g[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __expf(acc[i][j][r] - lse) - (hit == i * 16 + r ? 1.f : 0.f);
          g[r] = target < 0 || v + r >= a.w.extent ? 0.f : p * weight;
        }
        store_pack<T, 4>(static_cast<T *>(a.g) + row * a.g_ld + v, g);
      }
    } else {
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (hit == i * 16 + r) a.at_target[row] = acc[i][j][r];
          if (at.m + i * 16 + r >= a.w.extent) acc[i][j][r] = -INFINITY;
          top = fmaxf(top, acc[i][j][r]);
        }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float base = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) sum += __expf(acc[i][j][r] - base);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (inside && threadIdx.x % kWave < 16) a.parts[static_cast<int64_t>(part) * a.x.extent + row] = Part{top, sum};
    }
  }
}

// The parts of every row joined: 64 rows a workgroup, four threads a row.
__global__ __launch_bounds__(256) void join_kernel(const Part *parts, int32_t n_parts, int32_t rows, int32_t vocabulary, const int64_t *target,
                                                   const float *at_target, float *loss, float *lse) {
  __shared__ Part shared[3][64];
  const int lane = threadIdx.x % 64, share = threadIdx.x / 64;
  const int32_t row = blockIdx.x * 64 + lane;
  float top = -INFINITY, sum = 0.f;
  bool nan = false;
  if (row < rows) {
#pragma unroll 4
    for (int p = share; p < n_parts; p += 4) {
      const Part one = parts[static_cast<int64_t>(p) * rows + row];
      const float both = fmaxf(top, one.top);
      nan |= one.sum != one.sum;              // a maximum skips NaN, a sum does not
      if (both == -INFINITY) continue;
      sum = sum * __expf(top - both) + one.sum * __expf(one.top - both);
      top = both;
    }
  }
  if (nan) sum = __builtin_nanf("");
  if (share) shared[share - 1][lane] = Part{top, sum};
  __syncthreads();
  if (share || row >= rows) return;
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    const Part one = shared[s][lane];
    const float both = fmaxf(top, one.top);
    sum = both == -INFINITY ? sum + one.sum : sum * __expf(top - both) + one.sum * __expf(one.top - both);
    top = both;
  }
  const float all = top + logf(sum);
  const int64_t t = target[row];
  lse[row] = all;
  loss[row] = t < 0 ? 0.f : t >= vocabulary ? __builtin_nanf("") : all - at_target[row];
}

// Rows of two arrays copied with their columns padded with zeros; x's rows of ignored targets as zeros.  The last workgroup
// finds G's unit instead.
struct PackArgs {
  const uint16_t *from[2];
  uint16_t *to[2];
  int64_t from_ld[2];
  int32_t rows[2], cols, to_ld;
  const int64_t *target;                      // of the rows of array 0, or null
  const float *dloss;
  float *scale;
};
__global__ __launch_bounds__(256) void pack_kernel(PackArgs a) {
  if (a.scale && blockIdx.x == gridDim.x - 1) {
    __shared__ float part[4];
    float most = 0.f;
    for (int32_t i = threadIdx.x; i < a.rows[0]; i += 256)
      if (a.target[i] >= 0) most = fmaxf(most, fabsf(a.dloss[i]));
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) most = fmaxf(most, __shfl_xor(most, m));
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
      most = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
      const bool usable = most > 1e-30f && isfinite(most);
      a.scale[0] = usable ? 16384.f / most : 1.f;
      a.scale[1] = usable ? most / 16384.f : 1.f;
    }
    return;
  }
  const int64_t blocks = gridDim.x - (a.scale ? 1 : 0), pieces = a.to_ld / 8, total = (static_cast<int64_t>(a.rows[0]) + a.rows[1]) * pieces;
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
    *reinterpret_cast<Pack<uint16_t, 8> *>(a.to[which] + row * a.to_ld + c) = v;
  }
}

struct GradientArgs {
  Operand w_turned, g, x_turned, g_turned;
  const int64_t *target;
  const float *scale;
  float *sum;                                 // dx over the pieces so far, [rows][cols]
  void *dx, *dweight;                         // dweight: of the piece's first word
  int32_t cols, first, last;
};

// The tiles of dx first, then those of a piece's dW.
template <typename T, typename S>
__global__ __launch_bounds__(S::threads) void gradients_kernel(GradientArgs a) {
  __shared__ __align__(16) unsigned char lds[S::lds];
  const int32_t tm = (a.cols + S::BM - 1) / S::BM, of_dx = tm * ((a.g.extent + S::BN - 1) / S::BN);
  const float back = a.scale[1];
  const bool wide = a.cols % 4 == 0;
  const int32_t id = static_cast<int32_t>(blockIdx.x);
  Sums<S> acc;
  int32_t m, n;
  if (id < of_dx) {
    tile_of(id, of_dx, tm, of_dx / tm, m, n);
    product<T, true, false, S>(a.w_turned, a.g, m * S::BM, n * S::BN, lds, acc);
  } else {
    const int32_t of_dw = static_cast<int32_t>(gridDim.x) - of_dx;
    tile_of(id - of_dx, of_dw, tm, of_dw / tm, m, n);
    product<T, true, true, S>(a.x_turned, a.g_turned, m * S::BM, n * S::BN, lds, acc);
  }
  const Place<S> at(m * S::BM, n * S::BN);
#pragma unroll
  for (int j = 0; j < S::TN; ++j) {
    const int32_t row = at.n + j * 16;
    if (row >= (id < of_dx ? a.g.extent : a.g_turned.extent)) continue;
    const bool ignored = id < of_dx && a.target[row] < 0;
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int32_t c = at.m + i * 16;
      if (c >= a.cols) continue;
      const int64_t o = static_cast<int64_t>(row) * a.cols + c;
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = acc[i][j][r];
      if (id < of_dx && !a.first) {
#pragma unroll
        for (int r = 0; r < 4; ++r) if (c + r < a.cols) v[r] += a.sum[o + r];
      }
      if (id < of_dx && !a.last) {
        if (wide) store_pack<float, 4>(a.sum + o, v);
        else
#pragma unroll
          for (int r = 0; r < 4; ++r) if (c + r < a.cols) a.sum[o + r] = v[r];
        continue;
      }
      T *to = static_cast<T *>(id < of_dx ? a.dx : a.dweight) + o;
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = ignored ? 0.f : v[r] * back;
      if (wide) store_pack<T, 4>(to, v);
      else
#pragma unroll
        for (int r = 0; r < 4; ++r) if (c + r < a.cols) to[r] = static_cast<T>(v[r]);
    }
  }
}

// Large tiles where they are enough for most compute units, else small ones (four times as many, two a compute unit).
constexpr int64_t kEnoughTiles = 160;
bool large_tiles(int64_t m, int64_t n) { return ceil_div(m, Large::BM) * ceil_div(n, Large::BN) >= kEnoughTiles; }

struct LossPlan {
  int64_t cols8, parts, piece, pieces;
  bool large_logits, large_g, large_gradients;
  size_t x, w, part, at_target, forward;                       // offsets, and the bytes of the forward pass
  size_t g, sum, scale, backward;
};

LossPlan loss_plan(int64_t rows, int64_t cols, int64_t vocabulary, bool copies_x, bool copies_w) {
  LossPlan p{};
  p.cols8 = ceil_div(cols, 8) * 8;
  p.large_logits = large_tiles(vocabulary, rows);
  p.parts = p.large_logits ? ceil_div(vocabulary, Large::BM) * Large::WM : ceil_div(vocabulary, Small::BM) * Small::WM;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes); return at; };
  const size_t n = static_cast<size_t>(rows), d8 = static_cast<size_t>(p.cols8);
  p.x = take(copies_x ? n * d8 * 2 : 0);
  p.w = take(copies_w ? static_cast<size_t>(vocabulary) * d8 * 2 : 0);
  const size_t packed = off;
  p.part = take(static_cast<size_t>(p.parts) * n * sizeof(Part));
  p.at_target = take(n * 4);
  p.forward = off;
  off = packed;
  p.pieces = std::max<int64_t>(1, ceil_div(rows * ceil_div(vocabulary, 256) * 256 * 2, kPieceBytes));
  p.piece = ceil_div(ceil_div(vocabulary, p.pieces), 256) * 256;
  p.pieces = ceil_div(vocabulary, p.piece);
  p.large_g = large_tiles(p.piece, rows);
  p.large_gradients = ceil_div(cols, Large::BM) * (ceil_div(rows, Large::BN) + ceil_div(p.piece, Large::BN)) >= kEnoughTiles;
  p.g = take(n * static_cast<size_t>(p.piece) * 2);
  p.sum = take(p.pieces > 1 ? n * static_cast<size_t>(cols) * 4 : 0);
  p.scale = take(8);
  p.backward = off;
  return p;
}

int check_loss(int64_t rows, int64_t cols, int64_t vocabulary, int64_t x_stride, int64_t w_stride, int32_t type) {
  if (int rc = check_rows(rows, cols, x_stride)) return rc;
  if (int rc = check_rows(vocabulary, cols, w_stride)) return rc;
  if (cols < 1 || vocabulary < 1 || (type != ONES_F16 && type != ONES_BF16)) return ONES_E_INVALID_ARG;
  if (rows > ONES_MAX_LOSS_ROWS || vocabulary > ONES_MAX_VOCABULARY || cols > ONES_MAX_LOSS_COLUMNS) return ONES_E_BOUNDS;
  // tiles of a launch: at most 2^23, of 256 threads
  const int64_t n = ceil_div(rows, 128), v = ceil_div(vocabulary, 128), d = ceil_div(cols, 128);
  return std::max({n * v, d * n, d * v}) > (1 << 22) ? ONES_E_BOUNDS : ONES_OK;
}

// Rows that the products can load 16 bytes at a time.
bool loadable(const void *p, int64_t stride, int64_t cols) { return cols % 8 == 0 && stride % 8 == 0 && aligned(p, 16); }

void launch_pack(const PackArgs &a, hipStream_t s) {
  const int64_t total = (static_cast<int64_t>(a.rows[0]) + a.rows[1]) * (a.to_ld / 8);
  const int64_t blocks = std::min<int64_t>(ceil_div(total, 256), 4096) + (a.scale ? 1 : 0);
  if (blocks) hipLaunchKernelGGL(pack_kernel, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, s, a);
}

template <typename T, typename S, bool GRADIENT>
void launch_logits(const LossArgs &a, hipStream_t s) {
  const int64_t blocks = ceil_div(a.w.extent, S::BM) * ceil_div(a.x.extent, S::BN);
  hipLaunchKernelGGL((logits_kernel<T, S, GRADIENT>), dim3(static_cast<uint32_t>(blocks)), dim3(S::threads), 0, s, a);
}
template <bool GRADIENT>
void launch_logits(const LossArgs &a, int32_t type, bool large, hipStream_t s) {
  if (type == ONES_F16) large ? launch_logits<f16, Large, GRADIENT>(a, s) : launch_logits<f16, Small, GRADIENT>(a, s);
  else large ? launch_logits<bf16, Large, GRADIENT>(a, s) : launch_logits<bf16, Small, GRADIENT>(a, s);
}
template <typename T, typename S>
void launch_gradients(const GradientArgs &a, hipStream_t s) {
  const int64_t blocks = ceil_div(a.cols, S::BM) * (ceil_div(a.g.extent, S::BN) + ceil_div(a.g_turned.extent, S::BN));
  hipLaunchKernelGGL((gradients_kernel<T, S>), dim3(static_cast<uint32_t>(blocks)), dim3(S::threads), 0, s, a);
}
void launch_gradients(const GradientArgs &a, int32_t type, bool large, hipStream_t s) {
  if (type == ONES_F16) large ? launch_gradients<f16, Large>(a, s) : launch_gradients<f16, Small>(a, s);
  else large ? launch_gradients<bf16, Large>(a, s) : launch_gradients<bf16, Small>(a, s);
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

size_t ones_cross_entropy_forward_workspace_bytes(int64_t rows, int64_t cols, int64_t vocabulary, int32_t wide) {
  if (check_loss(rows, cols, vocabulary, cols, cols, ONES_BF16) != ONES_OK) return 0;
  return loss_plan(rows, cols, vocabulary, !wide, !wide).forward;
}
size_t ones_cross_entropy_backward_workspace_bytes(int64_t rows, int64_t cols, int64_t vocabulary, int32_t wide) {
  if (check_loss(rows, cols, vocabulary, cols, cols, ONES_BF16) != ONES_OK) return 0;
  return loss_plan(rows, cols, vocabulary, true, !wide).backward;
}

int ones_cross_entropy_forward(const void *x, int64_t x_stride, const void *weight, int64_t weight_stride, int64_t rows, int64_t cols,
                               int64_t vocabulary, int32_t type, const int64_t *target, float *loss, float *lse, void *d_workspace,
                               size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_loss(rows, cols, vocabulary, x_stride, weight_stride, type)) return rc;
  if (rows == 0) return ONES_OK;
  if (!x || !weight || !target || !loss || !lse) return ONES_E_INVALID_ARG;
  const bool copy_x = !loadable(x, x_stride, cols), copy_w = !loadable(weight, weight_stride, cols);
  const LossPlan p = loss_plan(rows, cols, vocabulary, copy_x, copy_w);
  if (int rc = check_workspace(d_workspace, workspace_bytes, p.forward)) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(d_workspace);
  const int32_t n = static_cast<int32_t>(rows), v = static_cast<int32_t>(vocabulary), d8 = static_cast<int32_t>(p.cols8);
  if (copy_x || copy_w) {
    PackArgs a{{static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(weight)},
               {reinterpret_cast<uint16_t *>(ws + p.x), reinterpret_cast<uint16_t *>(ws + p.w)}, {x_stride, weight_stride},
               {copy_x ? n : 0, copy_w ? v : 0}, static_cast<int32_t>(cols), d8, nullptr, nullptr, nullptr};
    launch_pack(a, s);
  }
  LossArgs a{};
  a.w = copy_w ? Operand{ws + p.w, d8, v, d8} : Operand{weight, weight_stride, v, static_cast<int32_t>(cols)};
  a.x = copy_x ? Operand{ws + p.x, d8, n, d8} : Operand{x, x_stride, n, static_cast<int32_t>(cols)};
  a.vocabulary = v;
  a.target = target;
  a.parts = reinterpret_cast<Part *>(ws + p.part);
  a.at_target = reinterpret_cast<float *>(ws + p.at_target);
  launch_logits<false>(a, type, p.large_logits, s);
  hipLaunchKernelGGL(join_kernel, dim3(static_cast<uint32_t>(ceil_div(rows, 64))), dim3(256), 0, s, a.parts, static_cast<int32_t>(p.parts), n, v,
                     target, a.at_target, loss, lse);
  return launched("cross entropy forward");
}

int ones_cross_entropy_backward(const float *dloss, const void *x, int64_t x_stride, const void *weight, int64_t weight_stride, int64_t rows,
                                int64_t cols, int64_t vocabulary, int32_t type, const int64_t *target, const float *lse, void *dx,
                                void *dweight, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_loss(rows, cols, vocabulary, x_stride, weight_stride, type)) return rc;
  if (!weight || !dweight || (rows && (!dloss || !x || !target || !lse || !dx))) return ONES_E_INVALID_ARG;
  const bool copy_w = !loadable(weight, weight_stride, cols);
  const LossPlan p = loss_plan(rows, cols, vocabulary, true, copy_w);
  if (int rc = check_workspace(d_workspace, workspace_bytes, p.backward)) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(d_workspace);
  const int32_t n = static_cast<int32_t>(rows), d8 = static_cast<int32_t>(p.cols8);
  float *scale = reinterpret_cast<float *>(ws + p.scale);
  PackArgs pack{{static_cast<const uint16_t *>(x), static_cast<const uint16_t *>(weight)},
                {reinterpret_cast<uint16_t *>(ws + p.x), reinterpret_cast<uint16_t *>(ws + p.w)}, {x_stride, weight_stride},
                {n, copy_w ? static_cast<int32_t>(vocabulary) : 0}, static_cast<int32_t>(cols), d8, target, dloss, scale};
  launch_pack(pack, s);
  const Operand xs{ws + p.x, d8, n, d8};
  const char *w = copy_w ? ws + p.w : static_cast<const char *>(weight);
  const int64_t w_ld = copy_w ? d8 : weight_stride;
  for (int64_t v0 = 0; v0 < vocabulary; v0 += p.piece) {
    const int32_t words = static_cast<int32_t>(std::min(p.piece, vocabulary - v0));
    const char *wp = w + v0 * w_ld * 2;
    LossArgs a{};
    a.w = Operand{wp, w_ld, words, d8};
    a.x = xs;
    a.v0 = static_cast<int32_t>(v0);
    a.vocabulary = static_cast<int32_t>(vocabulary);
    a.target = target; a.lse = lse; a.dloss = dloss; a.scale = scale;
    a.g = ws + p.g;
    a.g_ld = p.piece;
    if (rows) launch_logits<true>(a, type, p.large_g, s);
    GradientArgs b{};
    b.w_turned = Operand{wp, w_ld, d8, words};
    b.g = Operand{ws + p.g, p.piece, n, words};               // the rest of the last eight words is zeros
    b.x_turned = Operand{ws + p.x, d8, d8, n};
    b.g_turned = Operand{ws + p.g, p.piece, words, n};
    b.target = target; b.scale = scale;
    b.sum = reinterpret_cast<float *>(ws + p.sum);
    b.dx = dx;
    b.dweight = static_cast<char *>(dweight) + v0 * cols * 2;
    b.cols = static_cast<int32_t>(cols);
    b.first = v0 == 0;
    b.last = v0 + p.piece >= vocabulary;
    launch_gradients(b, type, p.large_gradients, s);
  }
  return launched("cross entropy backward");
}

}  // extern "C"

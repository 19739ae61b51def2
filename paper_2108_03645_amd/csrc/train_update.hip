// The orthogonalised update of weight matrices (ones_orthogonal_update): momentum, then Newton-Schulz products.
//
//   m = beta m + g, u = g + beta m (nesterov) or m, X = u / (|u| + eps)
//   steps times, with (a, b, c): A = X X^T, B = b A + c A^2, X = a X + B X
//
// X is held with the shorter side first (a tall u turned), r x q, r <= q: A is r x r.  A step is r^2 q + r^3 + 2 r^2 q operations
// when the symmetry of A and A^2 is used: only the tiles on and below the diagonal are computed, and written to both places.
//
// The operands are fp16 whatever the gradient's type: X's singular values stay near 1, so the range of bf16 is not needed, and
// three more bits keep the result of five steps next to a bf16 result's own rounding (each step rounds X, A and B).  They are held
// times 2^11 (X) and 2^10 (A, B): an element of X is at most 1.3 and typically (r q)^-1/2, of A typically r^-1 q^-1/2 off the diagonal.  For
// coefficients that keep the singular values below 7.9 nothing is too large for fp16.  At the other end, with both sides at their limit of
// 65536, X's elements are typically 2^-5 and A's 2^-14, where fp16's steps cease to shrink: an element is off by 2^-25 at most, as
// much as half a step is there, and by a larger share only where it is smaller than most.
//
// For a bf16 result that is 0.9e-3 to 1.8e-3 of the whole (sides 33 to 4100) next to the result's own rounding of 1.7e-3: mostly from X's
// roundings, which grow with the directions of small singular values; A's and B's diagonals kept apart in 32 bits took 3 to 28 % off that and
// cost 2 to 6 % of the time.  An fp16 result, whose own rounding is 2.1e-4, would be nearly ten times as far off as it has to be.  For it X, A
// and B are held in pairs (PAIRS), the second what the first was rounded by, and every product is three: 22 bits, which leaves the
// result's own rounding: 4100 x 3000 2.1e-4 in 2.70 ms, singly 1.5e-3 in 1.02 ms; eight of 256 x 256 159 us and 97.  (With only X, or only X
// and A, X and B in pairs: 0.8e-3 to 1.2e-3, 0.4e-3 to 0.6e-3.)
//
// Measured at 4100 x 3000: A 61 us and B 51 us (tiles of 192 x 128 on and below the diagonal, one round), X 96 us (0.77
// PFLOP/s, 204 tiles of 256 x 256 in one round), momentum 20 us and X's first form 34 us, both at memory's rate.  Eight of 256 x 256:
// 5 to 5.6 us each of 15 products, which is a launch, the operands' way from the cache and back, and four tiles of k.
//
// The first launch updates the momentum and sums the squares of u by workgroups; the second adds those sums up in a fixed order
// and writes X; then three products a step, the last of which writes the result in the caller's type and orientation.  All
// matrices of a call go through each launch together.
#include "train_host.h"
#include "train_matmul.h"

#include <algorithm>

namespace ones {
namespace train {
namespace {

constexpr float kUnitX = 2048.f, kUnitA = 1024.f;

struct MomentumArgs {
  const void *grad;
  float *momentum;                            // null: u = g
  double *squares;                            // [matrices][blocks]
  int64_t size;                               // elements of a matrix
  int32_t blocks;
  int32_t type, nesterov;
  float beta;
};

// u from the momentum as it was (first) or as it is now.
__device__ __forceinline__ float update_of(float g, float m, float beta, bool nesterov) { return nesterov ? g + beta * m : m; }

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

// The squares are summed in 64 bits: those of elements above 2^64 or below 2^-75 leave the range of 32 (a finite gradient would give an
// update of zeros, or NaN).  The kernel is bound by memory either way.
template <typename T, int V>
__global__ __launch_bounds__(256) void momentum_kernel(MomentumArgs a) {
  __shared__ double part[4];
  const T *grad = static_cast<const T *>(a.grad) + blockIdx.y * a.size;
  float *momentum = a.momentum ? a.momentum + blockIdx.y * a.size : nullptr;
  double sum = 0.;
  for (int64_t i = (blockIdx.x * 256ll + threadIdx.x) * V; i < a.size; i += a.blocks * 256ll * V) {
    const Pack<T, V> g = load_pack<T, V>(grad + i);
    float m[V];
    if (momentum) {
      const Pack<float, V> old = load_pack<float, V>(momentum + i);
#pragma unroll
      for (int k = 0; k < V; ++k) m[k] = a.beta * old.v[k] + static_cast<float>(g.v[k]);
      store_pack<float, V>(momentum + i, m);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float f = static_cast<float>(g.v[k]), u = momentum ? update_of(f, m[k], a.beta, a.nesterov) : f;
      sum = __builtin_fma(static_cast<double>(u), static_cast<double>(u), sum);
    }
  }
  sum = wave_sum64(sum);
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) a.squares[static_cast<int64_t>(blockIdx.y) * a.blocks + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// What v was rounded by.
__device__ __forceinline__ f16 rest_of(float v) { return static_cast<f16>(v - static_cast<float>(static_cast<f16>(v))); }

struct NormaliseArgs {
  MomentumArgs m;
  f16 *x;                                     // [matrices][r][q_ld]
  int64_t low;                                // elements from x to what it was rounded by; 0: not wanted
  int32_t rows, cols, r, q, q_ld;             // rows > cols: turned
  float eps;
};

// 64 x 64 elements of X a workgroup, through LDS where u is turned.  Columns up to the padded length are written as zeros.
template <typename T>
__global__ __launch_bounds__(256) void normalise_kernel(NormaliseArgs a) {
  __shared__ float tile[64][65];
  __shared__ double unit;
  const T *grad = static_cast<const T *>(a.m.grad) + blockIdx.z * a.m.size;
  const float *momentum = a.m.momentum ? a.m.momentum + blockIdx.z * a.m.size : nullptr;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  if (wave == 0) {
    double sum = 0.;
#pragma unroll 4
    for (int i = lane; i < a.m.blocks; i += 64) sum += a.m.squares[static_cast<int64_t>(blockIdx.z) * a.m.blocks + i];
    sum = wave_sum64(sum);
    if (lane == 0) unit = kUnitX / (sqrt(sum) + a.eps);
  }
  const bool turned = a.rows > a.cols;
  const int q0 = blockIdx.x * 64, r0 = blockIdx.y * 64;                    // of X
  const int row0 = turned ? q0 : r0, col0 = turned ? r0 : q0;              // of u
  for (int i = wave; i < 64; i += 4) {
    const int row = row0 + i, col = col0 + lane;
    float u = 0.f;
    if (row < a.rows && col < a.cols) {
      const int64_t at = static_cast<int64_t>(row) * a.cols + col;
      const float g = static_cast<float>(grad[at]);
      u = momentum ? update_of(g, momentum[at], a.m.beta, a.m.nesterov) : g;
    }
    tile[i][lane] = u;
  }
  __syncthreads();
  f16 *x = a.x + static_cast<int64_t>(blockIdx.z) * a.r * a.q_ld;
  for (int i = wave; i < 64; i += 4) {
    const int row = r0 + i, col = q0 + lane;
    if (row < a.r && col < a.q_ld) {
      const float v = static_cast<float>((turned ? tile[lane][i] : tile[i][lane]) * unit);
      f16 *to = x + static_cast<int64_t>(row) * a.q_ld + col;
      *to = static_cast<f16>(v);
      if (a.low) to[a.low] = rest_of(v);
    }
  }
}

struct ProductArgs {
  const f16 *x, *a;                           // [matrices][r][q_ld], [matrices][r][r_ld]
  f16 *to;
  void *out;                                  // the last step's result instead, [matrices][rows][cols]
  int64_t x_low, a_low;                       // PAIRS: elements from an array to what it was rounded by
  int32_t r, q, r_ld, q_ld, out_type, turned;
  float one, two;                             // coefficients
};

// Four elements next to each other, with what they were rounded by.
template <bool PAIRS>
__device__ __forceinline__ void load_four(const f16 *p, int64_t low, float *v) {
  const Pack<f16, 4> first = load_pack<f16, 4>(p);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = static_cast<float>(first.v[k]);
  if constexpr (PAIRS) {
    const Pack<f16, 4> second = load_pack<f16, 4>(p + low);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] += static_cast<float>(second.v[k]);
  }
}
template <bool PAIRS>
__device__ __forceinline__ void store_four(f16 *p, int64_t low, const float *v) {
  store_pack<f16, 4>(p, v);
  if constexpr (PAIRS) {
    float rest[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) rest[k] = v[k] - static_cast<float>(static_cast<f16>(v[k]));
    store_pack<f16, 4>(p + low, rest);
  }
}
template <bool PAIRS>
__device__ __forceinline__ void store_one(f16 *p, int64_t low, float v) {
  *p = static_cast<f16>(v);
  if constexpr (PAIRS) p[low] = rest_of(v);
}

// A = X X^T, or (POLY) B = b A + c A A; PAIRS: of and to arrays in pairs.  Only the elements on and below the diagonal are computed; each is written to both places.
template <typename S, bool POLY, bool PAIRS>
__global__ __launch_bounds__(S::threads, S::resident) void symmetric_kernel(ProductArgs a) {
  __shared__ __align__(16) unsigned char lds[S::lds];
  const int32_t tm = (a.r_ld + S::BM - 1) / S::BM, total = static_cast<int32_t>(gridDim.x), die = static_cast<int32_t>(blockIdx.x) % 8;
  int32_t m = die * (total / 8) + min(die, total % 8) + static_cast<int32_t>(blockIdx.x) / 8, n = 0;      // a run of tiles to each die
  for (int32_t in = tiles_in_row(0, tm, S::BM, S::BN); m >= in; in = tiles_in_row(++n, tm, S::BM, S::BN)) m -= in;
  const f16 *from = POLY ? a.a + static_cast<int64_t>(blockIdx.y) * a.r * a.r_ld : a.x + static_cast<int64_t>(blockIdx.y) * a.r * a.q_ld;
  const Operand o{from, POLY ? a.r_ld : a.q_ld, a.r, POLY ? a.r_ld : a.q_ld};
  Sums<S> acc;
  const int64_t low = POLY ? a.a_low : a.x_low;
  if constexpr (PAIRS) {
    const Operand both[] = {o, Operand{from + low, o.ld, o.extent, o.k}};
    product_of_pairs<f16, false, false, S>(both, both, m * S::BM, n * S::BN, 0, o.k, lds, acc);
  } else {
    product<f16, false, false, S>(o, o, m * S::BM, n * S::BN, 0, o.k, lds, acc);
  }
  f16 *to = a.to + static_cast<int64_t>(blockIdx.y) * a.r * a.r_ld;
  const Place<S> at(m * S::BM, n * S::BN);
  const bool below = (m + 1) * S::BM <= n * S::BN;
#pragma unroll
  for (int j = 0; j < S::TN; ++j) {
    const int32_t row = at.n + j * 16;
    if (row >= a.r_ld) continue;              // rows from r on come out as zeros, which are the columns beyond r of the others
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int32_t c = at.m + i * 16;
      if (c > row) continue;
      float v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = acc[i][j][k] * (POLY ? a.two / kUnitA : kUnitA / (kUnitX * kUnitX));
      if (POLY && row < a.r) {
        float first[4];
        load_four<PAIRS>(from + static_cast<int64_t>(row) * a.r_ld + c, low, first);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] += a.one * first[k];
      }
      if (below && row < a.r) store_four<PAIRS>(to + static_cast<int64_t>(row) * a.r_ld + c, a.a_low, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (c + k > row) continue;
        if (!below && row < a.r) store_one<PAIRS>(to + static_cast<int64_t>(row) * a.r_ld + c + k, a.a_low, v[k]);
        if (c + k < row && c + k < a.r) store_one<PAIRS>(to + static_cast<int64_t>(c + k) * a.r_ld + row, a.a_low, v[k]);
      }
    }
  }
}

// X = a X + B X.
template <typename S, bool PAIRS>
__global__ __launch_bounds__(S::threads, S::resident) void apply_kernel(ProductArgs a) {
  __shared__ __align__(16) unsigned char lds[S::lds];
  const int32_t tm = (a.q + S::BM - 1) / S::BM, tn = (a.r + S::BN - 1) / S::BN;
  int32_t m, n;
  tile_of(static_cast<int32_t>(blockIdx.x), tm * tn, tm, tn, m, n);
  const f16 *x = a.x + static_cast<int64_t>(blockIdx.y) * a.r * a.q_ld, *b = a.a + static_cast<int64_t>(blockIdx.y) * a.r * a.r_ld;
  Sums<S> acc;
  const Operand l{x, a.q_ld, a.q_ld, a.r}, r{b, a.r_ld, a.r, a.r_ld};
  if constexpr (PAIRS) {
    const Operand ls[] = {l, Operand{x + a.x_low, l.ld, l.extent, l.k}}, rs[] = {r, Operand{b + a.a_low, r.ld, r.extent, r.k}};
    product_of_pairs<f16, true, false, S>(ls, rs, m * S::BM, n * S::BN, 0, a.r, lds, acc);
  } else {
    product<f16, true, false, S>(l, r, m * S::BM, n * S::BN, 0, a.r, lds, acc);
  }
  const Place<S> at(m * S::BM, n * S::BN);
  const int64_t size = static_cast<int64_t>(a.r) * a.q;
#pragma unroll
  for (int j = 0; j < S::TN; ++j) {
    const int32_t row = at.n + j * 16;
    if (row >= a.r) continue;
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
      const int32_t c = at.m + i * 16;
      if (c >= a.q_ld) continue;
      const int64_t o = static_cast<int64_t>(row) * a.q_ld + c;
      float v[4];
      load_four<PAIRS>(x + o, a.x_low, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = a.one * v[k] + acc[i][j][k] * (1.f / kUnitA);
      if (!a.out) {
        store_four<PAIRS>(a.to + static_cast<int64_t>(blockIdx.y) * a.r * a.q_ld + o, a.x_low, v);
        continue;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (c + k < a.q) {
          const int64_t to = blockIdx.y * size + (a.turned ? static_cast<int64_t>(c + k) * a.r + row : static_cast<int64_t>(row) * a.q + c + k);
          store_as(a.out, a.out_type, to, v[k] * (1.f / kUnitX));
        }
    }
  }
}

template <typename T>
void launch_momentum(const MomentumArgs &a, int64_t count, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(a.blocks), static_cast<uint32_t>(count));
  const bool wide = a.size % 4 == 0 && aligned(a.grad, 4 * sizeof(T)) && (!a.momentum || aligned(a.momentum, 16));
  if (wide) hipLaunchKernelGGL((momentum_kernel<T, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((momentum_kernel<T, 1>), grid, dim3(256), 0, s, a);
}

template <typename S>
int64_t all_tiles(const ProductArgs &a) { return ceil_div(a.r, S::BN) * ceil_div(a.q, S::BM); }

template <typename S, bool POLY, bool PAIRS>
void launch_symmetric(const ProductArgs &a, int64_t count, hipStream_t s) {
  hipLaunchKernelGGL((symmetric_kernel<S, POLY, PAIRS>), dim3(static_cast<uint32_t>(symmetric_tiles(S::BM, S::BN, a.r_ld)), static_cast<uint32_t>(count)), dim3(S::threads), 0, s, a);
}
template <bool POLY, bool PAIRS>
void launch_symmetric(const ProductArgs &a, Tiles tiles, int64_t count, hipStream_t s) {
  switch (tiles) {
    case kLarge: return launch_symmetric<Large, POLY, PAIRS>(a, count, s);
    case kMiddle: return launch_symmetric<Middle, POLY, PAIRS>(a, count, s);
    case kDeep: return launch_symmetric<Deep, POLY, PAIRS>(a, count, s);
    case kSmall: return launch_symmetric<Small, POLY, PAIRS>(a, count, s);
    default: return launch_symmetric<Tiny, POLY, PAIRS>(a, count, s);
  }
}
template <typename S, bool PAIRS>
void launch_apply(const ProductArgs &a, int64_t count, hipStream_t s) {
  hipLaunchKernelGGL((apply_kernel<S, PAIRS>), dim3(static_cast<uint32_t>(all_tiles<S>(a)), static_cast<uint32_t>(count)), dim3(S::threads), 0, s, a);
}
template <bool PAIRS>
void launch_apply(const ProductArgs &a, Tiles tiles, int64_t count, hipStream_t s) {
  switch (tiles) {
    case kLarge: return launch_apply<Large, PAIRS>(a, count, s);
    case kMiddle: return launch_apply<MiddleTurned, PAIRS>(a, count, s);
    case kDeep: return launch_apply<Deep, PAIRS>(a, count, s);
    case kSmall: return launch_apply<Small, PAIRS>(a, count, s);
    default: return launch_apply<Tiny, PAIRS>(a, count, s);
  }
}

// The steps, from x[0] to `update`.
template <bool PAIRS>
void launch_steps(ProductArgs q, const UpdateTiles &tiles, f16 *const (&x)[2], f16 *const (&a)[2], const float *coefficients, int32_t steps, void *update,
                  int64_t count, hipStream_t s) {
  for (int32_t step = 0; step < steps; ++step) {
    q.x = x[step & 1];
    q.to = a[0];
    launch_symmetric<false, PAIRS>(q, tiles.gram, count, s);
    q.a = a[0];
    q.to = a[1];
    q.one = coefficients[1]; q.two = coefficients[2];
    launch_symmetric<true, PAIRS>(q, tiles.poly, count, s);
    q.a = a[1];
    q.to = x[(step & 1) ^ 1];
    q.out = step + 1 == steps ? update : nullptr;
    q.one = coefficients[0];
    launch_apply<PAIRS>(q, tiles.apply, count, s);
  }
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

size_t ones_orthogonal_update_workspace_bytes(int64_t count, int64_t rows, int64_t cols) {
  if (check_update(count, rows, cols) != ONES_OK || !count || !rows || !cols) return 0;
  return update_plan(count, rows, cols, true).total;
}

int ones_orthogonal_update(const void *grad, float *momentum, int64_t count, int64_t rows, int64_t cols, int32_t grad_type, float beta,
                           int32_t nesterov, int32_t steps, const float *coefficients, float eps, void *update, int32_t update_type,
                           void *d_workspace, size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_update(count, rows, cols)) return rc;
  if (!is_type(grad_type) || (update_type != ONES_F16 && update_type != ONES_BF16) || steps < 1 || steps > 100 || !coefficients || !(eps >= 0.f))
    return ONES_E_INVALID_ARG;
  if (!(beta >= 0.f && beta <= 1.f)) return ONES_E_INVALID_ARG;
  for (int i = 0; i < 3; ++i)
    if (!(coefficients[i] >= -16.f && coefficients[i] <= 16.f)) return ONES_E_BOUNDS;
  if (!count || !rows || !cols) return ONES_OK;
  if (!grad || !update) return ONES_E_INVALID_ARG;
  const bool pairs = update_type == ONES_F16;
  const UpdatePlan p = update_plan(count, rows, cols, pairs);
  if (int rc = check_workspace(d_workspace, workspace_bytes, p.total)) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  char *ws = static_cast<char *>(d_workspace);
  f16 *x[2] = {reinterpret_cast<f16 *>(ws + p.x[0]), reinterpret_cast<f16 *>(ws + p.x[1])};
  f16 *a[2] = {reinterpret_cast<f16 *>(ws + p.a[0]), reinterpret_cast<f16 *>(ws + p.a[1])};
  NormaliseArgs n{};
  n.m = MomentumArgs{grad, momentum, reinterpret_cast<double *>(ws + p.squares), rows * cols, static_cast<int32_t>(p.blocks), grad_type, nesterov, beta};
  n.x = x[0];
  n.low = p.x_low;
  n.rows = static_cast<int32_t>(rows); n.cols = static_cast<int32_t>(cols);
  n.r = static_cast<int32_t>(p.r); n.q = static_cast<int32_t>(p.q); n.q_ld = static_cast<int32_t>(p.q_ld);
  n.eps = eps;
  const dim3 grid(static_cast<uint32_t>(ceil_div(p.q_ld, 64)), static_cast<uint32_t>(ceil_div(p.r, 64)), static_cast<uint32_t>(count));
  if (grad_type == ONES_F32) {
    launch_momentum<float>(n.m, count, s);
    hipLaunchKernelGGL((normalise_kernel<float>), grid, dim3(256), 0, s, n);
  } else if (grad_type == ONES_F16) {
    launch_momentum<f16>(n.m, count, s);
    hipLaunchKernelGGL((normalise_kernel<f16>), grid, dim3(256), 0, s, n);
  } else {
    launch_momentum<bf16>(n.m, count, s);
    hipLaunchKernelGGL((normalise_kernel<bf16>), grid, dim3(256), 0, s, n);
  }
  ProductArgs q{};
  q.r = n.r; q.q = n.q; q.r_ld = static_cast<int32_t>(p.r_ld); q.q_ld = n.q_ld;
  q.out_type = update_type;
  q.turned = rows > cols;
  q.x_low = p.x_low;
  q.a_low = p.a_low;
  const UpdateTiles tiles = update_tiles(count, p.r, p.q, pairs);
  if (pairs) launch_steps<true>(q, tiles, x, a, coefficients, steps, update, count, s);
  else launch_steps<false>(q, tiles, x, a, coefficients, steps, update, count, s);
  return launched("orthogonal update");
}

}  // extern "C"

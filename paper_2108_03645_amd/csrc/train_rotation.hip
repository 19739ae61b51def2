// Norms of queries and keys for each head with the rotation by positions, in one pass (ones_head_norm_rotation_*).
//
//   n = x r w, r = (mean x^2 + eps)^-1/2 over a head's row; pairs of its first 2 F elements turn by position * frequency:
//   y1 = n1 cos - n2 sin, y2 = n2 cos + n1 sin
//   g = dy turned back, dw = sum over tokens and heads of g x r, u = g w, dx = r (u - x r mean(u x r))
//
// A wave takes a token: its cosines and sines are formed once, a lane each, and serve all heads, whose rows lie 4 to 64 lanes wide in the
// wave; a lane has the same pairs in every row, so that weights, cosines and the sums of the weights' gradients stay in registers.  Backward forms r
// again instead of reading it.  The sums of the workgroups are added up by a second launch.
//
// What bounds it is memory: 32768 tokens, 16 heads and 2 of 128, bf16: forward 54 us (302 MB, 5.6 TB/s), backward 97 us (453 MB, 4.7 TB/s) and 6 for the
// weights' sums; fp32: 115 us (604 MB, 5.3 TB/s), 163 (906 MB, 5.6 TB/s) and 6.  64 tokens: 4 us, a launch's own time and a chain of loads.
#include "train_device.h"
#include "train_host.h"

#include <hip/hip_runtime.h>

namespace ones {
namespace train {
namespace {

struct RotationArgs {
  const void *x[2], *dy[2];                   // of queries and keys
  void *out[2];                               // y, or dx
  int64_t stride[2], head[2], dy_stride[2], dy_head[2];
  const void *weight[2];
  void *dweight[2];
  float *partial;
  const int32_t *positions;
  const float *frequencies;
  int64_t tokens;
  int32_t heads[2], dim, turned, weight_type, parts;       // turned: pairs that turn; parts: waves of a token
  float eps;
  bool past;
};

// VEC pairs a lane, LANES lanes a row, PER times; NEIGHBOURS: pairs are (2 i, 2 i + 1), else (i, i + turned).  What does not turn is
// taken in pairs as well: of its first and second half, or of neighbours.
template <int VEC, int LANES, int PER, bool NEIGHBOURS>
struct Pairs {
  static constexpr int count = VEC * PER;
  int32_t dim, turned, lane;
  __device__ __forceinline__ int32_t pair(int j) const { return (j * LANES + lane) * VEC; }
  __device__ __forceinline__ int32_t first(int32_t p) const { return NEIGHBOURS ? 2 * p : p < turned ? p : turned + p; }
  __device__ __forceinline__ int32_t second(int32_t p) const {
    return NEIGHBOURS ? 2 * p + 1 : p < turned ? p + turned : p + turned + (dim - 2 * turned + 1) / 2;
  }
  __device__ __forceinline__ bool has(int32_t p) const { return 2 * p < dim; }
  // (a vector is there as a whole; of single elements an odd dim lacks the last second)
  template <typename T>
  __device__ __forceinline__ void load(const T *p, float (&a)[count], float (&b)[count]) const {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int32_t k = pair(j);
#pragma unroll
      for (int i = 0; i < VEC; ++i) a[j * VEC + i] = b[j * VEC + i] = 0.f;
      if (!has(k)) continue;
      if constexpr (VEC == 1) {
        a[j] = static_cast<float>(p[first(k)]);
        if (second(k) < dim) b[j] = static_cast<float>(p[second(k)]);
      } else {
        const Pack<T, VEC> u = load_pack<T, VEC>(p + first(k)), v = load_pack<T, VEC>(p + (NEIGHBOURS ? 2 * k + VEC : second(k)));
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if constexpr (NEIGHBOURS) {
            a[j * VEC + i] = static_cast<float>(2 * i < VEC ? u.v[2 * i % VEC] : v.v[2 * i % VEC]);
            b[j * VEC + i] = static_cast<float>(2 * i < VEC ? u.v[(2 * i + 1) % VEC] : v.v[(2 * i + 1) % VEC]);
          } else {
            a[j * VEC + i] = static_cast<float>(u.v[i]);
            b[j * VEC + i] = static_cast<float>(v.v[i]);
          }
        }
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void store(T *p, const float (&a)[count], const float (&b)[count], bool past) const {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int32_t k = pair(j);
      if (!has(k)) continue;
      if constexpr (VEC == 1) {
        p[first(k)] = static_cast<T>(a[j]);
        if (second(k) < dim) p[second(k)] = static_cast<T>(b[j]);
      } else {
        float u[VEC], v[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          if constexpr (NEIGHBOURS) {
            u[i] = (i & 1 ? b : a)[j * VEC + i / 2];
            v[i] = (i & 1 ? b : a)[j * VEC + VEC / 2 + i / 2];
          } else {
            u[i] = a[j * VEC + i];
            v[i] = b[j * VEC + i];
          }
        }
        store_pack<T, VEC>(p + first(k), u, past);
        store_pack<T, VEC>(p + (NEIGHBOURS ? 2 * k + VEC : second(k)), v, past);
      }
    }
  }
  __device__ __forceinline__ void load_weights(const void *w, int32_t type, float (&a)[count], float (&b)[count]) const {
    if (type == kF32) load(static_cast<const float *>(w), a, b);
    else if (type == kF16) load(static_cast<const f16 *>(w), a, b);
    else load(static_cast<const bf16 *>(w), a, b);
  }
};

// What `both` makes of the values of the LANES lanes of a row, for all of them: between neighbours, pairs, the halves of 8 (mirrored: what they hold is the
// same by then) and of 16, then between rows of 16 and between halves of the wave.
template <int PATTERN>
__device__ __forceinline__ float from_lane(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), PATTERN, 0xf, 0xf, true));
}
template <int LANES, class Both>
__device__ __forceinline__ float of_lanes(float v, Both both) {
  v = both(v, from_lane<0xb1>(v));
  v = both(v, from_lane<0x4e>(v));
  if constexpr (LANES > 4) v = both(v, from_lane<0x141>(v));
  if constexpr (LANES > 8) v = both(v, from_lane<0x140>(v));
  if constexpr (LANES > 16) {
    const uint32_t b = __float_as_uint(v);
    const auto h = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    v = both(__uint_as_float(h[0]), __uint_as_float(h[1]));
  }
  if constexpr (LANES > 32) {
    const uint32_t b = __float_as_uint(v);
    const auto h = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    v = both(__uint_as_float(h[0]), __uint_as_float(h[1]));
  }
  return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
  return of_lanes<LANES>(v, [](float a, float b) { return a + b; });
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) {
  return of_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}

constexpr int kMaxPairs = ONES_MAX_HEAD_DIM / 2;

// Cosines and sines of a token's pairs to LDS, a lane each.  The angle is formed in turns in 64 bits, so that far positions keep
// theirs, and is at most half a turn in 32.
__device__ __forceinline__ void turns(const RotationArgs &a, int64_t token, float2 *to) {
  if (a.turned == 0) return;                  // then there may be no positions
  const double position = a.positions[token];
  for (int p = threadIdx.x % kWave; p < a.turned; p += kWave) {
    const double t = position * static_cast<double>(a.frequencies[p]) * 0.15915494309189535;
    float s, c;
    sincospif(2.f * static_cast<float>(t - rint(t)), &s, &c);
    to[p] = make_float2(c, s);
  }
}

// Forward the grid is eight waves a SIMD, which have to fit at once: up to four pairs a lane do (22453 tokens of 15 x 88 fp16: 22.6 us; with 65 registers, and
// so seven waves, 25.8).
template <typename T, int VEC, int LANES, int PER, bool NEIGHBOURS, bool BACKWARD>
__global__ __launch_bounds__(256, !BACKWARD && VEC * PER <= 4 ? 8 : 1) void rotation_kernel(RotationArgs a) {
  using P = Pairs<VEC, LANES, PER, NEIGHBOURS>;
  constexpr int count = P::count, rows = kWave / LANES;      // rows of a wave at a time
  __shared__ float2 table[4][kMaxPairs];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  const P pairs{a.dim, a.turned, lane % LANES};
  float w[2][2][count], dw[BACKWARD ? 2 : 1][2][count];
#pragma unroll
  for (int k = 0; k < 2; ++k) pairs.load_weights(a.weight[k], a.weight_type, w[k][0], w[k][1]);
  if constexpr (BACKWARD) {
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < count; ++i) dw[k][0][i] = dw[k][1][i] = 0.f;
  }
  const float inverse = 1.f / static_cast<float>(a.dim);
  const uint32_t jobs = static_cast<uint32_t>(a.tokens) * a.parts;          // parts above 1 only with few tokens
  for (uint32_t job = blockIdx.x * 4 + wave; job < jobs; job += gridDim.x * 4) {
    const int64_t token = job / a.parts;
    const int part = static_cast<int>(job % a.parts);
    turns(a, token, table[wave]);
    __builtin_amdgcn_wave_barrier();
    float c[count], s[count];
#pragma unroll
    for (int j = 0; j < PER; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int32_t p = pairs.pair(j) + i;
        const float2 v = p < a.turned ? table[wave][p] : make_float2(1.f, 0.f);
        c[j * VEC + i] = v.x;
        s[j * VEC + i] = v.y;
      }
    __builtin_amdgcn_wave_barrier();
    int turn = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      for (int h0 = 0; h0 < a.heads[k]; h0 += rows, ++turn) {
        if (turn % a.parts != part) continue;
        const int h = h0 + lane / LANES;
        const bool live = h < a.heads[k];
        float x1[count], x2[count], square = 0.f;
        if (live) pairs.load(static_cast<const T *>(a.x[k]) + token * a.stride[k] + h * a.head[k], x1, x2);
        else {
#pragma unroll
          for (int i = 0; i < count; ++i) x1[i] = x2[i] = 0.f;
        }
        float g1[count], g2[count];
        if constexpr (BACKWARD) {
          if (live) pairs.load(static_cast<const T *>(a.dy[k]) + token * a.dy_stride[k] + h * a.dy_head[k], g1, g2);
          else {
#pragma unroll
            for (int i = 0; i < count; ++i) g1[i] = g2[i] = 0.f;
          }
        }
#pragma unroll
        for (int i = 0; i < count; ++i) square = __builtin_fmaf(x1[i], x1[i], __builtin_fmaf(x2[i], x2[i], square));
        float mean = lanes_sum<LANES>(square) * inverse + a.eps, unit = 1.f;
        // Rows whose squares 32 bits do not hold, or not with all of their bits, are taken in a unit of their own, a power of two by their largest element
        // (or eps), and every other row of the wave as it is.
        const bool beyond = live && !(mean > 0x1p-100f && mean < 0x1p100f);
        if (__builtin_expect(__any(beyond), 0)) {
          float most = sqrtf(a.eps);
#pragma unroll
          for (int i = 0; i < count; ++i) most = fmaxf(most, fmaxf(fabsf(x1[i]), fabsf(x2[i])));
          most = lanes_max<LANES>(most);
          if (beyond && most > 0.f && most < INFINITY) {
            int e;
            frexpf(most, &e);
            unit = ldexpf(1.f, min(-e, 126));
          }
          square = 0.f;
#pragma unroll
          for (int i = 0; i < count; ++i) {
            x1[i] *= unit;
            x2[i] *= unit;
            square = __builtin_fmaf(x1[i], x1[i], __builtin_fmaf(x2[i], x2[i], square));
          }
          square = lanes_sum<LANES>(square);
          if (unit != 1.f) mean = square * inverse + a.eps * unit * unit;
        }
        // What is no row has no norm: with eps 0 it would be infinite, and 0 times it NaN in the weights' gradients.
        const float r = live ? rsqrtf(mean) : 0.f;
        T *out = static_cast<T *>(a.out[k]) + (token * a.heads[k] + h) * a.dim;
        if constexpr (!BACKWARD) {
#pragma unroll
          for (int i = 0; i < count; ++i) {
            const float n1 = x1[i] * r * w[k][0][i], n2 = x2[i] * r * w[k][1][i];
            x1[i] = __builtin_fmaf(n1, c[i], -(n2 * s[i]));
            x2[i] = __builtin_fmaf(n2, c[i], n1 * s[i]);
          }
          if (live) pairs.store(out, x1, x2, a.past);
        } else {
          float dot = 0.f;
#pragma unroll
          for (int i = 0; i < count; ++i) {
            const float b1 = __builtin_fmaf(g1[i], c[i], g2[i] * s[i]), b2 = __builtin_fmaf(g2[i], c[i], -(g1[i] * s[i]));
            x1[i] *= r;
            x2[i] *= r;
            dw[k][0][i] = __builtin_fmaf(b1, x1[i], dw[k][0][i]);
            dw[k][1][i] = __builtin_fmaf(b2, x2[i], dw[k][1][i]);
            g1[i] = b1 * w[k][0][i];
            g2[i] = b2 * w[k][1][i];
            dot = __builtin_fmaf(g1[i], x1[i], __builtin_fmaf(g2[i], x2[i], dot));
          }
          dot = lanes_sum<LANES>(dot) * -inverse;
          const float of_x = r * unit;
#pragma unroll
          for (int i = 0; i < count; ++i) {
            g1[i] = of_x * __builtin_fmaf(x1[i], dot, g1[i]);
            g2[i] = of_x * __builtin_fmaf(x2[i], dot, g2[i]);
          }
          if (live) pairs.store(out, g1, g2, a.past);
        }
      }
    }
  }
  if constexpr (BACKWARD) {                   // the wave's rows, then the four waves, in order
    __shared__ float sums[4][2][2 * kMaxPairs];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int j = 0; j < PER; ++j)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float u = dw[k][0][j * VEC + i], v = dw[k][1][j * VEC + i];
#pragma unroll
          for (int m = LANES; m < kWave; m *= 2) { u += __shfl_xor(u, m); v += __shfl_xor(v, m); }
          const int32_t p = pairs.pair(j) + i;
          if (lane < LANES && pairs.has(p)) {
            sums[wave][k][pairs.first(p)] = u;
            if (pairs.second(p) < a.dim) sums[wave][k][pairs.second(p)] = v;
          }
        }
    __syncthreads();
    float *to = a.partial + static_cast<int64_t>(blockIdx.x) * 2 * a.dim;
    for (int i = threadIdx.x; i < 2 * a.dim; i += 256) {
      const int k = i >= a.dim, d = k ? i - a.dim : i;
      to[i] = (sums[0][k][d] + sums[1][k][d]) + (sums[2][k][d] + sums[3][k][d]);
    }
  }
}

// The weights' gradients from n rows of partial sums: 16 threads share 64 of the 2 dim columns.
__global__ __launch_bounds__(1024) void rotation_reduce_kernel(RotationArgs a, int32_t n) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x % 64, part = threadIdx.x / 64, c = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (c < 2 * a.dim) {
#pragma unroll 8
    for (int i = part; i < n; i += 16) s += a.partial[static_cast<int64_t>(i) * 2 * a.dim + c];
  }
  sums[part][lane] = s;
  __syncthreads();
  if (part || c >= 2 * a.dim) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += sums[i][lane];
  const int k = c >= a.dim;
  if (a.dweight[k]) store_as(a.dweight[k], a.weight_type, k ? c - a.dim : c, s);
}

template <typename T, int VEC, int LANES, int PER, bool NEIGHBOURS>
void launch(const RotationArgs &a, bool backward, int64_t blocks, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(blocks)), block(256);
  if (backward) hipLaunchKernelGGL((rotation_kernel<T, VEC, LANES, PER, NEIGHBOURS, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((rotation_kernel<T, VEC, LANES, PER, NEIGHBOURS, false>), grid, block, 0, s, a);
}

template <typename T, int VEC, bool NEIGHBOURS>
void launch_lanes(const RotationArgs &a, bool backward, const RotationPlan &p, hipStream_t s) {
  switch (p.lanes) {
    case 4: return launch<T, VEC, 4, 1, NEIGHBOURS>(a, backward, p.blocks, s);
    case 8: return launch<T, VEC, 8, 1, NEIGHBOURS>(a, backward, p.blocks, s);
    case 16: return launch<T, VEC, 16, 1, NEIGHBOURS>(a, backward, p.blocks, s);
    case 32: return launch<T, VEC, 32, 1, NEIGHBOURS>(a, backward, p.blocks, s);
    default: return launch<T, VEC, 64, 1, NEIGHBOURS>(a, backward, p.blocks, s);
  }
}
template <typename T, bool NEIGHBOURS>
void launch_vectors(RotationArgs a, bool backward, hipStream_t s) {
  const RotationPlan p = rotation_plan(a.tokens, a.heads[0], a.heads[1], a.dim, a.turned, sizeof(T), backward);
  a.parts = p.parts;
  if (p.vec == 16 / sizeof(T)) return launch_lanes<T, 16 / sizeof(T), NEIGHBOURS>(a, backward, p, s);
  if (p.vec == 8 / sizeof(T)) return launch_lanes<T, 8 / sizeof(T), NEIGHBOURS>(a, backward, p, s);
  if (p.per <= 2) return launch<T, 1, 16, 2, NEIGHBOURS>(a, backward, p.blocks, s);
  if (p.per <= 8) return launch<T, 1, 16, 8, NEIGHBOURS>(a, backward, p.blocks, s);
  launch<T, 1, 16, 16, NEIGHBOURS>(a, backward, p.blocks, s);
}

void launch_type(const RotationArgs &a, int32_t type, bool neighbours, bool backward, hipStream_t s) {
  if (type == ONES_F32) neighbours ? launch_vectors<float, true>(a, backward, s) : launch_vectors<float, false>(a, backward, s);
  else if (type == ONES_F16) neighbours ? launch_vectors<f16, true>(a, backward, s) : launch_vectors<f16, false>(a, backward, s);
  else neighbours ? launch_vectors<bf16, true>(a, backward, s) : launch_vectors<bf16, false>(a, backward, s);
}

RotationArgs arguments(const void *q, int64_t q_stride, int64_t q_head, const void *k, int64_t k_stride, int64_t k_head, int64_t tokens,
                       int64_t heads, int64_t kv_heads, int64_t dim, int32_t type, const void *q_weight, const void *k_weight,
                       int32_t weight_type, float eps, const int32_t *positions, const float *frequencies, int64_t turned) {
  RotationArgs a{};
  a.x[0] = q; a.x[1] = k;
  a.stride[0] = q_stride; a.stride[1] = k_stride; a.head[0] = q_head; a.head[1] = k_head;
  a.weight[0] = q_weight; a.weight[1] = k_weight;
  a.positions = positions; a.frequencies = frequencies; a.tokens = tokens;
  a.heads[0] = static_cast<int32_t>(heads); a.heads[1] = static_cast<int32_t>(kv_heads);
  a.dim = static_cast<int32_t>(dim); a.turned = static_cast<int32_t>(turned); a.weight_type = weight_type; a.eps = eps;
  a.past = tokens * (heads + kv_heads) * dim * type_bytes(type) >= (int64_t{64} << 20);
  return a;
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

int ones_head_norm_rotation_forward(const void *q, int64_t q_stride, int64_t q_head_stride, const void *k, int64_t k_stride,
                                    int64_t k_head_stride, int64_t tokens, int64_t heads, int64_t kv_heads, int64_t dim, int32_t type,
                                    const void *q_weight, const void *k_weight, int32_t weight_type, float eps, const int32_t *positions,
                                    const float *frequencies, int64_t pairs, int32_t neighbours, void *q_out, void *k_out, void *hip_stream) {
  if (int rc = check_rotation(tokens, heads, kv_heads, dim, type, weight_type, eps, pairs)) return rc;
  if (int rc = check_rows_of_heads(q_stride, q_head_stride)) return rc;
  if (int rc = check_rows_of_heads(k_stride, k_head_stride)) return rc;
  if (tokens == 0 || heads + kv_heads == 0) return ONES_OK;
  if ((heads && (!q || !q_weight || !q_out)) || (kv_heads && (!k || !k_weight || !k_out)) || (pairs && (!positions || !frequencies))) return ONES_E_INVALID_ARG;
  RotationArgs a = arguments(q, q_stride, q_head_stride, k, k_stride, k_head_stride, tokens, heads, kv_heads, dim, type, q_weight, k_weight,
                             weight_type, eps, positions, frequencies, pairs);
  if (!q_weight) a.weight[0] = k_weight;      // of no heads: anything readable
  if (!k_weight) a.weight[1] = q_weight;
  a.out[0] = q_out; a.out[1] = k_out;
  launch_type(a, type, neighbours != 0, false, static_cast<hipStream_t>(hip_stream));
  return launched("head norm and rotation forward");
}

size_t ones_head_norm_rotation_workspace_bytes(int64_t tokens, int64_t heads, int64_t kv_heads, int64_t dim) {
  if (check_rotation(tokens, heads, kv_heads, dim, ONES_F32, ONES_F32, 0.f, 0)) return 0;
  return align_up(static_cast<size_t>(kRotationBlocks) * 2 * static_cast<size_t>(dim) * 4);
}

int ones_head_norm_rotation_backward(const void *dq_out, int64_t dq_stride, int64_t dq_head_stride, const void *dk_out, int64_t dk_stride,
                                     int64_t dk_head_stride, const void *q, int64_t q_stride, int64_t q_head_stride, const void *k,
                                     int64_t k_stride, int64_t k_head_stride, int64_t tokens, int64_t heads, int64_t kv_heads, int64_t dim,
                                     int32_t type, const void *q_weight, const void *k_weight, int32_t weight_type, float eps,
                                     const int32_t *positions, const float *frequencies, int64_t pairs, int32_t neighbours, void *dq, void *dk,
                                     void *dq_weight, void *dk_weight, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_rotation(tokens, heads, kv_heads, dim, type, weight_type, eps, pairs)) return rc;
  if (int rc = check_rows_of_heads(q_stride, q_head_stride)) return rc;
  if (int rc = check_rows_of_heads(k_stride, k_head_stride)) return rc;
  if (int rc = check_rows_of_heads(dq_stride, dq_head_stride)) return rc;
  if (int rc = check_rows_of_heads(dk_stride, dk_head_stride)) return rc;
  const bool any = tokens && heads + kv_heads;
  if (any && ((heads && (!q || !q_weight || !dq || !dq_out)) || (kv_heads && (!k || !k_weight || !dk || !dk_out)) || (pairs && (!positions || !frequencies))))
    return ONES_E_INVALID_ARG;
  if (int rc = check_workspace(d_workspace, workspace_bytes, ones_head_norm_rotation_workspace_bytes(tokens, heads, kv_heads, dim))) return rc;
  RotationArgs a = arguments(q, q_stride, q_head_stride, k, k_stride, k_head_stride, tokens, heads, kv_heads, dim, type, q_weight, k_weight,
                             weight_type, eps, positions, frequencies, pairs);
  if (!q_weight) a.weight[0] = k_weight;
  if (!k_weight) a.weight[1] = q_weight;
  a.dy[0] = dq_out; a.dy[1] = dk_out;
  a.dy_stride[0] = dq_stride; a.dy_stride[1] = dk_stride; a.dy_head[0] = dq_head_stride; a.dy_head[1] = dk_head_stride;
  a.out[0] = dq; a.out[1] = dk;
  a.dweight[0] = dq_weight; a.dweight[1] = dk_weight;
  a.partial = static_cast<float *>(d_workspace);
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (any) launch_type(a, type, neighbours != 0, true, s);
  const RotationPlan p = rotation_plan(tokens, heads, kv_heads, dim, pairs, type_bytes(type), true);
  if (dq_weight || dk_weight)
    hipLaunchKernelGGL(rotation_reduce_kernel, dim3(static_cast<uint32_t>(ceil_div(2 * dim, 64))), dim3(1024), 0, s, a, any ? static_cast<int32_t>(p.blocks) : 0);
  return launched("head norm and rotation backward");
}

}  // extern "C"

// What the kernels of a scheduled job's training step share (train_*.hip; the boundary is include/ones_train.h): the element
// types, vectors of them, and sums over a wave and a workgroup.  All arithmetic is done in 32 bits; a value is rounded to 16 bits
// once, where it is stored (to nearest, ties to even).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ones {
namespace train {

using bf16 = __bf16;
using f16 = _Float16;
constexpr int kWave = 64;

template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  T v[N];
};

// N elements from p: one wide load.  (Global memory takes wide accesses at any multiple of an element's size; the copy says so to
// the compiler.)
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T *p) {
  Pack<T, N> v;
  __builtin_memcpy(&v, p, sizeof(v));
  return v;
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const float *v) {
  Pack<T, N> out;
#pragma unroll
  for (int i = 0; i < N; ++i) out.v[i] = static_cast<T>(v[i]);
  __builtin_memcpy(p, &out, sizeof(out));
}
// The same, and, if `past`, not kept in the caches: what is written would push out what is still to be read.  For results of
// kPastBytes and more, of which a next reader would not find much in the last-level cache of 256 MiB anyway (layer norm, bf16, 32768
// x 2048: 162 us to 144; recurrence 2 x 65521 x 512: 333 to 316, 16 x 2048 x 1024: 133 to 128).
constexpr int64_t kPastBytes = 64 << 20;
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const float *v, bool past) {
  if (!past) return store_pack<T, N>(p, v);
  typedef uint32_t Words __attribute__((ext_vector_type(sizeof(T) * N / 4)));
  typedef Words Loose __attribute__((aligned(sizeof(T))));
  Pack<T, N> out;
#pragma unroll
  for (int i = 0; i < N; ++i) out.v[i] = static_cast<T>(v[i]);
  __builtin_nontemporal_store(__builtin_bit_cast(Words, out), reinterpret_cast<Loose *>(p));
}
// The same where only the first n of the elements are there (n may be 0 or less, or more than N).
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_some(const T *p, int n) {
  if (n >= N) return load_pack<T, N>(p);
  Pack<T, N> v;
#pragma unroll
  for (int i = 0; i < N; ++i) v.v[i] = i < n ? p[i] : static_cast<T>(0.f);
  return v;
}
template <typename T, int N>
__device__ __forceinline__ void store_some(T *p, const float *v, int n, bool past = false) {
  if (n >= N) return store_pack<T, N>(p, v, past);
#pragma unroll
  for (int i = 0; i < N; ++i) if (i < n) p[i] = static_cast<T>(v[i]);
}

// An element of an array whose type is only known at run time (gradients of weights, an update).
enum : int { kF32 = 0, kF16 = 1, kBF16 = 2 };
__device__ __forceinline__ void store_as(void *p, int type, int64_t i, float v) {
  if (type == kF32) static_cast<float *>(p)[i] = v;
  else if (type == kF16) static_cast<f16 *>(p)[i] = static_cast<f16>(v);
  else static_cast<bf16 *>(p)[i] = static_cast<bf16>(v);
}

// v of the lane that lies n before in its row of 16, in a ring.
template <int N>
__device__ __forceinline__ float from_row(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + N, 0xf, 0xf, true));
}
// The sum over the wave, in every lane: rows of 16 by rotations, then the four rows.
__device__ __forceinline__ float wave_sum(float v) {
  v += from_row<8>(v);
  v += from_row<4>(v);
  v += from_row<2>(v);
  v += from_row<1>(v);
  float rows[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) rows[i] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16 * i));
  return (rows[0] + rows[1]) + (rows[2] + rows[3]);
}

// The sums of two values over the THREADS threads of a row, for all of them.  `part`: 2 * THREADS / 64 words of LDS, which the
// previous call must be done with: callers alternate between two such arrays.
template <int THREADS>
__device__ __forceinline__ void row_sum2(float &a, float &b, float *part) {
  a = wave_sum(a);
  b = wave_sum(b);
  if constexpr (THREADS > kWave) {
    constexpr int waves = THREADS / kWave;
    const int wave = threadIdx.x / kWave;
    if (threadIdx.x % kWave == 0) { part[wave] = a; part[waves + wave] = b; }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < waves; ++i) { a += part[i]; b += part[waves + i]; }
  }
}

}  // namespace train
}  // namespace ones

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

// N elements from p: one wide load (p aligned to the pack).
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T *p) {
  return *reinterpret_cast<const Pack<T, N> *>(p);
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const float *v) {
  Pack<T, N> out;
#pragma unroll
  for (int i = 0; i < N; ++i) out.v[i] = static_cast<T>(v[i]);
  *reinterpret_cast<Pack<T, N> *>(p) = out;
}

// An element of an array whose type is only known at run time (weights; read once a workgroup).
enum : int { kF32 = 0, kF16 = 1, kBF16 = 2 };
__device__ __forceinline__ float load_as(const void *p, int type, int64_t i) {
  if (type == kF32) return static_cast<const float *>(p)[i];
  if (type == kF16) return static_cast<float>(static_cast<const f16 *>(p)[i]);
  return static_cast<float>(static_cast<const bf16 *>(p)[i]);
}
__device__ __forceinline__ void store_as(void *p, int type, int64_t i, float v) {
  if (type == kF32) static_cast<float *>(p)[i] = v;
  else if (type == kF16) static_cast<f16 *>(p)[i] = static_cast<f16>(v);
  else static_cast<bf16 *>(p)[i] = static_cast<bf16>(v);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) v += __shfl_xor(v, m);
  return v;
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

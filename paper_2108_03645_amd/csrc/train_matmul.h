// The matrix product that the loss (train_loss.hip) and the orthogonalised update (train_update.hip) are made of:
//
//   C[n][m] = sum over k of L(m, k) R(n, k)        16-bit operands, 32-bit sums (v_mfma_f32_16x16x32)
//
// A workgroup computes a BM x BN tile of C in registers, 64 k at a time.  Either operand may lie as rows of k ("rows": L[m][k])
// or as rows of m or n ("turned": L[k][m]); both come to LDS as they lie, by direct loads of 16 bytes a lane, into two buffers in
// turn: the next 64 k arrive while the present ones are multiplied.  Rows are read back with 16 bytes a lane, turned operands with
// the transposing read (four k of a column to every lane).  So that the lanes of a read fall into different banks, the 16-byte
// pieces of an LDS row are exchanged by the row's number; a direct load writes LDS in lane order, so the exchange is made in
// the address that each lane loads from.  What lies outside an operand is loaded from a block of zeros.
//
// A wave's sums: acc[i][j][r] is C at m = 16 i + 4 (lane / 16) + r, n = 16 j + lane % 16 of the wave's part of the tile, so a
// lane holds runs of four m, which lie next to each other in C.
#pragma once

#include "train_device.h"

namespace ones {
namespace train {
namespace {

using f32x4 = __attribute__((ext_vector_type(4))) float;
using s16x4 = __attribute__((ext_vector_type(4))) short;
using s16x8 = __attribute__((ext_vector_type(8))) short;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using LdsBytes = __attribute__((address_space(3))) unsigned char;
using GlobalBytes = __attribute__((address_space(1))) const unsigned char;

constexpr int kK = 64;                        // k of a tile in LDS

// An operand: `extent` values of m (or n), `k` of k; rows `ld` elements apart.  Base and ld are multiples of 16 bytes, and the
// length of a row (k, or extent where it is turned) is read up to the next multiple of eight.
struct Operand {
  const void *p;
  int64_t ld;
  int32_t extent, k;
};

__device__ __align__(16) const uint32_t g_zeros[4] = {0, 0, 0, 0};

template <typename T>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (__is_same(T, bf16)) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// One operand's tile of B values of m (or n) by 64 k.
template <bool TURNED, int B, int THREADS>
struct Tile {
  static constexpr int bytes = B * kK * 2, loads = bytes / 16 / THREADS, pieces = B / 8;   // pieces: of a turned row
  static_assert(loads * 16 * THREADS == bytes);
  const unsigned char *at[loads];             // what this thread loads next
  int32_t left[loads];                        // k still to come where that is positive; negative: never inside
  int64_t step;

  __device__ __forceinline__ void start(const Operand &o, int32_t first) {
    step = TURNED ? o.ld * kK * 2 : kK * 2;
#pragma unroll
    for (int i = 0; i < loads; ++i) {
      const int u = i * THREADS + static_cast<int>(threadIdx.x);
      int32_t m, k;
      if constexpr (TURNED) {
        k = u / pieces;
        const int p = u % pieces;
        m = first + ((((p >> 1) ^ ((k & 3) | ((k >> 1) & 4))) << 1) | (p & 1)) * 8;
      } else {
        const int row = u / 8;
        m = first + row;
        k = ((u % 8) ^ (row & 7)) * 8;
      }
      left[i] = m < o.extent ? o.k - k : 0;
      at[i] = static_cast<const unsigned char *>(o.p) + 2 * (TURNED ? k * o.ld + m : m * o.ld + k);
    }
  }
  // The next 64 k, into LDS at `to` (the same for the whole workgroup).
  __device__ __forceinline__ void load(unsigned char *to) {
    const int wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
#pragma unroll
    for (int i = 0; i < loads; ++i) {
      const unsigned char *from = left[i] > 0 ? at[i] : reinterpret_cast<const unsigned char *>(g_zeros);
      __builtin_amdgcn_global_load_lds((GlobalBytes *)from, (LdsBytes *)(to + (i * THREADS + wave * kWave) * 16), 16, 0, 0);
      at[i] += step;
      left[i] -= kK;
    }
  }
  // Eight k of each of 16 values from `first` (a multiple of 16) of the tile on: k = 32 half + 8 (lane / 16) + 0..7.
  static __device__ __forceinline__ s16x8 fragment(const unsigned char *from, int first, int half, int lane) {
    if constexpr (TURNED) {
      const int q = lane >> 4, j = (lane >> 2) & 3, unit = (first >> 4) ^ (j | ((q & 1) << 2));
      const unsigned char *p = from + (half * 32 + q * 8 + j) * (B * 2) + unit * 32 + (lane & 3) * 8;
      typedef __attribute__((address_space(3))) s16x4 Lds;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)(p + 4 * B * 2));
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int row = first + (lane & 15);
      return *reinterpret_cast<const s16x8 *>(from + row * (kK * 2) + (((half * 4 + (lane >> 4)) ^ (lane & 7)) << 4));
    }
  }
};

// BM x BN tiles by WM x WN waves.
template <int BM_, int BN_, int WM_, int WN_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, threads = WM * WN * kWave;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;       // 16 x 16 products of a wave
  static constexpr int lds = 2 * (BM + BN) * kK * 2;
};
using Large = Shape<256, 256, 2, 4>;
using Small = Shape<128, 128, 2, 2>;

template <typename S>
using Sums = f32x4[S::TM][S::TN];

template <typename T, bool LT, bool RT, typename S>
__device__ __forceinline__ void product(const Operand &L, const Operand &R, int32_t m0, int32_t n0, unsigned char *lds, Sums<S> &acc) {
  constexpr int lbytes = S::BM * kK * 2, buffer = (S::BM + S::BN) * kK * 2;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int wm = (wave / S::WN) * (S::BM / S::WM), wn = (wave % S::WN) * (S::BN / S::WN);
  Tile<LT, S::BM, S::threads> l;
  Tile<RT, S::BN, S::threads> r;
  l.start(L, m0);
  r.start(R, n0);
#pragma unroll
  for (int i = 0; i < S::TM; ++i)
#pragma unroll
    for (int j = 0; j < S::TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int tiles = (L.k + kK - 1) / kK;
  if (tiles > 0) {
    l.load(lds);
    r.load(lds + lbytes);
  }
  for (int t = 0; t < tiles; ++t) {
    unsigned char *now = lds + (t & 1) * buffer, *next = lds + ((t & 1) ^ 1) * buffer;
    __syncthreads();                          // the present tile has arrived; the other buffer has been read by all
    if (t + 1 < tiles) {
      l.load(next);
      r.load(next + lbytes);
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      s16x8 a[S::TM], b[S::TN];
#pragma unroll
      for (int j = 0; j < S::TN; ++j) b[j] = r.fragment(now + lbytes, wn + j * 16, half, lane);
#pragma unroll
      for (int i = 0; i < S::TM; ++i) a[i] = l.fragment(now, wm + i * 16, half, lane);
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[i][j] = mfma<T>(a[i], b[j], acc[i][j]);
    }
  }
}

// Where a lane's runs of four m start, and its n: of sum (i, j), in the whole of C.
template <typename S>
struct Place {
  int32_t m, n;
  __device__ __forceinline__ Place(int32_t m0, int32_t n0) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    m = m0 + (wave / S::WN) * (S::BM / S::WM) + (lane >> 4) * 4;
    n = n0 + (wave % S::WN) * (S::BN / S::WN) + (lane & 15);
  }
};

// Tile `id` of tm x tn: ids go round the eight dies, whose L2s are separate, so each die takes a run of neighbouring tiles, by
// groups of four rows of tiles.
__device__ __forceinline__ void tile_of(int32_t id, int32_t total, int32_t tm, int32_t tn, int32_t &m, int32_t &n) {
  const int32_t each = total / 8, rest = total % 8, die = id % 8;
  const int32_t t = die * each + min(die, rest) + id / 8;
  const int32_t group = t / (4 * tm), in = t % (4 * tm), rows = min(4, tn - group * 4);
  n = group * 4 + in % rows;
  m = in / rows;
}

}  // namespace
}  // namespace train
}  // namespace ones

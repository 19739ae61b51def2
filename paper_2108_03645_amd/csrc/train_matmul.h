// The matrix product that the loss (train_loss.hip) and the orthogonalised update (train_update.hip) are made of:
//
//   C[n][m] = sum over k of L(m, k) R(n, k)        16-bit operands, 32-bit sums (v_mfma_f32_16x16x32)
//
// A workgroup computes a BM x BN tile of C in registers, 64 k at a time.  Either operand may lie as rows of k ("rows": L[m][k])
// or as rows of m or n ("turned": L[k][m]); both come to LDS as they lie, by direct loads of 16 bytes a lane, into two to
// four buffers in turn: the next k arrive while the present ones are multiplied.  Rows are read back with 16 bytes a lane, turned operands with
// the transposing read (four k of a column to every lane).  So that the lanes of a read fall into different banks, the 16-byte
// pieces of an LDS row are exchanged by the row's number; a direct load writes LDS in lane order, so the exchange is made in
// the address that each lane loads from.  What lies outside an operand comes as zeros, by the loads' own bounds.
//
// A wave's sums: acc[i][j][r] is C at m = 16 i + 4 (lane / 16) + r, n = 16 j + lane % 16 of the wave's part of the tile, so a
// lane holds runs of four m, which lie next to each other in C.
#pragma once

#include "train_device.h"
#include "train_plan.h"

namespace ones {
namespace train {
namespace {

using f32x4 = __attribute__((ext_vector_type(4))) float;
using s16x4 = __attribute__((ext_vector_type(4))) short;
using s16x8 = __attribute__((ext_vector_type(8))) short;
using bf16x8 = __attribute__((ext_vector_type(8))) __bf16;
using f16x8 = __attribute__((ext_vector_type(8))) _Float16;
using LdsBytes = __attribute__((address_space(3))) unsigned char;

// An operand: `extent` values of m (or n), `k` of k; rows `ld` elements apart.  Base and ld are multiples of 16 bytes, and the
// length of a row (k, or extent where it is turned) is read up to the next multiple of eight.  ld <= kMaxLoadableStride.
struct Operand {
  const void *p;
  int64_t ld;
  int32_t extent, k;
};

template <typename T>
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c) {
  if constexpr (__is_same(T, bf16)) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A value that is the same in all lanes, in a scalar register.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// A direct load of 16 bytes a lane to LDS: lane i's land at to + 16 i, zeros where `offset` is not below the `bytes` from base on that
// may be read.  Written as text: with the builtin in flight the compiler
// waits for all of LDS's reads where it needs the first of them (it takes the load for one that may return through either
// counter), and the reads ahead would be in vain.  It has no result in registers; meet() waits for it.
// (s_nop: a scalar register that a vector instruction wrote, a v_readlane of a spilled one among them, is read five cycles later at
// the earliest, m0 one instruction later; the compiler sees to neither inside text.)
__device__ __forceinline__ void load_to_lds(const unsigned char *base, uint32_t bytes, uint32_t offset, uint32_t to) {
  const uint64_t at = reinterpret_cast<uintptr_t>(base);
  typedef __attribute__((ext_vector_type(4))) uint32_t Descriptor;      // of a buffer of bytes: address, length, 32-bit data
  const Descriptor buffer{uniform(static_cast<uint32_t>(at)), uniform(static_cast<uint32_t>(at >> 32)), uniform(bytes), 0x00020000};
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer), "{m0}"(to) : "memory");
}

// The workgroup meets, and the direct loads to LDS of all its waves, but for the last PENDING of each, have arrived: a barrier
// alone does not wait for them.  (Memory operations are counted off in the order they were issued in; stores behind the loads
// make the wait longer, not shorter.)
template <int PENDING>
__device__ __forceinline__ void meet() {
  static_assert(PENDING < 64);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(PENDING) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// One operand's tile of B values of m (or n) by K of k.
template <bool TURNED, int B, int K, int THREADS>
struct Tile {
  static constexpr int bytes = B * K * 2, loads = bytes / 16 / THREADS;
  static constexpr int pieces = TURNED ? B / 8 : K / 8;            // 16-byte pieces of a row in LDS
  static constexpr int rows = THREADS / pieces;                    // LDS rows that one load of the workgroup fills
  static_assert(loads * 16 * THREADS == bytes && rows % (TURNED ? 16 : 8) == 0);
  static constexpr uint32_t kOutside = 0x80000000;
  const unsigned char *base;                  // of the next load: element (first, k); the same for all threads
  uint32_t row_bytes;                         // from an LDS row to the next in memory
  uint32_t offset;                            // from there to what this thread loads, in bytes; kOutside beyond a row's end
  int32_t piece;                              // k (m where turned) in the tile, of what this thread loads
  int32_t m_left, k_left;                     // what is left of the operand from base on, of m no more than a tile

  // The place of logical piece `p` of LDS row `row`, so that the lanes of a read meet different banks.  A read of rows takes the
  // same piece of eight rows at a time; a transposing read takes 32 bytes (a unit of two pieces) of rows k..k+3, and of k+8.
  static __device__ __forceinline__ int place(int row, int p) {
    if constexpr (TURNED) return p ^ ((((row & 3) | ((row >> 1) & 4)) & (B / 16 - 1)) << 1);
    else return p ^ (row & 7);
  }
  static_assert((TURNED ? K : B) * 2 * kMaxLoadableStride < kOutside);          // and so what is added to either never wraps
  // The loads of a thread lie `rows` LDS rows apart, a multiple of what place() goes by, so they share one offset.  Rows beyond the
  // operand's are kept out by the length of what may be read, the ends of rows by the offset.
  __device__ __forceinline__ void start(const Operand &o, int32_t first, int32_t k0) {
    const int row = static_cast<int>(threadIdx.x) / pieces;
    piece = place(row, static_cast<int>(threadIdx.x) % pieces) * 8;
    k_left = o.k - k0;
    m_left = min(o.extent - first, B);
    row_bytes = static_cast<uint32_t>(o.ld * 2);
    base = static_cast<const unsigned char *>(o.p) + 2 * (TURNED ? k0 * o.ld + first : first * o.ld + k0);
    offset = piece < (TURNED ? m_left : k_left) ? row * row_bytes + piece * 2 : kOutside;
  }
  // One of the loads of the next K, into LDS at `to` (the same for the whole workgroup); advance() behind the last.
  __device__ __forceinline__ void load_one(unsigned char *to, int i) {
    const uint32_t mine = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((LdsBytes *)to)) +
                          __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave) * (kWave * 16);
    const uint32_t inside = TURNED ? max(min(k_left, K), 0) : m_left;
    load_to_lds(base, inside * row_bytes, offset + i * rows * row_bytes, mine + i * THREADS * 16);
  }
  __device__ __forceinline__ void advance() {
    base += TURNED ? static_cast<uint64_t>(K) * row_bytes : K * 2;
    k_left -= K;
    if (!TURNED) offset = piece < k_left ? offset : kOutside;
  }
  __device__ __forceinline__ void load(unsigned char *to) {
#pragma unroll
    for (int i = 0; i < loads; ++i) load_one(to, i);
    advance();
  }
  // Eight k of each of 16 values from `first` (a multiple of 16) of the tile on: k = 32 half + 8 (lane / 16) + 0..7.
  static __device__ __forceinline__ s16x8 fragment(const unsigned char *from, int first, int half, int lane) {
    if constexpr (TURNED) {
      const int k = half * 32 + (lane >> 4) * 8 + ((lane >> 2) & 3);
      const unsigned char *p = from + k * (B * 2) + place(k, first >> 3) * 16 + (lane & 3) * 8;
      typedef __attribute__((address_space(3))) s16x4 Lds;
      const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)(p + 4 * B * 2));
      return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int row = first + (lane & 15);
      return *reinterpret_cast<const s16x8 *>(from + row * (K * 2) + place(lane & 15, half * 4 + (lane >> 4)) * 16);
    }
  }
};

// BM x BN tiles by WM x WN waves, K of k at a time in BUFFERS places of LDS; RESIDENT workgroups a compute unit.
template <int BM_, int BN_, int WM_, int WN_, int BUFFERS_, int RESIDENT_>
struct Shape {
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, K = 64, threads = WM * WN * kWave, buffers = BUFFERS_, resident = RESIDENT_;
  static constexpr int TM = BM / WM / 16, TN = BN / WN / 16;       // 16 x 16 products of a wave
  static constexpr int lds = buffers * (BM + BN) * K * 2;
};
// What carries them: two waves a SIMD at least (four waves of 64 x 64 on a tile of 128 x 128 take 1.2 times as long as eight of
// 64 x 32, although those read half as much again from LDS), and, where a compute unit holds one workgroup, four buffers
// instead of two (136 tiles of 128 x 128, k 2048: 21 us against 26).  An operand that is turned has 64, 128 or 256 values.
using Large = Shape<256, 256, 2, 4, 2, 1>;
using Middle = Shape<192, 128, 4, 2, 3, 1>;
using MiddleTurned = Shape<128, 192, 2, 4, 3, 1>;
using Deep = Shape<128, 128, 2, 4, 4, 1>;
using Small = Shape<128, 128, 2, 4, 2, 2>;
using Tiny = Shape<64, 64, 2, 2, 4, 2>;

// The plans (train_plan.h) count these.
template <typename S, Tiles T>
constexpr bool kCounted = S::BM == kTileCosts[T].bm && S::BN == kTileCosts[T].bn && S::resident * 256 == kTileCosts[T].places;
static_assert(kCounted<Large, kLarge> && kCounted<Middle, kMiddle> && kCounted<Deep, kDeep> && kCounted<Small, kSmall> && kCounted<Tiny, kTiny> &&
              MiddleTurned::BM == Middle::BN && MiddleTurned::BN == Middle::BM);
static_assert(Large::WM == 2 && Deep::WM == 2 && Small::WM == 2 && Tiny::WM == 2);      // parts of the loss: two a tile of logits

template <typename S>
using Sums = f32x4[S::TM][S::TN];

// The sums over k0 <= k < k1 (k0 a multiple of S::K; k1 the operands' k, or a multiple too).  begin() sets the loads of the first
// tiles of k off, run() multiplies; a workgroup may begin its next product before it deals with the sums of the last.
template <typename T, bool LT, bool RT, typename S>
struct Product {
  static constexpr int lbytes = S::BM * S::K * 2, buffer = (S::BM + S::BN) * S::K * 2;
  Tile<LT, S::BM, S::K, S::threads> l;
  Tile<RT, S::BN, S::K, S::threads> r;
  int tiles;

  __device__ __forceinline__ void begin(const Operand &L, const Operand &R, int32_t m0, int32_t n0, int32_t k0, int32_t k1, unsigned char *lds) {
    l.start(L, m0, k0);
    r.start(R, n0, k0);
    tiles = (k1 - k0 + S::K - 1) / S::K;
#pragma unroll
    for (int t = 0; t < S::buffers; ++t)
      if (t < tiles) {
        l.load(lds + t * buffer);
        r.load(lds + t * buffer + lbytes);
      }
  }

  static constexpr int kRows = S::TM <= 5 ? S::TM : S::TM / 2, groups = S::TM / kRows, phases = 2 * groups;
  static constexpr int l_loads = Tile<LT, S::BM, S::K, S::threads>::loads, r_loads = Tile<RT, S::BN, S::K, S::threads>::loads;
  static constexpr int of_tile = l_loads + r_loads;
  static_assert(S::K == 64 && S::TM % kRows == 0);

  // The products of one tile of k, in phases of up to five fragments of L by all of R.  The reads of the next phase, and the loads of a
  // later tile, are put between the rows of products of a phase: a wave issues in order, and behind a run of reads or
  // loads its products would wait for the queues that all eight waves fill at once.  The workgroup meets where the last fragments
  // of the tile have been read: from there on its buffer takes a later tile, and the next tile has arrived.
  template <bool MORE>                        // there is a tile to load
  __device__ __forceinline__ void multiply(unsigned char *now, unsigned char *next, int wm, int wn, int lane, s16x8 (&a)[2][kRows], s16x8 (&b)[2][S::TN],
                                           Sums<S> &acc) {
#pragma unroll
    for (int p = 0; p < phases; ++p) {
      const int half = p / groups, group = p % groups;
      const bool last = p + 1 == phases, turns = last || (p + 1) % groups == 0;            // turns: to the other half
      const unsigned char *from = last ? next : now;
      const int next_half = last ? 0 : (p + 1) / groups, next_group = (p + 1) % groups;
      if (last) meet<MORE ? (S::buffers - 2) * of_tile : 0>();
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int bs = turns ? S::TN : 0, n = bs + kRows;     // R's fragments first: the next phase begins with all of them
#pragma unroll
        for (int e = i * n / kRows; e < (i + 1) * n / kRows; ++e) {      // behind the last tile: of what lies there, not used
          if (e < bs) b[next_half][e] = r.fragment(from + lbytes, wn + e * 16, next_half, lane);
          else a[(p + 1) & 1][e - bs] = l.fragment(from, wm + (next_group * kRows + e - bs) * 16, next_half, lane);
        }
        if (MORE && last) {
#pragma unroll
          for (int e = i * l_loads / kRows; e < (i + 1) * l_loads / kRows; ++e) l.load_one(now, e);
#pragma unroll
          for (int e = i * r_loads / kRows; e < (i + 1) * r_loads / kRows; ++e) r.load_one(now + lbytes, e);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[group * kRows + i][j] = mfma<T>(a[p & 1][i], b[half][j], acc[group * kRows + i][j]);
        __builtin_amdgcn_sched_barrier(0);
      }
      if (MORE && last) {
        l.advance();
        r.advance();
      }
    }
  }

  template <bool ADDS = false>                // to what acc holds
  __device__ __forceinline__ void run(unsigned char *lds, Sums<S> &acc) {
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int wm = (wave / S::WN) * (S::BM / S::WM), wn = (wave % S::WN) * (S::BN / S::WN);
    if constexpr (!ADDS) {
#pragma unroll
      for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (tiles <= 0) return;
    s16x8 a[2][kRows], b[2][S::TN];
    if (tiles >= S::buffers) meet<(S::buffers - 1) * of_tile>();
    else meet<0>();
#pragma unroll
    for (int j = 0; j < S::TN; ++j) b[0][j] = r.fragment(lds + lbytes, wn + j * 16, 0, lane);
#pragma unroll
    for (int i = 0; i < kRows; ++i) a[0][i] = l.fragment(lds, wm + i * 16, 0, lane);
    unsigned char *now = lds, *const end = lds + S::buffers * buffer;
    auto after = [&](unsigned char *p) { return p + buffer == end ? lds : p + buffer; };
    int t = 0;
    for (; t + S::buffers < tiles; ++t, now = after(now)) multiply<true>(now, after(now), wm, wn, lane, a, b, acc);
    for (; t < tiles; ++t, now = after(now)) multiply<false>(now, after(now), wm, wn, lane, a, b, acc);
  }
};

template <typename T, bool LT, bool RT, typename S, bool ADDS = false>
__device__ __forceinline__ void product(const Operand &L, const Operand &R, int32_t m0, int32_t n0, int32_t k0, int32_t k1, unsigned char *lds,
                                        Sums<S> &acc) {
  Product<T, LT, RT, S> p;
  p.begin(L, R, m0, n0, k0, k1, lds);
  p.template run<ADDS>(lds, acc);
}
// The same of operands held in pairs, the second what the first was rounded by: three products, without that of the two seconds (2^-22).
template <typename T, bool LT, bool RT, typename S>
__device__ __forceinline__ void product_of_pairs(const Operand (&L)[2], const Operand (&R)[2], int32_t m0, int32_t n0, int32_t k0, int32_t k1,
                                                 unsigned char *lds, Sums<S> &acc) {
  product<T, LT, RT, S>(L[1], R[0], m0, n0, k0, k1, lds, acc);
  product<T, LT, RT, S, true>(L[0], R[1], m0, n0, k0, k1, lds, acc);
  product<T, LT, RT, S, true>(L[0], R[0], m0, n0, k0, k1, lds, acc);
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

// The runs of four of two sums (i, j) and (i + 1, j), rounded: lanes of even groups of 16 get the next eight of the first from their
// own and the next group's run, those of odd groups of the second.  (v_permlane16_swap: odd groups of one register for even ones of another.)
template <typename T>
__device__ __forceinline__ Pack<uint32_t, 4> swapped(f32x4 first, f32x4 second) {
  Pack<T, 4> a, b;
#pragma unroll
  for (int r = 0; r < 4; ++r) { a.v[r] = static_cast<T>(first[r]); b.v[r] = static_cast<T>(second[r]); }
  const uint2 wa = __builtin_bit_cast(uint2, a), wb = __builtin_bit_cast(uint2, b);
  const auto lo = __builtin_amdgcn_permlane16_swap(wa.x, wb.x, false, false), hi = __builtin_amdgcn_permlane16_swap(wa.y, wb.y, false, false);
  return Pack<uint32_t, 4>{{lo[0], hi[0], lo[1], hi[1]}};
}
// Where those eight start, from Place::m and for i = 0.
template <typename S>
__device__ __forceinline__ int32_t swapped_m(int32_t m) {
  static_assert(S::TM % 2 == 0);
  const int group = static_cast<int>(threadIdx.x) % kWave >> 4;
  return m - group * 4 + (group & 1) * 16 + (group >> 1) * 8;
}

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

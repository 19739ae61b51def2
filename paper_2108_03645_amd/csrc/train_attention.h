// What the attention kernels (train_attention.hip, train_attention_step.hip) share: tiles of rows in LDS that products read along
// the rows and across them, and the way from a workgroup's number to its rows of a sequence.
//
// A product C[m][n] = sum over k of A(m, k) B(n, k) is made of 16 x 16 x 32 matrix instructions: of A and B a lane gives eight k of
// m = n = lane % 16, of C it holds m = 4 (lane / 16) + 0..3 for n = lane % 16.  The kernels choose A and B so that what comes
// out of one product, scores with the rows of the long operand as m, is in place as B of the next one, whose k those rows are: of 32 rows a lane
// holds 4 g + 0..3 and 16 + 4 g + 0..3 (g = lane / 16), and since the order of k does not matter as long as A has the same, A's
// transposing reads fetch these rows.  So the scores never leave the registers.
#pragma once

#include "train_matmul.h"

namespace ones {
namespace train {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// fp16 keeps 2^-24 and up: the exponentials below the row's largest are held in units of 2^-8.
template <typename T>
constexpr float kShift = __is_same(T, f16) ? 8.f : 0.f;

// As load_to_lds, four bytes a lane.
__device__ __forceinline__ void load_words_to_lds(const unsigned char *base, uint32_t bytes, uint32_t offset, uint32_t to) {
  const uint64_t at = reinterpret_cast<uintptr_t>(base);
  typedef __attribute__((ext_vector_type(4))) uint32_t Descriptor;
  const Descriptor buffer{uniform(static_cast<uint32_t>(at)), uniform(static_cast<uint32_t>(at >> 32)), uniform(bytes), 0x00020000};
  asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(offset), "s"(buffer), "{m0}"(to) : "memory");
}

// A tile of ROWS rows of D elements (a head's rows of consecutive tokens).  The 16-byte pieces of a row are exchanged by the row's
// number so that the lanes of a read meet different banks (of 64, 256 bytes at a time), whichever way they read: two pieces of eight rows, or
// along the rows one piece of rows 0..3 and 12..15 with the next of rows 4..11 (lanes 0..3, 12..15 and 20..27 read at the same time).  (D 64: two
// rows are 256 bytes.)
// D: 32, 64, 96 or 128, of which dim may be less; a row has the room of 64 or 128.
template <int D>
constexpr int kPieces = D <= 64 ? 8 : 16;
template <int D, int ROWS, int THREADS>
struct RowTile {
  static constexpr int pieces = kPieces<D>, row = pieces * 16, bytes = ROWS * row, at_once = THREADS / pieces, loads = (ROWS + at_once - 1) / at_once;
  static_assert(at_once % 16 == 0 && ROWS % 16 == 0);
  static constexpr uint32_t kOutside = 0x80000000;
  const unsigned char *base;                  // of the next tile's first row; the same for all threads
  uint32_t row_bytes, offset;                 // between rows in memory; what this thread loads, kOutside beyond a row's end
  int32_t left;                               // rows from base on

  static __device__ __forceinline__ int exchange(int r) {
    return pieces > 8 ? ((r & 7) << 1) ^ (r & 8 ? 9 : 0) : (r & 6) ^ (r & 8 ? 5 : 0);
  }
  __device__ __forceinline__ void start(const void *first, int64_t stride, int32_t rows, int32_t dim) {
    const int r = static_cast<int>(threadIdx.x) / pieces, p = (static_cast<int>(threadIdx.x) % pieces) ^ exchange(r);
    base = static_cast<const unsigned char *>(first);
    row_bytes = static_cast<uint32_t>(stride * 2);
    offset = p * 8 < dim && r < ROWS ? r * row_bytes + p * 16 : kOutside;
    left = rows;
  }
  // The next tile to LDS at `to` (the same for the whole workgroup); rows beyond the last come as zeros.
  __device__ __forceinline__ void load(unsigned char *to) {
    const uint32_t wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
    const uint32_t mine = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((LdsBytes *)to)) + wave * (kWave * 16);
    const uint32_t inside = static_cast<uint32_t>(max(min(left, ROWS), 0)) * row_bytes;
#pragma unroll
    for (int i = 0; i < loads; ++i)
      if (at_once <= ROWS || wave * (kWave / pieces) < ROWS) load_to_lds(base, inside, offset + i * at_once * row_bytes, mine + i * THREADS * 16);
    base += static_cast<uint64_t>(ROWS) * row_bytes;
    left -= ROWS;
  }
  // A lane's place for reading along the rows (16 rows from a multiple of 16 on, elements 32 step + 8 (lane / 16) + 0..7)...
  static __device__ __forceinline__ int along(int lane, int step) {
    const int r = lane & 15;
    return r * row + (((step * 4 + (lane >> 4)) ^ exchange(r)) << 4);
  }
  static __device__ __forceinline__ s16x8 read_along(const unsigned char *from, int first, int place) {
    return *reinterpret_cast<const s16x8 *>(from + first * row + place);
  }
  // ... and across them: element 16 block + lane % 16 of rows 4 (lane / 16) + 0..3 and 16 + 4 (lane / 16) + 0..3 of 32.
  static __device__ __forceinline__ int across(int lane, int block) {
    const int r = (lane >> 4) * 4 + ((lane >> 2) & 3);
    return r * row + (((block * 2 + ((lane >> 1) & 1)) ^ exchange(r)) << 4) + (lane & 1) * 8;
  }
  static __device__ __forceinline__ s16x8 read_across(const unsigned char *from, int first, int place) {
    typedef __attribute__((address_space(3))) s16x4 Lds;
    const unsigned char *p = from + first * row + place;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds *)(p + 16 * row));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// Eight elements of row lane % 16 (of `rows`; others, and what lies beyond dim, zeros) for every 32 of a row: an operand in registers.
template <int D>
__device__ __forceinline__ void read_rows(const void *first, int64_t stride, int32_t rows, int32_t dim, int lane, s16x8 (&to)[D / 32]) {
  const int r = lane & 15;
#pragma unroll
  for (int s = 0; s < D / 32; ++s) {
    const int at = s * 32 + (lane >> 4) * 8;
    to[s] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
    if (r < rows && at < dim) to[s] = *reinterpret_cast<const s16x8 *>(static_cast<const short *>(first) + r * stride + at);
  }
}

// Eight scores of 32 rows (two C of 16) as eight k of an operand.
template <typename T>
__device__ __forceinline__ s16x8 rounded(f32x4 a, f32x4 b) {
  Pack<T, 8> v;
#pragma unroll
  for (int r = 0; r < 4; ++r) { v.v[r] = static_cast<T>(a[r]); v.v[4 + r] = static_cast<T>(b[r]); }
  return __builtin_bit_cast(s16x8, v);
}

// What the rounding took from them.
template <typename T>
__device__ __forceinline__ s16x8 remainder(f32x4 a, f32x4 b, s16x8 of) {
  const Pack<T, 8> w = __builtin_bit_cast(Pack<T, 8>, of);
#pragma unroll
  for (int r = 0; r < 4; ++r) { a[r] -= static_cast<float>(w.v[r]); b[r] -= static_cast<float>(w.v[4 + r]); }
  return rounded<T>(a, b);
}

template <int D, int TN>
__device__ __forceinline__ bool any_nan(const f32x4 (&acc)[D / 16][TN]) {
  bool found = false;
#pragma unroll
  for (int b = 0; b < D / 16; ++b)
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int r = 0; r < 4; ++r) found |= acc[b][n][r] != acc[b][n][r];
  return found;
}

// What is not finite among element d of the rows that a row sees, looked for as far as is asked, from the first row on; 16 at once, so that they are under
// way together.
struct Seen {
  float most = 0.f, least = 0.f;
  uint32_t size = 0;                          // the largest, as bits without the sign: NaN lies above infinity
  int32_t next = 0;
  __device__ __forceinline__ void add(float x) {
    most = fmaxf(most, x);
    least = fminf(least, x);
    size = max(size, __float_as_uint(x) & 0x7fffffff);
  }
  __device__ __forceinline__ bool up() const { return most == __builtin_inff(); }
  __device__ __forceinline__ bool down() const { return least == -__builtin_inff(); }
  __device__ __forceinline__ bool finite() const { return size < 0x7f800000; }
  // Whether a sum over it, with weights above 0, is NaN; whether it is one infinity.
  __device__ __forceinline__ bool no_number() const { return size > 0x7f800000 || (up() && down()); }
  __device__ __forceinline__ bool infinite() const { return size == 0x7f800000 && up() != down(); }
  template <typename T>
  __device__ __forceinline__ void through(const T *rows, int64_t stride, int32_t last, int d) {
    while (next <= last && !no_number()) {
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = static_cast<float>(rows[min(next + i, last) * stride + d]);
#pragma unroll
      for (int i = 0; i < 16; ++i) add(x[i]);
      next += 16;
    }
    next = min(next, last + 1);
  }
};

// Over the four lanes of a wave that hold the same n.
__device__ __forceinline__ float across_max(float v) {
  const uint32_t b = __float_as_uint(v);
  const auto h = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  v = fmaxf(__uint_as_float(h[0]), __uint_as_float(h[1]));
  const uint32_t c = __float_as_uint(v);
  const auto q = __builtin_amdgcn_permlane16_swap(c, c, false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float across_sum(float v) {
  const uint32_t b = __float_as_uint(v);
  const auto h = __builtin_amdgcn_permlane32_swap(b, b, false, false);
  v = __uint_as_float(h[0]) + __uint_as_float(h[1]);
  const uint32_t c = __float_as_uint(v);
  const auto q = __builtin_amdgcn_permlane16_swap(c, c, false, false);
  return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// Sequences lie one behind the other, offsets[s] .. offsets[s + 1] (pulled into 0 .. tokens).  Workgroups are numbered by slots of
// TILE rows: sequence s has the slots from offsets[s] / TILE + s + 1 on, which is enough room for its tiles whatever the offsets
// are (a partial tile fits into the one that is added for each sequence), so a slot's sequence is found by a search and nothing has
// to be planned ahead.  The rows in front of the first and behind the last sequence are sequences -1 and `sequences`.
__host__ __device__ inline int64_t slots_of(int64_t tokens, int64_t sequences, int64_t tile) { return tokens / tile + sequences + 2; }

struct Rows {
  int32_t sequence, first, length, at;        // the sequence: its first row, its rows; the slot's first row in it
  bool real;                                  // a sequence; or rows outside all of them
};
// The first slot of sequence s, which begins at row `first`.
template <int TILE>
__device__ __forceinline__ int32_t slot_of(int32_t s, int32_t first) { return s < 0 ? 0 : first / TILE + s + 1; }

template <int TILE>
__device__ __forceinline__ Rows rows_of(const int32_t *offsets, int32_t sequences, int32_t tokens, int32_t slot) {
  const int lane = static_cast<int>(threadIdx.x) % kWave;
  auto offset = [&](int32_t s) { return min(max(offsets[s], 0), tokens); };
  int32_t lo = 0, n = sequences + 1;          // the number of s whose first slot is not above this one, 64 probes at a time
  while (n > 0) {
    const int32_t stride = (n + kWave - 1) / kWave, mine = lane * stride + stride - 1;
    const bool below = mine < n && slot_of<TILE>(lo + mine, offset(lo + mine)) <= slot;
    const int32_t c = __popcll(__ballot(below));
    lo += c * stride;
    n = stride == 1 ? 0 : min(stride, n - c * stride);
  }
  const int32_t s = __builtin_amdgcn_readfirstlane(lo) - 1;
  Rows r;
  r.first = s < 0 ? 0 : offset(s);
  const int32_t end = s < 0 ? offset(0) : s >= sequences ? tokens : offset(s + 1);
  r.first = __builtin_amdgcn_readfirstlane(r.first);
  r.length = max(__builtin_amdgcn_readfirstlane(end) - r.first, 0);
  r.sequence = s;
  r.at = (slot - slot_of<TILE>(s, r.first)) * TILE;
  r.real = s >= 0 && s < sequences;
  return r;
}

// Which slot and head a workgroup takes.  Workgroups go round the eight dies, whose L2s are separate: heads that read the same keys follow
// each other in steps of kv_heads, so that a die mostly meets few of those.
struct Turn {
  int32_t slot, head, kv;
};
__device__ __forceinline__ Turn turn_of(uint32_t id, int32_t heads, int32_t kv_heads) {
  const int32_t in = static_cast<int32_t>(id % heads), kv = in % kv_heads;
  return Turn{static_cast<int32_t>(id / heads), kv * (heads / kv_heads) + in / kv_heads, kv};
}

// What rounding takes from x: nothing of an infinity.
template <typename T>
__device__ __forceinline__ float lost(float x) {
  const float r = static_cast<float>(static_cast<T>(x));
  return fabsf(r) == INFINITY ? 0.f : x - r;
}

// acc[block][n] is C with m = 16 block + ..., of an output's rows n: out[first + 16 n + lane % 16][m] = factor[n] * acc, rounded, and
// what the rounding took if `rest`.  Rows from `rows` on and elements from dim on are not there.
template <typename T, int D, int TN, bool REST = false>
__device__ __forceinline__ void write_rows(const f32x4 (&acc)[D / 16][TN], const float (&factor)[TN], T *out, T *rest, int64_t stride, int32_t rows,
                                           int32_t dim, int lane) {
#pragma unroll
  for (int n = 0; n < TN; ++n) {
    const int r = n * 16 + (lane & 15);
#pragma unroll
    for (int b = 0; b < D / 16; b += 2) {
      f32x4 x = acc[b][n] * factor[n], y = acc[b + 1][n] * factor[n];
      const Pack<uint32_t, 4> v = swapped<T>(x, y);
      const int at = b * 16 + ((lane >> 4) & 1) * 16 + (lane >> 5) * 8;
      const bool inside = r < rows && at < dim;
      if (inside) *reinterpret_cast<Pack<uint32_t, 4> *>(out + r * stride + at) = v;
      if constexpr (REST) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = lost<T>(x[i]); y[i] = lost<T>(y[i]); }
        const Pack<uint32_t, 4> w = swapped<T>(x, y);
        if (inside && rest) *reinterpret_cast<Pack<uint32_t, 4> *>(rest + r * stride + at) = w;
      }
    }
  }
}
// Zeros in rows at .. at + tile of an output.
template <typename T>
__device__ __forceinline__ void write_zeros(T *out, int64_t stride, int32_t rows, int32_t dim) {
  if (!out) return;
  const int pieces = dim / 8;
  for (int i = threadIdx.x; i < rows * pieces; i += blockDim.x)
    *reinterpret_cast<Pack<uint32_t, 4> *>(out + (i / pieces) * stride + (i % pieces) * 8) = Pack<uint32_t, 4>{{0, 0, 0, 0}};
}

}  // namespace
}  // namespace train
}  // namespace ones

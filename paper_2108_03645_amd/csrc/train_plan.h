// What the calls of the training operators launch and hold, from their sizes alone: which tiles of the matrix products, how a product
// is split, in which pieces the loss goes through the vocabulary, and the layout of the workspaces.  No HIP here: any C++17
// compiler takes it, so that the tests ask it which kernels a size reaches.
#pragma once

#include "ones.h"
#include "ones_train.h"

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>

namespace ones {
namespace train {

constexpr int64_t kMaxElements = int64_t{1} << 46;      // of one array: products of sizes stay far inside 64 bits
constexpr int64_t kMaxLoadableStride = 1 << 20;         // elements between rows that the matrix products load as they lie

inline bool is_type(int32_t t) { return t == ONES_F32 || t == ONES_F16 || t == ONES_BF16; }
inline int64_t type_bytes(int32_t t) { return t == ONES_F32 ? 4 : 2; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align_up(size_t v) { return (v + 255) & ~static_cast<size_t>(255); }

// The sizes of a two-dimensional array of `rows` rows of `cols` elements, rows `stride` elements apart.
inline int check_rows(int64_t rows, int64_t cols, int64_t stride) {
  if (rows < 0 || cols < 0 || stride < cols) return ONES_E_INVALID_ARG;
  if (rows && stride > kMaxElements / rows) return ONES_E_BOUNDS;
  return ONES_OK;
}

// ---------------------------------------------------------- the recurrence --------
constexpr int kV = 4, kTile = 128;            // channels of a thread, steps of a tile

constexpr int64_t kEnough = 192, kWanted = 512;
inline int64_t tiles_of(int64_t steps) { return ceil_div(steps, kTile); }

// How the work is cut.  Workgroups of 32 channels (8 lanes to a row) are twice as many as of 64, and two share every cache line
// of 128 bytes: on the same die, at about the same time.  Where they are enough for most compute units, or the tiles too few to
// split, they walk along whole sequences; backward (with five arrays instead of three) only along short ones, before two that
// share lines drift apart, and 64 channels along longer ones (us, 32 against 64 channels, bf16: forward 16 x 2048 x 1024 39 against
// 44, 64 x 256 x 1024 21 and 22, 8 x 512 x 512 8.7 and 11.5; backward 95 and 80, 33 and 42, 11.4 and 16.2).  Otherwise 64 channels, and
// as many segments as make two workgroups a compute unit (2 x 65521 x 512: 512 workgroups 141 and 220 us, 1024 152 and 231; with 32
// channels 179 and 250), which is 4.7 TB/s for what they read twice and write.
struct Cut {
  int32_t lanes, segments, tiles_each;
};
inline Cut cut_of(int64_t batch, int64_t steps, int64_t channels, bool backward) {
  const int64_t tiles = std::max<int64_t>(1, tiles_of(steps)), narrow = batch * ceil_div(channels, 32), chains = batch * ceil_div(channels, 64);
  const int32_t all = static_cast<int32_t>(tiles);
  if ((narrow >= kEnough || tiles < 8) && (!backward || tiles <= 8)) return Cut{8, 1, all};
  if (backward && chains >= kEnough) return Cut{16, 1, all};
  const int64_t each = ceil_div(tiles, std::min(tiles, ceil_div(kWanted, std::max<int64_t>(1, chains))));
  return Cut{16, static_cast<int32_t>(ceil_div(tiles, each)), static_cast<int32_t>(each)};
}
inline int64_t blocks_of(const Cut &cut, int64_t batch, int64_t channels) {
  const int64_t blocks = ceil_div(channels, cut.lanes * kV);
  return cut.lanes == 16 ? blocks * batch * cut.segments : ceil_div(ceil_div(blocks, 2) * batch * cut.segments, 8) * 16;
}

inline int check_sizes(int64_t batch, int64_t steps, int64_t channels, int32_t type) {
  if (batch < 0 || steps < 0 || channels < 0 || !is_type(type)) return ONES_E_INVALID_ARG;
  if (batch > ONES_MAX_BATCH || steps > ONES_MAX_STEPS || channels > ONES_MAX_CHANNELS) return ONES_E_BOUNDS;
  return steps && channels && batch > kMaxElements / (steps * channels) ? ONES_E_BOUNDS : ONES_OK;
}
inline int check_recurrence(int64_t batch, int64_t steps, int64_t channels, int32_t type) {
  if (int rc = check_sizes(batch, steps, channels, type)) return rc;
  // workgroups of a launch, numbered in 32 bits
  return std::max(blocks_of(cut_of(batch, steps, channels, false), batch, channels), blocks_of(cut_of(batch, steps, channels, true), batch, channels)) > (int64_t{1} << 31)
             ? ONES_E_BOUNDS : ONES_OK;
}
// Elements from a sequence to the next, and from a step to the next.
inline int check_strides(int64_t batch_stride, int64_t step_stride) {
  if (batch_stride < 0 || step_stride < 0) return ONES_E_INVALID_ARG;
  return batch_stride > (int64_t{1} << 40) || step_stride > (int64_t{1} << 32) ? ONES_E_BOUNDS : ONES_OK;
}
inline size_t carry_floats(int64_t batch, int64_t steps, int64_t channels) { return static_cast<size_t>(batch) * tiles_of(steps) * channels; }

// ------------------------------------------------- the matrix products --------
// The tiles of the matrix products (train_matmul.h), and how long a launch of them takes, by what was measured: so many
// microseconds for 64 k where every workgroup has a compute unit of its own, so many where `places` of them are at work, and so
// many for a workgroup's start and end.  From products of sides 256 to 4096 (k 4096, lower triangle of 4096 rows, us: large 92,
// middle 95, deep 109, small 106, tiny 160; of 3000 rows 93, 52, 67, 55, 90; of 2048, k 2048: 56, 30, 21, 26, 24; of 1024, k 4096:
// 90, 43, 29, 43, 16; eight of 256, k 256: 24, 16, 9, 9, 6; all tiles of 4096 x 4096, k 4096: 118, 146, 157, 141, 200).
enum Tiles : int { kLarge, kMiddle, kDeep, kSmall, kTiny };
struct TileCost {
  int64_t bm, bn, places;
  double alone, shared, fixed;
};
constexpr TileCost kTileCosts[] = {
    {256, 256, 256, 1.35, 1.45, 8.0}, {192, 128, 256, 0.72, 0.70, 6.0}, {128, 128, 256, 0.45, 0.47, 5.0}, {128, 128, 512, 0.62, 0.78, 5.0}, {64, 64, 512, 0.20, 0.38, 4.5}};

inline double item_time(const TileCost &c, int64_t items, int64_t k) { return ceil_div(k, 64) * (items <= 256 ? c.alone : c.shared) + c.fixed; }
inline double launch_time(const TileCost &c, int64_t items, int64_t k) { return ceil_div(items, c.places) * item_time(c, items, k); }

// ------------------------------------------------------------------ the loss --------
constexpr int64_t kPieceBytes = 128 << 20;

struct Part { float top, sum; };              // of some logits of a row: the largest, and the sum of exp(z - top)

// A product whose k is shared among `splits` workgroups a tile, `k_each` (a multiple of 64) each.
struct Split {
  int32_t splits, k_each;
};

// Which tiles, and into how many parts k is split: the estimate's least.
constexpr Tiles kUsed[] = {kLarge, kDeep, kSmall, kTiny};

inline Tiles logits_tiles(int64_t m, int64_t n, int64_t k) {
  auto time = [&](Tiles t) { return launch_time(kTileCosts[t], ceil_div(m, kTileCosts[t].bm) * ceil_div(n, kTileCosts[t].bn), k); };
  Tiles best = kLarge;
  for (Tiles t : kUsed) if (time(t) < time(best)) best = t;
  return best;
}

inline Split split_of(int64_t k, int64_t most) {
  const int64_t splits = std::max<int64_t>(1, ceil_div(k, most)), each = std::max<int64_t>(64, ceil_div(ceil_div(k, splits), 64) * 64);
  return Split{static_cast<int32_t>(std::max<int64_t>(1, ceil_div(k, each))), static_cast<int32_t>(each)};
}

// The gradients' operands are turned, which takes two reads from LDS a fragment instead of one, and their sums are written: what a tile
// takes longer for it, from the whole call's time with each of the tiles (rows, columns, words; large, deep, small, tiny, us, with the
// best split: 1003, 514, 10007: 94, 86, 89, 89; 2048, 512, 8000: 90, 77, 83, 88; 512, 768, 50000: 203, 185, 168, 212; 300, 2048, 16000: 138,
// 116, 107, 136; 4096, 4096, 4000: 372, 465, 413, 575; 8192, 1024, 32000: 1471, 1781, 1648, 2245).
inline TileCost turned_cost(Tiles t) {
  TileCost c = kTileCosts[t];
  const double times = t == kTiny ? 1.0 : t == kSmall ? 1.3 : 1.2;
  c.alone *= times;
  c.shared *= times;
  if (t == kLarge) c.fixed += 4.0;
  return c;
}

struct GradientPlan { Tiles tiles; Split of_dx, of_dw; };
inline GradientPlan gradient_plan(int64_t rows, int64_t cols, int64_t words) {
  GradientPlan best{};
  double best_time = INFINITY;
  for (Tiles t : kUsed) {
    const TileCost c = turned_cost(t);
    const int64_t tm = ceil_div(cols, c.bm), dx = tm * ceil_div(rows, c.bn), dw = tm * ceil_div(words, c.bn);
    for (int64_t most = std::max<int64_t>(128, ceil_div(std::max(rows, words), 64) * 64); most >= 128; most /= 2) {
      const GradientPlan p{t, split_of(words, most), split_of(rows, most)};
      if (p.of_dx.splits > 32 || p.of_dw.splits > 32) break;
      const int64_t dx_items = dx * p.of_dx.splits, dw_items = dw * p.of_dw.splits, items = dx_items + dw_items;
      const double dx_time = item_time(c, items, p.of_dx.k_each), dw_time = item_time(c, items, p.of_dw.k_each);
      // rounds of places, each as long as the items' mean, or the longest item
      double time = std::max(std::max(dx_time, dw_time), ceil_div(items, c.places) * (dx_items * dx_time + dw_items * dw_time) / items);
      double bytes = 0;                       // written and read again
      if (p.of_dx.splits > 1) bytes += 8.0 * p.of_dx.splits * rows * cols;
      if (p.of_dw.splits > 1) bytes += 8.0 * p.of_dw.splits * words * cols;
      if (bytes > 0) time += 4.0 + bytes / 4e6;
      if (time < best_time) { best = p; best_time = time; }
    }
  }
  return best;
}

// Backward: pieces of the vocabulary, each with all blocks of rows.
struct LossPlan {
  int64_t cols8, parts, piece, pieces, block, blocks;
  Tiles logits, logits_piece;
  GradientPlan gradients;
  size_t x, w, part, at_target, forward;                       // offsets, and the bytes of the forward pass
  size_t g, dx_sum, dw_sum, scale, backward;
};

inline LossPlan loss_plan(int64_t rows, int64_t cols, int64_t vocabulary, bool copies_x, bool copies_w, bool backward) {
  LossPlan p{};
  p.cols8 = ceil_div(cols, 8) * 8;
  p.logits = logits_tiles(vocabulary, rows, cols);
  p.parts = ceil_div(vocabulary, kTileCosts[p.logits].bm) * 2;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes); return at; };
  const size_t n = static_cast<size_t>(rows), d = static_cast<size_t>(cols), d8 = static_cast<size_t>(p.cols8);
  p.x = take(copies_x ? n * d8 * 2 : 0);
  p.w = take(copies_w ? static_cast<size_t>(vocabulary) * d8 * 2 : 0);
  const size_t packed = off;
  p.part = take(static_cast<size_t>(p.parts) * n * sizeof(Part));
  p.at_target = take(n * 4);
  p.forward = off;
  if (!backward) return p;
  off = packed;
  // a block's G of the smallest piece fills its bytes at most
  p.blocks = std::max<int64_t>(1, ceil_div(rows * 512, kPieceBytes));
  p.block = std::max<int64_t>(64, ceil_div(ceil_div(rows, p.blocks), 64) * 64);
  const int64_t at_once = std::min(rows, p.block);
  // G's rows are a piece apart, and the products load them as they lie
  const int64_t least_pieces = std::max(ceil_div(vocabulary, kMaxLoadableStride), ceil_div(at_once * ceil_div(vocabulary, 256) * 512, kPieceBytes));
  for (p.pieces = least_pieces;; ++p.pieces) {
    p.piece = ceil_div(ceil_div(vocabulary, p.pieces), 256) * 256;
    p.gradients = gradient_plan(at_once, cols, std::min(p.piece, vocabulary));
    const Split dx = p.gradients.of_dx, dw = p.gradients.of_dw;
    const int64_t sums = ((dx.splits - 1) * at_once + (dw.splits > 1 ? dw.splits * p.piece : 0)) * cols * 4;
    if (p.piece == 256 || at_once * p.piece * 2 + sums <= kPieceBytes) break;
  }
  p.pieces = ceil_div(vocabulary, p.piece);
  p.logits_piece = logits_tiles(p.piece, at_once, cols);
  p.g = take(static_cast<size_t>(at_once * p.piece) * 2);
  p.dx_sum = take(p.pieces > 1 || p.gradients.of_dx.splits > 1 ? p.gradients.of_dx.splits * n * d * 4 : 0);
  p.dw_sum = take(p.blocks > 1 || p.gradients.of_dw.splits > 1 ? static_cast<size_t>(p.gradients.of_dw.splits) * std::min(p.piece, vocabulary) * d * 4 : 0);
  p.scale = take(12);
  p.backward = off;
  return p;
}

inline int check_loss(int64_t rows, int64_t cols, int64_t vocabulary, int64_t x_stride, int64_t w_stride, int32_t type) {
  if (int rc = check_rows(rows, cols, x_stride)) return rc;
  if (int rc = check_rows(vocabulary, cols, w_stride)) return rc;
  if (cols < 1 || vocabulary < 1 || (type != ONES_F16 && type != ONES_BF16)) return ONES_E_INVALID_ARG;
  if (rows > ONES_MAX_LOSS_ROWS || vocabulary > ONES_MAX_VOCABULARY || cols > ONES_MAX_LOSS_COLUMNS) return ONES_E_BOUNDS;
  // The product of two sizes is at most 2^36, in tiles of 128 x 128 at most 2^22: the tiles that are chosen, with the parts that k is
  // split into and their 256 or 512 threads, then stay below the 2^32 threads of a launch.
  const int64_t n = ceil_div(rows, 128), v = ceil_div(vocabulary, 128), d = ceil_div(cols, 128);
  return std::max({n * v, d * n, d * v}) > (1 << 22) ? ONES_E_BOUNDS : ONES_OK;
}

// ------------------------------------------------ the orthogonalised update --------
constexpr int64_t kSumBlocks = 1024;          // workgroups that share a matrix's sum of squares, at most

// Tiles of rows n that begin at or below the diagonal (the first column is not beyond the last row), before tile row j.
constexpr int32_t tiles_in_row(int32_t j, int32_t tm, int32_t bm, int32_t bn) {
  const int32_t n = ((j + 1) * bn - 1) / bm + 1;
  return n < tm ? n : tm;
}
inline int64_t symmetric_tiles(int64_t bm, int64_t bn, int64_t r_ld) {
  int64_t tiles = 0;
  const int32_t tm = static_cast<int32_t>(ceil_div(r_ld, bm));
  for (int32_t j = 0; j < ceil_div(r_ld, bn); ++j) tiles += tiles_in_row(j, tm, static_cast<int32_t>(bm), static_cast<int32_t>(bn));
  return tiles;
}

// Which tiles each of a step's products takes: the estimate's least.  (kMiddle lies the other way round in X's own product.)
inline Tiles least(const int64_t (&items)[5], int64_t k) {
  Tiles best = kLarge;
  for (Tiles t : {kMiddle, kDeep, kSmall, kTiny})
    if (launch_time(kTileCosts[t], items[t], k) < launch_time(kTileCosts[best], items[best], k)) best = t;
  return best;
}
struct UpdateTiles { Tiles gram, poly, apply; };
inline UpdateTiles update_tiles(int64_t count, int64_t r, int64_t q, bool pairs) {
  const int64_t products = pairs ? 3 : 1;
  int64_t triangle[5], all[5];
  for (Tiles t : {kLarge, kMiddle, kDeep, kSmall, kTiny}) {
    const TileCost &c = kTileCosts[t];
    triangle[t] = count * symmetric_tiles(c.bm, c.bn, ceil_div(r, 8) * 8);
    all[t] = count * (t == kMiddle ? ceil_div(r, c.bm) * ceil_div(q, c.bn) : ceil_div(r, c.bn) * ceil_div(q, c.bm));
  }
  return UpdateTiles{least(triangle, products * q), least(triangle, products * r), least(all, products * r)};
}

// pairs: X and A are held in pairs, the second one behind all matrices' first.
struct UpdatePlan {
  int64_t r, q, r_ld, q_ld;
  int64_t blocks;
  int64_t x_low, a_low;                       // elements from a first to its second; 0 without
  size_t squares, x[2], a[2], total;
};
inline UpdatePlan update_plan(int64_t count, int64_t rows, int64_t cols, bool pairs) {
  UpdatePlan p{};
  p.r = std::min(rows, cols);
  p.q = std::max(rows, cols);
  p.r_ld = ceil_div(p.r, 8) * 8;
  p.q_ld = ceil_div(p.q, 8) * 8;
  size_t off = 0;
  auto take = [&](int64_t bytes) { const size_t at = off; off = align_up(off + static_cast<size_t>(bytes)); return at; };
  p.blocks = std::min(kSumBlocks, ceil_div(rows * cols, 4096));            // at least four runs of four elements a thread
  p.squares = take(count * p.blocks * 8);
  const int64_t x = count * p.r * p.q_ld, a = count * p.r * p.r_ld, bytes = pairs ? 4 : 2;
  p.x_low = pairs ? x : 0;
  p.a_low = pairs ? a : 0;
  p.x[0] = take(x * bytes);
  p.x[1] = take(x * bytes);
  p.a[0] = take(a * bytes);
  p.a[1] = take(a * bytes);
  p.total = off;
  return p;
}

inline int check_update(int64_t count, int64_t rows, int64_t cols) {
  if (count < 0 || rows < 0 || cols < 0) return ONES_E_INVALID_ARG;
  if (count > 65535 || rows > ONES_MAX_UPDATE_SIDE || cols > ONES_MAX_UPDATE_SIDE) return ONES_E_BOUNDS;
  return ONES_OK;
}

}  // namespace train
}  // namespace ones

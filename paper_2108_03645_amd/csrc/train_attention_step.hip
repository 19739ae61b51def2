// One more token of every sequence over its cache (ones_attention_step).
//
//   o = sum_{j <= n} p_j v_j, p = softmax(scale q . k_j), n the place of the new token
//
// A workgroup takes a part of one sequence's cache for up to 16 query heads of one key head, which are the columns of the products; its waves
// take tiles of 32 keys in turn, each by itself: the tiles come to the wave's own place in LDS by direct loads, the next while the present one is worked
// on.  The sums of the waves, then those of the parts, are joined at the end.  The new token's key and value are
// arguments; the wave that begins the cache begins with them, and the same workgroup writes them to the cache.
//
// What bounds it is memory: 32 sequences of 8192 places, 4 key heads of 128, 8 query heads each, bf16: 107 us and 6 for the joining launch, 537 MB, 5.0
// TB/s.  One sequence of 100003 places, 2 heads: 25 us and 5.  Eight short sequences: 8 us, a chain of loads one behind the other.
#include "train_attention.h"
#include "train_host.h"

#include <hip/hip_runtime.h>

#include <cmath>

namespace ones {
namespace train {
namespace {

struct StepArgs {
  const void *q, *k, *v;
  void *keys, *values, *o;
  int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head;
  int64_t keys_batch, keys_stride, keys_head, values_batch, values_stride, values_head;
  const int32_t *lengths;
  float *tops, *sums, *outputs;               // of the parts: [batch][heads][splits], outputs with dim
  int32_t batch, capacity, heads, kv_heads, dim, blocks_of_heads, splits;
  float scale;
};

// A wave's tile of 32 rows: like RowTile, but a load of the wave fills fewer than 16 rows, so that the exchange differs from load to load.
template <int D>
struct WaveTile {
  using Tile = RowTile<D, 32, 256>;           // places of the reads
  static constexpr int bytes = Tile::bytes, pieces = Tile::pieces, at_once = kWave / pieces, loads = 32 / at_once, kinds = 16 / at_once;
  static_assert(at_once == 4 || at_once == 8);
  uint32_t row_bytes, offset[kinds];
  __device__ __forceinline__ void start(int64_t stride, int32_t dim, int lane) {
    row_bytes = static_cast<uint32_t>(stride * 2);
#pragma unroll
    for (int i = 0; i < kinds; ++i) {
      const int r = lane / pieces + i * at_once, p = (lane % pieces) ^ Tile::exchange(r);
      offset[i] = p * 8 < dim ? r * row_bytes + p * 16 : Tile::kOutside;
    }
  }
  // Rows of which `left` are there.
  __device__ __forceinline__ void load(const unsigned char *base, int32_t left, unsigned char *to) const {
    const uint32_t mine = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>((LdsBytes *)to)));
    const uint32_t inside = static_cast<uint32_t>(max(min(left, 32), 0)) * row_bytes;
#pragma unroll
    for (int i = 0; i < loads; ++i)
      load_to_lds(base, inside, offset[i % kinds] + (i / kinds) * kinds * at_once * row_bytes, mine + i * kWave * 16);
  }
};

template <int PENDING>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PENDING) : "memory");
}

// The workgroup's tiles of a cache that part `split` of `splits` has: whole ones, evenly over the parts.  A part may have none; the first has the new
// token all the same.
struct Part {
  int32_t begin, end;
  __device__ __forceinline__ Part(int32_t length, int32_t split, int32_t splits) {
    const int64_t all = (length + kStepKeys * kStepWaves - 1) / (kStepKeys * kStepWaves);
    begin = static_cast<int32_t>(all * split / splits);
    end = static_cast<int32_t>(all * (split + 1) / splits);
  }
  __device__ __forceinline__ bool empty(int32_t split) const { return begin == end && split; }
};

template <typename T, int D>
__global__ __launch_bounds__(kStepWaves * 64) void step_kernel(StepArgs a) {
  using Load = WaveTile<D>;
  using Tile = typename Load::Tile;
  constexpr int waves = kStepWaves;
  __shared__ __attribute__((aligned(256))) unsigned char lds[waves * 4 * Load::bytes];
  __shared__ float tops[waves][16], sums[waves][16];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(static_cast<int>(threadIdx.x) / kWave);
  // key heads of a sequence follow each other, then the parts
  uint32_t id = blockIdx.x;
  const int32_t kv = id % a.kv_heads;
  id /= a.kv_heads;
  const int32_t of = id % a.blocks_of_heads;
  id /= a.blocks_of_heads;
  const int32_t split = id % a.splits, b = id / a.splits;
  const int32_t group = a.heads / a.kv_heads, head = kv * group + of * 16, heads = min(group - of * 16, 16);
  const int32_t length = a.lengths[b];
  const int64_t part0 = (static_cast<int64_t>(b) * a.heads + head) * a.splits + split;      // of the first head; `splits` apart
  T *const out = static_cast<T *>(a.o) + (static_cast<int64_t>(b) * a.heads + head) * a.dim;
  if (length < 0 || length >= a.capacity) {
    const float fill = length < 0 ? 0.f : NAN;
    if (split == 0)
      for (int i = threadIdx.x; i < heads * a.dim; i += kStepWaves * 64) out[i] = static_cast<T>(fill);
    return;
  }
  const Part part(length, split, a.splits);
  if (part.empty(split)) return;              // the joining launch knows
  const int32_t begin = part.begin, end = part.end;
  const T *const k_new = static_cast<const T *>(a.k) + b * a.k_stride + kv * a.k_head, *const v_new = static_cast<const T *>(a.v) + b * a.v_stride + kv * a.v_head;
  const unsigned char *ks = reinterpret_cast<const unsigned char *>(static_cast<const T *>(a.keys) + b * a.keys_batch + kv * a.keys_head);
  const unsigned char *vs = reinterpret_cast<const unsigned char *>(static_cast<const T *>(a.values) + b * a.values_batch + kv * a.values_head);
  Load k, v;
  k.start(a.keys_stride, a.dim, lane);
  v.start(a.values_stride, a.dim, lane);
  unsigned char *const mine = lds + wave * 4 * Load::bytes;
  auto load = [&](int32_t tile, int to) {     // the wave's tile of the workgroup's `tile`
    const int32_t first = (tile * waves + wave) * kStepKeys;
    k.load(ks + static_cast<int64_t>(first) * k.row_bytes, length - first, mine + to * 2 * Load::bytes);
    v.load(vs + static_cast<int64_t>(first) * v.row_bytes, length - first, mine + to * 2 * Load::bytes + Load::bytes);
  };
  if (begin < end) load(begin, 0);
  s16x8 q[D / 32];
  read_rows<D>(static_cast<const T *>(a.q) + b * a.q_stride + head * a.q_head, a.q_head, heads, a.dim, lane, q);
  const float c = a.scale * kLog2e;
  f32x4 acc[D / 16];
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (split == 0 && wave == 0) {              // the new token: row 0 of a product, weight 1
    s16x8 f[D / 32];
    read_rows<D>(k_new, 0, 1, a.dim, lane, f);
    f32x4 z{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < D / 32; ++s) z = mfma<T>(f[s], q[s], z);
    top = __shfl(z[0], lane & 15);
    const float weight = top == -INFINITY ? 0.f : top - top == 0.f ? __builtin_amdgcn_exp2f(kShift<T>) : NAN;
    if (lane < 16) sum = weight;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = i * 16 + (lane >> 4) * 4 + r;
        acc[i][r] = d < a.dim && weight != 0.f ? static_cast<float>(v_new[d]) * weight : 0.f;
      }
  }
  if (split == 0 && of == 0 && threadIdx.x < 2 * Tile::pieces) {
    const int which = threadIdx.x / Tile::pieces, d = threadIdx.x % Tile::pieces * 8;
    T *to = which ? static_cast<T *>(a.values) + b * a.values_batch + length * a.values_stride + kv * a.values_head
                  : static_cast<T *>(a.keys) + b * a.keys_batch + length * a.keys_stride + kv * a.keys_head;
    if (d < a.dim) *reinterpret_cast<Pack<uint32_t, 4> *>(to + d) = *reinterpret_cast<const Pack<uint32_t, 4> *>((which ? v_new : k_new) + d);
  }
  int along[D / 32], across[D / 16];
#pragma unroll
  for (int s = 0; s < D / 32; ++s) along[s] = Tile::along(lane, s);
#pragma unroll
  for (int i = 0; i < D / 16; ++i) across[i] = Tile::across(lane, i);
  for (int32_t tile = begin; tile < end; ++tile) {
    const int now = (tile - begin) & 1;
    if (tile + 1 < end) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // its place has been read
      load(tile + 1, now ^ 1);
      arrived<2 * Load::loads>();
    } else {
      arrived<0>();
    }
    const int32_t left = length - (tile * waves + wave) * kStepKeys;
    if (left <= 0) continue;
    const unsigned char *kt = mine + now * 2 * Load::bytes, *vt = kt + Load::bytes;
    f32x4 z[2];
    float most = top;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      z[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < D / 32; ++s) z[i] = mfma<T>(Tile::read_along(kt, i * 16, along[s]), q[s], z[i]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if (i * 16 + (lane >> 4) * 4 + r >= left) z[i][r] = -INFINITY;
        most = fmaxf(most, z[i][r]);
      }
    }
    most = across_max(most);
    if (__any(most > top)) {
      const float factor = most == top ? 1.f : __builtin_amdgcn_exp2f((top - most) * c);
      sum *= factor;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) acc[i] *= factor;
      top = most;
    }
    const float base = (top == -INFINITY ? 0.f : top * c) - kShift<T>;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        z[i][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[i][r], c, -base));
        sum += z[i][r];
      }
    const s16x8 p = rounded<T>(z[0], z[1]);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) acc[i] = mfma<T>(Tile::read_across(vt, 0, across[i]), p, acc[i]);
  }
  sum = across_sum(sum);
  __syncthreads();                            // the tiles' places take the sums
  float *const parts = reinterpret_cast<float *>(lds);        // [wave][head][D]
  if (lane < 16) {
    tops[wave][lane] = top;
    sums[wave][lane] = sum;
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
    *reinterpret_cast<f32x4 *>(parts + ((wave * 16 + (lane & 15)) * D + i * 16 + (lane >> 4) * 4)) = acc[i];
  __syncthreads();
  Seen seen;                                  // among the values of element of_d
  int of_d = -1;
  for (int i = threadIdx.x; i < heads * D; i += kStepWaves * 64) {
    const int h = i / D, d = i % D;
    float most = tops[0][h];
#pragma unroll
    for (int w = 1; w < waves; ++w) most = fmaxf(most, tops[w][h]);
    float all_sum = 0.f, x = 0.f;
#pragma unroll
    for (int w = 0; w < waves; ++w) {
      const float f = tops[w][h] == most ? 1.f : __builtin_amdgcn_exp2f((tops[w][h] - most) * c);
      all_sum += sums[w][h] * f;
      x += parts[(w * 16 + h) * D + d] * f;
    }
    if (d >= a.dim) continue;
    if (a.splits == 1) {
      x /= all_sum;
      if (x != x && all_sum > 0.f) {          // a weight that is 0 in 32 bits is above 0 all the same: one infinity that it met is the result, not NaN
        if (d != of_d) seen = Seen();
        of_d = d;
        seen.add(static_cast<float>(v_new[d]));
        seen.through(reinterpret_cast<const T *>(vs), a.values_stride, length - 1, d);
        if (seen.infinite()) x = seen.up() ? __builtin_inff() : -__builtin_inff();
      }
      out[h * a.dim + d] = static_cast<T>(x);
    } else {
      const int64_t at = part0 + static_cast<int64_t>(h) * a.splits;
      a.outputs[at * a.dim + d] = x;
      if (d == 0) { a.tops[at] = most; a.sums[at] = all_sum; }
    }
  }
}

// The parts of a head: 128 elements by 8 groups of parts, added up in order.  Parts without keys left nothing behind; all others count, also where their
// factor is 0: 0 times NaN is NaN.
template <typename T>
__global__ __launch_bounds__(1024) void step_join_kernel(StepArgs a) {
  __shared__ float factors[kStepMaxSplits], most_of[16], sums[8], outputs[8][128];
  const int32_t b = blockIdx.x / a.heads, length = a.lengths[b];
  if (length < 0 || length >= a.capacity) return;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * a.splits;
  const int i = threadIdx.x, d = i % 128, group = i / 128;
  const bool empty = i >= a.splits || Part(length, i, a.splits).empty(i);
  const float top = empty ? -INFINITY : a.tops[at + i];
  float most = across_max(top);
#pragma unroll
  for (int m = 1; m < 16; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
  if (i % kWave == 0) most_of[i / kWave] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) most = fmaxf(most, most_of[w]);
  if (i < a.splits) factors[i] = empty ? -1.f : top == most ? 1.f : __builtin_amdgcn_exp2f((top - most) * (a.scale * kLog2e));
  __syncthreads();
  float sum = 0.f, x = 0.f;
  const int e = min(d, a.dim - 1);
#pragma unroll 4
  for (int p = group; p < a.splits; p += 8) {
    const float f = factors[p], s = a.sums[at + p], y = a.outputs[(at + p) * a.dim + e];
    sum += f < 0.f ? 0.f : s * f;
    x += f < 0.f ? 0.f : y * f;
  }
  outputs[group][d] = x;
  if (d == 0) sums[group] = sum;
  __syncthreads();
  if (group || d >= a.dim) return;
  sum = sums[0];
#pragma unroll
  for (int g = 1; g < 8; ++g) { x += outputs[g][d]; sum += sums[g]; }
  x /= sum;
  if (x != x && sum > 0.f) {                  // as in step_kernel; the new token's value is in its place by now
    Seen seen;
    seen.through(static_cast<const T *>(a.values) + b * a.values_batch + (blockIdx.x % a.heads) / (a.heads / a.kv_heads) * a.values_head, a.values_stride, length, d);
    if (seen.infinite()) x = seen.up() ? __builtin_inff() : -__builtin_inff();
  }
  static_cast<T *>(a.o)[static_cast<int64_t>(blockIdx.x) * a.dim + d] = static_cast<T>(x);
}

template <typename T>
void launch(const StepArgs &a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(a.batch) * a.splits * a.blocks_of_heads * a.kv_heads)), block(kStepWaves * 64);
  if (a.dim <= 32) hipLaunchKernelGGL((step_kernel<T, 32>), grid, block, 0, s, a);
  else if (a.dim <= 64) hipLaunchKernelGGL((step_kernel<T, 64>), grid, block, 0, s, a);
  else if (a.dim <= 96) hipLaunchKernelGGL((step_kernel<T, 96>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((step_kernel<T, 128>), grid, block, 0, s, a);
  if (a.splits > 1) hipLaunchKernelGGL((step_join_kernel<T>), dim3(static_cast<uint32_t>(a.batch * a.heads)), dim3(1024), 0, s, a);
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

size_t ones_attention_step_workspace_bytes(int64_t batch, int64_t capacity, int64_t heads, int64_t kv_heads, int64_t dim) {
  if (check_step(batch, capacity, heads, kv_heads, dim, ONES_F16, 1.f)) return 0;
  return step_plan(batch, capacity, heads, kv_heads, dim).bytes;
}

int ones_attention_step(const void *q, int64_t q_stride, int64_t q_head_stride, const void *k, int64_t k_stride, int64_t k_head_stride,
                        const void *v, int64_t v_stride, int64_t v_head_stride, void *keys, int64_t keys_batch_stride, int64_t keys_stride,
                        int64_t keys_head_stride, void *values, int64_t values_batch_stride, int64_t values_stride, int64_t values_head_stride,
                        const int32_t *lengths, int64_t batch, int64_t capacity, int64_t heads, int64_t kv_heads, int64_t dim, int32_t type,
                        float scale, void *o, void *d_workspace, size_t workspace_bytes, void *hip_stream) {
  if (int rc = check_step(batch, capacity, heads, kv_heads, dim, type, scale)) return rc;
  if (batch == 0) return ONES_OK;
  if (int rc = check_token_rows(q, q_stride, q_head_stride, batch, heads)) return rc;
  if (int rc = check_token_rows(k, k_stride, k_head_stride, batch, kv_heads)) return rc;
  if (int rc = check_token_rows(v, v_stride, v_head_stride, batch, kv_heads)) return rc;
  if (!lengths || !o || !aligned(o, 16)) return ONES_E_INVALID_ARG;
  if (capacity) {
    if (int rc = check_head_rows(keys, keys_stride, keys_head_stride, kv_heads, dim)) return rc;
    if (int rc = check_head_rows(values, values_stride, values_head_stride, kv_heads, dim)) return rc;
  }
  for (const int64_t stride : {keys_batch_stride, values_batch_stride})
    if (batch > 1 && (stride < 0 || stride % 8)) return ONES_E_INVALID_ARG;
    else if (batch > 1 && stride > kMaxElements / batch) return ONES_E_BOUNDS;
  if (capacity && batch) {                    // places are written: no two may be one
    const Places of_keys(batch, keys_batch_stride, keys_stride, keys_head_stride, capacity, kv_heads, dim);
    const Places of_values(batch, values_batch_stride, values_stride, values_head_stride, capacity, kv_heads, dim);
    const int64_t behind = (reinterpret_cast<intptr_t>(values) - reinterpret_cast<intptr_t>(keys)) / 2;
    if (!of_keys.apart() || !of_values.apart() || !of_keys.apart_from(of_values, behind)) return ONES_E_INVALID_ARG;
  }
  const StepPlan plan = step_plan(batch, capacity, heads, kv_heads, dim);
  if (int rc = check_workspace(d_workspace, workspace_bytes, plan.bytes)) return rc;
  unsigned char *const w = static_cast<unsigned char *>(d_workspace);
  StepArgs a{};
  a.q = q; a.k = k; a.v = v; a.keys = keys; a.values = values; a.o = o;
  a.q_stride = q_stride; a.q_head = q_head_stride; a.k_stride = k_stride; a.k_head = k_head_stride; a.v_stride = v_stride; a.v_head = v_head_stride;
  a.keys_batch = keys_batch_stride; a.keys_stride = keys_stride; a.keys_head = keys_head_stride;
  a.values_batch = values_batch_stride; a.values_stride = values_stride; a.values_head = values_head_stride;
  a.lengths = lengths;
  if (plan.splits > 1) {
    a.tops = reinterpret_cast<float *>(w + plan.tops);
    a.sums = reinterpret_cast<float *>(w + plan.sums);
    a.outputs = reinterpret_cast<float *>(w + plan.outputs);
  }
  a.batch = static_cast<int32_t>(batch); a.capacity = static_cast<int32_t>(capacity); a.heads = static_cast<int32_t>(heads);
  a.kv_heads = static_cast<int32_t>(kv_heads); a.dim = static_cast<int32_t>(dim);
  a.blocks_of_heads = static_cast<int32_t>(plan.blocks_of_heads); a.splits = static_cast<int32_t>(plan.splits); a.scale = scale;
  if (type == ONES_F16) launch<f16>(a, static_cast<hipStream_t>(hip_stream));
  else launch<bf16>(a, static_cast<hipStream_t>(hip_stream));
  return launched("attention step");
}

}  // extern "C"

// The gated linear recurrence over the steps of a sequence, channel by channel (ones_recurrence_*).
//
//   a_t = sigmoid(gate_t), h_t = a_t h_{t-1} + (1 - a_t) x_t
//   l_t = dh_t + a_{t+1} l_{t+1}, dx_t = (1 - a_t) l_t, dgate_t = l_t (h_{t-1} - x_t) a_t (1 - a_t), dstate = a_0 l_0
//
// Steps t past a sequence's length keep the state: a_t = 1, no input, h_t written as 0, no gradients.
//
// A run of steps acts on the state as h -> A h + H (A the product of its gates), and on what comes back from behind as
// r -> A r + Q (r_t = a_t l_t); two runs one after another compose.  A workgroup owns 64 (or 32) channels of one sequence and
// takes tiles of 128 steps: a thread keeps eight (or four) steps of four channels in registers and forms its run's A and H, one
// wave composes the runs of the tile's thread groups through LDS, and every thread walks its steps again from the state before
// them.  gate, x and dh are read once and everything is written once.  The state before every tile is kept in 32 bits (one for 128
// elements): backward recomputes h from it, which is neither rounded to 16 bits nor read.  What bounds it is memory; next to it
// the arithmetic (an exponential and a reciprocal an element) and the chain through a tile's groups.
//
// Measured at 16 x 2048 x 1024 bf16: forward 39 us (206 MB with the carry, 5.2 TB/s; a copy of 4 GiB runs at 4.65), backward 65 us (340
// MB, 5.2 TB/s).  One step of 64 x 1024 is 3 us, a launch's own time.
//
// Where sequences and channels are too few for the compute units, the steps are split into segments of whole tiles as well.  A
// first launch forms each segment's A and H (or Q), a small second one turns them into the state before (what comes from behind)
// each, and the third walks along the segments side by side: the inputs are read twice then.  The first launch goes through a segment
// against the third's direction, so that what it read last, and the caches still have, is what the third reads first (316 us for
// 2 x 65521 x 512 forward and backward, 328 in the same direction; the launches take 51, 5 and 62 us
// forward, 43, 5 and 143 us backward).  No workgroup waits for another, and the order of all sums is fixed.
#include "train_device.h"
#include "train_host.h"

#include <algorithm>
#include <type_traits>

namespace ones {
namespace train {
namespace {

constexpr int kThreads = 256;

struct RecurrenceArgs {
  const void *gate, *x, *dh;
  void *h, *dgate, *dx;
  const float *state, *dlast;      // may be null: zeros
  float *last, *dstate;            // may be null
  const int32_t *lengths;          // may be null: all steps
  float *carry;                    // [batch][tiles][channels]: the state before every tile; forward may be null
  float *segments;                 // [batch][segments][2][channels]: A and H (Q) of each, then the state before it (from behind it) for H
  int64_t gate_batch, gate_step, x_batch, x_step, dh_batch, dh_step;
  int32_t batch, steps, channels, tiles, n_segments, tiles_per_segment;
};

__device__ __forceinline__ int length_of(const RecurrenceArgs &a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.steps) : a.steps;
}

// The S steps of kV channels of this thread's run, as read; zeros from step `len` on and beyond the last channel.  EDGE: the
// channels are no multiple of kV.
template <typename T, int S, bool EDGE>
struct Run {
  Pack<T, kV> p[S];
  __device__ __forceinline__ void load(const T *base, int64_t step_stride, int t0, int c, int len, int channels) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const T *from = base + (t0 + i) * step_stride + c;
      if (EDGE) p[i] = load_some<T, kV>(from, t0 + i < len ? channels - c : 0);
      else if (t0 + i < len && c < channels) p[i] = load_pack<T, kV>(from);
      else
#pragma unroll
        for (int k = 0; k < kV; ++k) p[i].v[k] = static_cast<T>(0.f);
    }
  }
};
template <typename T, bool EDGE, bool PAST>
__device__ __forceinline__ void store_run(T *base, int channels, int t0, int steps, int c, int i, const float *v) {
  T *to = base + static_cast<int64_t>(t0 + i) * channels + c;
  if (EDGE) { if (t0 + i < steps) store_some<T, kV>(to, v, channels - c, PAST); }
  else if (t0 + i < steps && c < channels) store_pack<T, kV>(to, v, PAST);
}

// a = sigmoid(g) and 1 - a, which keeps its digits where a is close to 1.  (The reciprocal is off by one place of 32 bits at most.)
__device__ __forceinline__ void gate_of(float g, float &a, float &keep) {
  const float e = __expf(-g);
  a = __builtin_amdgcn_rcpf(1.f + e);
  keep = e > 1.f ? 1.f - a : e * a;
}

// Which channels, sequence and segment.  Two blocks of 32 channels share cache lines: they go to one die, one right after the
// other (ids go round the eight dies).
struct Work {
  int32_t c0, b, segment;
  bool any;
};
template <int LANES>
__device__ __forceinline__ Work work_of(const RecurrenceArgs &a) {
  const uint32_t id = blockIdx.y * gridDim.x + blockIdx.x, blocks = (a.channels + LANES * kV - 1) / (LANES * kV);
  uint32_t rest, block;
  if constexpr (LANES == 16) {
    rest = id / blocks;
    block = id % blocks;
  } else {
    const uint32_t pair = id / 16 * 8 + id % 8, pairs = (blocks + 1) / 2;
    rest = pair / pairs;
    block = pair % pairs * 2 + id % 16 / 8;
  }
  const uint32_t b = rest % static_cast<uint32_t>(a.batch), segment = rest / static_cast<uint32_t>(a.batch);
  return Work{static_cast<int32_t>(block * LANES * kV), static_cast<int32_t>(b), static_cast<int32_t>(segment),
              block < blocks && segment < static_cast<uint32_t>(a.n_segments)};
}

template <typename T, int LANES, bool EDGE, bool FORM, bool PAST>     // FORM: only the segments' A and H; PAST: h goes past the caches
__global__ __launch_bounds__(kThreads) void recurrence_forward_kernel(RecurrenceArgs a) {
  constexpr int V = kV, kChannels = LANES * V, groups = kThreads / LANES, S = kTile / groups;
  __shared__ float sa[groups][kChannels], sh[groups][kChannels];
  const Work work = work_of<LANES>(a);
  const int b = work.b, segment = work.segment, c0 = work.c0;
  if (!work.any || (FORM && segment == a.n_segments - 1)) return;   // nothing comes after the last
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, c = c0 + lane * V;
  const int len = length_of(a, b);
  const T *gate = static_cast<const T *>(a.gate) + b * a.gate_batch, *x = static_cast<const T *>(a.x) + b * a.x_batch;
  T *h = FORM ? nullptr : static_cast<T *>(a.h) + static_cast<int64_t>(b) * a.steps * a.channels;
  const int first = segment * a.tiles_per_segment, end = min(a.tiles, first + a.tiles_per_segment);
  // thread c of the first wave keeps channel c0 + c's state, and the segment's product of gates where that is asked for
  const int own = c0 + static_cast<int>(threadIdx.x);
  const bool keeps = threadIdx.x < kChannels && own < a.channels;
  float state = 0.f, through = 1.f;
  if (!FORM && keeps) {
    if (segment) state = a.segments[((static_cast<int64_t>(b) * a.n_segments + segment) * 2 + 1) * a.channels + own];
    else if (a.state) state = a.state[static_cast<int64_t>(b) * a.channels + own];
  }
  constexpr int turn = FORM ? -1 : 1;            // FORM goes from the segment's end to its start
  const int start = FORM ? end - 1 : first, stop = FORM ? first - 1 : end;
  Run<T, S, EDGE> g, u;
  g.load(gate, a.gate_step, start * kTile + group * S, c, len, a.channels);
  u.load(x, a.x_step, start * kTile + group * S, c, len, a.channels);
  auto body = [&](int tile, auto whole) {          // whole: no step of the tile is past the length
    constexpr bool all = decltype(whole)::value;
    const int t0 = tile * kTile + group * S;
    float ga[S][V], in[S][V], A[V], H[V];
#pragma unroll
    for (int k = 0; k < V; ++k) { A[k] = 1.f; H[k] = 0.f; }
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const bool live = all || t0 + i < len;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float r, q;
        gate_of(static_cast<float>(g.p[i].v[k]), r, q);
        ga[i][k] = live ? r : 1.f;
        in[i][k] = live ? q * static_cast<float>(u.p[i].v[k]) : 0.f;
        A[k] *= ga[i][k];
        H[k] = __builtin_fmaf(ga[i][k], H[k], in[i][k]);
      }
    }
    if (tile + turn != stop) {                   // the next tile's rows arrive while this one is put together
      g.load(gate, a.gate_step, t0 + turn * kTile, c, len, a.channels);
      u.load(x, a.x_step, t0 + turn * kTile, c, len, a.channels);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) { sa[group][lane * V + k] = A[k]; sh[group][lane * V + k] = H[k]; }
    __syncthreads();
    if (threadIdx.x < kChannels) {
      if (!FORM && keeps && a.carry) a.carry[(static_cast<int64_t>(b) * a.tiles + tile) * a.channels + own] = state;
      float as[groups], hs[groups];              // all read before the chain
#pragma unroll
      for (int s = 0; s < groups; ++s) { as[s] = sa[s][threadIdx.x]; hs[s] = sh[s][threadIdx.x]; }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (FORM) {
        float tile_h = 0.f, tile_a = 1.f;
#pragma unroll
        for (int s = 0; s < groups; ++s) {
          tile_h = __builtin_fmaf(as[s], tile_h, hs[s]);
          tile_a *= as[s];
        }
        state = __builtin_fmaf(through, tile_h, state);      // the tile, then those behind it
        through *= tile_a;
      } else {
#pragma unroll
        for (int s = 0; s < groups; ++s) {
          sh[s][threadIdx.x] = state;            // before the group's first step
          state = __builtin_fmaf(as[s], state, hs[s]);
        }
      }
    }
    __syncthreads();
    if constexpr (!FORM) {
      float now[V];
#pragma unroll
      for (int k = 0; k < V; ++k) now[k] = sh[group][lane * V + k];
#pragma unroll
      for (int i = 0; i < S; ++i) {
        float out[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          now[k] = __builtin_fmaf(ga[i][k], now[k], in[i][k]);
          out[k] = all || t0 + i < len ? now[k] : 0.f;
        }
        store_run<T, EDGE, PAST>(h, a.channels, t0, a.steps, c, i, out);
      }
      __syncthreads();                           // sh is written anew
    }
  };
  for (int tile = start; tile != stop; tile += turn) {
    if ((tile + 1) * kTile <= len) body(tile, std::true_type{});
    else body(tile, std::false_type{});
  }
  if (!keeps) return;
  if (FORM) {
    float *seg = a.segments + (static_cast<int64_t>(b) * a.n_segments + segment) * 2 * a.channels + own;
    seg[0] = through;
    seg[a.channels] = state;
  } else if (a.last && end == a.tiles) {
    a.last[static_cast<int64_t>(b) * a.channels + own] = state;
  }
}

template <typename T, int LANES, bool EDGE, bool FORM, bool PAST>     // FORM: only the segments' A and Q; PAST: dgate and dx go past the caches
__global__ __launch_bounds__(kThreads) void recurrence_backward_kernel(RecurrenceArgs a) {
  constexpr int V = kV, kChannels = LANES * V, groups = kThreads / LANES, S = kTile / groups;
  __shared__ float sa[groups][kChannels], sh[groups][kChannels], sq[groups][kChannels];
  const Work work = work_of<LANES>(a);
  const int b = work.b, segment = work.segment, c0 = work.c0;
  if (!work.any || (FORM && segment == 0)) return;                  // nothing comes before the first
  const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES, c = c0 + lane * V;
  const int len = length_of(a, b);
  const T *gate = static_cast<const T *>(a.gate) + b * a.gate_batch, *x = static_cast<const T *>(a.x) + b * a.x_batch;
  const T *dh = static_cast<const T *>(a.dh) + b * a.dh_batch;
  const int64_t out = static_cast<int64_t>(b) * a.steps * a.channels;
  const int first = segment * a.tiles_per_segment, end = min(a.tiles, first + a.tiles_per_segment);
  // the second wave keeps what comes back from behind, the first composes the states
  const int at = static_cast<int>(threadIdx.x) % kWave, own = c0 + at;
  const bool second = threadIdx.x / kWave == 1, keeps = second && at < kChannels && own < a.channels;
  float back = 0.f, through = 1.f;
  if (!FORM && keeps) {
    if (segment + 1 < a.n_segments) back = a.segments[((static_cast<int64_t>(b) * a.n_segments + segment) * 2 + 1) * a.channels + own];
    else if (a.dlast) back = a.dlast[static_cast<int64_t>(b) * a.channels + own];
  }
  Run<T, S, EDGE> g, u, d;
  float carry = 0.f;                             // of the first wave's threads
  auto load_carry = [&](int tile) {
    if (!FORM && threadIdx.x < kChannels && own < a.channels) carry = a.carry[(static_cast<int64_t>(b) * a.tiles + tile) * a.channels + own];
  };
  constexpr int turn = FORM ? 1 : -1;            // FORM goes from the segment's start to its end
  const int start = FORM ? first : end - 1, stop = FORM ? end : first - 1;
  if (end > first) {                             // always, but for sequences of no steps
    load_carry(start);
    const int t0 = start * kTile + group * S;
    g.load(gate, a.gate_step, t0, c, len, a.channels);
    if (!FORM) u.load(x, a.x_step, t0, c, len, a.channels);
    d.load(dh, a.dh_step, t0, c, len, a.channels);
  }
  auto body = [&](int tile, auto whole) {          // whole: no step of the tile is past the length
    constexpr bool all = decltype(whole)::value;
    const int t0 = tile * kTile + group * S;
    float ga[S][V], keep[S][V], A[V], H[V], Q[V];
    const Run<T, S, EDGE> u0 = u, d0 = d;                // as read: half the registers
    auto xs = [&](int i, int k) { return static_cast<float>(u0.p[i].v[k]); };
    auto ds = [&](int i, int k) { return static_cast<float>(d0.p[i].v[k]); };
#pragma unroll
    for (int k = 0; k < V; ++k) { A[k] = 1.f; H[k] = Q[k] = 0.f; }
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const bool live = all || t0 + i < len;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float r, q;
        gate_of(static_cast<float>(g.p[i].v[k]), r, q);
        ga[i][k] = live ? r : 1.f;
        keep[i][k] = live ? q : 0.f;
        A[k] *= ga[i][k];
        if (!FORM) H[k] = __builtin_fmaf(ga[i][k], H[k], live ? keep[i][k] * xs(i, k) : 0.f);
      }
    }
#pragma unroll
    for (int i = S - 1; i >= 0; --i)
#pragma unroll
      for (int k = 0; k < V; ++k) Q[k] = ga[i][k] * (ds(i, k) + Q[k]);
    if (tile + turn != stop) {
      g.load(gate, a.gate_step, t0 + turn * kTile, c, len, a.channels);
      if (!FORM) u.load(x, a.x_step, t0 + turn * kTile, c, len, a.channels);
      d.load(dh, a.dh_step, t0 + turn * kTile, c, len, a.channels);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      sa[group][lane * V + k] = A[k];
      sq[group][lane * V + k] = Q[k];
      if (!FORM) sh[group][lane * V + k] = H[k];
    }
    __syncthreads();
    if (second && threadIdx.x % kWave < kChannels) {
      float as[groups], qs[groups];              // all read before the chain
#pragma unroll
      for (int s = 0; s < groups; ++s) { as[s] = sa[s][at]; qs[s] = sq[s][at]; }
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (FORM) {
        float tile_q = 0.f, tile_a = 1.f;
#pragma unroll
        for (int s = groups - 1; s >= 0; --s) {
          tile_q = __builtin_fmaf(as[s], tile_q, qs[s]);
          tile_a *= as[s];
        }
        back = __builtin_fmaf(through, tile_q, back);        // the tile, then those before it
        through *= tile_a;
      } else {
#pragma unroll
        for (int s = groups - 1; s >= 0; --s) {
          sq[s][at] = back;                      // from behind the group's last step
          back = __builtin_fmaf(as[s], back, qs[s]);
        }
      }
    } else if (!FORM && threadIdx.x < kChannels) {
      float state = carry, as[groups], hs[groups];
#pragma unroll
      for (int s = 0; s < groups; ++s) { as[s] = sa[s][at]; hs[s] = sh[s][at]; }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < groups; ++s) {
        sh[s][at] = state;
        state = __builtin_fmaf(as[s], state, hs[s]);
      }
      if (tile > first) load_carry(tile - 1);
    }
    __syncthreads();
    if constexpr (!FORM) {
      float before[S][V], r[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float now = sh[group][lane * V + k];
        r[k] = sq[group][lane * V + k];
#pragma unroll
        for (int i = 0; i < S; ++i) {
          before[i][k] = now;
          now = __builtin_fmaf(ga[i][k], now, all || t0 + i < len ? keep[i][k] * xs(i, k) : 0.f);
        }
      }
#pragma unroll
      for (int i = S - 1; i >= 0; --i) {
        const bool live = all || t0 + i < len;
        float dg[V], dx[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float l = ds(i, k) + r[k];
          r[k] = ga[i][k] * l;
          dx[k] = live ? keep[i][k] * l : 0.f;
          dg[k] = live ? r[k] * keep[i][k] * (before[i][k] - xs(i, k)) : 0.f;
        }
        store_run<T, EDGE, PAST>(static_cast<T *>(a.dgate) + out, a.channels, t0, a.steps, c, i, dg);
        store_run<T, EDGE, PAST>(static_cast<T *>(a.dx) + out, a.channels, t0, a.steps, c, i, dx);
      }
    }
    __syncthreads();
  };
  for (int tile = start; tile != stop; tile += turn) {
    if ((tile + 1) * kTile <= len) body(tile, std::true_type{});
    else body(tile, std::false_type{});
  }
  if (!keeps) return;
  if (FORM) {
    float *seg = a.segments + (static_cast<int64_t>(b) * a.n_segments + segment) * 2 * a.channels + own;
    seg[0] = through;
    seg[a.channels] = back;
  } else if (a.dstate && first == 0) {
    a.dstate[static_cast<int64_t>(b) * a.channels + own] = back;
  }
}

// The second launch of the split form: the A and H of the segments of 64 channels of a sequence, in sixteen parts; each
// segment's H becomes the state before it, or (BACK) what comes from behind it.
constexpr int kParts = 16;
template <bool BACK>
__global__ __launch_bounds__(64 * kParts) void recurrence_join_kernel(RecurrenceArgs a) {
  __shared__ float sa[kParts][64], sh[kParts][64];
  const int lane = threadIdx.x % 64, part = threadIdx.x / 64, c = blockIdx.x * 64 + lane, b = blockIdx.y;
  const bool inside = c < a.channels;
  const int each = (a.n_segments + kParts - 1) / kParts, lo = part * each, n = max(0, min(a.n_segments, lo + each) - lo);
  float *seg = a.segments + static_cast<int64_t>(b) * a.n_segments * 2 * a.channels + c;
  // the i-th segment of the part in the order they are passed through; the last one of all passes nothing on
  auto at = [&](int i) { return seg + static_cast<int64_t>(BACK ? a.n_segments - 1 - (lo + i) : lo + i) * 2 * a.channels; };
  auto passes = [&](int i) { return lo + i + 1 < a.n_segments; };
  float A = 1.f, H = 0.f;
  if (inside) {
#pragma unroll 8
    for (int i = 0; i < n; ++i) {
      const float as = passes(i) ? at(i)[0] : 1.f, hs = passes(i) ? at(i)[a.channels] : 0.f;
      H = __builtin_fmaf(as, H, hs);
      A *= as;
    }
  }
  sa[part][lane] = A;
  sh[part][lane] = H;
  __syncthreads();
  if (!inside) return;
  const float *given = BACK ? a.dlast : a.state;
  float state = given ? given[static_cast<int64_t>(b) * a.channels + c] : 0.f;
  for (int s = 0; s < part; ++s) state = __builtin_fmaf(sa[s][lane], state, sh[s][lane]);
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    float *p = at(i);
    const float as = passes(i) ? p[0] : 1.f, hs = passes(i) ? p[a.channels] : 0.f;
    p[a.channels] = state;
    state = __builtin_fmaf(as, state, hs);
  }
}

// One step, the state updated in place: four channels a thread.
template <typename T>
__global__ __launch_bounds__(kThreads) void recurrence_step_kernel(const T *gate, const T *x, float *state, T *h, int64_t batch, int32_t channels,
                                                                  int64_t gate_stride, int64_t x_stride) {
  const int32_t packs = (channels + kV - 1) / kV;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < batch * packs; i += static_cast<int64_t>(gridDim.x) * kThreads) {
    const int64_t b = i / packs;
    const int c = static_cast<int>(i - b * packs) * kV, have = channels - c;
    const Pack<T, kV> g = load_some<T, kV>(gate + b * gate_stride + c, have), u = load_some<T, kV>(x + b * x_stride + c, have);
    float *s = state + b * channels + c;
    const Pack<float, kV> old = load_some<float, kV>(s, have);
    float now[kV];
#pragma unroll
    for (int k = 0; k < kV; ++k) {
      float r, q;
      gate_of(static_cast<float>(g.v[k]), r, q);
      now[k] = r * old.v[k] + q * static_cast<float>(u.v[k]);
    }
    store_some<float, kV>(s, now, have);
    store_some<T, kV>(h + b * channels + c, now, have);
  }
}

template <typename T, int LANES, bool EDGE, bool FORM, bool PAST>
void launch_recurrence(const RecurrenceArgs &a, int64_t blocks, bool backward, hipStream_t s) {
  // more workgroups than one dimension takes (2^32 threads): rows of them, the last of which goes past the end
  const int64_t across = std::min<int64_t>(blocks, 1 << 20);
  const dim3 grid(static_cast<uint32_t>(across), static_cast<uint32_t>(ceil_div(blocks, across)));
  if (backward) hipLaunchKernelGGL((recurrence_backward_kernel<T, LANES, EDGE, FORM, PAST>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((recurrence_forward_kernel<T, LANES, EDGE, FORM, PAST>), grid, dim3(kThreads), 0, s, a);
}
// PAST is a choice at compile time: as a branch at every store it costs more than it gives (16 x 2048 x 1024: 136 us against 128).
template <typename T, bool EDGE, bool PAST>
void launch_recurrence(const RecurrenceArgs &a, const Cut &cut, bool backward, hipStream_t s) {
  const int64_t blocks = blocks_of(cut, a.batch, a.channels);
  if (cut.lanes == 8) return launch_recurrence<T, 8, EDGE, false, PAST>(a, blocks, backward, s);
  if (cut.segments > 1) {
    launch_recurrence<T, 16, EDGE, true, false>(a, blocks, backward, s);
    const dim3 grid(static_cast<uint32_t>(ceil_div(a.channels, 64)), static_cast<uint32_t>(a.batch));
    if (backward) hipLaunchKernelGGL((recurrence_join_kernel<true>), grid, dim3(64 * kParts), 0, s, a);
    else hipLaunchKernelGGL((recurrence_join_kernel<false>), grid, dim3(64 * kParts), 0, s, a);
  }
  launch_recurrence<T, 16, EDGE, false, PAST>(a, blocks, backward, s);
}
template <typename T>
void launch_recurrence(const RecurrenceArgs &a, const Cut &cut, bool backward, hipStream_t s) {
  const bool past = static_cast<int64_t>(a.batch) * a.steps * a.channels * static_cast<int64_t>(sizeof(T)) >= kPastBytes;
  if (a.channels % kV) past ? launch_recurrence<T, true, true>(a, cut, backward, s) : launch_recurrence<T, true, false>(a, cut, backward, s);
  else past ? launch_recurrence<T, false, true>(a, cut, backward, s) : launch_recurrence<T, false, false>(a, cut, backward, s);
}

void launch_recurrence_type(RecurrenceArgs &a, int32_t type, bool backward, hipStream_t s) {
  const Cut cut = cut_of(a.batch, a.steps, a.channels, backward);
  a.n_segments = cut.segments;
  a.tiles_per_segment = cut.tiles_each;
  if (type == ONES_F32) launch_recurrence<float>(a, cut, backward, s);
  else if (type == ONES_F16) launch_recurrence<f16>(a, cut, backward, s);
  else launch_recurrence<bf16>(a, cut, backward, s);
}

template <typename T>
void launch_step(const void *gate, int64_t gate_stride, const void *x, int64_t x_stride, int64_t batch, int64_t channels, float *state, void *h,
                 hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(ceil_div(batch * ceil_div(channels, kV), kThreads), 1 << 16)));
  hipLaunchKernelGGL((recurrence_step_kernel<T>), grid, dim3(kThreads), 0, s, static_cast<const T *>(gate), static_cast<const T *>(x), state,
                     static_cast<T *>(h), batch, static_cast<int32_t>(channels), gate_stride, x_stride);
}

}  // namespace
}  // namespace train
}  // namespace ones

using namespace ones::train;

extern "C" {

size_t ones_recurrence_carry_bytes(int64_t batch, int64_t steps, int64_t channels) {
  if (check_recurrence(batch, steps, channels, ONES_F32) != ONES_OK) return 0;
  return carry_floats(batch, steps, channels) * 4;
}

size_t ones_recurrence_workspace_bytes(int64_t batch, int64_t steps, int64_t channels) {
  if (check_recurrence(batch, steps, channels, ONES_F32) != ONES_OK) return 0;
  const int64_t n = std::max(cut_of(batch, steps, channels, false).segments, cut_of(batch, steps, channels, true).segments);
  return n > 1 ? align_up(static_cast<size_t>(batch * n * 2 * channels * 4)) : 0;
}

int ones_recurrence_forward(const void *gate, int64_t gate_batch_stride, int64_t gate_step_stride, const void *x, int64_t x_batch_stride,
                            int64_t x_step_stride, int64_t batch, int64_t steps, int64_t channels, int32_t type, const float *state,
                            const int32_t *lengths, void *h, float *last, float *carry, void *d_workspace, size_t workspace_bytes,
                            void *hip_stream) {
  if (int rc = check_recurrence(batch, steps, channels, type)) return rc;
  if (int rc = check_strides(gate_batch_stride, gate_step_stride)) return rc;
  if (int rc = check_strides(x_batch_stride, x_step_stride)) return rc;
  if (batch == 0 || channels == 0) return ONES_OK;
  if (steps && (!gate || !x || !h)) return ONES_E_INVALID_ARG;
  if (int rc = check_workspace(d_workspace, workspace_bytes, ones_recurrence_workspace_bytes(batch, steps, channels))) return rc;
  RecurrenceArgs a{};
  a.gate = gate; a.x = x; a.h = h; a.state = state; a.last = last; a.lengths = lengths; a.carry = carry;
  a.segments = static_cast<float *>(d_workspace);
  a.gate_batch = gate_batch_stride; a.gate_step = gate_step_stride; a.x_batch = x_batch_stride; a.x_step = x_step_stride;
  a.batch = static_cast<int32_t>(batch); a.steps = static_cast<int32_t>(steps); a.channels = static_cast<int32_t>(channels);
  a.tiles = static_cast<int32_t>(tiles_of(steps));
  launch_recurrence_type(a, type, false, static_cast<hipStream_t>(hip_stream));
  return launched("recurrence forward");
}

int ones_recurrence_backward(const void *dh, int64_t dh_batch_stride, int64_t dh_step_stride, const float *dlast, const void *gate,
                             int64_t gate_batch_stride, int64_t gate_step_stride, const void *x, int64_t x_batch_stride,
                             int64_t x_step_stride, int64_t batch, int64_t steps, int64_t channels, int32_t type, const float *carry,
                             const int32_t *lengths, void *dgate, void *dx, float *dstate, void *d_workspace, size_t workspace_bytes,
                             void *hip_stream) {
  if (int rc = check_recurrence(batch, steps, channels, type)) return rc;
  if (int rc = check_strides(dh_batch_stride, dh_step_stride)) return rc;
  if (int rc = check_strides(gate_batch_stride, gate_step_stride)) return rc;
  if (int rc = check_strides(x_batch_stride, x_step_stride)) return rc;
  if (batch == 0 || channels == 0) return ONES_OK;
  if (steps && (!dh || !gate || !x || !carry || !dgate || !dx)) return ONES_E_INVALID_ARG;
  if (int rc = check_workspace(d_workspace, workspace_bytes, ones_recurrence_workspace_bytes(batch, steps, channels))) return rc;
  RecurrenceArgs a{};
  a.gate = gate; a.x = x; a.dh = dh; a.dgate = dgate; a.dx = dx; a.dlast = dlast; a.dstate = dstate; a.lengths = lengths;
  a.carry = const_cast<float *>(carry);
  a.segments = static_cast<float *>(d_workspace);
  a.gate_batch = gate_batch_stride; a.gate_step = gate_step_stride; a.x_batch = x_batch_stride; a.x_step = x_step_stride;
  a.dh_batch = dh_batch_stride; a.dh_step = dh_step_stride;
  a.batch = static_cast<int32_t>(batch); a.steps = static_cast<int32_t>(steps); a.channels = static_cast<int32_t>(channels);
  a.tiles = static_cast<int32_t>(tiles_of(steps));
  launch_recurrence_type(a, type, true, static_cast<hipStream_t>(hip_stream));
  return launched("recurrence backward");
}

int ones_recurrence_step(const void *gate, int64_t gate_stride, const void *x, int64_t x_stride, int64_t batch, int64_t channels, int32_t type,
                         float *state, void *h, void *hip_stream) {
  if (int rc = check_sizes(batch, 1, channels, type)) return rc;
  if (int rc = check_strides(gate_stride, 0)) return rc;
  if (int rc = check_strides(x_stride, 0)) return rc;
  if (batch == 0 || channels == 0) return ONES_OK;
  if (!gate || !x || !state || !h) return ONES_E_INVALID_ARG;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (type == ONES_F32) launch_step<float>(gate, gate_stride, x, x_stride, batch, channels, state, h, s);
  else if (type == ONES_F16) launch_step<f16>(gate, gate_stride, x, x_stride, batch, channels, state, h, s);
  else launch_step<bf16>(gate, gate_stride, x, x_stride, batch, channels, state, h, s);
  return launched("recurrence step");
}

}  // extern "C"

// The gated linear recurrence over the steps of a sequence, channel by channel (ones_recurrence_*).
//
//   a_t = sigmoid(gate_t), h_t = a_t h_{t-1} + (1 - a_t) x_t
//   l_t = dh_t + a_{t+1} l_{t+1}, dx_t = (1 - a_t) l_t, dgate_t = l_t (h_{t-1} - x_t) a_t (1 - a_t), dstate = a_0 l_0
//
// Steps t past a sequence's length keep the state: a_t = 1, no input, h_t written as 0, no gradients.
//
// A run of steps acts on the state as h -> A h + H (A the product of its gates), and on what comes back from behind as
// r -> A r + Q (r_t = a_t l_t); two runs one after another compose.  A workgroup owns 64 channels of one sequence and takes tiles
// of 128 steps: a thread keeps eight steps of four channels in registers (32 steps of one where the rows do not allow wide
// loads) and forms its run's A and H, one wave composes the runs of the tile's thread groups through LDS, and every thread walks
// its steps again from the state before them.  gate, x and dh are read once and everything is written once.  The state before
// every tile is kept in 32 bits (1/32 of the bytes of a 16-bit h): backward recomputes h from it, which is neither rounded to 16
// bits nor read.
//
// Where sequences and channels are too few for the compute units, the steps are split into segments of whole tiles as well.  A
// first launch forms each segment's A and H (or Q), and the workgroups of the second compose those of the segments before (or
// behind) their own: the inputs are read twice then.  No workgroup waits for another, and the order of all sums is fixed.
#include "train_device.h"
#include "train_host.h"

#include <algorithm>

namespace ones {
namespace train {
namespace {

constexpr int kThreads = 256, kChannels = 64, kTile = 128;

struct RecurrenceArgs {
  const void *gate, *x, *dh;
  void *h, *dgate, *dx;
  const float *state, *dlast;      // may be null: zeros
  float *last, *dstate;            // may be null
  const int32_t *lengths;          // may be null: all steps
  float *carry;                    // [batch][tiles][channels]: the state before every tile; forward may be null
  float *segments;                 // [batch][segments][2][channels]
  int64_t gate_batch, gate_step, x_batch, x_step, dh_batch, dh_step;
  int32_t batch, steps, channels, tiles, n_segments, tiles_per_segment;
};

__device__ __forceinline__ int length_of(const RecurrenceArgs &a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.steps) : a.steps;
}

// The S steps x V channels of this thread's run, as read.
template <typename T, int S, int V>
struct Run {
  Pack<T, V> p[S];
  __device__ __forceinline__ void load(const T *base, int64_t step_stride, int t0, int c, int len, int channels) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      if (t0 + i < len && c < channels) p[i] = load_pack<T, V>(base + (t0 + i) * step_stride + c);
      else
#pragma unroll
        for (int k = 0; k < V; ++k) p[i].v[k] = static_cast<T>(0.f);
    }
  }
};

// a = sigmoid(g) and 1 - a, which keeps its digits where a is close to 1.
__device__ __forceinline__ void gate_of(float g, float &a, float &keep) {
  const float e = __expf(-g);
  a = 1.f / (1.f + e);
  keep = isinf(e) ? 1.f : e * a;
}

template <typename T, int V, bool FORM>     // FORM: only the segments' A and H
__global__ __launch_bounds__(kThreads) void recurrence_forward_kernel(RecurrenceArgs a) {
  constexpr int lanes = kChannels / V, groups = kThreads / lanes, S = kTile / groups;
  __shared__ float sa[groups][kChannels], sh[groups][kChannels];
  const int b = blockIdx.y, segment = blockIdx.z, c0 = blockIdx.x * kChannels;
  if (FORM && segment == a.n_segments - 1) return;   // nothing comes after it
  const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes, c = c0 + lane * V;
  const int len = length_of(a, b);
  const T *gate = static_cast<const T *>(a.gate) + b * a.gate_batch, *x = static_cast<const T *>(a.x) + b * a.x_batch;
  T *h = FORM ? nullptr : static_cast<T *>(a.h) + static_cast<int64_t>(b) * a.steps * a.channels;
  const int first = segment * a.tiles_per_segment, end = min(a.tiles, first + a.tiles_per_segment);
  // thread c of the first wave keeps channel c0 + c's state, and the segment's product of gates where that is asked for
  const int own = c0 + static_cast<int>(threadIdx.x);
  const bool keeps = threadIdx.x < kChannels && own < a.channels;
  float state = 0.f, through = 1.f;
  if (!FORM && keeps) {
    if (a.state) state = a.state[static_cast<int64_t>(b) * a.channels + own];
    const float *seg = a.segments + static_cast<int64_t>(b) * a.n_segments * 2 * a.channels + own;
#pragma unroll 4
    for (int s = 0; s < segment; ++s, seg += 2 * a.channels) state = seg[0] * state + seg[a.channels];
  }
  Run<T, S, V> g, u;
  g.load(gate, a.gate_step, first * kTile + group * S, c, len, a.channels);
  u.load(x, a.x_step, first * kTile + group * S, c, len, a.channels);
  for (int tile = first; tile < end; ++tile) {
    const int t0 = tile * kTile + group * S;
    float ga[S][V], in[S][V], A[V], H[V];
#pragma unroll
    for (int k = 0; k < V; ++k) { A[k] = 1.f; H[k] = 0.f; }
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const bool live = t0 + i < len;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float r, q;
        gate_of(static_cast<float>(g.p[i].v[k]), r, q);
        ga[i][k] = live ? r : 1.f;
        in[i][k] = live ? q * static_cast<float>(u.p[i].v[k]) : 0.f;
        A[k] *= ga[i][k];
        H[k] = ga[i][k] * H[k] + in[i][k];
      }
    }
    if (tile + 1 < end) {                        // the next tile's rows arrive while this one is put together
      g.load(gate, a.gate_step, t0 + kTile, c, len, a.channels);
      u.load(x, a.x_step, t0 + kTile, c, len, a.channels);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) { sa[group][lane * V + k] = A[k]; sh[group][lane * V + k] = H[k]; }
    __syncthreads();
    if (threadIdx.x < kChannels) {
      if (!FORM && keeps && a.carry) a.carry[(static_cast<int64_t>(b) * a.tiles + tile) * a.channels + own] = state;
#pragma unroll
      for (int s = 0; s < groups; ++s) {
        const float as = sa[s][threadIdx.x], hs = sh[s][threadIdx.x];
        sh[s][threadIdx.x] = state;              // before the group's first step
        state = as * state + hs;
        if (FORM) through *= as;
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
          now[k] = ga[i][k] * now[k] + in[i][k];
          out[k] = t0 + i < len ? now[k] : 0.f;
        }
        if (t0 + i < a.steps && c < a.channels) store_pack<T, V>(h + static_cast<int64_t>(t0 + i) * a.channels + c, out);
      }
      __syncthreads();                           // sh is written anew
    }
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

template <typename T, int V, bool FORM>     // FORM: only the segments' A and Q
__global__ __launch_bounds__(kThreads) void recurrence_backward_kernel(RecurrenceArgs a) {
  constexpr int lanes = kChannels / V, groups = kThreads / lanes, S = kTile / groups;
  __shared__ float sa[groups][kChannels], sh[groups][kChannels], sq[groups][kChannels];
  const int b = blockIdx.y, segment = blockIdx.z, c0 = blockIdx.x * kChannels;
  if (FORM && segment == 0) return;                  // nothing comes before it
  const int lane = threadIdx.x % lanes, group = threadIdx.x / lanes, c = c0 + lane * V;
  const int len = length_of(a, b);
  const T *gate = static_cast<const T *>(a.gate) + b * a.gate_batch, *x = static_cast<const T *>(a.x) + b * a.x_batch;
  const T *dh = static_cast<const T *>(a.dh) + b * a.dh_batch;
  const int64_t out = static_cast<int64_t>(b) * a.steps * a.channels;
  const int first = segment * a.tiles_per_segment, end = min(a.tiles, first + a.tiles_per_segment);
  // the second wave keeps what comes back from behind, the first composes the states
  const int own = c0 + static_cast<int>(threadIdx.x % kChannels);
  const bool second = threadIdx.x / kChannels == 1, keeps = second && own < a.channels;
  float back = 0.f, through = 1.f;
  if (!FORM && keeps) {
    if (a.dlast) back = a.dlast[static_cast<int64_t>(b) * a.channels + own];
    const float *seg = a.segments + (static_cast<int64_t>(b) * a.n_segments + a.n_segments - 1) * 2 * a.channels + own;
#pragma unroll 4
    for (int s = a.n_segments - 1; s > segment; --s, seg -= 2 * a.channels) back = seg[0] * back + seg[a.channels];
  }
  Run<T, S, V> g, u, d;
  if (end > first) {                             // always, but for sequences of no steps
    const int t0 = (end - 1) * kTile + group * S;
    g.load(gate, a.gate_step, t0, c, len, a.channels);
    if (!FORM) u.load(x, a.x_step, t0, c, len, a.channels);
    d.load(dh, a.dh_step, t0, c, len, a.channels);
  }
  for (int tile = end - 1; tile >= first; --tile) {
    const int t0 = tile * kTile + group * S;
    float ga[S][V], keep[S][V], xs[S][V], ds[S][V], A[V], H[V], Q[V];
#pragma unroll
    for (int k = 0; k < V; ++k) { A[k] = 1.f; H[k] = Q[k] = 0.f; }
#pragma unroll
    for (int i = 0; i < S; ++i) {
      const bool live = t0 + i < len;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float r, q;
        gate_of(static_cast<float>(g.p[i].v[k]), r, q);
        ga[i][k] = live ? r : 1.f;
        keep[i][k] = live ? q : 0.f;
        ds[i][k] = static_cast<float>(d.p[i].v[k]);
        A[k] *= ga[i][k];
        if (!FORM) {
          xs[i][k] = static_cast<float>(u.p[i].v[k]);
          H[k] = ga[i][k] * H[k] + (live ? keep[i][k] * xs[i][k] : 0.f);
        }
      }
    }
#pragma unroll
    for (int i = S - 1; i >= 0; --i)
#pragma unroll
      for (int k = 0; k < V; ++k) Q[k] = ga[i][k] * (ds[i][k] + Q[k]);
    if (tile > first) {
      g.load(gate, a.gate_step, t0 - kTile, c, len, a.channels);
      if (!FORM) u.load(x, a.x_step, t0 - kTile, c, len, a.channels);
      d.load(dh, a.dh_step, t0 - kTile, c, len, a.channels);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
      sa[group][lane * V + k] = A[k];
      sq[group][lane * V + k] = Q[k];
      if (!FORM) sh[group][lane * V + k] = H[k];
    }
    __syncthreads();
    if (second) {
#pragma unroll
      for (int s = groups - 1; s >= 0; --s) {
        const float as = sa[s][threadIdx.x % kChannels], qs = sq[s][threadIdx.x % kChannels];
        sq[s][threadIdx.x % kChannels] = back;   // from behind the group's last step
        back = as * back + qs;
        if (FORM) through *= as;
      }
    } else if (!FORM && threadIdx.x < kChannels) {
      float state = own < a.channels ? a.carry[(static_cast<int64_t>(b) * a.tiles + tile) * a.channels + own] : 0.f;
#pragma unroll
      for (int s = 0; s < groups; ++s) {
        const float as = sa[s][threadIdx.x], hs = sh[s][threadIdx.x];
        sh[s][threadIdx.x] = state;
        state = as * state + hs;
      }
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
          now = ga[i][k] * now + (t0 + i < len ? keep[i][k] * xs[i][k] : 0.f);
        }
      }
#pragma unroll
      for (int i = S - 1; i >= 0; --i) {
        const bool live = t0 + i < len;
        float dg[V], dx[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float l = ds[i][k] + r[k];
          r[k] = ga[i][k] * l;
          dx[k] = live ? keep[i][k] * l : 0.f;
          dg[k] = live ? r[k] * keep[i][k] * (before[i][k] - xs[i][k]) : 0.f;
        }
        if (t0 + i < a.steps && c < a.channels) {
          store_pack<T, V>(static_cast<T *>(a.dgate) + out + static_cast<int64_t>(t0 + i) * a.channels + c, dg);
          store_pack<T, V>(static_cast<T *>(a.dx) + out + static_cast<int64_t>(t0 + i) * a.channels + c, dx);
        }
      }
    }
    __syncthreads();
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

// One step, the state updated in place: an element a thread (four with wide rows).
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void recurrence_step_kernel(const T *gate, const T *x, float *state, T *h, int64_t batch, int32_t channels,
                                                                  int64_t gate_stride, int64_t x_stride) {
  const int32_t packs = (channels + V - 1) / V;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (i >= batch * packs) return;
  const int64_t b = i / packs;
  const int c = static_cast<int>(i - b * packs) * V;
  const Pack<T, V> g = load_pack<T, V>(gate + b * gate_stride + c), u = load_pack<T, V>(x + b * x_stride + c);
  float *s = state + b * channels + c;
  const Pack<float, V> old = load_pack<float, V>(s);
  float now[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float r, q;
    gate_of(static_cast<float>(g.v[k]), r, q);
    now[k] = r * old.v[k] + q * static_cast<float>(u.v[k]);
  }
  store_pack<float, V>(s, now);
  store_pack<T, V>(h + b * channels + c, now);
}

int64_t tiles_of(int64_t steps) { return ceil_div(steps, kTile); }

// Segments: as many as fill the compute units with a few workgroups each, of four tiles at least.
void split(int64_t batch, int64_t steps, int64_t channels, int32_t &n, int32_t &tiles_each) {
  const int64_t tiles = tiles_of(steps), chains = batch * ceil_div(channels, kChannels);
  int64_t want = chains >= 192 ? 1 : std::min(ceil_div(1024, std::max<int64_t>(chains, 1)), tiles / 4);
  want = std::max<int64_t>(1, want);
  tiles_each = static_cast<int32_t>(std::max<int64_t>(1, ceil_div(tiles, want)));
  n = static_cast<int32_t>(std::max<int64_t>(1, ceil_div(tiles, tiles_each)));
}

template <typename T, int V>
void launch_recurrence(const RecurrenceArgs &a, bool backward, hipStream_t s) {
  const uint32_t blocks = static_cast<uint32_t>(ceil_div(a.channels, kChannels));
  const dim3 grid(blocks, static_cast<uint32_t>(a.batch), static_cast<uint32_t>(a.n_segments));
  if (backward) {
    if (a.n_segments > 1) hipLaunchKernelGGL((recurrence_backward_kernel<T, V, true>), grid, dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL((recurrence_backward_kernel<T, V, false>), grid, dim3(kThreads), 0, s, a);
  } else {
    if (a.n_segments > 1) hipLaunchKernelGGL((recurrence_forward_kernel<T, V, true>), grid, dim3(kThreads), 0, s, a);
    hipLaunchKernelGGL((recurrence_forward_kernel<T, V, false>), grid, dim3(kThreads), 0, s, a);
  }
}

template <typename T>
void launch_recurrence_vec(const RecurrenceArgs &a, bool backward, hipStream_t s) {
  const int64_t bytes = 4 * sizeof(T);
  bool wide = a.channels % 4 == 0 && a.gate_batch % 4 == 0 && a.gate_step % 4 == 0 && a.x_batch % 4 == 0 && a.x_step % 4 == 0 &&
              aligned(a.gate, bytes) && aligned(a.x, bytes);
  if (backward) wide = wide && a.dh_batch % 4 == 0 && a.dh_step % 4 == 0 && aligned(a.dh, bytes) && aligned(a.dgate, bytes) && aligned(a.dx, bytes);
  else wide = wide && aligned(a.h, bytes);
  if (wide) launch_recurrence<T, 4>(a, backward, s);
  else launch_recurrence<T, 1>(a, backward, s);
}

void launch_recurrence_type(const RecurrenceArgs &a, int32_t type, bool backward, hipStream_t s) {
  if (type == ONES_F32) launch_recurrence_vec<float>(a, backward, s);
  else if (type == ONES_F16) launch_recurrence_vec<f16>(a, backward, s);
  else launch_recurrence_vec<bf16>(a, backward, s);
}

int check_recurrence(int64_t batch, int64_t steps, int64_t channels, int32_t type) {
  if (batch < 0 || steps < 0 || channels < 0 || !is_type(type)) return ONES_E_INVALID_ARG;
  if (batch > ONES_MAX_BATCH || steps > ONES_MAX_STEPS || channels > ONES_MAX_CHANNELS) return ONES_E_BOUNDS;
  return steps && channels && batch > kMaxElements / (steps * channels) ? ONES_E_BOUNDS : ONES_OK;
}
// Rows of `channels` elements, `step` elements apart and sequences `batch` elements apart.
int check_strides(int64_t batch_stride, int64_t step_stride, int64_t channels) {
  if (batch_stride < 0 || step_stride < 0) return ONES_E_INVALID_ARG;
  return batch_stride > (int64_t{1} << 40) || step_stride > (int64_t{1} << 32) ? ONES_E_BOUNDS : ONES_OK;
}

template <typename T>
void launch_step(const void *gate, int64_t gate_stride, const void *x, int64_t x_stride, int64_t batch, int64_t channels, float *state, void *h,
                 hipStream_t s) {
  const bool wide = channels % 4 == 0 && gate_stride % 4 == 0 && x_stride % 4 == 0 && aligned(gate, 4 * sizeof(T)) && aligned(x, 4 * sizeof(T)) &&
                    aligned(h, 4 * sizeof(T)) && aligned(state, 16);
  const int64_t packs = batch * (wide ? channels / 4 : channels);
  const dim3 grid(static_cast<uint32_t>(ceil_div(packs, kThreads)));
  const T *g = static_cast<const T *>(gate), *u = static_cast<const T *>(x);
  if (wide) hipLaunchKernelGGL((recurrence_step_kernel<T, 4>), grid, dim3(kThreads), 0, s, g, u, state, static_cast<T *>(h), batch, static_cast<int32_t>(channels), gate_stride, x_stride);
  else hipLaunchKernelGGL((recurrence_step_kernel<T, 1>), grid, dim3(kThreads), 0, s, g, u, state, static_cast<T *>(h), batch, static_cast<int32_t>(channels), gate_stride, x_stride);
}

size_t carry_floats(int64_t batch, int64_t steps, int64_t channels) { return static_cast<size_t>(batch) * tiles_of(steps) * channels; }

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
  int32_t n, each;
  split(batch, steps, channels, n, each);
  return n > 1 ? align_up(static_cast<size_t>(batch) * n * 2 * channels * 4) : 0;
}

int ones_recurrence_forward(const void *gate, int64_t gate_batch_stride, int64_t gate_step_stride, const void *x, int64_t x_batch_stride,
                            int64_t x_step_stride, int64_t batch, int64_t steps, int64_t channels, int32_t type, const float *state,
                            const int32_t *lengths, void *h, float *last, float *carry, void *d_workspace, size_t workspace_bytes,
                            void *hip_stream) {
  if (int rc = check_recurrence(batch, steps, channels, type)) return rc;
  if (int rc = check_strides(gate_batch_stride, gate_step_stride, channels)) return rc;
  if (int rc = check_strides(x_batch_stride, x_step_stride, channels)) return rc;
  if (batch == 0 || channels == 0) return ONES_OK;
  if (steps && (!gate || !x || !h)) return ONES_E_INVALID_ARG;
  if (int rc = check_workspace(d_workspace, workspace_bytes, ones_recurrence_workspace_bytes(batch, steps, channels))) return rc;
  RecurrenceArgs a{};
  a.gate = gate; a.x = x; a.h = h; a.state = state; a.last = last; a.lengths = lengths; a.carry = carry;
  a.segments = static_cast<float *>(d_workspace);
  a.gate_batch = gate_batch_stride; a.gate_step = gate_step_stride; a.x_batch = x_batch_stride; a.x_step = x_step_stride;
  a.batch = static_cast<int32_t>(batch); a.steps = static_cast<int32_t>(steps); a.channels = static_cast<int32_t>(channels);
  a.tiles = static_cast<int32_t>(tiles_of(steps));
  split(batch, steps, channels, a.n_segments, a.tiles_per_segment);
  launch_recurrence_type(a, type, false, static_cast<hipStream_t>(hip_stream));
  return launched("recurrence forward");
}

int ones_recurrence_backward(const void *dh, int64_t dh_batch_stride, int64_t dh_step_stride, const float *dlast, const void *gate,
                             int64_t gate_batch_stride, int64_t gate_step_stride, const void *x, int64_t x_batch_stride,
                             int64_t x_step_stride, int64_t batch, int64_t steps, int64_t channels, int32_t type, const float *carry,
                             const int32_t *lengths, void *dgate, void *dx, float *dstate, void *d_workspace, size_t workspace_bytes,
                             void *hip_stream) {
  if (int rc = check_recurrence(batch, steps, channels, type)) return rc;
  if (int rc = check_strides(dh_batch_stride, dh_step_stride, channels)) return rc;
  if (int rc = check_strides(gate_batch_stride, gate_step_stride, channels)) return rc;
  if (int rc = check_strides(x_batch_stride, x_step_stride, channels)) return rc;
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
  split(batch, steps, channels, a.n_segments, a.tiles_per_segment);
  launch_recurrence_type(a, type, true, static_cast<hipStream_t>(hip_stream));
  return launched("recurrence backward");
}

int ones_recurrence_step(const void *gate, int64_t gate_stride, const void *x, int64_t x_stride, int64_t batch, int64_t channels, int32_t type,
                         float *state, void *h, void *hip_stream) {
  if (int rc = check_recurrence(batch, 1, channels, type)) return rc;
  if (int rc = check_strides(gate_stride, 0, channels)) return rc;
  if (int rc = check_strides(x_stride, 0, channels)) return rc;
  if (batch == 0 || channels == 0) return ONES_OK;
  if (!gate || !x || !state || !h) return ONES_E_INVALID_ARG;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (type == ONES_F32) launch_step<float>(gate, gate_stride, x, x_stride, batch, channels, state, h, s);
  else if (type == ONES_F16) launch_step<f16>(gate, gate_stride, x, x_stride, batch, channels, state, h, s);
  else launch_step<bf16>(gate, gate_stride, x, x_stride, batch, channels, state, h, s);
  return launched("recurrence step");
}

}  // extern "C"

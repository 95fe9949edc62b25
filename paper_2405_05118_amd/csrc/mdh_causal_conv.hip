// A causal convolution of W taps along the tokens, a filter for each channel: y_t = act(bias + sum_j w_j X_{t-W+1+j}), X the
// window that came in and the tokens behind it.  2 W operations a value: bound by memory, or by a launch.  4 x 2048 x 4096 bf16, 4 taps: forward 33 us
// (134 MB, 4.1 TB/s), backward 62 (201 MB, 3.2 TB/s; the rows of d_z are added up and the activation's slope is taken besides) and 5 for the
// filters' sums.
//
// A lane owns V channels of a run of tokens, and the last W - 1 values of each in registers: a row is read once by the run that owns
// it and once by the next.  The rows of a run are read kAhead at a time, the next ones while these are worked on.  The backward
// call computes the values before the activation again, from the same window; a row of d_z = d_y act'(z) is spread over the W
// rows of gradients that a lane holds open.  Sums for the filter's gradients are a lane's own, added up over the runs of a workgroup
// in LDS; one row of the workspace for each workgroup, added up in order by a second launch.
#include "mdh_act.h"
#include "mdh_internal.h"
#include "mdh_vec.h"

namespace mdh {
namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;  // rows whose loads are under way together

// lanes along the channels (2^k of them), the other lanes of a workgroup are runs; then blocks of channels, runs, sequences
struct Grid {
  int k, run;              // tokens of a run
  int64_t blocks, groups;  // of channels; workgroups along the tokens
};
struct Place {
  int64_t b, group, t0, slot;  // slot: of the windows, -1: none
  int ch, left;
  int64_t len;
};

template <int V>
__device__ __forceinline__ Place place(const ConvCall& c, const Grid& g) {
  Place p;
  unsigned i = xcd_order(blockIdx.x, gridDim.x);
  p.ch = (int)((i % (unsigned)g.blocks << g.k) + (threadIdx.x & ((1 << g.k) - 1))) * V, i /= (unsigned)g.blocks;
  p.left = c.C - p.ch;
  p.group = i % (unsigned)g.groups;
  p.b = i / (unsigned)g.groups;
  p.t0 = (p.group * (kThreads >> g.k) + (threadIdx.x >> g.k)) * g.run;
  p.len = c.lengths ? min(max((int64_t)c.lengths[p.b], (int64_t)0), c.T) : c.T;
  p.slot = c.slots ? (int64_t)c.slots[p.b] : p.b;
  if (c.slots && (p.slot < 0 || p.slot >= c.n_slots)) p.slot = -1;
  return p;
}
template <typename T>
__device__ __forceinline__ T* at(const TokenView& v, int64_t b, int64_t t, int ch) {
  return (T*)const_cast<void*>(v.p) + b * v.sb + t * v.st + ch;
}
template <typename T>
__device__ __forceinline__ T* window_at(const ConvCall& c, const void* base, int64_t slot, int64_t row, int ch) {
  return (T*)const_cast<void*>(base) + (slot * (c.W - 1) + row) * c.C + ch;
}
// X_t: a token, what came in before the first one (zeros without), zeros from the length on
template <typename T, int V>
__device__ __forceinline__ RowWords<T, V> line(const ConvCall& c, const Place& p, int64_t t) {
  if (t >= 0 && t < p.len) return load_row<T, V>(at<T>(c.x, p.b, t, p.ch), p.left);
  if (t < 0 && c.s_in && p.slot >= 0) return load_row<T, V>(window_at<T>(c, c.s_in, p.slot, c.W - 1 + t, p.ch), p.left);
  return 0;
}
// N rows from p on, those before `end`; as they are wanted, part_of() each
template <typename T, int V, int N>
__device__ __forceinline__ void rows_of(const TokenView& v, const Place& p, int64_t t, int64_t end, RowWords<T, V> (&w)[N]) {
  const T* from = at<T>(v, p.b, t, p.ch);
#pragma unroll
  for (int u = 0; u < N; ++u) {
    w[u] = 0;
    if (t + u < end) w[u] = load_part<T, V>(from + u * v.st, p.left, p.ch >= V);
  }
}
template <typename T, int W, int V>
__device__ __forceinline__ void filter(const ConvCall& c, const Place& p, float (&w)[W][V], float (&bias)[V]) {
  float flat[V * W];
  load_params<V * W>(c.weight + (int64_t)p.ch * W, p.left * W, 0.f, flat);
  load_params<V>(c.bias ? c.bias + p.ch : nullptr, p.left, 0.f, bias);
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) w[j][i] = flat[i * W + j];
}
// window[j] <- window[j + 1], the last one <- x
template <int W, int V>
__device__ __forceinline__ void shift(float (&window)[W][V], const float (&x)[V]) {
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) window[j][i] = j + 1 < W ? window[j + 1 < W ? j + 1 : j][i] : x[i];
}
template <int W, int V>
__device__ __forceinline__ void taps(const float (&w)[W][V], const float (&bias)[V], const float (&window)[W][V], float (&z)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    z[i] = bias[i];
#pragma unroll
    for (int j = 0; j < W; ++j) z[i] = fmaf(w[j][i], window[j][i], z[i]);
  }
}

template <typename T, int W, int V>
__global__ __launch_bounds__(kThreads) void conv_kernel(ConvCall c, Grid g) {
  const Place p = place<V>(c, g);
  const int64_t t1 = min(p.t0 + g.run, c.T), end = min(t1, p.len);
  if (p.left <= 0 || (p.t0 >= c.T && p.t0)) return;
  RowWords<T, V> next[kAhead];
  rows_of<T, V>(c.x, p, p.t0, end, next);
  float window[W][V], w[W][V], bias[V];
#pragma unroll
  for (int j = 0; j < W; ++j) unpack_row<T, V>(j ? line<T, V>(c, p, p.t0 - W + j) : (RowWords<T, V>)0, window[j]);
  filter<T, W, V>(c, p, w, bias);
  if (p.t0 == 0 && c.s_out && p.slot >= 0) {
    // all reads of the window that came in are this lane's, and before its writes: both may be one buffer
    RowWords<T, V> last[W];
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) last[j] = line<T, V>(c, p, p.len - (W - 1) + j);
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) store_row<T, V>(window_at<T>(c, c.s_out, p.slot, j, p.ch), p.left, last[j]);
  }
  T* to = at<T>(c.y, p.b, p.t0, p.ch);
  for (int64_t t = p.t0; t < t1; t += kAhead) {
    RowWords<T, V> raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) raw[u] = next[u];
    if (t + kAhead < end) rows_of<T, V>(c.x, p, t + kAhead, end, next);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (t + u >= t1) break;
      float x[V], z[V], y[V];
      unpack_row<T, V>(part_of<T, V>(raw[u], p.left, p.ch >= V), x);
      shift<W, V>(window, x);
      taps<W, V>(w, bias, window, z);
      act_of<V>(c.act, z, y);
      store_row<T, V>(to + u * c.y.st, p.left, t + u < end ? pack_row<T, V>(y) : (RowWords<T, V>)0);
    }
    to += kAhead * c.y.st;
  }
}

// open[j]: gradient of X_{t-W+1+j} as far as the tokens up to t give it
template <typename T, int W, int V>
__global__ __launch_bounds__(kThreads) void conv_backward_kernel(ConvCall c, Grid g) {
  constexpr int AHEAD = sizeof(T) == 2 ? 8 : 4;  // (rows ahead: four of bf16 65 us for 62; eight of fp32 leave one wavefront a SIMD)
  const Place p = place<V>(c, g);
  // rows of the gradient: this run's, the window's before the first run's
  const int64_t t1 = min(p.t0 + g.run, c.T), first = p.t0 ? p.t0 : -(int64_t)(W - 1), end = t1 + W - 1;
  float dw[W][V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    db[i] = 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j][i] = 0.f;
  }
  if (p.left > 0 && (p.t0 < c.T || p.t0 == 0)) {
    RowWords<T, V> next_x[AHEAD], next_dy[AHEAD];
    const int64_t readable = min(end, p.len);
    rows_of<T, V>(c.x, p, p.t0, readable, next_x);
    rows_of<T, V>(c.y, p, p.t0, readable, next_dy);
    float window[W][V], w[W][V], bias[V], open[W][V];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      unpack_row<T, V>(j ? line<T, V>(c, p, p.t0 - W + j) : (RowWords<T, V>)0, window[j]);
#pragma unroll
      for (int i = 0; i < V; ++i) open[j][i] = 0.f;
    }
    filter<T, W, V>(c, p, w, bias);
    for (int64_t t = p.t0; t < end; t += AHEAD) {
      RowWords<T, V> rx[AHEAD], ry[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) rx[u] = next_x[u], ry[u] = next_dy[u];
      if (t + AHEAD < end) {
        rows_of<T, V>(c.x, p, t + AHEAD, readable, next_x);
        rows_of<T, V>(c.y, p, t + AHEAD, readable, next_dy);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (t + u >= end) break;
        float x[V], dy[V], z[V], y[V], slope[V];
        unpack_row<T, V>(part_of<T, V>(rx[u], p.left, p.ch >= V), x);
        unpack_row<T, V>(part_of<T, V>(ry[u], p.left, p.ch >= V), dy);
        shift<W, V>(window, x);
        taps<W, V>(w, bias, window, z);
        act_slope<V>(c.act, z, y, slope);
        const float zero[V] = {};
        shift<W, V>(open, zero);
        const bool live = t + u < p.len, own = t + u < t1;
        float dz[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          dz[i] = live ? dy[i] * slope[i] : 0.f;
#pragma unroll
          for (int j = 0; j < W; ++j) open[j][i] = fmaf(w[j][i], dz[i], open[j][i]);
        }
        // (0 times a window that no valid token reads, one before a sequence of no tokens, may be NaN)
        if (live && own)
#pragma unroll
          for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j][i] = fmaf(dz[i], window[j][i], dw[j][i]);
            db[i] += dz[i];
          }
        const int64_t s = t + u - (W - 1);  // complete now
        if (s < first) continue;
        const int64_t tail = s - (p.len - (W - 1));  // row of the window that went out
        if (c.d_out && tail >= 0 && tail < W - 1) {
          float d[V];
          unpack_row<T, V>(load_row<T, V>(window_at<T>(c, c.d_out, p.b, tail, p.ch), p.left), d);
#pragma unroll
          for (int i = 0; i < V; ++i) open[0][i] += d[i];
        }
        if (s >= 0)
          store_row<T, V>(at<T>(c.dx, p.b, s, p.ch), p.left, s < p.len ? pack_row<T, V>(open[0]) : (RowWords<T, V>)0);
        else if (c.d_in)
          store_row<T, V>(window_at<T>(c, c.d_in, p.b, s + W - 1, p.ch), p.left, pack_row<T, V>(open[0]));
      }
    }
  }
  if (!c.part) return;
  // over the runs of the workgroup: those of a wavefront, then the wavefronts
  for (int d = 1 << g.k; d < 64; d *= 2)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      db[i] += __shfl_xor(db[i], d);
#pragma unroll
      for (int j = 0; j < W; ++j) dw[j][i] += __shfl_xor(dw[j][i], d);
    }
  constexpr int N = V * (W + 1);
  __shared__ float sums[kThreads / 64][N][64];
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < V; ++i) {
#pragma unroll
    for (int j = 0; j < W; ++j) sums[threadIdx.x >> 6][i * W + j][lane] = dw[j][i];
    sums[threadIdx.x >> 6][V * W + i][lane] = db[i];
  }
  __syncthreads();
  const int lanes = 1 << g.k;  // (at most 64)
  if ((int)threadIdx.x >= lanes || p.left <= 0) return;
  float all[N];
#pragma unroll
  for (int n = 0; n < N; ++n) all[n] = (sums[0][n][lane] + sums[1][n][lane]) + (sums[2][n][lane] + sums[3][n][lane]);
  float* part = c.part + (p.b * g.groups + p.group) * (int64_t)(W + 1) * c.C;
  float flat[V * W], bias[V];
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (n < V * W)
      flat[n < V * W ? n : 0] = all[n];
    else
      bias[n - V * W] = all[n];
  store_params<V * W>(part + (int64_t)p.ch * W, p.left * W, flat);
  store_params<V>(part + (int64_t)c.C * W + p.ch, p.left, bias);
}

// one token: X is the window and x, the window moves on by one
template <typename T, int W, int V>
__global__ __launch_bounds__(kThreads) void conv_step_kernel(ConvCall c, Grid g) {
  const Place p = place<V>(c, g);
  if (p.left <= 0 || p.t0 > 0) return;
  T* y = at<T>(c.y, p.b, 0, p.ch);
  if (p.slot < 0) {
    store_row<T, V>(y, p.left, (RowWords<T, V>)0);
    return;
  }
  RowWords<T, V> raw[W];
#pragma unroll
  for (int j = 0; j < W; ++j)
    raw[j] = j + 1 < W ? load_row<T, V>(window_at<T>(c, c.s_out, p.slot, j, p.ch), p.left)
                       : load_row<T, V>(at<T>(c.x, p.b, 0, p.ch), p.left);
  float window[W][V], w[W][V], bias[V], z[V], out[V];
  filter<T, W, V>(c, p, w, bias);
#pragma unroll
  for (int j = 0; j < W; ++j) unpack_row<T, V>(raw[j], window[j]);
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) store_row<T, V>(window_at<T>(c, c.s_out, p.slot, j, p.ch), p.left, raw[j + 1 < W ? j + 1 : j]);
  taps<W, V>(w, bias, window, z);
  act_of<V>(c.act, z, out);
  store_row<T, V>(y, p.left, pack_row<T, V>(out));
}

enum Which { kForward, kBackward, kStep };
// Channels of a lane.  (8 of bf16, which are 16 bytes, hold twice the filters: then 103 registers became 164 and more, 6 x 1021 x 2500
// 16.6 us become 30, 4 x 2048 x 4096 33 become 34.)
constexpr int kValues = 4;

Grid grid_of(const ConvCall& c, Which which) {
  Grid g;
  const int64_t lanes = cdiv(c.C, kValues);
  g.k = 0;
  while (g.k < (which == kStep ? 8 : which == kBackward ? 5 : 6) && 1 << g.k < lanes) ++g.k;
  g.blocks = cdiv(lanes, 1 << g.k);
  const auto groups = [&](int64_t run) { return c.T ? cdiv(c.T, run * (kThreads >> g.k)) : 1; };
  // runs of 64 tokens, shorter ones while there are fewer than three wavefronts a SIMD
  g.run = which == kStep ? 1 : 64;
  while (which == kForward && g.run > 8 && lanes * c.B * cdiv(c.T, g.run) < 1024 * 64 * 3) g.run /= 2;
  // Backward two workgroups a compute unit are at work, and some left over take as long as all of them (4 x 2048 x 4104 in runs of 64:
  // 528 workgroups, 130 us; 4096 channels are 512, 62): the run with the least rounds of them times its rows, 12 of them
  // for the start and the rows of the run before.  (By registers it is three for bf16 of 3 taps and fp32 of 1, and one for fp32 of 7 and 8 taps:
  // 4 x 2048 x 4096 117 and 127 us; 4 taps 87.)
  if (which == kBackward) {
    int64_t least = 0;
    for (int run = 8; run <= 128; run += 8) {
      const int64_t time = cdiv(g.blocks * groups(run) * c.B, 512) * (run + 12);
      if (run == 8 || time <= least) g.run = run, least = time;
    }
  }
  g.groups = groups(g.run);
  return g;
}

template <typename T, int W>
void go(const ConvCall& c, Which which, const Grid& g, unsigned blocks, hipStream_t st) {
  if (which == kForward)
    conv_kernel<T, W, kValues><<<blocks, kThreads, 0, st>>>(c, g);
  else if (which == kBackward)
    conv_backward_kernel<T, W, kValues><<<blocks, kThreads, 0, st>>>(c, g);
  else
    conv_step_kernel<T, W, kValues><<<blocks, kThreads, 0, st>>>(c, g);
}
template <typename T>
void taps_of(const ConvCall& c, Which which, const Grid& g, unsigned blocks, hipStream_t st) {
  switch (c.W) {
    case 1: return go<T, 1>(c, which, g, blocks, st);
    case 2: return go<T, 2>(c, which, g, blocks, st);
    case 3: return go<T, 3>(c, which, g, blocks, st);
    case 4: return go<T, 4>(c, which, g, blocks, st);
    case 5: return go<T, 5>(c, which, g, blocks, st);
    case 6: return go<T, 6>(c, which, g, blocks, st);
    case 7: return go<T, 7>(c, which, g, blocks, st);
    default: return go<T, 8>(c, which, g, blocks, st);
  }
}
mdh_status launch(const ConvCall& c, Which which, hipStream_t st) {
  const Grid g = grid_of(c, which);
  const int64_t blocks = g.blocks * g.groups * c.B;
  if (blocks >= 1 << 24) return MDH_ERR_SIZE;  // 2^32 lanes
  // a run reads the last rows of the run before it, which are another lane's to write
  if (c.W > 1 && c.T > 0 && which != kStep) {
    const bool here = which == kForward ? c.y.p == c.x.p : c.dx.p == c.x.p || c.dx.p == c.y.p;
    if (here) return MDH_ERR_UNSUPPORTED;
  }
  clear_stale_error();
  if (c.dtype == MDH_BF16)
    taps_of<bf16>(c, which, g, (unsigned)blocks, st);
  else
    taps_of<float>(c, which, g, (unsigned)blocks, st);
  return launch_status();
}

int64_t parts(const ConvCall& c) { return c.B && c.T ? c.B * grid_of(c, kBackward).groups : 0; }

}  // namespace

size_t conv_workspace(const ConvCall& c) { return (size_t)parts(c) * (size_t)(c.W + 1) * (size_t)c.C * sizeof(float); }
mdh_status launch_conv(const ConvCall& c, hipStream_t st) { return launch(c, kForward, st); }
mdh_status launch_conv_step(const ConvCall& c, hipStream_t st) { return launch(c, kStep, st); }
mdh_status launch_conv_backward(const ConvCall& call, hipStream_t st) {
  ConvCall c = call;
  const bool sums = c.dweight || c.dbias;
  if (!sums || c.T == 0) c.part = nullptr;
  if (c.B && (c.T || c.d_in)) {
    const mdh_status r = launch(c, kBackward, st);
    if (r != MDH_OK) return r;
  }
  if (!sums) return MDH_OK;
  const int64_t n = (int64_t)c.W * c.C;
  return launch_sum_rows(c.part, parts(c), n + c.C, {{c.dweight, n}, {c.dbias, c.C}, {nullptr, 0}}, st);
}

}  // namespace mdh

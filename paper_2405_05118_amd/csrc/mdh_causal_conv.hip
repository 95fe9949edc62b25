// A causal convolution of W taps along the tokens, a filter for each channel: y_t = act(bias + sum_j w_j X_{t-W+1+j}), X the
// window that came in and the tokens behind it.  2 W operations a value: bound by memory, or by a launch.
//
// A lane owns V channels (16 bytes) of a run of tokens, and the last W - 1 values of each in registers: a row is read once by
// the run that owns it and once by the next.  The backward call computes the values before the activation again, from the same
// window; a row of d_z = d_y act'(z) is spread over the W rows of gradients that a lane holds open.  Sums for the filter's gradients
// are a lane's own, one row of the workspace for each run, added up in order by a second launch.
#include "mdh_act.h"
#include "mdh_internal.h"
#include "mdh_vec.h"

namespace mdh {
namespace {

constexpr int kThreads = 256;

struct Place {
  int64_t b, seg, slot;  // slot: of the windows, -1: none
  int ch, left;
  int64_t len;
};

// lanes along the channels first, then runs, then sequences
template <typename T>
__device__ __forceinline__ bool place(const ConvCall& c, int64_t nseg, Place* p) {
  constexpr int V = kLaneValues<T>;
  const int nc = (c.C + V - 1) / V;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  p->ch = (int)(i % nc) * V;
  p->left = c.C - p->ch;
  p->seg = i / nc % nseg;
  p->b = i / nc / nseg;
  if (p->b >= c.B) return false;
  p->len = c.lengths ? min(max((int64_t)c.lengths[p->b], (int64_t)0), c.T) : c.T;
  p->slot = c.slots ? (int64_t)c.slots[p->b] : p->b;
  if (c.slots && (p->slot < 0 || p->slot >= c.n_slots)) p->slot = -1;
  return true;
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
template <typename T>
__device__ __forceinline__ Word4 line(const ConvCall& c, const Place& p, int64_t t) {
  if (t >= 0 && t < p.len) return load_row<T>(at<T>(c.x, p.b, t, p.ch), p.left);
  if (t < 0 && c.s_in && p.slot >= 0) return load_row<T>(window_at<T>(c, c.s_in, p.slot, c.W - 1 + t, p.ch), p.left);
  return (Word4){0, 0, 0, 0};
}
template <typename T, int W>
__device__ __forceinline__ void filter(const ConvCall& c, const Place& p, float (&w)[W][kLaneValues<T>], float (&bias)[kLaneValues<T>]) {
  constexpr int V = kLaneValues<T>;
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

constexpr int kAhead = 8;  // rows whose loads are under way together; a run has a multiple of them

template <typename T, int W>
__global__ __launch_bounds__(kThreads) void conv_kernel(ConvCall c, int64_t nseg, int run) {
  constexpr int V = kLaneValues<T>;
  Place p;
  if (!place<T>(c, nseg, &p)) return;
  const int64_t t0 = p.seg * run, t1 = min(t0 + run, c.T);
  float window[W][V], w[W][V], bias[V];
#pragma unroll
  for (int j = 0; j < W; ++j) unpack_row<T>(j ? line<T>(c, p, t0 - W + j) : (Word4){0, 0, 0, 0}, window[j]);
  filter<T, W>(c, p, w, bias);
  if (p.seg == 0 && c.s_out && p.slot >= 0) {
    // all reads of the window that came in are this lane's, and before its writes: both may be one buffer
    Word4 last[W];
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) last[j] = line<T>(c, p, p.len - (W - 1) + j);
#pragma unroll
    for (int j = 0; j + 1 < W; ++j) store_row<T>(window_at<T>(c, c.s_out, p.slot, j, p.ch), p.left, last[j]);
  }
  for (int64_t t = t0; t < t1; t += kAhead) {
    Word4 raw[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) raw[u] = t + u < t1 ? line<T>(c, p, t + u) : (Word4){0, 0, 0, 0};
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (t + u >= t1) break;
      float x[V], z[V], y[V];
      unpack_row<T>(raw[u], x);
      shift<W, V>(window, x);
      taps<W, V>(w, bias, window, z);
      act_of<V>(c.act, z, y);
      store_row<T>(at<T>(c.y, p.b, t + u, p.ch), p.left, t + u < p.len ? pack_row<T>(y) : (Word4){0, 0, 0, 0});
    }
  }
}

// open[j]: gradient of X_{t-W+1+j} as far as the tokens up to t give it
template <typename T, int W>
__global__ __launch_bounds__(kThreads) void conv_backward_kernel(ConvCall c, int64_t nseg, int run) {
  constexpr int V = kLaneValues<T>;
  Place p;
  if (!place<T>(c, nseg, &p)) return;
  const int64_t t0 = p.seg * run, t1 = min(t0 + run, c.T);
  const int64_t first = p.seg ? t0 : -(int64_t)(W - 1);  // rows of the gradient: this run's, the window's before the first run's
  float window[W][V], w[W][V], bias[V], open[W][V], dw[W][V], db[V];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    unpack_row<T>(j ? line<T>(c, p, t0 - W + j) : (Word4){0, 0, 0, 0}, window[j]);
#pragma unroll
    for (int i = 0; i < V; ++i) open[j][i] = dw[j][i] = db[i] = 0.f;
  }
  filter<T, W>(c, p, w, bias);
  const int64_t end = t1 + W - 1;
  for (int64_t t = t0; t < end; ++t) {
    const bool live = t < p.len;
    float x[V], dy[V], z[V], y[V], slope[V];
    unpack_row<T>(line<T>(c, p, t), x);
    unpack_row<T>(live ? load_row<T>(at<T>(c.y, p.b, t, p.ch), p.left) : (Word4){0, 0, 0, 0}, dy);
    shift<W, V>(window, x);
    taps<W, V>(w, bias, window, z);
    act_slope<V>(c.act, z, y, slope);
    const float zero[V] = {};
    shift<W, V>(open, zero);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float dz = live ? dy[i] * slope[i] : 0.f;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        open[j][i] = fmaf(w[j][i], dz, open[j][i]);
        if (t < t1) dw[j][i] = fmaf(dz, window[j][i], dw[j][i]);
      }
      if (t < t1) db[i] += dz;
    }
    const int64_t s = t - (W - 1);  // complete now
    if (s < first) continue;
    const int64_t tail = s - (p.len - (W - 1));  // row of the window that went out
    if (c.d_out && tail >= 0 && tail < W - 1) {
      float d[V];
      unpack_row<T>(load_row<T>(window_at<T>(c, c.d_out, p.b, tail, p.ch), p.left), d);
#pragma unroll
      for (int i = 0; i < V; ++i) open[0][i] += d[i];
    }
    if (s >= 0)
      store_row<T>(at<T>(c.dx, p.b, s, p.ch), p.left, s < p.len ? pack_row<T>(open[0]) : (Word4){0, 0, 0, 0});
    else if (c.d_in)
      store_row<T>(window_at<T>(c, c.d_in, p.b, s + W - 1, p.ch), p.left, pack_row<T>(open[0]));
  }
  if (c.T == 0) return;
  float* part = c.part + (p.b * nseg + p.seg) * (int64_t)(W + 1) * c.C;
  float flat[V * W];
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) flat[i * W + j] = dw[j][i];
  store_params<V * W>(part + (int64_t)p.ch * W, p.left * W, flat);
  store_params<V>(part + (int64_t)c.C * W + p.ch, p.left, db);
}

// one token: X is the window and x, the window moves on by one
template <typename T, int W>
__global__ __launch_bounds__(kThreads) void conv_step_kernel(ConvCall c) {
  constexpr int V = kLaneValues<T>;
  Place p;
  if (!place<T>(c, 1, &p)) return;
  T* y = at<T>(c.y, p.b, 0, p.ch);
  if (p.slot < 0) {
    store_row<T>(y, p.left, (Word4){0, 0, 0, 0});
    return;
  }
  Word4 raw[W];
#pragma unroll
  for (int j = 0; j < W; ++j)
    raw[j] = j + 1 < W ? load_row<T>(window_at<T>(c, c.s_out, p.slot, j, p.ch), p.left) : load_row<T>(at<T>(c.x, p.b, 0, p.ch), p.left);
  float window[W][V], w[W][V], bias[V], z[V], out[V];
  filter<T, W>(c, p, w, bias);
#pragma unroll
  for (int j = 0; j < W; ++j) unpack_row<T>(raw[j], window[j]);
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) store_row<T>(window_at<T>(c, c.s_out, p.slot, j, p.ch), p.left, raw[j + 1 < W ? j + 1 : j]);
  taps<W, V>(w, bias, window, z);
  act_of<V>(c.act, z, out);
  store_row<T>(y, p.left, pack_row<T>(out));
}

int64_t lanes_of(const ConvCall& c) { return cdiv(c.C, c.dtype == MDH_BF16 ? 8 : 4); }
// Runs of 32 tokens where that fills the chip, else of 8 (a run reads W - 1 rows of the one before it)
int run_of(const ConvCall& c, bool backward) {
  (void)backward;
  const int64_t lanes = lanes_of(c) * c.B;
  int run = 64;
  while (run > kAhead && lanes * cdiv(c.T, run) < 256 * 4 * 64 * 4) run /= 2;
  return run;
}
int64_t runs(const ConvCall& c, bool backward) { return c.T ? cdiv(c.T, run_of(c, backward)) : 1; }
bool too_many(int64_t lanes) { return lanes >= ((int64_t)1 << 32) - kThreads; }

enum Which { kForward, kBackward, kStep };
template <typename T, int W>
void go(const ConvCall& c, Which which, int64_t nseg, int run, unsigned blocks, hipStream_t st) {
  if (which == kForward)
    conv_kernel<T, W><<<blocks, kThreads, 0, st>>>(c, nseg, run);
  else if (which == kBackward)
    conv_backward_kernel<T, W><<<blocks, kThreads, 0, st>>>(c, nseg, run);
  else
    conv_step_kernel<T, W><<<blocks, kThreads, 0, st>>>(c);
}
template <typename T>
void taps_of(const ConvCall& c, Which which, int64_t nseg, int run, unsigned blocks, hipStream_t st) {
  switch (c.W) {
    case 1: return go<T, 1>(c, which, nseg, run, blocks, st);
    case 2: return go<T, 2>(c, which, nseg, run, blocks, st);
    case 3: return go<T, 3>(c, which, nseg, run, blocks, st);
    case 4: return go<T, 4>(c, which, nseg, run, blocks, st);
    case 5: return go<T, 5>(c, which, nseg, run, blocks, st);
    case 6: return go<T, 6>(c, which, nseg, run, blocks, st);
    case 7: return go<T, 7>(c, which, nseg, run, blocks, st);
    default: return go<T, 8>(c, which, nseg, run, blocks, st);
  }
}
mdh_status launch(const ConvCall& c, Which which, hipStream_t st) {
  const int64_t nseg = which == kStep ? 1 : runs(c, which == kBackward);
  const int run = run_of(c, which == kBackward);
  const int64_t lanes = lanes_of(c) * nseg * c.B;
  if (too_many(lanes)) return MDH_ERR_SIZE;
  const unsigned blocks = (unsigned)cdiv(lanes, kThreads);
  clear_stale_error();
  if (c.dtype == MDH_BF16)
    taps_of<bf16>(c, which, nseg, run, blocks, st);
  else
    taps_of<float>(c, which, nseg, run, blocks, st);
  return launch_status();
}

}  // namespace

size_t conv_workspace(const ConvCall& c) {
  return c.B && c.T ? (size_t)(c.B * runs(c, true)) * (size_t)(c.W + 1) * (size_t)c.C * sizeof(float) : 0;
}
mdh_status launch_conv(const ConvCall& c, hipStream_t st) { return launch(c, kForward, st); }
mdh_status launch_conv_step(const ConvCall& c, hipStream_t st) { return launch(c, kStep, st); }
mdh_status launch_conv_backward(const ConvCall& c, hipStream_t st) {
  if (c.B && (c.T || c.d_in)) {
    const mdh_status r = launch(c, kBackward, st);
    if (r != MDH_OK) return r;
  }
  if (!c.dweight && !c.dbias) return MDH_OK;
  const int64_t rows = c.T ? c.B * runs(c, true) : 0, n = (int64_t)c.W * c.C;
  return launch_sum_rows(c.part, rows, n + c.C, {{c.dweight, n}, {c.dbias, c.C}, {nullptr, 0}}, st);
}

}  // namespace mdh

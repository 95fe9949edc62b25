// The selective state space scan: h_t = e^(delta_t A) h_{t-1} + delta_t x_t b_t, y_t = (c_t . h_t + skip x_t) silu(gate_t), for every
// channel and its N states -- the prefix-sum operator on pairs (a, u): (a1, u1) op (a2, u2) = (a1 a2, a2 u1 + u2), whose a a token gives.
//
// 1 exponential and 4 multiplications a step (token, channel, state), on 8 bytes a token and channel (bf16, N = 16): bound by the
// vector ALU.  Measured on this chip, cycles of a wavefront instruction with four wavefronts a SIMD: v_exp_f32 11.3, fma 3.8,
// multiplication 3.4, the same with a lane of the row broadcast to it (DPP) 5.2.
//
// De-composition.  A row of 16 lanes is a channel, a lane one state of every 16; a wavefront has four channels, a workgroup 16.
// Tokens are walked in tiles of 16.  Lane j loads x, dt and gate of token j, takes the softplus, and a step's delta reaches the row's
// other lanes as a modifier of the multiplication.  c_t . h_t: every lane's term goes to LDS, lane j adds up token j's.
// b and c of a tile lie in LDS as fp32.  With too few channels for the chip, tokens are cut into segments: what each leaves from
// a state of zeros and the sum of its deltas (its decay is e^(A sum)), a prefix sum over the segments, the pass itself.
#include "mdh_selective.h"

namespace mdh {
namespace {

constexpr int kThreads = 256, kChannels = kThreads / 16;

// what the segments leave: h of (b, seg, d, n) and the sum of deltas of (b, seg, d)
struct Segments {
  float *h, *sum;
  int n;
  int64_t tiles;  // of one
};

// STATES_ONLY: a segment's own state and sum of deltas.  Else the pass.
template <typename T, int NS, bool STATES_ONLY>
__global__ __launch_bounds__(kThreads) void scan_kernel(ScanCall c, Segments segs, int blocks) {
  constexpr int S = NS * 16;
  __shared__ float bs[S * kPitch], cs[STATES_ONLY ? 1 : S * kPitch], sums[STATES_ONLY ? 1 : kThreads / 64][kSumFloats];
  const ScanPlace p = scan_place(c, blocks, segs.n, segs.tiles);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int e = p.block * kChannels + p.row;
  const bool mine = e < c.E;
  const int64_t d = (int64_t)p.g * c.E + e, slot = scan_slot(c, p.b);
  float A[NS], h[NS], skip = 0.f, dt_bias = 0.f, total = 0.f;
  const int64_t seg_state = ((p.b * segs.n + p.seg) * c.D + d) * c.N;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int n = s * 16 + p.j;
    const bool has = mine && n < c.N;
    A[s] = has ? c.A[d * c.N + n] * kLog2e : 0.f;
    h[s] = 0.f;
    if (!STATES_ONLY && has) {
      if (segs.n > 1)
        h[s] = segs.h[seg_state + n];
      else if (c.s_in && slot >= 0)
        h[s] = c.s_in[(slot * c.D + d) * c.N + n];
    }
  }
  if (mine) {
    skip = c.skip ? c.skip[d] : 0.f;
    dt_bias = c.dt_bias ? c.dt_bias[d] : 0.f;
  }
  for (int64_t tile = p.first; tile < p.last; ++tile) {
    const int64_t t0 = tile * kTile, t = t0 + p.j;
    if (t0 >= p.len) {  // nothing is left of the sequence
      if (!STATES_ONLY && mine && t < c.T) *at<T>(c.y, p.b, t, d) = from_float<T>(0.f);
      continue;
    }
    if (!STATES_ONLY && c.checkpoints)
#pragma unroll
      for (int s = 0; s < NS; ++s)
        if (mine && s * 16 + p.j < c.N) c.checkpoints[((p.b * c.tiles + tile) * c.D + d) * c.N + s * 16 + p.j] = h[s];
    const bool live = mine && t < p.len;
    const Token k = token_of<T>(c, live, at<T>(c.x, p.b, t, d), at<T>(c.dt, p.b, t, d), dt_bias);
    const float gate = !STATES_ONLY && c.gate.p && live ? to_float(*at<T>(c.gate, p.b, t, d)) : 0.f;
    const float in = k.delta * k.x;
    total += k.delta;
    __syncthreads();
    stage_shared<T, S, kThreads>(c, c.b, p, t0, bs);
    if (!STATES_ONLY) stage_shared<T, S, kThreads>(c, c.c, p, t0, cs);
    __syncthreads();
    float y[kTile];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float bt[kTile], ct[kTile];
      tile_of(bs, s * 16 + p.j, bt);
      if (!STATES_ONLY) tile_of(cs, s * 16 + p.j, ct);
      unroll<kTile>([&](auto i) {
        constexpr int I = decltype(i)::value;
        const float a = exp2_of(lane_of_row<I>(k.delta) * A[s]);
        h[s] = fmaf(a, h[s], lane_of_row<I>(in) * bt[I]);
        if (!STATES_ONLY) y[I] = s ? fmaf(ct[I], h[s], y[I]) : ct[I] * h[s];
      });
    }
    if (!STATES_ONLY) {
      wave_fence();
#pragma unroll
      for (int i = 0; i < kTile; ++i) sums[wave][i * kSumPitch + lane] = y[i];
      wave_fence();
      float v = row_sum(sums[wave], lane) + skip * k.x;
      if (c.gate.p) v *= gate * sigmoid(gate);
      if (mine && t < c.T) *at<T>(c.y, p.b, t, d) = from_float<T>(live ? v : 0.f);
    }
  }
  if (!mine) return;
  if (STATES_ONLY) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (s * 16 + p.j < c.N) segs.h[seg_state + s * 16 + p.j] = h[s];
#pragma unroll
    for (int k = 1; k < 16; k *= 2) total += __shfl_xor(total, k);
    if (p.j == 0) segs.sum[(p.b * segs.n + p.seg) * c.D + d] = total;
  } else if (p.seg == segs.n - 1 && c.s_out && slot >= 0) {
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (s * 16 + p.j < c.N) c.s_out[(slot * c.D + d) * c.N + s * 16 + p.j] = h[s];
  }
}

// The prefix sum over the segments, in place: afterwards h holds the states that the segments begin with.  rev: from the last one,
// for the gradients of the states that the segments end with.
__global__ __launch_bounds__(256) void segments_kernel(ScanCall c, Segments segs, const float* start, bool rev) {
  const int64_t per = (int64_t)c.D * c.N, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= c.B * per) return;
  const int64_t b = i / per, dn = i % per, d = dn / c.N, slot = rev ? b : scan_slot(c, b);
  const float A = c.A[dn] * kLog2e;
  float h = start && slot >= 0 ? start[slot * per + dn] : 0.f;
  for (int k = 0; k < segs.n; ++k) {
    const int64_t seg = b * segs.n + (rev ? segs.n - 1 - k : k);
    float* at = segs.h + seg * per + dn;
    const float own = *at;
    *at = h;
    h = fmaf(exp2_of(A * segs.sum[seg * c.D + d]), h, own);
  }
}

// One token, states in place.  V adjacent states a lane, L lanes a channel (all states at once: V L >= N).
template <typename T, int V, int L>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanCall c) {
  typedef float fv __attribute__((ext_vector_type(V)));
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t d = i / L % c.D, b = i / L / c.D;
  const int n = (int)(i % L) * V;
  const bool live = b < c.B;
  const int64_t slot = live ? scan_slot(c, b) : -1;
  float y = 0.f, x = 0.f;
  if (slot >= 0) {
    const int g = (int)(d / c.E);
    const Token k = token_of<T>(c, true, at<T>(c.x, b, 0, d), at<T>(c.dt, b, 0, d), c.dt_bias ? c.dt_bias[d] : 0.f);
    x = k.x;
    if (n < c.N) {
      float* state = c.s_out + (slot * c.D + d) * c.N + n;
      fv h = *(const fv*)state;
      const fv A = *(const fv*)(c.A + d * c.N + n);
      const T *pb = at<T>(c.b, b, 0, g, n), *pc = at<T>(c.c, b, 0, g, n);
#pragma unroll
      for (int s = 0; s < V; ++s) {
        h[s] = fmaf(exp2_of(k.delta * (A[s] * kLog2e)), h[s], k.delta * k.x * to_float(pb[s]));
        y = fmaf(to_float(pc[s]), h[s], y);
      }
      *(fv*)state = h;
    }
  }
#pragma unroll
  for (int k = 1; k < L; k *= 2) y += __shfl_xor(y, k);
  if (!live || i % L) return;
  if (slot >= 0) {
    if (c.skip) y = fmaf(c.skip[d], x, y);
    if (c.gate.p) {
      const float gate = to_float(*at<T>(c.gate, b, 0, d));
      y *= gate * sigmoid(gate);
    }
  }
  *at<T>(c.y, b, 0, d) = from_float<T>(y);
}

int states_of(const ScanCall& c) { return c.N <= 16 ? 1 : c.N <= 32 ? 2 : 4; }
int blocks_of(const ScanCall& c) { return (int)cdiv(c.E, kChannels); }

// Segments: as many as give the chip two wavefronts a SIMD, of 4 tiles at least
int segments(const ScanCall& c, int64_t* tiles_of_one) {
  const int64_t tiles = cdiv(c.T, kTile), groups = c.B * c.G * blocks_of(c);
  int64_t n = groups ? 512 / groups : 1;
  n = n < 1 ? 1 : n;
  const int64_t most = cdiv(tiles, 4);
  if (n > most) n = most > 0 ? most : 1;
  *tiles_of_one = tiles > 0 ? cdiv(tiles, n) : 1;
  return tiles > 0 ? (int)cdiv(tiles, *tiles_of_one) : 1;
}

template <typename T, int NS>
mdh_status pass(const ScanCall& c, const Segments& segs, hipStream_t st) {
  const int blocks = blocks_of(c);
  const int64_t grid = c.B * segs.n * c.G * blocks;
  if (grid >= 1 << 24) return MDH_ERR_SIZE;
  clear_stale_error();
  if (segs.n > 1) {
    scan_kernel<T, NS, true><<<(unsigned)grid, kThreads, 0, st>>>(c, segs, blocks);
    mdh_status r = launch_status();
    if (r != MDH_OK) return r;
    r = launch_scan_segments(c, segs.h, segs.sum, segs.n, c.s_in, false, st);
    if (r != MDH_OK) return r;
  }
  scan_kernel<T, NS, false><<<(unsigned)grid, kThreads, 0, st>>>(c, segs, blocks);
  return launch_status();
}
template <typename T>
mdh_status pass_of(const ScanCall& c, const Segments& segs, hipStream_t st) {
  switch (states_of(c)) {
    case 1: return pass<T, 1>(c, segs, st);
    case 2: return pass<T, 2>(c, segs, st);
    default: return pass<T, 4>(c, segs, st);
  }
}

template <typename T, int V, int L>
void step(const ScanCall& c, hipStream_t st) {
  scan_step_kernel<T, V, L><<<(unsigned)cdiv(c.B * c.D * L, 256), 256, 0, st>>>(c);
}
template <typename T>
mdh_status step_of(const ScanCall& c, hipStream_t st) {
  const bool vec = c.N % 4 == 0 && ((uintptr_t)c.s_out | (uintptr_t)c.A) % 16 == 0;
  const int V = vec ? 4 : 1, lanes = (int)cdiv(c.N, V);
  if (c.B * c.D >= (int64_t)1 << 25) return MDH_ERR_SIZE;  // (64 lanes a channel at the most)
  clear_stale_error();
  if (vec) {
    if (lanes <= 1) step<T, 4, 1>(c, st);
    else if (lanes <= 4) step<T, 4, 4>(c, st);
    else step<T, 4, 16>(c, st);
  } else {
    if (lanes <= 4) step<T, 1, 4>(c, st);
    else if (lanes <= 16) step<T, 1, 16>(c, st);
    else step<T, 1, 64>(c, st);
  }
  return launch_status();
}

}  // namespace

mdh_status launch_scan_segments(const ScanCall& c, float* h, float* sum, int n, const float* start, bool rev, hipStream_t st) {
  const int64_t blocks = cdiv(c.B * c.D * c.N, 256);
  if (blocks >= 1 << 24) return MDH_ERR_SIZE;
  clear_stale_error();
  segments_kernel<<<(unsigned)blocks, 256, 0, st>>>(c, Segments{h, sum, n, 0}, start, rev);
  return launch_status();
}

size_t scan_workspace(const ScanCall& c) {
  int64_t tiles;
  const int n = segments(c, &tiles);
  return n > 1 ? (size_t)(c.B * n) * (size_t)c.D * (size_t)(c.N + 1) * sizeof(float) : 0;
}
mdh_status launch_scan_forward(const ScanCall& c, hipStream_t st) {
  Segments segs{};
  segs.n = segments(c, &segs.tiles);
  segs.h = (float*)c.ws;
  segs.sum = segs.h + c.B * segs.n * (int64_t)c.D * c.N;
  return c.dtype == MDH_BF16 ? pass_of<bf16>(c, segs, st) : pass_of<float>(c, segs, st);
}
mdh_status launch_scan_step(const ScanCall& c, hipStream_t st) { return c.dtype == MDH_BF16 ? step_of<bf16>(c, st) : step_of<float>(c, st); }

}  // namespace mdh

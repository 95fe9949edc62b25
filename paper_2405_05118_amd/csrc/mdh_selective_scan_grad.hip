// Gradients of the selective scan.  With d_p = d_y silu(gate) (p: the sum before the gate), E_T the gradient of the final state,
//   G_t = E_t + d_p c_t,  E_{t-1} = a_t G_t;   d_c = sum_d d_p h_t,  d_b = sum_d G_t delta x,  r = sum_n G_t b_t,  q = G_t a_t h_{t-1}
//   d_x = delta r + skip d_p,  d_delta = sum_n q A + x r,  d_A = sum_t q delta,  d_skip = sum d_p x,  d_gate = d_y p silu'(gate)
// from the last token to the first.  The states h come from the forward call's checkpoints, one for every tile of 16 tokens:
// a tile's a_t and h_t are computed again and stay in registers while it is walked back.
//
// 1 exponential and 15 multiplications a step: bound by the vector ALU.  De-composition as in the forward pass (a row of 16 lanes is a
// channel, a lane a state); a workgroup has 64 channels, a row two of them one after the other.  Sums over the states (p, r,
// sum q A) go through LDS, token j's to lane j.  Sums over the channels (d_b, d_c): a lane adds up its channels in registers, the
// workgroup its rows in LDS at the end of a tile, a second launch the workgroups, in order.  Sums over tokens (d_A, d_skip, d_dt_bias)
// stay in registers to the end of the segment.
#include "mdh_selective.h"

namespace mdh {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64, kRows = kThreads / 16, kTimes = 2, kChannels = kRows * kTimes;

struct Parts {
  float *e, *sum;     // gradients of the states that the segments end with; sums of deltas of the segments
  float *shared;      // d_b, then d_c: (block, b, t, g, n)
  float *params;      // (b, seg): d_A, d_skip, d_dt_bias
  int n;
  int64_t tiles;
};

__device__ __forceinline__ float gate_of(float g) { return g * sigmoid(g); }

// what a segment hands to the one before it, from zeros behind it
constexpr int kSegThreads = 256;
template <typename T, int NS>
__global__ __launch_bounds__(kSegThreads) void grad_segments_kernel(ScanCall c, Parts w, int blocks) {
  constexpr int S = NS * 16;
  __shared__ float cs[S * kPitch];
  const ScanPlace p = scan_place(c, blocks, w.n, w.tiles);
  const int e0 = p.block * (kSegThreads / 16) + p.row;
  const bool mine = e0 < c.E;
  const int64_t d = (int64_t)p.g * c.E + e0;
  float A[NS], e[NS], total = 0.f;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    A[s] = mine && s * 16 + p.j < c.N ? c.A[d * c.N + s * 16 + p.j] * kLog2e : 0.f;
    e[s] = 0.f;
  }
  const float dt_bias = mine && c.dt_bias ? c.dt_bias[d] : 0.f;
  for (int64_t tile = p.last - 1; tile >= p.first; --tile) {
    const int64_t t0 = tile * kTile, t = t0 + p.j;
    if (t0 >= p.len) continue;
    const bool live = mine && t < p.len;
    const Token k = token_of<T>(c, live, at<T>(c.x, p.b, t, d), at<T>(c.dt, p.b, t, d), dt_bias);
    float dp = live ? to_float(*at<T>(c.y, p.b, t, d)) : 0.f;
    if (c.gate.p && live) dp *= gate_of(to_float(*at<T>(c.gate, p.b, t, d)));
    total += k.delta;
    __syncthreads();
    stage_shared<T, S, kSegThreads>(c, c.c, p, t0, cs);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float ct[kTile];
      tile_of(cs, s * 16 + p.j, ct);
      unroll<kTile>([&](auto i) {
        constexpr int I = kTile - 1 - decltype(i)::value;
        e[s] = exp2_of(lane_of_row<I>(k.delta) * A[s]) * fmaf(lane_of_row<I>(dp), ct[I], e[s]);
      });
    }
  }
  if (!mine) return;
  const int64_t seg = p.b * w.n + p.seg;
#pragma unroll
  for (int s = 0; s < NS; ++s)
    if (s * 16 + p.j < c.N) w.e[(seg * c.D + d) * c.N + s * 16 + p.j] = e[s];
#pragma unroll
  for (int k = 1; k < 16; k *= 2) total += __shfl_xor(total, k);
  if (p.j == 0) w.sum[seg * c.D + d] = total;
}

template <typename T, int NS>
__global__ __launch_bounds__(kThreads) void scan_backward_kernel(ScanCall c, Parts w, int blocks) {
  constexpr int S = NS * 16;
  __shared__ float bs[S * kPitch], cs[S * kPitch], sums[kWaves][kSumFloats];
  const ScanPlace p = scan_place(c, blocks, w.n, w.tiles);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t seg = p.b * w.n + p.seg;
  int64_t d[kTimes];
  bool mine[kTimes];
  float A[kTimes][NS], e[kTimes][NS], dA[kTimes][NS], skip[kTimes], dt_bias[kTimes], d_skip[kTimes], d_bias[kTimes];
#pragma unroll
  for (int m = 0; m < kTimes; ++m) {
    const int ch = p.block * kChannels + m * kRows + p.row;
    mine[m] = ch < c.E;
    d[m] = (int64_t)p.g * c.E + ch;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int n = s * 16 + p.j;
      const bool has = mine[m] && n < c.N;
      A[m][s] = has ? c.A[d[m] * c.N + n] * kLog2e : 0.f;
      e[m][s] = dA[m][s] = 0.f;
      if (has && w.n > 1)
        e[m][s] = w.e[(seg * c.D + d[m]) * c.N + n];
      else if (has && c.s_in)
        e[m][s] = c.s_in[(p.b * c.D + d[m]) * c.N + n];
    }
    skip[m] = mine[m] && c.skip ? c.skip[d[m]] : 0.f;
    dt_bias[m] = mine[m] && c.dt_bias ? c.dt_bias[d[m]] : 0.f;
    d_skip[m] = d_bias[m] = 0.f;
  }
  for (int64_t tile = p.last - 1; tile >= p.first; --tile) {
    const int64_t t0 = tile * kTile, t = t0 + p.j;
    if (t0 >= p.len) {
#pragma unroll
      for (int m = 0; m < kTimes; ++m)
        if (mine[m] && t < c.T) {
          *at<T>(c.dx, p.b, t, d[m]) = from_float<T>(0.f);
          *at<T>(c.ddt, p.b, t, d[m]) = from_float<T>(0.f);
          if (c.dgate.p) *at<T>(c.dgate, p.b, t, d[m]) = from_float<T>(0.f);
        }
      continue;
    }
    Token k[kTimes];
    float gate[kTimes], dy[kTimes], dp[kTimes], sp[kTimes], sr[kTimes], sq[kTimes];
#pragma unroll
    for (int m = 0; m < kTimes; ++m) {
      const bool live = mine[m] && t < p.len;
      k[m] = token_of<T>(c, live, at<T>(c.x, p.b, t, d[m]), at<T>(c.dt, p.b, t, d[m]), dt_bias[m]);
      dp[m] = dy[m] = live ? to_float(*at<T>(c.y, p.b, t, d[m])) : 0.f;
      gate[m] = 0.f;
      if (c.gate.p && live) {
        gate[m] = to_float(*at<T>(c.gate, p.b, t, d[m]));
        dp[m] *= gate_of(gate[m]);
      }
      sp[m] = sr[m] = sq[m] = 0.f;
    }
    __syncthreads();
    stage_shared<T, S, kThreads>(c, c.b, p, t0, bs);
    stage_shared<T, S, kThreads>(c, c.c, p, t0, cs);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float bt[kTile], ct[kTile], db[kTile], dc[kTile];
      tile_of(bs, s * 16 + p.j, bt);
      tile_of(cs, s * 16 + p.j, ct);
#pragma unroll
      for (int i = 0; i < kTile; ++i) db[i] = dc[i] = 0.f;
#pragma unroll
      for (int m = 0; m < kTimes; ++m) {
        const float in = k[m].delta * k[m].x;
        float h[kTile + 1], a[kTile];
        h[0] = mine[m] && s * 16 + p.j < c.N ? c.checkpoints[((p.b * c.tiles + tile) * c.D + d[m]) * c.N + s * 16 + p.j] : 0.f;
        wave_fence();
        unroll<kTile>([&](auto i) {
          constexpr int I = decltype(i)::value;
          a[I] = exp2_of(lane_of_row<I>(k[m].delta) * A[m][s]);
          h[I + 1] = fmaf(a[I], h[I], lane_of_row<I>(in) * bt[I]);
          sums[wave][I * kSumPitch + lane] = ct[I] * h[I + 1];
        });
        wave_fence();
        sp[m] += row_sum(sums[wave], lane);
        wave_fence();
        float q[kTile];
        unroll<kTile>([&](auto i) {
          constexpr int I = kTile - 1 - decltype(i)::value;
          const float g = fmaf(lane_of_row<I>(dp[m]), ct[I], e[m][s]);
          dc[I] = fmaf(lane_of_row<I>(dp[m]), h[I + 1], dc[I]);
          db[I] = fmaf(lane_of_row<I>(in), g, db[I]);
          sums[wave][I * kSumPitch + lane] = g * bt[I];
          e[m][s] = a[I] * g;
          const float gh = e[m][s] * h[I];
          dA[m][s] = fmaf(lane_of_row<I>(k[m].delta), gh, dA[m][s]);
          q[I] = gh * A[m][s];
        });
        wave_fence();
        sr[m] += row_sum(sums[wave], lane);
        wave_fence();
#pragma unroll
        for (int i = 0; i < kTile; ++i) sums[wave][i * kSumPitch + lane] = q[i];
        wave_fence();
        sq[m] += row_sum(sums[wave], lane);
      }
      // over the rows of the workgroup
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        wave_fence();
#pragma unroll
        for (int i = 0; i < kTile; ++i) sums[wave][i * kSumPitch + lane] = which ? dc[i] : db[i];
        __syncthreads();
        const int i = threadIdx.x / 16, n = s * 16 + p.j;
        if (threadIdx.x < 256) {
          float v = 0.f;
#pragma unroll
          for (int x = 0; x < kWaves; ++x)
#pragma unroll
            for (int r = 0; r < 4; ++r) v += sums[x][i * kSumPitch + r * 16 + p.j];
          if (n < c.N && t0 + i < p.len)
            w.shared[(((which * (int64_t)blocks + p.block) * c.B + p.b) * c.T + t0 + i) * c.G * c.N + (int64_t)p.g * c.N + n] = v;
        }
        __syncthreads();
      }
    }
#pragma unroll
    for (int m = 0; m < kTimes; ++m) {
      if (!mine[m] || t >= c.T) continue;
      const bool live = t < p.len;
      const float d_delta = fmaf(k[m].x, sr[m], sq[m] * kLn2);
      const float d_dt = c.softplus ? d_delta * sigmoid(k[m].raw) : d_delta;
      d_skip[m] = fmaf(dp[m], k[m].x, d_skip[m]);
      if (live) d_bias[m] += d_dt;
      *at<T>(c.dx, p.b, t, d[m]) = from_float<T>(live ? fmaf(k[m].delta, sr[m], skip[m] * dp[m]) : 0.f);
      *at<T>(c.ddt, p.b, t, d[m]) = from_float<T>(live ? d_dt : 0.f);
      if (c.dgate.p) {
        const float f = sigmoid(gate[m]);
        *at<T>(c.dgate, p.b, t, d[m]) =
            from_float<T>(live ? dy[m] * fmaf(skip[m], k[m].x, sp[m]) * f * (1.f + gate[m] * (1.f - f)) : 0.f);
      }
    }
  }
  float* row = w.params + seg * c.D * (c.N + 2);
#pragma unroll
  for (int m = 0; m < kTimes; ++m) {
#pragma unroll
    for (int k = 1; k < 16; k *= 2) d_skip[m] += __shfl_xor(d_skip[m], k), d_bias[m] += __shfl_xor(d_bias[m], k);
    if (!mine[m]) continue;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const int n = s * 16 + p.j;
      if (n >= c.N) continue;
      row[d[m] * c.N + n] = dA[m][s];
      if (p.seg == 0 && c.s_out) c.s_out[(p.b * c.D + d[m]) * c.N + n] = e[m][s];
    }
    if (p.j == 0) row[(int64_t)c.D * c.N + d[m]] = d_skip[m], row[(int64_t)c.D * (c.N + 1) + d[m]] = d_bias[m];
  }
}

// d_b and d_c: the blocks of channels of each group, in order
template <typename T>
__global__ __launch_bounds__(256) void shared_sums_kernel(ScanCall c, const float* part, int blocks) {
  const int64_t per = c.B * c.T * c.G * c.N, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= per) return;
  const int n = (int)(i % c.N), g = (int)(i / c.N % c.G);
  const int64_t t = i / c.N / c.G % c.T, b = i / c.N / c.G / c.T;
  const bool live = t < scan_length(c, b);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float* p = part + which * (int64_t)blocks * per + i;
    float v = 0.f;
    if (live)
      for (int k = 0; k < blocks; ++k) v += p[k * per];
    *at<T>(which ? c.dc : c.db, b, t, g, n) = from_float<T>(v);
  }
}

int states_of(const ScanCall& c) { return c.N <= 16 ? 1 : c.N <= 32 ? 2 : 4; }
int blocks_of(const ScanCall& c) { return (int)cdiv(c.E, kChannels); }

// Segments: as many as give the chip two wavefronts a SIMD, of 4 tiles at least
int segments(const ScanCall& c, int64_t* tiles_of_one) {
  const int64_t tiles = cdiv(c.T, kTile), groups = c.B * c.G * blocks_of(c);
  int64_t n = groups ? 256 / groups : 1;
  n = n < 1 ? 1 : n;
  const int64_t most = cdiv(tiles, 4);
  if (n > most) n = most > 0 ? most : 1;
  *tiles_of_one = tiles > 0 ? cdiv(tiles, n) : 1;
  return tiles > 0 ? (int)cdiv(tiles, *tiles_of_one) : 1;
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
// bytes of: states and sums of the segments, d_b and d_c of the blocks, parameters' rows
size_t seg_bytes(const ScanCall& c, int n) { return n > 1 ? up16((size_t)c.B * n * c.D * (c.N + 1) * sizeof(float)) : 0; }
size_t shared_bytes(const ScanCall& c) { return up16((size_t)2 * blocks_of(c) * c.B * c.T * c.G * c.N * sizeof(float)); }
size_t param_bytes(const ScanCall& c, int n) { return (size_t)c.B * n * c.D * (c.N + 2) * sizeof(float); }

template <typename T, int NS>
mdh_status pass(const ScanCall& c, const Parts& w, hipStream_t st) {
  const int blocks = blocks_of(c), seg_blocks = (int)cdiv(c.E, kSegThreads / 16);
  const int64_t grid = c.B * w.n * c.G * blocks, seg_grid = c.B * w.n * c.G * seg_blocks, outs = cdiv(c.B * c.T * c.G * c.N, 256);
  if (grid >= 1 << 23 || (w.n > 1 && seg_grid >= 1 << 24) || outs >= 1 << 24) return MDH_ERR_SIZE;
  clear_stale_error();
  if (w.n > 1) {
    grad_segments_kernel<T, NS><<<(unsigned)seg_grid, kSegThreads, 0, st>>>(c, w, seg_blocks);
    mdh_status r = launch_status();
    if (r != MDH_OK) return r;
    r = launch_scan_segments(c, w.e, w.sum, w.n, c.s_in, true, st);
    if (r != MDH_OK) return r;
  }
  scan_backward_kernel<T, NS><<<(unsigned)grid, kThreads, 0, st>>>(c, w, blocks);
  mdh_status r = launch_status();
  if (r != MDH_OK || outs == 0) return r;
  shared_sums_kernel<T><<<(unsigned)outs, 256, 0, st>>>(c, w.shared, blocks);
  return launch_status();
}
template <typename T>
mdh_status pass_of(const ScanCall& c, const Parts& w, hipStream_t st) {
  switch (states_of(c)) {
    case 1: return pass<T, 1>(c, w, st);
    case 2: return pass<T, 2>(c, w, st);
    default: return pass<T, 4>(c, w, st);
  }
}

}  // namespace

size_t scan_backward_workspace(const ScanCall& c) {
  if (c.B == 0) return 0;
  int64_t tiles;
  const int n = segments(c, &tiles);
  return seg_bytes(c, n) + shared_bytes(c) + param_bytes(c, n);
}
mdh_status launch_scan_backward(const ScanCall& c, hipStream_t st) {
  Parts w{};
  w.n = segments(c, &w.tiles);
  int64_t rows = 0;
  if (c.B) {
    w.e = (float*)c.ws, w.sum = w.e + c.B * w.n * (int64_t)c.D * c.N;
    w.shared = (float*)((char*)c.ws + seg_bytes(c, w.n));
    w.params = (float*)((char*)w.shared + shared_bytes(c));
    rows = c.B * w.n;
    const mdh_status r = c.dtype == MDH_BF16 ? pass_of<bf16>(c, w, st) : pass_of<float>(c, w, st);
    if (r != MDH_OK) return r;
  }
  const int64_t states = (int64_t)c.D * c.N;
  return launch_sum_rows(w.params, rows, states + 2 * (int64_t)c.D, {{c.dA, states}, {c.dskip, c.D}, {c.ddt_bias, c.D}}, st);
}

}  // namespace mdh

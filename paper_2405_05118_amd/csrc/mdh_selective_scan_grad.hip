// Gradients of the selective scan.  With d_p = d_y silu(gate) (p: the sum before the gate), E_T the gradient of the final state,
//   G_t = E_t + d_p c_t,  E_{t-1} = a_t G_t;   d_c = sum_d d_p h_t,  d_b = sum_d G_t delta x,  r = sum_n G_t b_t,  q = G_t a_t h_{t-1}
//   d_x = delta r + skip d_p,  d_delta = sum_n q A + x r,  d_A = sum_t q delta,  d_skip = sum d_p x,  d_gate = d_y p silu'(gate)
// from the last token to the first.  The states h come from the forward call's checkpoints, one for every tile of 16 tokens:
// a tile's a_t and h_t are computed again and stay in registers while it is walked back; E goes over a block
// of 32 tokens by the block's own factor.
//
// 1 exponential and 16 multiplications a step: bound by the vector ALU (28 of its instructions a step, sums and staging with them).
// 4 x 2048 tokens of 4096 channels with 16 states, bf16: 546 us, 557 to 586 in a kernel trace, 26 for the sums of d_b and d_c.
// De-composition as in the forward pass (a row of 16 lanes is a channel, a lane a state); a workgroup has 32 channels.  Sums over the
// states (p, r, sum q A) go through LDS, token j's to lane j.  Sums over the channels (d_b, d_c): rows of the wavefront exchange halves, then
// LDS over the workgroup's wavefronts, in two places by turns: one barrier a tile (with all five sums through LDS and two barriers 721
// us where this took 646); a second launch adds up the workgroups, in order.  Sums over tokens (d_A, d_skip, d_dt_bias)
// stay in registers to the end of the segment.
#include "mdh_selective.h"

namespace mdh {
namespace {

constexpr int kThreads = 256, kRows = kThreads / 16;  // of the kernel over segments

struct Parts {
  float *e, *sum;     // gradients of the states that the segments end with; sums of deltas of the segments
  float *shared;      // d_b, then d_c: (block, b, t, g, n)
  float *params;      // (b, seg): d_A, d_skip, d_dt_bias
  int n;
  int64_t tokens;  // of a segment
};

__device__ __forceinline__ float gate_of(float g) { return g * sigmoid(g); }
// the last block of tokens that has a valid one
__device__ __forceinline__ int64_t last_block(const ScanPlace& p, int block) {
  return p.alive > p.first ? p.first + (p.alive - p.first - 1) / block * block : p.first - block;
}

constexpr int kTokens = 32;  // of a block

// what a segment hands to the one before it, from zeros behind it
template <typename T, int NS>
__global__ __launch_bounds__(kThreads) void grad_segments_kernel(ScanCall c, Parts w, int blocks) {
  constexpr int S = NS * 16;
  typedef Stage<T, 3, 1, kRows, S, kTokens, kThreads> In;
  __shared__ T raw[3 * kTokens * kRows] __attribute__((aligned(16)));
  __shared__ float cs[In::kFloats] __attribute__((aligned(16)));
  T *const dts = raw, *const gates = raw + kTokens * kRows, *const dys = raw + 2 * kTokens * kRows;
  const ScanPlace p = scan_place(c, blocks, w.n, w.tokens);
  const int e0 = p.block * kRows, width = min(kRows, c.E - e0);
  const bool mine = p.row < width;
  const int64_t d0 = (int64_t)p.g * c.E + e0, d = d0 + p.row;
  In in;
  int64_t t0 = last_block(p, kTokens);
  in.begin(c.in + 1, c.bc + 1, p, t0, -1, d0, width, c.N);
  if (t0 >= p.first) in.load(p.alive - t0);
  float A[NS], e[NS], total = 0.f;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    A[s] = mine && s * 16 + p.j < c.N ? in_powers_of_2(c.A[d * c.N + s * 16 + p.j]) : 0.f;
    e[s] = 0.f;
  }
  const float dt_bias = mine && c.dt_bias ? c.dt_bias[d] : 0.f;
  for (; t0 >= p.first; t0 -= kTokens) {
    in.stage(raw, cs);
    __syncthreads();
    if (t0 > p.first) in.load(kTokens);
    const int tokens = (int)min((int64_t)kTokens, p.alive - t0);
    for (int i0 = (tokens - 1) / kTile * kTile; i0 >= 0; i0 -= kTile) {
      const int at = place_of<T, kRows>(i0 + p.j, p.row);
      const Token k = token_of(c, 0.f, to_float(dts[at]), i0 + p.j < tokens, dt_bias);
      float dp = to_float(dys[at]);
      if (c.in[2].p) dp *= gate_of(to_float(gates[at]));
      total += k.delta;
      const float sum = sum_of_row(k.delta);
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        float own = 0.f;
        unroll<kTile / 4>([&](auto quarter) {
          constexpr int Q = kTile - 4 - decltype(quarter)::value * 4;
          const Float4 ct = four_of(cs + (s * 16 + p.j) * In::kPitch + i0 + Q);
          unroll<4>([&](auto i) {
            constexpr int I = 3 - decltype(i)::value;
            own = exp2_of(lane_of_row<Q + I>(k.delta) * A[s]) * fmaf(lane_of_row<Q + I>(dp), ct[I], own);
          });
        });
        e[s] = fmaf(factor_of(sum, A[s]), e[s], own);
      }
    }
    __syncthreads();
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

// A lane owns one channel's state of every 16; WAVES wavefronts are CH = 4 WAVES channels.
template <typename T, int NS, int WAVES>
__global__ __launch_bounds__(64 * WAVES, NS == 1 && sizeof(T) == 2 ? 4 : 2) void scan_backward_kernel(ScanCall c, Parts w, int blocks) {
  constexpr int S = NS * 16, CH = 4 * WAVES, THREADS = 64 * WAVES, TILES = kTokens / kTile;
  typedef Stage<T, 4, 2, CH, S, kTokens, THREADS> In;
  typedef Outputs<T, 3, CH, kTokens, THREADS> Out;
  __shared__ T raw[4 * kTokens * CH] __attribute__((aligned(16)));
  __shared__ float bc[2 * In::kFloats] __attribute__((aligned(16))), sums[WAVES][kSumFloats] __attribute__((aligned(16))), meet[2][WAVES][512];
  T *const xs = raw, *const dts = raw + kTokens * CH, *const gates = raw + 2 * kTokens * CH, *const dys = raw + 3 * kTokens * CH;
  const ScanPlace p = scan_place(c, blocks, w.n, w.tokens);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t seg = p.b * w.n + p.seg;
  const int e0 = p.block * CH, width = min(CH, c.E - e0);
  const bool mine = p.row < width;
  const int64_t d0 = (int64_t)p.g * c.E + e0, d = d0 + p.row;
  In in;
  int64_t t0 = last_block(p, kTokens);
  in.begin(c.in, c.bc, p, t0, -1, d0, width, c.N);
  float A[NS], e[NS], dA[NS], next_h[TILES][NS], d_skip = 0.f, d_bias = 0.f;
  const int64_t all_states = (int64_t)c.D * c.N, state_at = d * c.N + p.j;
  auto load = [&](int64_t from) {
    in.load(p.alive - from);
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        next_h[i][s] = 0.f;
        if (mine && s * 16 + p.j < c.N && from + i * kTile < p.alive)
          next_h[i][s] = (c.checkpoints + (p.b * c.tiles + from / kTile + i) * all_states + s * 16)[state_at];
      }
  };
  if (t0 >= p.first) load(t0);
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int n = s * 16 + p.j;
    const bool has = mine && n < c.N;
    A[s] = has ? in_powers_of_2(c.A[d * c.N + n]) : 0.f;
    e[s] = dA[s] = 0.f;
    if (has && w.n > 1)
      e[s] = w.e[(seg * c.D + d) * c.N + n];
    else if (has && c.s_in)
      e[s] = c.s_in[(p.b * c.D + d) * c.N + n];
  }
  const float skip = mine && c.skip ? c.skip[d] : 0.f, dt_bias = mine && c.dt_bias ? c.dt_bias[d] : 0.f;
  for (int i = 0; i < 3; ++i)
    if (c.out[i].p) store_zeros<T, CH, THREADS>(c.out[i], p, d0, width, kTokens);
  Out out;
  out.begin(c.out, p, t0, -1, d0, width);
  // of the 512 sums of a tile (d_b and d_c of 16 tokens and 16 states) a thread adds up its own over the wavefronts
  static_assert(THREADS == 512, "a thread's sum of d_b or d_c");
  const int shared_t = (int)threadIdx.x / 16 % 4 * 4 + (int)threadIdx.x / 64 % 4, shared_n = p.j, per_token = c.G * c.N;
  // (B T G N < 2^31: of a token that there is, less than that)
  const unsigned shared_at = (unsigned)shared_t * (unsigned)per_token + (unsigned)shared_n;
  const int which = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 256);
  float* const shared_to = w.shared + ((which * (int64_t)blocks + p.block) * c.B + p.b) * c.T * per_token + (int64_t)p.g * c.N;
  int turn = 0;
  bool behind = false;  // a block's gradients lie in LDS
  for (; t0 >= p.first; t0 -= kTokens) {
    if (behind) out.take(raw);
    in.stage(raw, bc);
    float h0[TILES][NS];
#pragma unroll
    for (int i = 0; i < TILES; ++i)
#pragma unroll
      for (int s = 0; s < NS; ++s) h0[i][s] = next_h[i][s];
    __syncthreads();
    // (stores go out behind the wait for the block's loads: what is waited for next has been under way for long)
    if (behind) out.store(p.last - t0 - kTokens);
    behind = true;
    if (t0 > p.first) load(t0 - kTokens);
    const int tokens = (int)min((int64_t)kTokens, p.alive - t0);
    // of the block: what it is walked back from, the product of its factors, a lane's share of its deltas
    float behind_it[NS], all[NS], deltas = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) behind_it[s] = e[s], all[s] = 1.f;
#pragma unroll
    for (int tile = TILES - 1; tile >= 0; --tile) {
      const int i0 = tile * kTile;
      if (i0 >= tokens) continue;
      const bool live = i0 + p.j < tokens;
      const int at = place_of<T, CH>(i0 + p.j, p.row);
      const Token k = token_of(c, to_float(xs[at]), to_float(dts[at]), live, dt_bias);
      const float dy = to_float(dys[at]), dp = c.in[2].p ? dy * gate_of(to_float(gates[at])) : dy, u = k.delta * k.x;
      deltas += k.delta;
      float sp = 0.f, sr = 0.f, sq = 0.f;
      float* own = sums[wave];
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const float* bs = bc + (s * 16 + p.j) * In::kPitch + i0;
        float h[kTile + 1], a[kTile], g[kTile];
        h[0] = h0[tile][s];
        unroll<kTile / 4>([&](auto quarter) {
          constexpr int Q = decltype(quarter)::value * 4;
          const Float4 bt = four_of(bs + Q), ct = four_of(bs + In::kFloats + Q);
          unroll<4>([&](auto i) {
            constexpr int I = Q + decltype(i)::value;
            a[I] = exp2_of(lane_of_row<I>(k.delta) * A[s]);
            all[s] *= a[I];
            h[I + 1] = fmaf(a[I], h[I], lane_of_row<I>(u) * bt[I - Q]);
            own[I * kSumPitch + lane] = ct[I - Q] * h[I + 1];
          });
        });
        settle(all[s]);
        wave_fence();
        sp += row_sum(own, lane);
        settle(sp);
        wave_fence();
        const float dp2 = again(dp), delta2 = again(k.delta), u2 = again(u);
        float terms[kTile];
        unroll<kTile>([&](auto i) {
          constexpr int I = decltype(i)::value;
          terms[I] = lane_of_row<I>(dp) * h[I + 1];
        });
        Float4 dc = over_rows(terms);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float v = dc[i];
          settle(v);
          dc[i] = v;
        }
        unroll<kTile / 4>([&](auto quarter) {
          constexpr int Q = kTile - 4 - decltype(quarter)::value * 4;
          const Float4 bt = four_of(bs + Q), ct = four_of(bs + In::kFloats + Q);
          unroll<4>([&](auto i) {
            constexpr int I = Q + 3 - decltype(i)::value;
            g[I] = e[s];
            add_lane_of_row<I>(g[I], dp2, ct[I - Q]);
            own[I * kSumPitch + lane] = g[I] * bt[I - Q];
            e[s] = a[I] * g[I];
            a[I] = e[s] * h[I];  // (the factor is done with)
            add_lane_of_row<I>(dA[s], delta2, a[I]);
          });
        });
        wave_fence();
        sr += row_sum(own, lane);
        settle(sr), settle(dA[s]), settle(e[s]);
        wave_fence();
        unroll<kTile>([&](auto i) {
          constexpr int I = decltype(i)::value;
          g[I] *= lane_of_row<I>(u2);
        });
        const Float4 db = over_rows(g);
#pragma unroll
        for (int i = 0; i < kTile; ++i) own[i * kSumPitch + lane] = a[i] * A[s];
        wave_fence();
        sq += row_sum(own, lane);
        settle(sq);
        wave_fence();
        // over the wavefronts
#pragma unroll
        for (int i = 0; i < 4; ++i) meet[turn][wave][i * 64 + lane] = db[i], meet[turn][wave][256 + i * 64 + lane] = dc[i];
        __syncthreads();
        float sum = meet[turn][0][threadIdx.x];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += meet[turn][v][threadIdx.x];
        if (s * 16 + shared_n < c.N && i0 + shared_t < tokens) (shared_to + (t0 + i0) * per_token + s * 16)[shared_at] = sum;
        turn ^= 1;  // (whoever writes there again has been past another barrier)
      }
      const float d_delta = fmaf(k.x, sr, sq * kLn2), d_dt = c.softplus ? d_delta * sigmoid(k.raw) : d_delta;
      d_skip = fmaf(dp, k.x, d_skip);
      if (live) d_bias += d_dt;
      // gradients take the places of what they are the gradients of
      xs[at] = from_float<T>(live ? fmaf(k.delta, sr, skip * dp) : 0.f);
      dts[at] = from_float<T>(live ? d_dt : 0.f);
      if (c.out[2].p) {
        const float g = to_float(gates[at]), f = sigmoid(g);
        gates[at] = from_float<T>(live ? dy * fmaf(skip, k.x, sp) * f * (1.f + g * (1.f - f)) : 0.f);
      }
    }
    deltas = sum_of_row(deltas);
#pragma unroll
    for (int s = 0; s < NS; ++s) e[s] += put_right(factor_of(deltas, A[s]), all[s], behind_it[s]);
    __syncthreads();
  }
  if (behind) {
    out.take(raw);
    out.store(p.last - p.first);
  }
  float* row = w.params + seg * c.D * (c.N + 2);
#pragma unroll
  for (int k = 1; k < 16; k *= 2) d_skip += __shfl_xor(d_skip, k), d_bias += __shfl_xor(d_bias, k);
  if (!mine) return;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int n = s * 16 + p.j;
    if (n >= c.N) continue;
    row[d * c.N + n] = dA[s];
    if (p.seg == 0 && c.s_out) c.s_out[(p.b * c.D + d) * c.N + n] = e[s];
  }
  if (p.j == 0) row[(int64_t)c.D * c.N + d] = d_skip, row[(int64_t)c.D * (c.N + 1) + d] = d_bias;
}

// d_b and d_c: the blocks of channels of each group, in order.  blockIdx.y: which of the two
template <typename T>
__global__ __launch_bounds__(256) void shared_sums_kernel(ScanCall c, const float* part, int blocks) {
  const int64_t per = c.B * c.T * c.G * c.N, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= per) return;
  const int n = (int)(i % c.N), g = (int)(i / c.N % c.G);
  const int64_t t = i / c.N / c.G % c.T, b = i / c.N / c.G / c.T;
  const float* p = part + blockIdx.y * (int64_t)blocks * per + i;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (t < scan_length(c, b)) {
    int k = 0;
    for (; k + 3 < blocks; k += 4)
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] += p[(k + u) * per];
    for (; k < blocks; ++k) v[0] += p[k * per];
  }
  *at<T>(c.dbc[blockIdx.y], b, t, g, n) = from_float<T>((v[0] + v[1]) + (v[2] + v[3]));
}

// Wavefronts of a workgroup (the more, the fewer the rows of partial sums of d_b and d_c), and segments: of the tokens, as many as
// give the chip two wavefronts a SIMD, whole blocks of tokens.
struct Shape {
  int NS, waves, blocks, n;  // blocks of 4 * waves channels of a group, segments
  int64_t tokens;            // of a segment
};
Shape shape_of(const ScanCall& c) {
  Shape z;
  z.NS = c.N <= 16 ? 1 : c.N <= 32 ? 2 : 4;
  z.waves = 8;
  z.blocks = (int)cdiv(c.E, 4 * z.waves);
  const int block = kTokens;
  const int64_t in_all = cdiv(c.T, block), groups = c.B * c.G * z.blocks;
  int64_t n = groups ? 256 / groups : 1;
  if (n > in_all) n = in_all;
  if (n < 1) n = 1;
  const int64_t each = in_all ? cdiv(in_all, n) : 1;
  z.tokens = each * block;
  z.n = in_all ? (int)cdiv(in_all, each) : 1;
  return z;
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
// bytes of: states and sums of the segments, d_b and d_c of the blocks, parameters' rows
size_t seg_bytes(const ScanCall& c, const Shape& z) { return z.n > 1 ? up16((size_t)c.B * z.n * c.D * (c.N + 1) * sizeof(float)) : 0; }
size_t shared_bytes(const ScanCall& c, const Shape& z) { return up16((size_t)2 * z.blocks * c.B * c.T * c.G * c.N * sizeof(float)); }
size_t param_bytes(const ScanCall& c, const Shape& z) { return (size_t)c.B * z.n * c.D * (c.N + 2) * sizeof(float); }

template <typename T, int NS, int WAVES>
mdh_status pass(const ScanCall& c, const Shape& z, const Parts& w, hipStream_t st) {
  const int seg_blocks = (int)cdiv(c.E, kRows);
  const int64_t grid = c.B * z.n * c.G * z.blocks, seg_grid = c.B * z.n * c.G * seg_blocks, outs = cdiv(c.B * c.T * c.G * c.N, 256);
  if (grid * z.waves >= 1 << 26 || (z.n > 1 && seg_grid >= 1 << 24) || outs >= 1 << 23) return MDH_ERR_SIZE;  // 2^32 lanes
  clear_stale_error();
  if (z.n > 1) {
    grad_segments_kernel<T, NS><<<(unsigned)seg_grid, kThreads, 0, st>>>(c, w, seg_blocks);
    mdh_status r = launch_status();
    if (r != MDH_OK) return r;
    r = launch_scan_segments(c, w.e, w.sum, w.n, c.s_in, true, st);
    if (r != MDH_OK) return r;
  }
  scan_backward_kernel<T, NS, WAVES><<<(unsigned)grid, 64 * WAVES, 0, st>>>(c, w, z.blocks);
  const mdh_status r = launch_status();
  if (r != MDH_OK || outs == 0) return r;
  shared_sums_kernel<T><<<dim3((unsigned)outs, 2), 256, 0, st>>>(c, w.shared, z.blocks);
  return launch_status();
}
template <typename T>
mdh_status pass_of(const ScanCall& c, const Shape& z, const Parts& w, hipStream_t st) {
  switch (z.NS) {
    case 1: return pass<T, 1, 8>(c, z, w, st);
    case 2: return pass<T, 2, 8>(c, z, w, st);
    default: return pass<T, 4, 8>(c, z, w, st);
  }
}

}  // namespace

size_t scan_backward_workspace(const ScanCall& c) {
  const Shape z = shape_of(c);
  return c.B ? seg_bytes(c, z) + shared_bytes(c, z) + param_bytes(c, z) : 0;
}
mdh_status launch_scan_backward(const ScanCall& c, hipStream_t st) {
  const Shape z = shape_of(c);
  Parts w{};
  w.n = z.n, w.tokens = z.tokens;
  int64_t rows = 0;
  if (c.B) {
    w.e = (float*)c.ws, w.sum = w.e + c.B * w.n * (int64_t)c.D * c.N;
    w.shared = (float*)((char*)c.ws + seg_bytes(c, z));
    w.params = (float*)((char*)w.shared + shared_bytes(c, z));
    rows = c.B * w.n;
    const mdh_status r = c.dtype == MDH_BF16 ? pass_of<bf16>(c, z, w, st) : pass_of<float>(c, z, w, st);
    if (r != MDH_OK) return r;
  }
  const int64_t states = (int64_t)c.D * c.N;
  return launch_sum_rows(w.params, rows, states + 2 * (int64_t)c.D, {{c.dA, states}, {c.dskip, c.D}, {c.ddt_bias, c.D}}, st);
}

}  // namespace mdh

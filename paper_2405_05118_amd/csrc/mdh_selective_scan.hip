// The selective state space scan: h_t = e^(delta_t A) h_{t-1} + delta_t x_t b_t, y_t = (c_t . h_t + skip x_t) silu(gate_t), for every
// channel and its N states -- the prefix-sum operator on pairs (a, u): (a1, u1) op (a2, u2) = (a1 a2, a2 u1 + u2), whose a a token gives.
//
// 1 exponential and 4 multiplications a step (token, channel, state), on 8 bytes a token and channel (bf16, N = 16): bound by the
// vector ALU.  Measured on this chip, cycles of a wavefront instruction with four wavefronts a SIMD: v_exp_f32 8.4, fma and
// multiplication 2.6 to 3.2, with a lane of the row broadcast to it (DPP) 4.4; a step of all of them 24 to 27 (with two wavefronts 31,
// with one 57).  Times (bf16, N = 16): 2048 tokens of 4096 channels 81 us; 32768 tokens of 1536 channels 492 us.
//
// De-composition.  A row of 16 lanes is a channel, a lane one state of every 16; a wavefront has four channels, a workgroup 8 or 16.
// Tokens are walked in tiles of 16.  Lane j loads x, dt and gate of token j, takes the softplus, and a step's delta reaches the row's
// other lanes as a modifier of the multiplication.  c_t . h_t: every lane's term goes to LDS, lane j adds up token j's.
// b and c of a tile lie in LDS as fp32.  A state goes over a block of tokens by the block's own factor (mdh_selective.h): in turn that is
// another multiplication a step, the product of the factors that it went by (4 x 2048 tokens of 4096 channels 205 us, so 215; tile by
// tile 219).  With too few channels for the chip, tokens are cut into segments: what each leaves from
// a state of zeros and the sum of its deltas (its decay is e^(A sum)), a prefix sum over the segments, the pass itself.
#include "mdh_selective.h"

namespace mdh {
namespace {

// what the segments leave: h of (b, seg, d, n) and the sum of deltas of (b, seg, d)
struct Segments {
  float *h, *sum;
  int n;
  int64_t tokens;  // of one
};

// A workgroup has CH channels, and W tiles of tokens at once (W = 1: one after the other).  Tiles at once: every wavefront walks its own
// from a state of zeros, keeping h and the product of the factors for every token; the tiles' ends meet in LDS, and h + product *
// (state before the tile) is what the walk from there would give: 6 multiplications a step for which no token is walked twice.
template <int NS, int CH_, int W_, int TOKENS_>
struct Form {
  static constexpr int CH = CH_, W = W_, TOKENS = TOKENS_, THREADS = 16 * CH * W;
  static_assert(W == 1 || TOKENS == W * kTile, "a wavefront has one tile of a block");
};
template <int NS>
using InTurn = Form<NS, 16, 1, NS == 4 ? 32 : 64>;
template <int NS>
using AtOnce = Form<NS, 8, 4, 64>;
template <int NS>
using ManyAtOnce = Form<NS, 8, 8, 128>;

// STATES_ONLY: a segment's own state and sum of deltas.  Else the pass.
template <typename T, int NS, typename F, bool STATES_ONLY>
__global__ __launch_bounds__(F::THREADS, NS == 4 && sizeof(T) == 4 ? 3 : 1) void scan_kernel(ScanCall c, Segments segs, int blocks) {
  constexpr int S = NS * 16, CH = F::CH, W = F::W, TOKENS = F::TOKENS, NA = STATES_ONLY ? 2 : 3, NB = STATES_ONLY ? 1 : 2;
  typedef Stage<T, NA, NB, CH, S, TOKENS, F::THREADS> In;
  typedef Outputs<T, 1, CH, TOKENS, F::THREADS> Out;
  // two buffers where they do not cost a workgroup its place: the next block is staged while one is worked on, one barrier less
  constexpr int BUFFERS = W > 1 && NS == 1 ? 2 : 1, RAW = NA * TOKENS * CH, BC = NB * In::kFloats;
  __shared__ T raws[BUFFERS * RAW] __attribute__((aligned(16)));
  __shared__ float bcs[BUFFERS * BC] __attribute__((aligned(16)));
  __shared__ float sums[STATES_ONLY ? 1 : F::THREADS / 64][STATES_ONLY ? 4 : kSumFloats] __attribute__((aligned(16)));
  __shared__ float2 ends[W > 1 ? W : 1][W > 1 ? CH * S : 1];
  ScanPlace p = scan_place(c, blocks, segs.n, segs.tokens);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tile = W > 1 ? __builtin_amdgcn_readfirstlane(p.row / CH) : 0;
  p.row %= CH;
  const int e0 = p.block * CH, width = min(CH, c.E - e0);
  const bool mine = p.row < width;
  const int64_t d0 = (int64_t)p.g * c.E + e0, d = d0 + p.row, slot = scan_slot(c, p.b);
  In in;
  in.begin(c.in, c.bc, p, p.first, 1, d0, width, c.N);
  if (p.first < p.alive) in.load(p.alive - p.first);
  float A[NS], h[NS], skip = 0.f, dt_bias = 0.f, total = 0.f;
  const int64_t seg_state = ((p.b * segs.n + p.seg) * c.D + d) * c.N;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int n = s * 16 + p.j;
    const bool has = mine && n < c.N;
    A[s] = has ? in_powers_of_2(c.A[d * c.N + n]) : 0.f;
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
  const int64_t all_states = (int64_t)c.D * c.N, state_at = d * c.N + p.j;
  auto keep = [&](int64_t t, const float (&state)[NS]) {
    if (STATES_ONLY || !c.checkpoints || t >= p.alive) return;
    float* to = c.checkpoints + (p.b * c.tiles + t / kTile) * all_states;  // (the same for the wavefront)
#pragma unroll
    for (int s = 0; s < NS; ++s)
      if (mine && s * 16 + p.j < c.N) (to + s * 16)[state_at] = state[s];
  };
  Out out;
  if (!STATES_ONLY) out.begin(c.out, p, p.first, 1, d0, width);
  if (p.first < p.alive) {
    in.stage(raws, bcs);
    __syncthreads();
    if (p.first + TOKENS < p.alive) in.load(p.alive - p.first - TOKENS);
  }
  int turn = 0;
  for (int64_t t0 = p.first; t0 < p.alive; t0 += TOKENS) {
    T* const raw = raws + turn * RAW;
    const float* const bc = bcs + turn * BC;
    T *const xs = raw, *const dts = raw + TOKENS * CH, *const gates = raw + 2 * TOKENS * CH;
    const bool more = t0 + TOKENS < p.alive;
    const int tokens = (int)min((int64_t)TOKENS, p.alive - t0);
    // in turn: of the block, what it begins with, the product of its factors, a lane's share of its deltas
    float before[NS], all[NS], sum = 0.f;
    if constexpr (W == 1)
#pragma unroll
      for (int s = 0; s < NS; ++s) before[s] = h[s], all[s] = 1.f, h[s] = STATES_ONLY ? 0.f : h[s];
    for (int i0 = tile * kTile; i0 < (W > 1 ? (tile + 1) * kTile : tokens); i0 += kTile) {
      const int at = place_of<T, CH>(i0 + p.j, p.row);
      const bool live = i0 + p.j < tokens;
      const Token k = token_of(c, to_float(xs[at]), to_float(dts[at]), live, dt_bias);
      const float u = k.delta * k.x;
      total += k.delta;
      float y[kTile];
      const float* bs = bc + p.j * In::kPitch + i0;
      if constexpr (W == 1) {
        keep(t0 + i0, h);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          unroll<kTile / 4>([&](auto quarter) {
            constexpr int Q = decltype(quarter)::value * 4;
            const Float4 bt = four_of(bs + s * 16 * In::kPitch + Q), ct = four_of(bs + (STATES_ONLY ? 0 : In::kFloats) + s * 16 * In::kPitch + Q);
            unroll<4>([&](auto i) {
              constexpr int I = decltype(i)::value;
              const float a = exp2_of(lane_of_row<Q + I>(k.delta) * A[s]);
              h[s] = fmaf(a, h[s], lane_of_row<Q + I>(u) * bt[I]);
              if (!STATES_ONLY) all[s] *= a, y[Q + I] = s ? fmaf(ct[I], h[s], y[Q + I]) : ct[I] * h[s];
            });
          });
          if (!STATES_ONLY) settle(all[s]);  // (one block of states after the other: all at once take up to 40 registers more)
        }
        sum += k.delta;
      } else {
        float own[NS][kTile], product[NS][kTile];
        const float deltas = sum_of_row(k.delta);
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          float from_zero = 0.f, all = 1.f;
          unroll<kTile / 4>([&](auto quarter) {
            constexpr int Q = decltype(quarter)::value * 4;
            const Float4 bt = four_of(bs + s * 16 * In::kPitch + Q);
            unroll<4>([&](auto i) {
              constexpr int I = decltype(i)::value;
              const float a = exp2_of(lane_of_row<Q + I>(k.delta) * A[s]);
              from_zero = fmaf(a, from_zero, lane_of_row<Q + I>(u) * bt[I]);
              all *= a;
              own[s][Q + I] = from_zero, product[s][Q + I] = all;
            });
          });
          ends[tile][(s * CH + p.row) * 16 + p.j] = make_float2(from_zero, factor_of(deltas, A[s]));
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          before[s] = h[s];
#pragma unroll
          for (int v = 0; v < W; ++v) {
            const float2 end = ends[v][(s * CH + p.row) * 16 + p.j];
            if (v == tile) before[s] = h[s];
            h[s] = fmaf(end.y, h[s], end.x);
          }
        }
        keep(t0 + i0, before);
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int q = 0; q < kTile; q += 4) {
            const Float4 ct = four_of(bs + In::kFloats + s * 16 * In::kPitch + q);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float v = fmaf(product[s][q + i], before[s], own[s][q + i]);
              y[q + i] = s ? fmaf(ct[i], v, y[q + i]) : ct[i] * v;
            }
          }
      }
      if (!STATES_ONLY) {
        wave_fence();
#pragma unroll
        for (int i = 0; i < kTile; ++i) sums[wave][i * kSumPitch + lane] = y[i];
        wave_fence();
        float v = row_sum(sums[wave], lane) + skip * k.x;
        if (c.in[2].p) {
          const float g = to_float(gates[at]);
          v *= g * sigmoid(g);
        }
        xs[at] = from_float<T>(live ? v : 0.f);  // where x was
      }
    }
    if constexpr (W == 1) {
      const float deltas = sum_of_row(sum);
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        const float factor = factor_of(deltas, A[s]);
        h[s] = STATES_ONLY ? fmaf(factor, before[s], h[s]) : h[s] + put_right(factor, all[s], before[s]);
      }
    }
    if (BUFFERS == 2) turn ^= 1;
    if (BUFFERS == 2 && more) in.stage(raws + turn * RAW, bcs + turn * BC);
    __syncthreads();
    if (!STATES_ONLY) out.take(raw);  // (a lane's own pieces, before it stages others in their place)
    if (BUFFERS == 1 && more) {
      in.stage(raws, bcs);
      __syncthreads();
    }
    // (stores go out behind the wait for the block's loads: what is waited for next has been under way for long)
    if (!STATES_ONLY) out.store(p.last - t0);
    if (t0 + 2 * TOKENS < p.alive) in.load(p.alive - t0 - 2 * TOKENS);
  }
  if (!STATES_ONLY) {
    store_zeros<T, CH, F::THREADS>(c.out[0], p, d0, width, TOKENS);
  }
  if (!mine || tile) return;
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
  const float A = in_powers_of_2(c.A[dn]);
  float h = start && slot >= 0 ? start[slot * per + dn] : 0.f;
  for (int k = 0; k < segs.n; ++k) {
    const int64_t seg = b * segs.n + (rev ? segs.n - 1 - k : k);
    float* at = segs.h + seg * per + dn;
    const float own = *at;
    *at = h;
    h = fmaf(exp2_of(A * __builtin_amdgcn_fmed3f(segs.sum[seg * c.D + d], -3e38f, 3e38f)), h, own);  // (infinite times 0 is NaN)
  }
}

// One token, states in place.  V adjacent states a lane, L lanes a channel (all states at once: V L >= N).  Bound by the states'
// way in and out: 250 sequences of 4096 channels with 16 states, 138 MB, 29 us (4.8 TB/s; with the indexes in 64 bits 33).
// Two, four and eight sequences a lane, A read once for them: 29.5, 35, 61 us; non-temporal accesses: 35.
// ROWS: a workgroup is of one sequence, `blocks` of them each (else lanes go over sequences: a division for each lane, 31 us).
template <typename T, int V, int L, bool ROWS>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanCall c, unsigned blocks) {
  typedef float fv __attribute__((ext_vector_type(V)));
  const unsigned row = ROWS ? blockIdx.x / blocks : 0, i = (blockIdx.x - row * blocks) * 256 + threadIdx.x;
  const unsigned at_b = ROWS ? row : i / L / (unsigned)c.D, d = ROWS ? i / L : i / L - at_b * (unsigned)c.D;
  const int64_t b = at_b;
  if (b >= c.B || d >= (unsigned)c.D) return;  // (all lanes of a channel)
  const int64_t slot = scan_slot(c, b);
  const int n = (int)(i % L) * V;
  float y = 0.f;
  if (slot >= 0) {
    const float x = to_float(*at<T>(c.in[0], b, 0, d)), dt = to_float(*at<T>(c.in[1], b, 0, d));
    if (n < c.N) {
      const int g = (int)(d / (unsigned)c.E);
      float* state = c.s_out + (slot * c.D + d) * c.N + n;
      fv h = *(const fv*)state;
      const fv A = *(const fv*)(c.A + (int64_t)d * c.N + n);
      const T *pb = at<T>(c.bc[0], b, 0, g, n), *pc = at<T>(c.bc[1], b, 0, g, n);
      float bt[V], ct[V];
      if constexpr (V == 4) {
        unpack_row<T, V>(load_row<T, V>(pb, V), bt);
        unpack_row<T, V>(load_row<T, V>(pc, V), ct);
      } else {
        bt[0] = to_float(*pb), ct[0] = to_float(*pc);
      }
      const Token k = token_of(c, x, dt, true, c.dt_bias ? c.dt_bias[d] : 0.f);
      const float steps = __builtin_amdgcn_fmed3f(k.delta * kLog2e, -3.4e38f, 3.4e38f);  // (infinite, it would make NaN of an A of 0)
#pragma unroll
      for (int s = 0; s < V; ++s) {
        h[s] = fmaf(factor_of(steps, A[s]), h[s], k.delta * k.x * bt[s]);
        y = fmaf(ct[s], h[s], y);
      }
      *(fv*)state = h;
    }
#pragma unroll
    for (int k = 1; k < L; k *= 2) y += __shfl_xor(y, k);
    if (i % L) return;
    if (c.skip) y = fmaf(c.skip[d], x, y);
    if (c.in[2].p) {
      const float gate = to_float(*at<T>(c.in[2], b, 0, d));
      y *= gate * sigmoid(gate);
    }
  }
  if (i % L == 0) *at<T>(c.out[0], b, 0, d) = from_float<T>(y);
}

int states_of(const ScanCall& c) { return c.N <= 16 ? 1 : c.N <= 32 ? 2 : 4; }

// Tiles at once (1: in turn) and segments
struct Plan {
  int W, n;
  int64_t tokens;  // of a segment
};
// The least of estimated times, in cycles for 16 states.  In turn: 55 a token and 60 for every wavefront of a SIMD (one of them: 2048
// tokens of 4096 channels 118 us; four: 4 x 2048 of 4096 216).  At once: 98 a token with two workgroups of 8 wavefronts a compute unit
// (2048 of 4096: 82), 65 with one (2048 of 2048: 56), 60 with one of 16 (32768 of 1536: 853).  Segments: 92 a step whatever the shape, and two more launches
// (32768 of 1536: 492; 2048 of 4096: 105), 15 us in all.  Where that misses: more than 16 states are more cycles a token, of which the rule
// knows nothing (300 tokens of 1024 channels with 64 states go in turn, 42 us; segments 29); 2048 of 1536 and 8192 of 4096 go in segments (57
// and 334; at once 47 and 292).
Plan plan(const ScanCall& c) {
  const int ns = states_of(c);
  const int64_t T = c.T, eights = c.B * c.G * cdiv(c.E, 8), groups = c.B * c.G * cdiv(c.E, 16);
  const int64_t turn = T * (55 + (groups <= 256 ? 60 : groups * 60 / 256)), four = T * (eights <= 256 ? 65 : 98 * cdiv(eights, 512)), eight = T * 60 * cdiv(eights, 256);
  if (groups == 0) return {1, 1, T};  // (no sequences: no channels to share segments out over)
  const int64_t cut = T * groups * 92 / 256 + 36000;
  Plan z{1, 1, 0};
  int64_t best = turn;
  if (ns < 4 && four < best) z.W = 4, best = four;
  if (ns < 4 && eight < best) z.W = 8, best = eight;
  if (cut < best) z.W = 1;
  const int block = z.W == 8 ? 128 : ns == 4 ? 32 : 64;
  const int64_t in_all = cdiv(T, block);
  int64_t n = cut < best ? cdiv(12 * 256, groups) : 1;  // (twelve workgroups a compute unit)
  if (n > in_all) n = in_all;
  if (n < 1) n = 1;
  const int64_t each = in_all ? cdiv(in_all, n) : 1;
  z.tokens = each * block;
  z.n = in_all ? (int)cdiv(in_all, each) : 1;
  return z;
}

template <typename T, int NS, typename F, bool STATES_ONLY>
mdh_status pass(const ScanCall& c, const Segments& segs, hipStream_t st) {
  const int blocks = (int)cdiv(c.E, F::CH);
  const int64_t grid = c.B * segs.n * c.G * blocks;
  if (grid * F::THREADS >= (int64_t)1 << 32) return MDH_ERR_SIZE;
  clear_stale_error();
  scan_kernel<T, NS, F, STATES_ONLY><<<(unsigned)grid, F::THREADS, 0, st>>>(c, segs, blocks);
  return launch_status();
}
template <typename T, int NS>
mdh_status passes(const ScanCall& c, const Plan& z, const Segments& segs, hipStream_t st) {
  if (segs.n > 1) {
    mdh_status r = pass<T, NS, InTurn<NS>, true>(c, segs, st);
    if (r == MDH_OK) r = launch_scan_segments(c, segs.h, segs.sum, segs.n, c.s_in, false, st);
    if (r != MDH_OK) return r;
  }
  if constexpr (NS < 4) {
    if (z.W == 4) return pass<T, NS, AtOnce<NS>, false>(c, segs, st);
    if (z.W == 8) return pass<T, NS, ManyAtOnce<NS>, false>(c, segs, st);
  }
  return pass<T, NS, InTurn<NS>, false>(c, segs, st);
}
template <typename T>
mdh_status pass_of(const ScanCall& c, const Plan& z, const Segments& segs, hipStream_t st) {
  switch (states_of(c)) {
    case 1: return passes<T, 1>(c, z, segs, st);
    case 2: return passes<T, 2>(c, z, segs, st);
    default: return passes<T, 4>(c, z, segs, st);
  }
}

template <typename T, int V, int L>
mdh_status step(const ScanCall& c, hipStream_t st) {
  if (c.B * c.D >= (int64_t)1 << 25) return MDH_ERR_SIZE;  // (64 lanes a channel at the most: 2^31)
  clear_stale_error();
  const int64_t lanes = (int64_t)c.D * L, blocks = cdiv(lanes, 256);
  if (lanes >= 2048)  // (an eighth of the lanes without a channel at the most)
    scan_step_kernel<T, V, L, true><<<(unsigned)(c.B * blocks), 256, 0, st>>>(c, (unsigned)blocks);
  else
    scan_step_kernel<T, V, L, false><<<(unsigned)cdiv(c.B * lanes, 256), 256, 0, st>>>(c, 0);
  return launch_status();
}
template <typename T>
mdh_status step_of(const ScanCall& c, hipStream_t st) {
  const bool vec = c.N % 4 == 0 && ((uintptr_t)c.s_out | (uintptr_t)c.A) % 16 == 0;
  const int V = vec ? 4 : 1, lanes = (int)cdiv(c.N, V);
  if (vec) {
    if (lanes <= 1) return step<T, 4, 1>(c, st);
    if (lanes <= 4) return step<T, 4, 4>(c, st);
    return step<T, 4, 16>(c, st);
  }
  if (lanes <= 4) return step<T, 1, 4>(c, st);
  if (lanes <= 16) return step<T, 1, 16>(c, st);
  return step<T, 1, 64>(c, st);
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
  const int n = plan(c).n;
  return n > 1 ? (size_t)(c.B * n) * (size_t)c.D * (size_t)(c.N + 1) * sizeof(float) : 0;
}
mdh_status launch_scan_forward(const ScanCall& c, hipStream_t st) {
  const Plan z = plan(c);
  Segments segs{};
  segs.n = z.n, segs.tokens = z.tokens;
  segs.h = (float*)c.ws;
  segs.sum = segs.h + c.B * segs.n * (int64_t)c.D * c.N;
  return c.dtype == MDH_BF16 ? pass_of<bf16>(c, z, segs, st) : pass_of<float>(c, z, segs, st);
}
mdh_status launch_scan_step(const ScanCall& c, hipStream_t st) { return c.dtype == MDH_BF16 ? step_of<bf16>(c, st) : step_of<float>(c, st); }

}  // namespace mdh

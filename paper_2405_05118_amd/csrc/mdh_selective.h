// What the kernels of the selective scan share: places of lanes, time steps, sums over a row of lanes.
#pragma once
#include <utility>

#include "mdh_act.h"
#include "mdh_internal.h"
#include "mdh_vec.h"

namespace mdh {

// 16 lanes (a row of a wavefront) are one channel, each lane one state of every 16; tokens are walked 16 at a time.
constexpr int kTile = kScanTile, kWaveChannels = 4;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

template <int... I, typename F>
__device__ __forceinline__ void unroll_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
// f(0) .. f(N-1) with the number as a constant
template <int N, typename F>
__device__ __forceinline__ void unroll(F f) {
  unroll_of(std::make_integer_sequence<int, N>{}, f);
}

// lane J's value in all 16 lanes of its row (an operand's modifier: no instruction of its own)
template <int J>
__device__ __forceinline__ float lane_of_row(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x150 + J, 0xf, 0xf, true));
}
// lane J's value of `v` times x, added to sum.  (The compiler broadcasts to a register first; the two wait states are those between
// an instruction that writes a register and a broadcast of it.)
template <int J>
__device__ __forceinline__ void add_lane_of_row(float& sum, float v, float x) {
  asm("s_nop 1\n\tv_fmac_f32_dpp %0, %1, %2 row_newbcast:%3 row_mask:0xf bank_mask:0xf" : "+v"(sum) : "v"(v), "v"(x), "n"(J));
}
// computed here, not behind the next barrier with all that it is computed from in registers until there
__device__ __forceinline__ void settle(float& v) { asm volatile("" : "+v"(v)); }
// The same value to be broadcast at another place: where the compiler knows that two broadcasts are one, it keeps their result in
// a register of its own, 16 for a tile, and both lose the modifier.
__device__ __forceinline__ float again(float v) {
  asm("" : "+v"(v));
  return v;
}
// 2^x by the hardware (1 ulp; 0 below 2^-126)
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// A for powers of 2.  The largest numbers stay as they are: infinite, they would make NaN of a time step of 0.  (NaN stays, too.)
__device__ __forceinline__ float in_powers_of_2(float A) {
  const float v = A * kLog2e;
  return v < -3.4e38f || v > 3.4e38f ? A : v;
}

// A state that decays slowly multiplies thousands of factors just below 1, each of them rounded, and v_exp_f32 is besides too small by
// 0.12 2^-24 on average there (a million arguments from -1e-2 to -1e-5; no more than 0.7 2^-24 at any).  So a state goes over a block of
// tokens (a tile, or the 32 or 64 that are staged together) by the factor of the block, e^(A sum of deltas), one exponential for them all:
// what the tokens' own factors are off by does not add up beyond their block, and states that do not decay, or by less than 32 bits can
// tell for a token, are held.  1e-8 more in the exponent makes up for the mean (2^0 stays 1).
__device__ __forceinline__ float factor_of(float delta, float A) { return exp2_of(fmaf(delta, A, 1e-8f)); }
// the sum of the 16 lanes of a row, the same bits in all of them
template <int N>
__device__ __forceinline__ float add_rotated(float v) {
  return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x120 + N, 0xf, 0xf, true));
}
// the sum of a block's deltas, bounded: of steps near the largest number it would be infinite, and NaN times an A of 0
__device__ __forceinline__ float sum_of_row(float delta) {
  return add_rotated<1>(add_rotated<2>(add_rotated<4>(add_rotated<8>(__builtin_amdgcn_fmed3f(delta, -1e37f, 1e37f)))));
}
// What is to be added to a state behind a block that began with `before` and was multiplied by `product` where `factor` is right.
// (An infinite state is infinite behind the block too; its difference of factors may be 0.)
__device__ __forceinline__ float put_right(float factor, float product, float before) {
  return (factor - product) * __builtin_amdgcn_fmed3f(before, -3e38f, 3e38f);
}

// e^v with the rounding of v log2(e) put right (0 and infinity stay: v log2(e) may be infinite there, and its rounding NaN)
__device__ __forceinline__ float exp_of(float v) {
  const float p = v * kLog2e, r = fmaf(v, kLog2e, -p) + v * 1.92596299e-8f;  // log2(e) = kLog2e + 1.926e-8
  const float e = exp2_of(p);
  return e > 0.f && e < 3e38f ? fmaf(e, r * kLn2, e) : e;
}
// log(1 + e^v).  log(1 + e) = 2 artanh(e / (2 + e)), whose series of five terms is off by less than 2^-26 up to e = 0.4
// (s = 1/6: s^10 / 11); beyond, 1 + e is rounded by 2^-24 of a logarithm above 0.33.
__device__ __forceinline__ float softplus_of(float v) {
  const float e = exp_of(v);
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  const float near = 2.f * s * fmaf(q, fmaf(q, fmaf(q, fmaf(q, 1.f / 9, 1.f / 7), 1.f / 5), 1.f / 3), 1.f);
  const float far = kLn2 * __builtin_amdgcn_logf(1.f + e), both = e <= 0.4f ? near : far;
  return v > 20.f ? v : both;  // (e^-20 is below half an ulp of 20; NaN stays)
}

struct ScanPlace {
  int64_t b, len;
  int64_t first, last, alive;  // tokens of the segment; up to its last valid one
  int seg, g, block;           // block: of the group's channels
  int row, j;                  // the lane: row of its workgroup, place in the row
};

__device__ __forceinline__ int64_t scan_length(const ScanCall& c, int64_t b) {
  return c.lengths ? min(max((int64_t)c.lengths[b], (int64_t)0), c.T) : c.T;
}
__device__ __forceinline__ int64_t scan_slot(const ScanCall& c, int64_t b) {
  if (!c.slots) return b;
  const int64_t s = c.slots[b];
  return s >= 0 && s < c.n_slots ? s : -1;
}
// workgroup id -> (batch, segment, group, block), blocks fastest (neighbours read the same lines: xcd_order)
__device__ __forceinline__ ScanPlace scan_place(const ScanCall& c, int blocks, int nseg, int64_t seg_tokens) {
  ScanPlace p;
  unsigned i = xcd_order(blockIdx.x, gridDim.x);
  p.block = (int)(i % (unsigned)blocks), i /= (unsigned)blocks;
  p.g = (int)(i % (unsigned)c.G), i /= (unsigned)c.G;
  p.seg = (int)(i % (unsigned)nseg);
  p.b = i / (unsigned)nseg;
  p.len = scan_length(c, p.b);
  p.first = p.seg * seg_tokens;
  p.last = min(p.first + seg_tokens, c.T);
  p.alive = min(p.last, p.len);
  p.j = threadIdx.x & 15;
  p.row = threadIdx.x >> 4;
  return p;
}
template <typename T>
__device__ __forceinline__ T* at(const TokenView& v, int64_t b, int64_t t, int64_t ch) {
  return (T*)const_cast<void*>(v.p) + b * v.sb + t * v.st + ch;
}
template <typename T>
__device__ __forceinline__ T* at(const SharedView& v, int64_t b, int64_t t, int g, int n) {
  return (T*)const_cast<void*>(v.p) + b * v.sb + t * v.st + g * v.sg + n;
}

// Tokens are staged in LDS in blocks: the loads of the next block are under way while one is worked on.  All operands of a block are
// one list of pieces of 16 bytes, dealt out to the lanes of the workgroup (read element by element, the 16 tokens of a tile cost the
// caches an access for each token and wavefront, 1.4e8 for 8192 tokens of 4096 channels: one a cycle, as much as all the rest;
// operand by operand, most of the lanes had nothing to do).
//   token operands   (x, dt, ..) CH channels, in LDS as they are in memory: piece q at raw + q; gradients and outputs take the places
//                    of the first ones, and a lane stores the pieces that it stages
//   shared operands  (b, c) in LDS as fp32, state by state
// Zeros from the end of the valid tokens on, and past the last channel or state.  The pieces of a token are exchanged so that a
// channel's 16 tokens lie in different banks.
template <int PA>
__device__ __forceinline__ int swizzle(int q) {
  const int t = q / PA;
  return q ^ (t / (16 / PA) & (PA - 1));
}
// where channel ch of token t of a block of CH channels is
template <typename T, int CH>
__device__ __forceinline__ int place_of(int t, int ch) {
  constexpr int V = kLaneValues<T>, PA = CH / V;
  return swizzle<PA>(t * PA + ch / V) * V + ch % V;
}
template <typename T, int NA, int NB, int CH, int STATES, int TOKENS, int THREADS>
struct Stage {
  static constexpr int V = kLaneValues<T>, PA = CH / V, QA = TOKENS * PA, PB = STATES / V, QB = TOKENS * PB;
  static constexpr int PIECES = NA * QA + NB * QB, SLOTS = (PIECES + THREADS - 1) / THREADS;
  static constexpr int kPitch = TOKENS + 4, kFloats = STATES * kPitch;  // (16 lanes that read 16 bytes each reach all 64 banks)
  static_assert(QA % 64 == 0 && QB % 64 == 0 && THREADS % 64 == 0, "a wavefront's pieces are of one operand");
  Word4 w[SLOTS];
  const T* at[SLOTS];   // of the block that is loaded next
  int64_t step[SLOTS];  // to the one after it
  int left[SLOTS];      // channels or states from there on

  // which operand a wavefront's pieces are of (PIECES / .. and on: none)
  __device__ __forceinline__ static int operand(int k) {
    const int q = __builtin_amdgcn_readfirstlane(k * THREADS + (int)threadIdx.x);
    return q < NA * QA ? q / QA : NA + (q - NA * QA) / QB;
  }
  __device__ __forceinline__ static int token(int k) {
    const int q = k * THREADS + (int)threadIdx.x;
    return operand(k) < NA ? q % QA / PA : (q - NA * QA) % QB / PB;
  }
  // token operands that are not there have null pointers
  // way: 1 from the first block to the last, -1 back
  __device__ __forceinline__ void begin(const TokenView* va, const SharedView* vb, const ScanPlace& p, int64_t t0, int way, int64_t d0, int width,
                                        int N) {
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      const int o = operand(k), q = k * THREADS + (int)threadIdx.x;
      at[k] = nullptr, step[k] = 0, left[k] = 0;
      if (o < NA) {
        const int ch = q % QA % PA * V;
        at[k] = (const T*)va[o].p + p.b * va[o].sb + (t0 + token(k)) * va[o].st + d0 + ch;
        step[k] = way * TOKENS * va[o].st;
        left[k] = va[o].p ? width - ch : 0;
      } else if (o < NA + NB) {
        const int n = (q - NA * QA) % QB % PB * V;
        const SharedView& v = vb[o - NA];
        at[k] = (const T*)v.p + p.b * v.sb + (t0 + token(k)) * v.st + p.g * v.sg + n;
        step[k] = way * TOKENS * v.st;
        left[k] = N - n;
      }
    }
  }
  // `tokens` valid ones of the block; then on to the next one
  __device__ __forceinline__ void load(int64_t tokens) {
    const int valid = (int)min(tokens, (int64_t)TOKENS);
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      w[k] = (Word4){0, 0, 0, 0};
      if (left[k] > 0 && token(k) < valid) w[k] = load_row<T>(at[k], left[k]);
      at[k] += step[k];
    }
  }
  __device__ __forceinline__ void stage(T* raw, float* shared) const {
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      const int o = operand(k), q = k * THREADS + (int)threadIdx.x;
      if (o < NA) {
        ((Word4*)raw)[q / QA * QA + swizzle<PA>(q % QA)] = w[k];
      } else if (o < NA + NB) {
        float x[V];
        unpack_row<T>(w[k], x);
        float* to = shared + (o - NA) * kFloats + (q - NA * QA) % QB % PB * V * kPitch + token(k);
#pragma unroll
        for (int i = 0; i < V; ++i) to[i * kPitch] = x[i];
      }
    }
  }
};

// Outputs of a block, NO of them, in the places of the first token operands of a Stage
template <typename T, int NO, int CH, int TOKENS, int THREADS>
struct Outputs {
  static constexpr int V = kLaneValues<T>, PA = CH / V, QA = TOKENS * PA, SLOTS = (NO * QA + THREADS - 1) / THREADS;
  Word4 w[SLOTS];
  T* at[SLOTS];
  int64_t step[SLOTS];
  int left[SLOTS];
  __device__ __forceinline__ static int operand(int k) { return __builtin_amdgcn_readfirstlane(k * THREADS + (int)threadIdx.x) / QA; }
  __device__ __forceinline__ void begin(const TokenView* to, const ScanPlace& p, int64_t t0, int way, int64_t d0, int width) {
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      const int o = operand(k), q = (k * THREADS + (int)threadIdx.x) % QA, ch = q % PA * V;
      at[k] = nullptr, step[k] = 0, left[k] = 0;
      if (o < NO && to[o].p) {
        at[k] = (T*)const_cast<void*>(to[o].p) + p.b * to[o].sb + (t0 + q / PA) * to[o].st + d0 + ch;
        step[k] = way * TOKENS * to[o].st;
        left[k] = width - ch;
      }
    }
  }
  __device__ __forceinline__ void take(const T* raw) {
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      const int q = k * THREADS + (int)threadIdx.x;
      if (NO * QA % THREADS == 0 || q < NO * QA) w[k] = ((const Word4*)raw)[q / QA * QA + swizzle<PA>(q % QA)];
    }
  }
  // `tokens` of the block are the segment's; then on to the next one
  __device__ __forceinline__ void store(int64_t tokens) {
    const int valid = (int)min(tokens, (int64_t)TOKENS);
#pragma unroll
    for (int k = 0; k < SLOTS; ++k) {
      if (left[k] > 0 && (k * THREADS + (int)threadIdx.x) % QA / PA < valid) store_row<T>(at[k], left[k], w[k]);
      at[k] += step[k];
    }
  }
};
// zeros behind the block of tokens that the length is in
template <typename T, int CH, int THREADS>
__device__ __forceinline__ void store_zeros(const TokenView& v, const ScanPlace& p, int64_t d0, int width, int block) {
  constexpr int V = kLaneValues<T>, P = CH / V;
  const int64_t from = p.alive > p.first ? p.first + (p.alive - p.first + block - 1) / block * block : p.first;
  for (int64_t t = from + (int)threadIdx.x / P; t < p.last; t += THREADS / P) {
    const int ch = (int)threadIdx.x % P * V;
    if (ch < width) store_row<T>((T*)const_cast<void*>(v.p) + p.b * v.sb + t * v.st + d0 + ch, width - ch, (Word4){0, 0, 0, 0});
  }
}
__device__ __forceinline__ Float4 four_of(const float* lds) { return *(const Float4*)lds; }

// Sums over the 16 lanes of a row, for 16 tokens at once: every lane leaves its value for token t at t * 68 + lane and lane j
// adds up token j's (68: 16 lanes that read 16 bytes each reach all 64 banks).  A wavefront's own part of LDS, in order.
constexpr int kSumPitch = 68, kSumFloats = kTile * kSumPitch;
__device__ __forceinline__ float row_sum(const float* lds, int lane) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  const f4* p = (const f4*)(lds + (lane & 15) * kSumPitch + (lane & 48));
  const f4 s = (p[0] + p[1]) + (p[2] + p[3]);
  return (s[0] + s[1]) + (s[2] + s[3]);
}
// A lane's 16 values, of a token each, summed over the four rows of a wavefront: lane (r, j) those of lanes j for tokens 4 r + 0 .. 3
__device__ __forceinline__ Float4 over_rows(const float (&v)[kTile]) {
  float half[8];
  Float4 s;
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[t]), __float_as_uint(v[t + 8]), false, false);
    half[t] = __uint_as_float(x[0]) + __uint_as_float(x[1]);  // rows 0 and 1: token t, 2 and 3: t + 8
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(half[t]), __float_as_uint(half[t + 4]), false, false);
    s[t] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
  }
  return s;
}
// between a wavefront's stores to LDS and other lanes' loads of them, and back
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// what lane j of a row has of token j
struct Token {
  float x, delta, raw;  // raw: before the softplus
};
__device__ __forceinline__ Token token_of(const ScanCall& c, float x, float dt, bool live, float dt_bias) {
  Token k;
  k.x = x;
  k.raw = dt + dt_bias;
  const float delta = c.softplus ? softplus_of(k.raw) : k.raw;
  k.delta = live ? delta : 0.f;
  return k;
}

}  // namespace mdh

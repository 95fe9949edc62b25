// What the kernels of the selective scan share: places of lanes, time steps, sums over a row of lanes.
#pragma once
#include <utility>

#include "mdh_act.h"
#include "mdh_internal.h"
#include "mdh_types.h"

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
// 2^x by the hardware (1 ulp; 0 below 2^-126)
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// e^v with the rounding of v log2(e) put right
__device__ __forceinline__ float exp_of(float v) {
  const float p = v * kLog2e, r = fmaf(v, kLog2e, -p) + v * 1.92596299e-8f;  // log2(e) = kLog2e + 1.926e-8
  const float e = exp2_of(p);
  return e < 3e38f ? fmaf(e, r * kLn2, e) : e;
}
// log(1 + e^v).  log(1 + e) = 2 artanh(e / (2 + e)), whose series of five terms is off by less than 2^-26 up to e = 0.4
// (s = 1/6: s^10 / 11); beyond, 1 + e is rounded by 2^-24 of a logarithm above 0.33.
__device__ __forceinline__ float softplus_of(float v) {
  if (v > 20.f) return v;  // e^-20 is below half an ulp of 20
  const float e = exp_of(v);
  const float s = e * __builtin_amdgcn_rcpf(2.f + e), q = s * s;
  const float near = 2.f * s * fmaf(q, fmaf(q, fmaf(q, fmaf(q, 1.f / 9, 1.f / 7), 1.f / 5), 1.f / 3), 1.f);
  return e <= 0.4f ? near : kLn2 * __builtin_amdgcn_logf(1.f + e);
}

struct ScanPlace {
  int64_t b, seg, len, first, last;  // tiles first <= t < last, those of them before the length
  int g, block;                      // group, block of its channels
  int row, j;                        // the lane: row of its workgroup, place in the row
};

// channels of a workgroup of `waves` wavefronts, walked `times` channels a row
__device__ __forceinline__ int64_t scan_length(const ScanCall& c, int64_t b) {
  return c.lengths ? min(max((int64_t)c.lengths[b], (int64_t)0), c.T) : c.T;
}
__device__ __forceinline__ int64_t scan_slot(const ScanCall& c, int64_t b) {
  if (!c.slots) return b;
  const int64_t s = c.slots[b];
  return s >= 0 && s < c.n_slots ? s : -1;
}
// workgroup id -> (batch, segment, group, block), blocks fastest (neighbours read the same lines: xcd_order)
__device__ __forceinline__ ScanPlace scan_place(const ScanCall& c, int blocks, int nseg, int64_t seg_tiles) {
  ScanPlace p;
  int64_t i = xcd_order(blockIdx.x, gridDim.x);
  p.block = (int)(i % blocks), i /= blocks;
  p.g = (int)(i % c.G), i /= c.G;
  p.seg = i % nseg;
  p.b = i / nseg;
  p.len = scan_length(c, p.b);
  const int64_t tiles = (c.T + kTile - 1) / kTile;
  p.first = p.seg * seg_tiles;
  p.last = min(p.first + seg_tiles, tiles);
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

// b or c of a tile in LDS as fp32, state by state with kTile tokens each; zeros past the length and past N.
constexpr int kPitch = kTile + 4;  // (16 lanes that read 16 bytes each: all 64 banks)
template <typename T, int STATES, int THREADS>
__device__ __forceinline__ void stage_shared(const ScanCall& c, const SharedView& v, const ScanPlace& p, int64_t t0, float* lds) {
#pragma unroll
  for (int i0 = 0; i0 < STATES * kTile; i0 += THREADS) {
    const int i = i0 + threadIdx.x, n = i % STATES, t = i / STATES;
    if (i < STATES * kTile) lds[n * kPitch + t] = n < c.N && t0 + t < p.len ? to_float(*at<T>(v, p.b, t0 + t, p.g, n)) : 0.f;
  }
}
__device__ __forceinline__ void tile_of(const float* lds, int n, float (&x)[kTile]) {
  typedef float f4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < kTile / 4; ++i) {
    const f4 v = ((const f4*)(lds + n * kPitch))[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
  }
}

// Sums over the 16 lanes of a row, for 16 tokens at once: every lane leaves its value for token t at t * 68 + lane and lane j
// adds up token j's (68: 16 lanes that read 16 bytes each reach all 64 banks).  A wavefront's own part of LDS, in order.
constexpr int kSumPitch = 68, kSumFloats = kTile * kSumPitch;
__device__ __forceinline__ float row_sum(const float* lds, int lane) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  const f4* p = (const f4*)(lds + (lane & 15) * kSumPitch + (lane & 48));
  const f4 s = (p[0] + p[1]) + (p[2] + p[3]);
  return (s[0] + s[1]) + (s[2] + s[3]);
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
template <typename T>
__device__ __forceinline__ Token token_of(const ScanCall& c, bool live, const T* x, const T* dt, float dt_bias) {
  Token k{0.f, 0.f, 0.f};
  if (!live) return k;
  k.x = to_float(*x);
  k.raw = to_float(*dt) + dt_bias;
  k.delta = c.softplus ? softplus_of(k.raw) : k.raw;
  return k;
}

}  // namespace mdh

// Element types of the sequence layers in device code.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mdh {

struct bf16 {
  uint16_t bits;
};
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }

// two values rounded to nearest even (NaN stays NaN)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}

template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) {
  return x;
}
template <>
__device__ __forceinline__ bf16 from_float<bf16>(float x) {
  return bf16{(uint16_t)pack_bf16(x, 0.f)};
}

// l^n for a decay given as its natural logarithm, as the sum of two floats.  A state is multiplied by it once for every run
// of tokens: rounded to one float, l^n is off by up to 2^-25 in the same direction each time, which a memory of thousands
// of tokens adds up (2000 tokens, one at a time: 8e-6 of the results against 64 bits, 8e-7 with both).
struct Decay {
  float hi, lo;
  __device__ __forceinline__ float operator*(float x) const { return fmaf(x, hi, x * lo); }
};
__device__ __forceinline__ Decay decay_power(float log_decay, int64_t n) {
  const double v = n == 0 ? 1.0 : exp((double)log_decay * (double)n);  // (-infinity, l = 0, has l^0 = 1 too)
  const float hi = (float)v;
  return Decay{hi, (float)(v - (double)hi)};
}

}  // namespace mdh

// Activations of the group norm and their slopes, in fp32, on the values of a lane.  Which one is a number that is the same
// for the whole launch: one branch for all values.
#pragma once
#include <hip/hip_runtime.h>
#include "mdh.h"

namespace mdh {

// 1 / (1 + e^-z): e^-z may overflow, its reciprocal is then 0.  (The hardware's reciprocal, off by 1 ulp at most: a division is
// ten instructions, and made the group norm of 8 x 128 x 128 x 256 values a third slower.)
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }
// (a product with 0 would make NaN of -infinity; NaN itself is not less than 0 and stays)
__device__ __forceinline__ float relu(float z) { return z < 0.f ? 0.f : z; }
__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * (1.f + erff(z * 0.70710678118654752440f)); }

template <int N>
__device__ __forceinline__ void act_of(int act, const float (&z)[N], float (&out)[N]) {
  if (act == MDH_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = z[i] * sigmoid(z[i]);
  } else if (act == MDH_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = z[i] * normal_cdf(z[i]);
  } else if (act == MDH_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = relu(z[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = z[i];
  }
}

// the activation and its slope
template <int N>
__device__ __forceinline__ void act_slope(int act, const float (&z)[N], float (&out)[N], float (&slope)[N]) {
  if (act == MDH_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float p = sigmoid(z[i]);
      out[i] = z[i] * p;
      slope[i] = p * (1.f + z[i] * (1.f - p));
    }
    asm volatile("; silu");  // (the branches end differently: the compiler would make one store of their last ones, to an
                             // address that depends on the branch, and with it keep the arrays in memory)
  } else if (act == MDH_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float p = normal_cdf(z[i]);
      out[i] = z[i] * p;
      slope[i] = p + z[i] * 0.39894228040143267794f * __expf(-0.5f * z[i] * z[i]);
    }
    asm volatile("; gelu");
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      slope[i] = act == MDH_ACT_RELU ? (z[i] > 0.f ? 1.f : 0.f) : 1.f;
      out[i] = act == MDH_ACT_RELU ? relu(z[i]) : z[i];
    }
    asm volatile("; others");
  }
}

}  // namespace mdh

// Activations of the group norm and their slopes, in fp32.
#pragma once
#include <hip/hip_runtime.h>
#include "mdh.h"

namespace mdh {

// 1 / (1 + e^-z): e^-z may overflow, its reciprocal is then 0
__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + __expf(-z)); }

template <int ACT>
__device__ __forceinline__ float act(float z) {
  if constexpr (ACT == MDH_ACT_RELU) return z > 0.f ? z : z - z;  // NaN and not 0 where z is NaN
  if constexpr (ACT == MDH_ACT_SILU) return z * sigmoid(z);
  if constexpr (ACT == MDH_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752440f));
  return z;
}

template <int ACT>
__device__ __forceinline__ float slope(float z) {
  if constexpr (ACT == MDH_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if constexpr (ACT == MDH_ACT_SILU) {
    const float p = sigmoid(z);
    return p * (1.f + z * (1.f - p));
  }
  if constexpr (ACT == MDH_ACT_GELU)
    return 0.5f * (1.f + erff(z * 0.70710678118654752440f)) + z * 0.39894228040143267794f * __expf(-0.5f * z * z);
  return 1.f;
}

}  // namespace mdh

// Rows of V = 16 / sizeof(T) channels a lane, at any alignment that the type has: 16 bytes at a time (the hardware reads and
// writes unaligned ones, in one or two pieces), the last channels of a row that has no V left one by one.
#pragma once
#include "mdh_types.h"

namespace mdh {

typedef uint32_t Word4 __attribute__((ext_vector_type(4)));
typedef Word4 AnyWord4 __attribute__((aligned(2)));
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef Float4 AnyFloat4 __attribute__((aligned(4)));

template <typename T>
constexpr int kLaneValues = 16 / (int)sizeof(T);

template <typename T>
__device__ __forceinline__ Word4 load_row(const T* p, int left) {
  constexpr int V = kLaneValues<T>;
  if (left >= V) return *(const AnyWord4*)p;
  Word4 w = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < V - 1; ++i)
    if (i < left) {
      if constexpr (sizeof(T) == 4)
        w[i] = ((const uint32_t*)p)[i];
      else
        w[i / 2] |= (uint32_t)((const uint16_t*)p)[i] << 16 * (i & 1);
    }
  return w;
}
template <typename T>
__device__ __forceinline__ void store_row(T* p, int left, const Word4& w) {
  constexpr int V = kLaneValues<T>;
  if (left >= V) {
    *(AnyWord4*)p = w;
    return;
  }
#pragma unroll
  for (int i = 0; i < V - 1; ++i)
    if (i < left) {
      if constexpr (sizeof(T) == 4)
        ((uint32_t*)p)[i] = w[i];
      else
        ((uint16_t*)p)[i] = (uint16_t)(w[i / 2] >> 16 * (i & 1));
    }
}
template <typename T>
__device__ __forceinline__ void unpack_row(const Word4& w, float (&x)[kLaneValues<T>]) {
#pragma unroll
  for (int i = 0; i < kLaneValues<T>; ++i) {
    if constexpr (sizeof(T) == 4)
      x[i] = __uint_as_float(w[i]);
    else
      x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
}
template <typename T>
__device__ __forceinline__ Word4 pack_row(const float (&x)[kLaneValues<T>]) {
  Word4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4)
      w[i] = __float_as_uint(x[i]);
    else
      w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
  }
  return w;
}
// `left` of N parameters (the others: fill), all fill where there are none
template <int N>
__device__ __forceinline__ void load_params(const float* p, int left, float fill, float (&x)[N]) {
  if (p && left >= N && N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const Float4 f = ((const AnyFloat4*)p)[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * i + e] = f[e];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = p && i < left ? p[i] : fill;
}
template <int N>
__device__ __forceinline__ void store_params(float* p, int left, const float (&x)[N]) {
  if (left >= N && N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) ((AnyFloat4*)p)[i] = (Float4){x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < left) p[i] = x[i];
}

}  // namespace mdh

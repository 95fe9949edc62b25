// Rows of V channels a lane (16 bytes, or 8), at any alignment that the type has: all at a time (the hardware reads and
// writes unaligned ones, in one or two pieces), the last channels of a row that has no V left one by one.
#pragma once
#include "mdh_types.h"

namespace mdh {

template <int N>
struct WordsOf {
  typedef uint32_t type __attribute__((ext_vector_type(N)));
  typedef type any __attribute__((aligned(2)));
};
template <int N>
using Words = typename WordsOf<N>::type;
typedef Words<4> Word4;
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef Float4 AnyFloat4 __attribute__((aligned(4)));

template <typename T>
constexpr int kLaneValues = 16 / (int)sizeof(T);
// V values of a lane as they are in memory
template <typename T, int V>
using RowWords = Words<V * (int)sizeof(T) / 4>;

template <typename T, int V = kLaneValues<T>>
__device__ __forceinline__ RowWords<T, V> load_row(const T* p, int left) {
  if (left >= V) return *(const typename WordsOf<V * (int)sizeof(T) / 4>::any*)p;
  RowWords<T, V> w = 0;
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
// The same for loads that other work goes on beside: the last values of a row come as the V that end there, in one access (value by value a
// wavefront waits for each before it goes on), and part_of() moves them to their places when they are wanted
// (a row's last lane, backward: norm of 8192 x 4097 111 us, so 79; convolution of 4 x 2048 x 4097 fp32 160, so 99).
// inside: V values or more lie in the row before p.
template <typename T, int V = kLaneValues<T>>
__device__ __forceinline__ RowWords<T, V> load_part(const T* p, int left, bool inside) {
  if (left < V && !inside) return load_row<T, V>(p, left);
  return *(const typename WordsOf<V * (int)sizeof(T) / 4>::any*)(p - (left < V ? V - left : 0));
}
template <typename T, int V = kLaneValues<T>>
__device__ __forceinline__ RowWords<T, V> part_of(RowWords<T, V> w, int left, bool inside) {
  if (left <= 0 || left >= V || !inside) return w;
  const int bits = (V - left) * (int)sizeof(T) * 8;
  uint64_t low = (uint64_t)w[1] << 32 | w[0];
  if constexpr (V * sizeof(T) == 8) {
    low >>= bits;
  } else {
    const uint64_t high = (uint64_t)w[3] << 32 | w[2];
    low = bits < 64 ? low >> bits | high << (64 - bits) : high >> (bits - 64);
    const uint64_t rest = bits < 64 ? high >> bits : 0;
    w[2] = (uint32_t)rest, w[3] = (uint32_t)(rest >> 32);
  }
  w[0] = (uint32_t)low, w[1] = (uint32_t)(low >> 32);
  return w;
}
template <typename T, int V = kLaneValues<T>>
__device__ __forceinline__ void store_row(T* p, int left, const RowWords<T, V>& w) {
  if (left >= V) {
    *(typename WordsOf<V * (int)sizeof(T) / 4>::any*)p = w;
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
template <typename T, int V = kLaneValues<T>>
__device__ __forceinline__ void unpack_row(const RowWords<T, V>& w, float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (sizeof(T) == 4)
      x[i] = __uint_as_float(w[i]);
    else
      x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
}
template <typename T, int V = kLaneValues<T>>
__device__ __forceinline__ RowWords<T, V> pack_row(const float (&x)[V]) {
  RowWords<T, V> w;
#pragma unroll
  for (int i = 0; i < V * (int)sizeof(T) / 4; ++i) {
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

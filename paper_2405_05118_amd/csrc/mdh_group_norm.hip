// Group norm with an activation, channels last.
//
// A workgroup owns one group of one entry and reads it three times (mean, variance, result); gradients of weight and bias
// have a workgroup for each channel.
#include "mdh_act.h"
#include "mdh_internal.h"
#include "mdh_types.h"

#include <type_traits>

namespace mdh {
namespace {

__device__ __forceinline__ float workgroup_sum(float v, float* red) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

template <typename T>
__device__ __forceinline__ const T* row(const RowView& v, int64_t r) {
  return (const T*)v.p + r * v.stride;
}

template <typename T, int ACT, bool GATE>
__global__ __launch_bounds__(256) void group_norm_kernel(GroupNormCall c) {
  __shared__ float red[4];
  const int64_t n = blockIdx.x / c.G, r0 = n * c.S;
  const int g = blockIdx.x % c.G, D = c.C / c.G;
  const int64_t m = c.S * D;
  float sum = 0.f;
  for (int64_t i = threadIdx.x; i < m; i += 256) sum += to_float(row<T>(c.x, r0 + i / D)[g * D + i % D]);
  const float mean = workgroup_sum(sum, red) / (float)m;
  float sq = 0.f;
  for (int64_t i = threadIdx.x; i < m; i += 256) {
    const float d = to_float(row<T>(c.x, r0 + i / D)[g * D + i % D]) - mean;
    sq += d * d;
  }
  const float rstd = 1.f / sqrtf(workgroup_sum(sq, red) / (float)m + c.eps);
  for (int64_t i = threadIdx.x; i < m; i += 256) {
    const int ch = g * D + (int)(i % D);
    const int64_t r = r0 + i / D;
    const float xh = (to_float(row<T>(c.x, r)[ch]) - mean) * rstd;
    const float z = xh * (c.weight ? c.weight[ch] : 1.f) + (c.bias ? c.bias[ch] : 0.f);
    const float y = GATE ? z * act<ACT>(to_float(row<T>(c.gate, r)[ch])) : act<ACT>(z);
    const_cast<T*>(row<T>(c.y, r))[ch] = from_float<T>(y);
  }
  if (threadIdx.x == 0) {
    if (c.mean) c.mean[blockIdx.x] = mean;
    if (c.rstd) c.rstd[blockIdx.x] = rstd;
  }
}

// gradient of z, and of the gate
template <typename T, int ACT, bool GATE>
__device__ __forceinline__ float grad_z(const GroupNormCall& c, int64_t r, int ch, float xh, float* dgate) {
  const float dy = to_float(row<T>(c.y, r)[ch]);
  const float z = xh * (c.weight ? c.weight[ch] : 1.f) + (c.bias ? c.bias[ch] : 0.f);
  if constexpr (GATE) {
    const float g = to_float(row<T>(c.gate, r)[ch]);
    *dgate = dy * z * slope<ACT>(g);
    return dy * act<ACT>(g);
  }
  return dy * slope<ACT>(z);
}

template <typename T, int ACT, bool GATE>
__global__ __launch_bounds__(256) void group_norm_dx_kernel(GroupNormCall c) {
  __shared__ float red[4];
  const int64_t n = blockIdx.x / c.G, r0 = n * c.S;
  const int g = blockIdx.x % c.G, D = c.C / c.G;
  const int64_t m = c.S * D;
  const float mean = c.mean[blockIdx.x], rstd = c.rstd[blockIdx.x];
  float t1 = 0.f, t2 = 0.f, dg = 0.f;
  for (int64_t i = threadIdx.x; i < m; i += 256) {
    const int ch = g * D + (int)(i % D);
    const int64_t r = r0 + i / D;
    const float xh = (to_float(row<T>(c.x, r)[ch]) - mean) * rstd;
    const float t = grad_z<T, ACT, GATE>(c, r, ch, xh, &dg) * (c.weight ? c.weight[ch] : 1.f);
    t1 += t;
    t2 += t * xh;
  }
  t1 = workgroup_sum(t1, red) / (float)m;
  t2 = workgroup_sum(t2, red) / (float)m;
  for (int64_t i = threadIdx.x; i < m; i += 256) {
    const int ch = g * D + (int)(i % D);
    const int64_t r = r0 + i / D;
    const float xh = (to_float(row<T>(c.x, r)[ch]) - mean) * rstd;
    const float t = grad_z<T, ACT, GATE>(c, r, ch, xh, &dg) * (c.weight ? c.weight[ch] : 1.f);
    const_cast<T*>(row<T>(c.dx, r))[ch] = from_float<T>(rstd * (t - t1 - xh * t2));
    if (GATE) const_cast<T*>(row<T>(c.dgate, r))[ch] = from_float<T>(dg);
  }
}

template <typename T, int ACT, bool GATE>
__global__ __launch_bounds__(256) void group_norm_dw_kernel(GroupNormCall c) {
  __shared__ float red[4];
  const int ch = blockIdx.x, g = ch / (c.C / c.G);
  float dw = 0.f, db = 0.f, dg = 0.f;
  for (int64_t r = threadIdx.x; r < c.N * c.S; r += 256) {
    const int64_t ng = r / c.S * c.G + g;
    const float xh = (to_float(row<T>(c.x, r)[ch]) - c.mean[ng]) * c.rstd[ng];
    const float dz = grad_z<T, ACT, GATE>(c, r, ch, xh, &dg);
    dw += dz * xh;
    db += dz;
  }
  dw = workgroup_sum(dw, red);
  db = workgroup_sum(db, red);
  if (threadIdx.x == 0) {
    if (c.dweight) c.dweight[ch] = dw;
    if (c.dbias) c.dbias[ch] = db;
  }
}

// f(ACT, GATE) with both as types
template <typename F>
void with_act(int act, bool gate, F f) {
  auto g = [&](auto a) {
    if (gate)
      f(a, std::true_type{});
    else
      f(a, std::false_type{});
  };
  if (act == MDH_ACT_RELU)
    g(std::integral_constant<int, MDH_ACT_RELU>{});
  else if (act == MDH_ACT_SILU)
    g(std::integral_constant<int, MDH_ACT_SILU>{});
  else if (act == MDH_ACT_GELU)
    g(std::integral_constant<int, MDH_ACT_GELU>{});
  else
    g(std::integral_constant<int, MDH_ACT_NONE>{});
}

template <typename T>
void forward(const GroupNormCall& c, hipStream_t st) {
  with_act(c.act, c.gate.p != nullptr, [&](auto a, auto g) {
    group_norm_kernel<T, a.value, g.value><<<dim3((unsigned)(c.N * c.G)), 256, 0, st>>>(c);
  });
}

template <typename T>
void backward(const GroupNormCall& c, hipStream_t st) {
  with_act(c.act, c.gate.p != nullptr, [&](auto a, auto g) {
    if (c.N && c.S) group_norm_dx_kernel<T, a.value, g.value><<<dim3((unsigned)(c.N * c.G)), 256, 0, st>>>(c);
    group_norm_dw_kernel<T, a.value, g.value><<<dim3((unsigned)c.C), 256, 0, st>>>(c);
  });
}

}  // namespace

size_t group_norm_workspace(const GroupNormCall&, bool) { return 0; }

mdh_status launch_group_norm(const GroupNormCall& c, hipStream_t st) {
  clear_stale_error();
  if (c.dtype == MDH_BF16)
    forward<bf16>(c, st);
  else
    forward<float>(c, st);
  return launch_status();
}

mdh_status launch_group_norm_backward(const GroupNormCall& c, hipStream_t st) {
  clear_stale_error();
  if (c.dtype == MDH_BF16)
    backward<bf16>(c, st);
  else
    backward<float>(c, st);
  return launch_status();
}

}  // namespace mdh

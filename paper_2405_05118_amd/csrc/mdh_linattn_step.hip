// One token of linear attention, the state in place: state <- l state + k v^T, o = scale state^T q.
//
// 2 * dk * dv multiply-adds on dk * dv numbers that are read and written once: bound by the memory that holds the states,
// or, with few of them, by one trip to it.  A workgroup owns W columns of one state (whole rows where there are states
// enough to fill the chip, 16 columns where not), a lane 4 columns of every 1024/W-th row: the sum over the rows that q
// asks for stays in the workgroup.
#include "mdh_internal.h"
#include "mdh_types.h"

namespace mdh {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

struct StepArgs {
  LinattnCall c;
  HeadView q, k, v, o;
  int dk, dv;
  float scale;
  float* state;
};

// V: columns of a lane, LW: lanes along the columns (W = V * LW)
template <typename T, int V, int LW>
__global__ __launch_bounds__(256) void linattn_step_kernel(StepArgs s) {
  constexpr int RP = 256 / LW;  // rows at once
  __shared__ float ks[256], qs[256], red[256 / 64][V * LW];
  const int h = blockIdx.x % s.c.H;
  const int64_t b = blockIdx.x / s.c.H;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = blockIdx.y * V * LW + (threadIdx.x % LW) * V, row = threadIdx.x / LW;
  const int64_t slot = s.c.slots ? (int64_t)s.c.slots[b] : b;
  T* o = (T*)s.o.p + b * s.o.sb + h * s.o.sh;
  if (s.c.slots && (slot < 0 || slot >= s.c.n_slots)) {
    if (row == 0)
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (col + e < s.dv) o[col + e] = from_float<T>(0.f);
    return;
  }
  const Decay l = decay_power(s.c.log_decay[h], 1);
  if ((int)threadIdx.x < s.dk) {
    ks[threadIdx.x] = to_float(((const T*)s.k.p + b * s.k.sb + (h / s.k.group) * s.k.sh)[threadIdx.x]);
    qs[threadIdx.x] = to_float(((const T*)s.q.p + b * s.q.sb + (h / s.q.group) * s.q.sh)[threadIdx.x]);
  }
  const T* pv = (const T*)s.v.p + b * s.v.sb + (h / s.v.group) * s.v.sh;
  float v[V], sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    v[e] = col + e < s.dv ? to_float(pv[col + e]) : 0.f;
    sum[e] = 0.f;
  }
  __syncthreads();
  float* st = s.state + ((slot * s.c.H + h) * s.dk) * (int64_t)s.dv + col;
  if (col < s.dv) {
#pragma unroll 8
    for (int r = row; r < s.dk; r += RP) {
      float* at = st + (int64_t)r * s.dv;
      float x[V];
      if constexpr (V == 4) {
        const f4 w = *(const f4*)at;
        for (int e = 0; e < 4; ++e) x[e] = w[e];
      } else {
        x[0] = at[0];
      }
      const float kr = ks[r], qr = qs[r];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[e] = l * x[e] + kr * v[e];
        sum[e] += qr * x[e];
      }
      if constexpr (V == 4)
        *(f4*)at = (f4){x[0], x[1], x[2], x[3]};
      else
        at[0] = x[0];
    }
  }
  // rows: over the lanes of a wavefront that share columns, then over the wavefronts
#pragma unroll
  for (int d = LW; d < 64; d *= 2)
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] += __shfl_xor(sum[e], d);
  if (lane < LW)
#pragma unroll
    for (int e = 0; e < V; ++e) red[wave][lane * V + e] = sum[e];
  __syncthreads();
  if (threadIdx.x < V * LW) {
    const int cc = blockIdx.y * V * LW + threadIdx.x;
    if (cc < s.dv)
      o[cc] = from_float<T>(s.scale * ((red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x])));
  }
}

template <typename T>
void step(const StepArgs& s, bool vec, hipStream_t st) {
  const unsigned states = (unsigned)(s.c.B * s.c.H);
  auto grid = [&](int w) { return dim3(states, (s.dv + w - 1) / w); };
  if (!vec)
    linattn_step_kernel<T, 1, 64><<<grid(64), 256, 0, st>>>(s);
  else
    linattn_step_kernel<T, 4, 32><<<grid(128), 256, 0, st>>>(s);
}

}  // namespace

mdh_status launch_linattn_step(const LinattnCall& c, const HeadView& q, const HeadView& k, const HeadView& v,
                               const HeadView& o, int dk, int dv, float scale, float* state, int dtype, hipStream_t st) {
  if (c.B * c.H > 0x7fffffff) return MDH_ERR_SIZE;
  const StepArgs s{c, q, k, v, o, dk, dv, scale, state};
  const bool vec = dv % 4 == 0 && (uintptr_t)state % 16 == 0;
  clear_stale_error();
  if (dtype == MDH_BF16)
    step<bf16>(s, vec, st);
  else
    step<float>(s, vec, st);
  return launch_status();
}

}  // namespace mdh

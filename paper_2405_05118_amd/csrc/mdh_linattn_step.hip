// One token of linear attention, the state in place: state <- l state + k v^T, o = scale state^T q.
//
// 2 * dk * dv multiply-adds on dk * dv numbers that are read and written once: bound by the memory that holds the states,
// or, with few of them, by one trip to it.  A workgroup owns W columns of one state, a lane 4 columns
// of every 1024/W-th row: the sum over the rows that q asks for stays in the workgroup.  A lane's first eight loads are
// under way before anything is waited for.  W is 64 where that gives the chip two workgroups a compute unit, else 16.
// Loads and stores leave the caches to others: between two tokens of one layer come all the other layers, whose states push
// its own out (cached / not, the states cold: 32 of 128 x 128 4.4 / 4.0 us, 512 17.3 / 12.4, 1024 32.3 / 26.0, 4096 113.7 /
// 102.4 = 5.2 TB/s; of one layer called again and again 3.8 / 3.8, 10.5 / 10.0, 24.8 / 22.8, 89.6 / 101.8).
// Measured in a graph, W = 64 / 16, states of 128 x 128: 32 of them 5.3 / 4.0 us, 128 6.3 / 6.1, 256 7.9 / 11.8, 1024
// 26.0 / 47.1; W = 128: 9.7, 10.8, 12.6, 25.4.  Where dv is no multiple of 4, or the states are not 16-byte aligned, a lane has one
// column and W is 16: 250 x 16 states of 128 x 127 501 us.
#include "mdh_internal.h"
#include "mdh_types.h"

namespace mdh {
namespace {

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
  typedef float fv __attribute__((ext_vector_type(V)));
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
  constexpr int U = 8;
  float* st = s.state + ((slot * s.c.H + h) * s.dk) * (int64_t)s.dv + col;
  fv x[U];
  auto read = [&](int r0) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (col < s.dv && r0 + u * RP < s.dk) x[u] = __builtin_nontemporal_load((const fv*)(st + (int64_t)(r0 + u * RP) * s.dv));
  };
  read(row);
  const T* pv = (const T*)s.v.p + b * s.v.sb + (h / s.v.group) * s.v.sh;
  float v[V], sum[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    v[e] = col + e < s.dv ? to_float(pv[col + e]) : 0.f;
    sum[e] = 0.f;
  }
  if ((int)threadIdx.x < s.dk) {
    ks[threadIdx.x] = to_float(((const T*)s.k.p + b * s.k.sb + (h / s.k.group) * s.k.sh)[threadIdx.x]);
    qs[threadIdx.x] = to_float(((const T*)s.q.p + b * s.q.sb + (h / s.q.group) * s.q.sh)[threadIdx.x]);
  }
  const Decay l = decay_power(s.c.log_decay[h], 1);
  __syncthreads();
  for (int r0 = row; r0 < s.dk; r0 += U * RP) {
    if (r0 != row) read(r0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int r = r0 + u * RP;
      if (col >= s.dv || r >= s.dk) continue;
      const float kr = ks[r], qr = qs[r];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[u][e] = l * x[u][e] + kr * v[e];
        sum[e] += qr * x[u][e];
      }
      __builtin_nontemporal_store(x[u], (fv*)(st + (int64_t)r * s.dv));
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
    linattn_step_kernel<T, 1, 16><<<grid(16), 256, 0, st>>>(s);
  else if ((int64_t)states * ((s.dv + 63) / 64) >= 512)
    linattn_step_kernel<T, 4, 16><<<grid(64), 256, 0, st>>>(s);
  else
    linattn_step_kernel<T, 4, 4><<<grid(16), 256, 0, st>>>(s);
}

}  // namespace

mdh_status launch_linattn_step(const LinattnCall& c, const HeadView& q, const HeadView& k, const HeadView& v,
                               const HeadView& o, int dk, int dv, float scale, float* state, int dtype, hipStream_t st) {
  if (c.B * c.H >= 1 << 24) return MDH_ERR_SIZE;  // 2^32 lanes
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

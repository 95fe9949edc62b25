// Linear attention with a decay for each head: md_hom(k v^T, (++, ++, prefix-sum)) over (b, h, t) whose prefix-sum operator
// combines matrices, S <- l^n S + S'.  One kernel evaluates a pass over the tokens (LinattnPass); the forward call is one
// pass, the backward call three.
//
// A workgroup owns 64 columns of the state of one (b, h) and walks the tokens one at a time, the state in registers: four
// wavefronts have a quarter of its rows each.  Two barriers and a reduction over the wavefronts per token are what it
// spends its time on.
#include "mdh_internal.h"
#include "mdh_types.h"

namespace mdh {
namespace {

constexpr int kRows = 64;  // rows of a state that a lane holds: 4 wavefronts x 64 = 256

struct Passes {
  LinattnPass p[3];
};

__device__ __forceinline__ int64_t slot_of(const LinattnCall& c, int64_t b) {
  if (!c.slots) return b;
  const int64_t s = c.slots[b];
  return s >= 0 && s < c.n_slots ? s : -1;
}

template <typename T>
__global__ __launch_bounds__(256) void linattn_tokens_kernel(LinattnCall c, Passes ps) {
  const LinattnPass& p = ps.p[blockIdx.z];
  const int col = blockIdx.y * 64 + (threadIdx.x & 63), wave = threadIdx.x >> 6;
  if ((int)blockIdx.y * 64 >= p.dc) return;
  const int h = blockIdx.x % c.H;
  const int64_t b = blockIdx.x / c.H;
  const int da = p.da, dc = p.dc;
  const bool mine = col < dc;
  const int64_t n = c.lengths ? min(max((int64_t)c.lengths[b], (int64_t)0), c.T) : c.T;
  const Decay l = decay_power(c.log_decay[h], 1);
  const int64_t slot = slot_of(c, b), at = (slot * c.H + h) * (int64_t)da * dc;
  __shared__ float as[256], bs[256], red[4][64];

  float S[kRows];
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const int i = 4 * j + wave;
    S[j] = p.s_in && slot >= 0 && mine && i < da ? p.s_in[at + (p.s_in_t ? (int64_t)col * da + i : (int64_t)i * dc + col)] : 0.f;
  }
  const T* pa = (const T*)p.a.p + b * p.a.sb + (h / p.a.group) * p.a.sh;
  const T* pb = (const T*)p.b.p + b * p.b.sb + (h / p.b.group) * p.b.sh;
  const T* pc = (const T*)p.c.p + b * p.c.sb + (h / p.c.group) * p.c.sh;
  const int64_t out0 = b * p.out.sb + (h / p.out.group) * p.out.sh + col;
  auto put = [&](int64_t t, float v) {
    if (p.out_f32)
      ((float*)p.out.p)[out0 + t * p.out.st] = v;
    else
      ((T*)p.out.p)[out0 + t * p.out.st] = from_float<T>(v);
  };
  for (int64_t i = 0; i < n; ++i) {
    const int64_t t = p.rev ? n - 1 - i : i;
    __syncthreads();
    if ((int)threadIdx.x < da) {
      as[threadIdx.x] = to_float(pa[t * p.a.st + threadIdx.x]);
      bs[threadIdx.x] = to_float(pb[t * p.b.st + threadIdx.x]);
    }
    const float x = mine ? p.scale_u * to_float(pc[t * p.c.st + col]) : 0.f;
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < kRows; ++j) {
      const int r = 4 * j + wave;
      if (r < da) {
        S[j] = (p.shift ? l * S[j] : S[j]) + bs[r] * x;
        sum += as[r] * S[j];
        if (!p.shift) S[j] = l * S[j];
      }
    }
    red[wave][threadIdx.x & 63] = sum;
    __syncthreads();
    if (wave == 0 && mine) put(t, p.scale_r * (red[0][threadIdx.x] + red[1][threadIdx.x] + red[2][threadIdx.x] + red[3][threadIdx.x]));
  }
  for (int64_t t = n + wave; t < c.T; t += 4)
    if (mine) put(t, 0.f);
  if (p.s_out && slot >= 0 && mine)
#pragma unroll
    for (int j = 0; j < kRows; ++j)
      if (4 * j + wave < da) p.s_out[at + (int64_t)(4 * j + wave) * dc + col] = S[j];
}

template <typename T>
__global__ __launch_bounds__(256) void linattn_share_kernel(const float* __restrict__ src, HeadView dst, int64_t T_, int H, int heads,
                                                            int d, int64_t total) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;  // (b, t, shared head, channel)
  if (i >= total) return;
  const int ch = (int)(i % d), g = H / heads;
  const int64_t r = i / d, hs = r % heads, bt = r / heads;
  float sum = 0.f;
  for (int j = 0; j < g; ++j) sum += src[(bt * H + hs * g + j) * d + ch];
  ((T*)dst.p)[bt / T_ * dst.sb + bt % T_ * dst.st + hs * dst.sh + ch] = from_float<T>(sum);
}

}  // namespace

mdh_status launch_linattn_pass(const LinattnCall& c, const LinattnPass* passes, int n, int dtype, hipStream_t st) {
  Passes ps;
  int dc = 0;
  for (int i = 0; i < n; ++i) {
    ps.p[i] = passes[i];
    if (passes[i].dc > dc) dc = passes[i].dc;
  }
  if (c.B * c.H > 0x7fffffff) return MDH_ERR_SIZE;
  const dim3 grid((unsigned)(c.B * c.H), (dc + 63) / 64, n);
  clear_stale_error();
  if (dtype == MDH_BF16)
    linattn_tokens_kernel<bf16><<<grid, 256, 0, st>>>(c, ps);
  else
    linattn_tokens_kernel<float><<<grid, 256, 0, st>>>(c, ps);
  return launch_status();
}

mdh_status launch_linattn_share(const LinattnCall& c, const float* src, int d, const HeadView& dst, int heads, int dtype,
                                hipStream_t st) {
  const int64_t total = c.B * c.T * heads * d;
  if (total == 0) return MDH_OK;
  const int64_t blocks = cdiv(total, 256);
  if (blocks > 0x7fffffff) return MDH_ERR_SIZE;
  clear_stale_error();
  if (dtype == MDH_BF16)
    linattn_share_kernel<bf16><<<dim3((unsigned)blocks), 256, 0, st>>>(src, dst, c.T, c.H, heads, d, total);
  else
    linattn_share_kernel<float><<<dim3((unsigned)blocks), 256, 0, st>>>(src, dst, c.T, c.H, heads, d, total);
  return launch_status();
}

}  // namespace mdh

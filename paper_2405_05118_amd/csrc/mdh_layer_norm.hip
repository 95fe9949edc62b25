// Layer norm of rows, with the sum that a residual stream takes in front of it: s = x + residual, y = (s - mean) rstd w + b.
// A few operations a value: bound by memory, or by a launch.  16384 rows of 4096 bf16 with the stream: forward 101 us, backward 111
// (537 MB each: 5.3 and 4.8 TB/s), 5 for the parameters' sums.
//
// A row is read once: L lanes (8 to 1024) hold it, P pieces of 16 bytes each, and exchange two sums.  Where the mean
// is large against the spread it is put right by the sum of the differences: equal values have that value as their mean and the
// variance 0 whatever their sum was rounded to.  Wider rows than
// 16384 are read again for every sum.  In the backward call a workgroup keeps its columns and walks the rows, the next one's loads under
// way, its share of the gradients of weight and bias in registers; one row of the workspace for each workgroup, added up in order by a second launch.
#include "mdh_internal.h"
#include "mdh_vec.h"

namespace mdh {
namespace {

constexpr int kRegisterRow = 16384;  // widest row that lanes hold

template <typename T>
__device__ __forceinline__ T* at(const RowView& v, int64_t row, int ch) {
  return (T*)const_cast<void*>(v.p) + row * v.stride + ch;
}

// sums of two values over the L lanes of a row, the same for all of them.  `turn` alternates between two places in LDS.
template <int L>
__device__ __forceinline__ void row_sums(float& a, float& b, int& turn) {
#pragma unroll
  for (int d = 1; d < (L < 64 ? L : 64); d *= 2) a += __shfl_xor(a, d), b += __shfl_xor(b, d);
  if constexpr (L > 64) {
    __shared__ float part[2][2][L / 64];
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) part[turn][0][wave] = a, part[turn][1][wave] = b;
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int i = 0; i < L / 64; ++i) a += part[turn][0][i], b += part[turn][1][i];
    turn ^= 1;
  }
}

struct Moments {
  float mean, rstd;
};
// from the sum of a row: `differ` gives the lane's sums of differences from a mean and of their squares, `scaled` that of its values
// times a factor, for rows whose sum is past the largest number
template <int L, typename F, typename G>
__device__ __forceinline__ Moments moments(float sum, int C, float eps, int& turn, F differ, G scaled) {
  constexpr float kLargest = 3.40282347e38f;
  float none = 0.f, d = 0.f, d2 = 0.f;
  row_sums<L>(sum, none, turn);
  const float over = 1.f / (float)C;
  float mean = sum * over;
  if (!(fabsf(sum) <= kLargest)) {  // (the same for all lanes of the row)
    float half = scaled(0.5f * over);
    row_sums<L>(half, none, turn);
    mean = fabsf(half) <= kLargest ? fminf(fmaxf(2.f * half, -kLargest), kLargest) : half;  // (infinity and NaN stay)
  }
  asm("" : "+v"(mean));  // (rounded here: fused into the differences, it would be another number than the one that is put right)
  differ(mean, d, d2);
  row_sums<L>(d, d2, turn);
  float off = d * over;
  if (!(d2 <= kLargest)) {
    // squares past the largest number: of values that far apart (a variance of infinity), or of what the mean's rounding came to, which
    // is put right first
    if (fabsf(off) <= kLargest) mean += off;
    d = d2 = 0.f;
    differ(mean, d, d2);
    row_sums<L>(d, d2, turn);
    off = 0.f;
  }
  const float var = fmaxf(d2 * over - off * off, 0.f);
  // (means within 16 times the spread are right as they are: the differences' own roundings would be added to them)
  if (mean * mean > 256.f * var) mean += off;
  // NaN and infinity stay: fmaxf would drop NaN
  return Moments{mean, 1.f / sqrtf((d2 == d2 ? var : d2) + eps)};
}

template <typename T, int L, int P>
__global__ __launch_bounds__(L > 256 ? L : 256) void layer_norm_kernel(LayerNormCall c) {
  constexpr int V = kLaneValues<T>, R = (L > 256 ? L : 256) / L;
  const int l = threadIdx.x % L;
  const int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L;
  int turn = 0;
  const bool live = row < c.rows;
  Word4 raw[P], res[P];
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int ch = (k * L + l) * V, left = live ? c.C - ch : 0;
    raw[k] = left > 0 ? load_row<T>(at<T>(c.x, row, ch), left) : (Word4){0, 0, 0, 0};
    if (c.residual.p) res[k] = left > 0 ? load_row<T>(at<T>(c.residual, row, ch), left) : (Word4){0, 0, 0, 0};
  }
  float x[P][V], sum = 0.f;
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int ch = (k * L + l) * V, left = live ? c.C - ch : 0;
    unpack_row<T>(raw[k], x[k]);
    if (c.residual.p) {
      float r[V];
      unpack_row<T>(res[k], r);
#pragma unroll
      for (int i = 0; i < V; ++i) x[k][i] += r[i];
      raw[k] = pack_row<T>(x[k]);  // the stream in its own type is what is normalised
      unpack_row<T>(raw[k], x[k]);
      if (left > 0) store_row<T>(at<T>(c.total, row, ch), left, raw[k]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sum += x[k][i];
  }
  const Moments m = moments<L>(sum, c.C, c.eps, turn, [&](float mean, float& d, float& d2) {
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i)
        if ((k * L + l) * V + i < c.C) {
          const float e = x[k][i] - mean;
          d += e, d2 = fmaf(e, e, d2);
        }
  }, [&](float factor) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) s = fmaf(x[k][i], factor, s);
    return s;
  });
  if (!live) return;
  if (l == 0) {
    if (c.mean) c.mean[row] = m.mean;
    if (c.rstd) c.rstd[row] = m.rstd;
  }
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int ch = (k * L + l) * V, left = c.C - ch;
    if (left <= 0) continue;
    float w[V], b[V], y[V];
    load_params<V>(c.weight ? c.weight + ch : nullptr, left, 1.f, w);
    load_params<V>(c.bias ? c.bias + ch : nullptr, left, 0.f, b);
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] = fmaf((x[k][i] - m.mean) * m.rstd, w[i], b[i]);
    store_row<T>(at<T>(c.y, row, ch), left, pack_row<T>(y));
  }
}

// rows of any width, read three times
constexpr int kWide = 1024;
template <typename T>
__global__ __launch_bounds__(kWide) void layer_norm_wide_kernel(LayerNormCall c) {
  constexpr int V = kLaneValues<T>;
  const int64_t row = blockIdx.x;
  int turn = 0;
  float sum = 0.f;
  for (int ch = threadIdx.x * V; ch < c.C; ch += kWide * V) {
    const int left = c.C - ch;
    float x[V];
    unpack_row<T>(load_row<T>(at<T>(c.x, row, ch), left), x);
    if (c.residual.p) {
      float r[V];
      unpack_row<T>(load_row<T>(at<T>(c.residual, row, ch), left), r);
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] += r[i];
      const Word4 s = pack_row<T>(x);
      unpack_row<T>(s, x);
      store_row<T>(at<T>(c.total, row, ch), left, s);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sum += x[i];
  }
  const RowView& from = c.residual.p ? c.total : c.x;  // a lane reads what it wrote itself
  const Moments m = moments<kWide>(sum, c.C, c.eps, turn, [&](float mean, float& d, float& d2) {
    for (int ch = threadIdx.x * V; ch < c.C; ch += kWide * V) {
      float x[V];
      unpack_row<T>(load_row<T>(at<T>(from, row, ch), c.C - ch), x);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (ch + i < c.C) {
          const float e = x[i] - mean;
          d += e, d2 = fmaf(e, e, d2);
        }
    }
  }, [&](float factor) {
    float s = 0.f;
    for (int ch = threadIdx.x * V; ch < c.C; ch += kWide * V) {
      float x[V];
      unpack_row<T>(load_row<T>(at<T>(from, row, ch), c.C - ch), x);
#pragma unroll
      for (int i = 0; i < V; ++i) s = fmaf(x[i], factor, s);
    }
    return s;
  });
  if (threadIdx.x == 0) {
    if (c.mean) c.mean[row] = m.mean;
    if (c.rstd) c.rstd[row] = m.rstd;
  }
  for (int ch = threadIdx.x * V; ch < c.C; ch += kWide * V) {
    const int left = c.C - ch;
    float x[V], w[V], b[V], y[V];
    unpack_row<T>(load_row<T>(at<T>(from, row, ch), left), x);
    load_params<V>(c.weight ? c.weight + ch : nullptr, left, 1.f, w);
    load_params<V>(c.bias ? c.bias + ch : nullptr, left, 0.f, b);
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] = fmaf((x[i] - m.mean) * m.rstd, w[i], b[i]);
    store_row<T>(at<T>(c.y, row, ch), left, pack_row<T>(y));
  }
}

// ---- gradients: t = d_y w, d_s = rstd (t - mean(t) - xh mean(t xh)) + d_total
template <typename T, int L, int P>
__global__ __launch_bounds__(L > 256 ? L : 256) void layer_norm_backward_kernel(LayerNormCall c) {
  constexpr int V = kLaneValues<T>, NT = L > 256 ? L : 256, R = NT / L;
  const int l = threadIdx.x % L;
  int turn = 0;
  float w[P][V], dw[P][V], db[P][V];
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int ch = (k * L + l) * V, left = c.C - ch;
    load_params<V>(c.weight && left > 0 ? c.weight + ch : nullptr, left, 1.f, w[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0.f;
  }
  const float over = 1.f / (float)c.C;
  struct Row {
    Word4 x[P], y[P], t[P];
    float mean, rstd;
  };
  // the next row is under way while one is worked on
  auto load = [&](Row& r, int64_t row) {
    const bool live = row < c.rows;
    r.mean = live ? c.mean[row] : 0.f, r.rstd = live ? c.rstd[row] : 0.f;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const int ch = (k * L + l) * V, left = live ? c.C - ch : 0;
      r.x[k] = r.y[k] = r.t[k] = (Word4){0, 0, 0, 0};
      if (left <= 0) continue;
      r.x[k] = load_part<T>(at<T>(c.x, row, ch), left, ch >= V);
      r.y[k] = load_part<T>(at<T>(c.y, row, ch), left, ch >= V);
      if (c.dtotal.p) r.t[k] = load_part<T>(at<T>(c.dtotal, row, ch), left, ch >= V);
    }
  };
  constexpr bool AHEAD = L < 1024;  // (1024 lanes have 128 registers each)
  const int64_t step = (int64_t)gridDim.x * R;
  int64_t first = (int64_t)blockIdx.x * R;
  Row next;
  if (AHEAD && first < c.rows) load(next, first + threadIdx.x / L);
  for (; first < c.rows; first += step) {
    const int64_t row = first + threadIdx.x / L;
    if (!AHEAD) load(next, row);
    Row r = next;
    if (row < c.rows)
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const int ch = (k * L + l) * V, left = c.C - ch;
        r.x[k] = part_of<T>(r.x[k], left, ch >= V), r.y[k] = part_of<T>(r.y[k], left, ch >= V), r.t[k] = part_of<T>(r.t[k], left, ch >= V);
      }
    if (AHEAD && first + step < c.rows) load(next, row + step);
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      float x[V], dy[V];
      unpack_row<T>(r.x[k], x);
      unpack_row<T>(r.y[k], dy);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float xh = (k * L + l) * V + i < c.C ? (x[i] - r.mean) * r.rstd : 0.f, t = dy[i] * w[k][i];
        s1 += t, s2 = fmaf(t, xh, s2);
        dw[k][i] = fmaf(dy[i], xh, dw[k][i]), db[k][i] += dy[i];
      }
    }
    row_sums<L>(s1, s2, turn);
    s1 *= over, s2 *= over;
    if (row >= c.rows) continue;
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const int ch = (k * L + l) * V, left = c.C - ch;
      if (left <= 0) continue;
      float x[V], dy[V], dt[V], dx[V];
      unpack_row<T>(r.x[k], x);
      unpack_row<T>(r.y[k], dy);
      unpack_row<T>(r.t[k], dt);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float xh = (x[i] - r.mean) * r.rstd;
        dx[i] = fmaf(r.rstd, dy[i] * w[k][i] - s1 - xh * s2, dt[i]);
      }
      store_row<T>(at<T>(c.dx, row, ch), left, pack_row<T>(dx));
    }
  }
  if (!c.dweight && !c.dbias) return;
  // the rows that a workgroup has at once, in order
  float* part = (float*)c.ws + (int64_t)blockIdx.x * 2 * c.C;
  __shared__ float sums[R > 1 ? NT / 64 : 1][R > 1 ? 64 : 1][V];
#pragma unroll
  for (int k = 0; k < P; ++k) {
    const int ch = (k * L + l) * V, left = c.C - ch;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float v[V];
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = which ? db[k][i] : dw[k][i];
      if constexpr (R > 1) {
#pragma unroll
        for (int d = L; d < 64; d *= 2)
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] += __shfl_xor(v[i], d);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) sums[threadIdx.x >> 6][threadIdx.x & 63][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (sums[0][l][i] + sums[1][l][i]) + (sums[2][l][i] + sums[3][l][i]);
      }
      if ((int)threadIdx.x < L && left > 0) store_params<V>(part + which * (int64_t)c.C + ch, left, v);
    }
  }
}

// rows of any width: read twice, a lane's columns of the workspace's row added to row by row
template <typename T>
__global__ __launch_bounds__(kWide) void layer_norm_wide_backward_kernel(LayerNormCall c) {
  constexpr int V = kLaneValues<T>;
  int turn = 0;
  const float over = 1.f / (float)c.C;
  const bool sums = c.dweight || c.dbias;
  float* part = (float*)c.ws + (int64_t)blockIdx.x * 2 * c.C;
  for (int64_t row = blockIdx.x; row < c.rows; row += gridDim.x) {
    const float mean = c.mean[row], rstd = c.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int ch = threadIdx.x * V; ch < c.C; ch += kWide * V) {
      const int left = c.C - ch;
      float x[V], dy[V], w[V], dw[V], db[V];
      unpack_row<T>(load_row<T>(at<T>(c.x, row, ch), left), x);
      unpack_row<T>(load_row<T>(at<T>(c.y, row, ch), left), dy);
      load_params<V>(c.weight ? c.weight + ch : nullptr, left, 1.f, w);
      const bool more = sums && row != blockIdx.x;
      load_params<V>(more ? part + ch : nullptr, left, 0.f, dw);
      load_params<V>(more ? part + c.C + ch : nullptr, left, 0.f, db);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float xh = ch + i < c.C ? (x[i] - mean) * rstd : 0.f, t = dy[i] * w[i];
        s1 += t, s2 = fmaf(t, xh, s2);
        dw[i] = fmaf(dy[i], xh, dw[i]), db[i] += dy[i];
      }
      if (sums) {
        store_params<V>(part + ch, left, dw);
        store_params<V>(part + c.C + ch, left, db);
      }
    }
    row_sums<kWide>(s1, s2, turn);
    s1 *= over, s2 *= over;
    for (int ch = threadIdx.x * V; ch < c.C; ch += kWide * V) {
      const int left = c.C - ch;
      float x[V], dy[V], w[V], dt[V], dx[V];
      unpack_row<T>(load_row<T>(at<T>(c.x, row, ch), left), x);
      unpack_row<T>(load_row<T>(at<T>(c.y, row, ch), left), dy);
      unpack_row<T>(c.dtotal.p ? load_row<T>(at<T>(c.dtotal, row, ch), left) : (Word4){0, 0, 0, 0}, dt);
      load_params<V>(c.weight ? c.weight + ch : nullptr, left, 1.f, w);
#pragma unroll
      for (int i = 0; i < V; ++i) dx[i] = fmaf(rstd, dy[i] * w[i] - s1 - (x[i] - mean) * rstd * s2, dt[i]);
      store_row<T>(at<T>(c.dx, row, ch), left, pack_row<T>(dx));
    }
  }
}

// Lanes of a row and pieces of a lane: the fewest that hold it
struct Shape {
  int L, P;  // L = 0: wider than lanes hold
};
Shape shape_of(const LayerNormCall& c, bool backward) {
  if (c.C > kRegisterRow) return {0, 0};
  const int n = (int)cdiv(c.C, c.dtype == MDH_BF16 ? 8 : 4);
  if (n <= 8) return {8, 1};
  if (n <= 32) return {32, 1};
  if (n <= 64) return {64, 1};
  if (n <= 128) return {64, 2};
  // (backward a lane holds its weights and two sums besides: one piece each where that can be)
  if (n <= 256) return backward ? Shape{256, 1} : Shape{64, 4};
  if (n <= 512) return backward ? Shape{512, 1} : Shape{256, 2};
  if (n <= 1024) return backward ? Shape{512, 2} : Shape{256, 4};
  if (n <= 2048) return {1024, 2};
  return backward ? Shape{0, 0} : Shape{1024, 4};
}
int64_t row_groups(const LayerNormCall& c, bool backward) {  // workgroups that have a row
  const Shape s = shape_of(c, backward);
  return s.L && s.L < 256 ? cdiv(c.rows, 256 / s.L) : c.rows;
}
int64_t backward_groups(const LayerNormCall& c) {
  const int64_t n = row_groups(c, true);
  return n < 512 ? n : 512;
}

template <typename T, int L, int P>
void go(const LayerNormCall& c, bool backward, unsigned blocks, hipStream_t st) {
  constexpr int NT = L > 256 ? L : 256;
  if (backward)
    layer_norm_backward_kernel<T, L, P><<<blocks, NT, 0, st>>>(c);
  else
    layer_norm_kernel<T, L, P><<<blocks, NT, 0, st>>>(c);
}
template <typename T>
mdh_status launch(const LayerNormCall& c, bool backward, hipStream_t st) {
  const Shape s = shape_of(c, backward);
  const int64_t n = backward ? backward_groups(c) : row_groups(c, false);
  if (n * (s.L == 0 || s.L > 256 ? 1024 : 256) >= (int64_t)1 << 32) return MDH_ERR_SIZE;
  const unsigned blocks = (unsigned)n;
  clear_stale_error();
  switch (s.L * 8 + s.P) {
    case 8 * 8 + 1: go<T, 8, 1>(c, backward, blocks, st); break;
    case 32 * 8 + 1: go<T, 32, 1>(c, backward, blocks, st); break;
    case 64 * 8 + 1: go<T, 64, 1>(c, backward, blocks, st); break;
    case 64 * 8 + 2: go<T, 64, 2>(c, backward, blocks, st); break;
    case 64 * 8 + 4: layer_norm_kernel<T, 64, 4><<<blocks, 256, 0, st>>>(c); break;
    case 256 * 8 + 2: layer_norm_kernel<T, 256, 2><<<blocks, 256, 0, st>>>(c); break;
    case 256 * 8 + 4: layer_norm_kernel<T, 256, 4><<<blocks, 256, 0, st>>>(c); break;
    case 256 * 8 + 1: layer_norm_backward_kernel<T, 256, 1><<<blocks, 256, 0, st>>>(c); break;
    case 512 * 8 + 1: layer_norm_backward_kernel<T, 512, 1><<<blocks, 512, 0, st>>>(c); break;
    case 512 * 8 + 2: layer_norm_backward_kernel<T, 512, 2><<<blocks, 512, 0, st>>>(c); break;
    case 1024 * 8 + 2: go<T, 1024, 2>(c, backward, blocks, st); break;
    case 1024 * 8 + 4:
      if constexpr (sizeof(T) == 4) layer_norm_kernel<T, 1024, 4><<<blocks, 1024, 0, st>>>(c);  // (bf16 rows of that many pieces are wide)
      break;
    default:
      if (backward)
        layer_norm_wide_backward_kernel<T><<<blocks, kWide, 0, st>>>(c);
      else
        layer_norm_wide_kernel<T><<<blocks, kWide, 0, st>>>(c);
  }
  return launch_status();
}

}  // namespace

size_t layer_norm_workspace(const LayerNormCall& c) {
  return c.rows ? (size_t)backward_groups(c) * 2 * (size_t)c.C * sizeof(float) : 0;
}
mdh_status launch_layer_norm(const LayerNormCall& c, hipStream_t st) {
  return c.dtype == MDH_BF16 ? launch<bf16>(c, false, st) : launch<float>(c, false, st);
}
mdh_status launch_layer_norm_backward(const LayerNormCall& c, hipStream_t st) {
  if (c.rows) {
    const mdh_status r = c.dtype == MDH_BF16 ? launch<bf16>(c, true, st) : launch<float>(c, true, st);
    if (r != MDH_OK) return r;
  }
  if (!c.dweight && !c.dbias) return MDH_OK;
  return launch_sum_rows((const float*)c.ws, c.rows ? backward_groups(c) : 0, 2 * (int64_t)c.C,
                         {{c.dweight, c.C}, {c.dbias, c.C}, {nullptr, 0}}, st);
}

}  // namespace mdh

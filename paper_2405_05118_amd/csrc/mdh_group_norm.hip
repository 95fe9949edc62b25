// Group norm with an activation and a gate, channels last: md_hom over (n, s, c) whose statistics combine (count, mean, sum of
// squared differences) of parts.  A few operations a value: bound by memory, or by a launch where there is little of it.
//
// Two de-compositions.  P = D / V: pieces of a group of D channels, V channels each (16 bytes where alignment and D allow).
//   teams  (S = 1, P <= 256: the heads of tokens) a group of a row is 1 to 64 lanes with up to four pieces each: read once,
//          statistics by exchanges between lanes, written.  In the backward call a team keeps its group and walks rows, its
//          channels' share of the gradients of weight and bias in registers.
//   slabs  (images, and rows of very wide groups) a workgroup owns up to 256 pieces of channels -- whole groups, or a part of
//          one -- of a share of the positions.  A first launch leaves its statistics (backward: its sums) in the workspace, the
//          second combines the shares of its groups and writes.  What was read is still in the chip's cache for images of up
//          to some hundred MB.
// Sums over shares are taken in a fixed order.  Gradients of weight and bias: one row of the workspace for each share, summed
// by the workgroups of the second launch that come after those for the images (teams: a launch of their own).
//
// Measured, bf16 unless said, three sets of inputs in turn.  Teams: 16384 rows of 4096 in 32 groups with a gate 77 us (5.2 TB/s),
// their gradients 148 (4.5 TB/s over five tensors); one such row 3.4 in its kernel.  Slabs: 8 x 128 x 128 x 256 in 32 groups, silu,
// 51 us (67 MB read, read again and written: 3.9 TB/s), trained 143, of which a kernel trace gives 24 + 31 to the forward call and 43 +
// 47 to the gradients; fp32 16 x 56 x 56 x 64 in 32 groups 17 (7 + 11).  Stores that leave the caches alone are up to a
// tenth faster (16384 rows, trained: 5 %) and cost whoever reads the output next as much (2048 rows and a sum after it: 20.1 us for
// 19.5): not taken.
#include "mdh_act.h"
#include "mdh_internal.h"
#include "mdh_types.h"

#include <type_traits>

namespace mdh {
namespace {

constexpr int kLanes = 256;

// ---- V values of a lane
template <int BYTES>
struct Bits;
template <>
struct Bits<2> { typedef uint16_t type; };
template <>
struct Bits<4> { typedef uint32_t type; };
template <>
struct Bits<8> { typedef uint32_t type __attribute__((ext_vector_type(2))); };
template <>
struct Bits<16> { typedef uint32_t type __attribute__((ext_vector_type(4))); };

template <int W, typename B>
__device__ __forceinline__ uint32_t word(const B& b, int i) {
  if constexpr (W == 1)
    return (uint32_t)b;
  else
    return b[i];
}
template <typename T, int V>
using Raw = typename Bits<sizeof(T) * V>::type;  // as they are in memory
template <typename T, int V>
__device__ __forceinline__ void expand(const Raw<T, V>& b, float (&x)[V]) {
  constexpr int W = sizeof(T) * V < 4 ? 1 : sizeof(T) * V / 4;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (sizeof(T) == 4)
      x[i] = __uint_as_float(word<W>(b, i));
    else
      x[i] = __uint_as_float(i & 1 ? word<W>(b, i / 2) & 0xffff0000u : word<W>(b, i / 2) << 16);
  }
}
template <typename T, int V>
__device__ __forceinline__ void load(const T* p, float (&x)[V]) {
  expand<T, V>(*(const Raw<T, V>*)p, x);
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const float (&x)[V]) {
  typedef typename Bits<sizeof(T) * V>::type B;
  B b;
  if constexpr (V == 1) {
    b = sizeof(T) == 4 ? (B)__float_as_uint(x[0]) : (B)pack_bf16(x[0], 0.f);
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] = __float_as_uint(x[i]);
  } else if constexpr (V == 2) {
    b = pack_bf16(x[0], x[1]);
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 2) b[i / 2] = pack_bf16(x[i], x[i + 1]);
  }
  *(B*)p = b;
}
template <int V>
__device__ __forceinline__ void params(const float* p, int ch, float fill, float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = p ? p[ch + i] : fill;
}
template <typename T>
__device__ __forceinline__ T* at(const RowView& v, int64_t row, int ch) {
  return (T*)const_cast<void*>(v.p) + row * v.stride + ch;
}

// ---- what a value gives: forward
template <typename T, int V>
__device__ __forceinline__ void result(const GroupNormCall& c, int64_t row, int ch, const float (&x)[V], const Raw<T, V>& gate,
                                       float mean, float rstd, const float (&w)[V], const float (&b)[V]) {
  float z[V], in[V], y[V];
#pragma unroll
  for (int i = 0; i < V; ++i) z[i] = in[i] = (x[i] - mean) * rstd * w[i] + b[i];
  if (c.gate.p) expand<T, V>(gate, in);
  act_of<V>(c.act, in, y);
  if (c.gate.p)
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] *= z[i];
  store<T, V>(at<T>(c.y, row, ch), y);
}

// ---- and backward: gradient of z; the gate's where there is one
template <typename T, int V>
__device__ __forceinline__ void grad_z(const GroupNormCall& c, int64_t row, int ch, const float (&xh)[V], const float (&dy)[V],
                                       const float (&g)[V], const float (&w)[V], const float (&b)[V], float (&dz)[V], bool write_gate) {
  float z[V], in[V], a[V], s[V];
  const bool gated = c.gate.p != nullptr;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    z[i] = xh[i] * w[i] + b[i];
    const float gi = g[i], zi = z[i];  // (values: a choice of places would put the arrays in memory)
    in[i] = gated ? gi : zi;
  }
  act_slope<V>(c.act, in, a, s);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float ai = a[i], si = s[i];
    dz[i] = dy[i] * (gated ? ai : si);
    s[i] *= dy[i] * z[i];
  }
  if (gated && write_gate) store<T, V>(at<T>(c.dgate, row, ch), s);
}

// Statistics.  A mean from one sum is off by some ulps, and a group that is almost one value (a large mean, a variance below eps)
// gets that times rstd.  The sum of the differences from it says by how much: it puts the mean right to half an ulp -- to the value
// itself where there is only one.  (The mean is rounded before it is subtracted, so that the sum belongs to what was rounded.)
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// ============================================================================================ teams

struct Teams {
  int L;         // lanes of a team, a power of two
  int across;    // teams side by side, of neighbouring groups; kLanes / (L * across) rows at once
  int rows;      // rows of a workgroup
  int shares;    // workgroups along the rows
  float* parts;  // backward: [share][2][C]
};

__device__ __forceinline__ float team_sum(float v, int L) {
  for (int d = 1; d < L; d *= 2) v += __shfl_xor(v, d);
  return v;
}

template <typename T, int V, int NP>
__global__ __launch_bounds__(kLanes) void teams_forward_kernel(GroupNormCall c, Teams t) {
  const int D = c.C / c.G, P = D / V, l = threadIdx.x % t.L, team = threadIdx.x / t.L;
  const int g = blockIdx.x * t.across + team % t.across, step = kLanes / (t.L * t.across);
  if (g >= c.G || team >= t.across * step) return;
  const int64_t first = (int64_t)blockIdx.y * t.rows + team / t.across, end = min(c.N, (int64_t)(blockIdx.y + 1) * t.rows);
  const float per = 1.f / (float)D;
  // a row's operands, read while the row before it is worked on
  struct Row {
    Raw<T, V> x[NP], gate[NP];
  };
  auto read = [&](int64_t r, Row& row) {
    if (r >= end) return;
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      if (l + k * t.L >= P) continue;
      row.x[k] = *(const Raw<T, V>*)at<T>(c.x, r, g * D + (l + k * t.L) * V);
      if (c.gate.p) row.gate[k] = *(const Raw<T, V>*)at<T>(c.gate, r, g * D + (l + k * t.L) * V);
    }
  };
  Row next;
  read(first, next);
  float w[NP][V], b[NP][V];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int ch = g * D + min(l + k * t.L, P - 1) * V;
    params<V>(c.weight, ch, 1.f, w[k]);
    params<V>(c.bias, ch, 0.f, b[k]);
  }
  for (int64_t r = first; r < end; r += step) {
    const Row row = next;
    read(r + step, next);
    float x[NP][V];
#pragma unroll
    for (int k = 0; k < NP; ++k)
      if (l + k * t.L < P) expand<T, V>(row.x[k], x[k]);
    auto sum = [&](auto term) {  // of the group
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < NP; ++k)
        if (l + k * t.L < P)
#pragma unroll
          for (int i = 0; i < V; ++i) s += term(x[k][i]);
      return team_sum(s, t.L);
    };
    float mean = rounded_product(sum([](float v) { return v; }), per);
    auto square = [&](float v) { return (v - mean) * (v - mean); };
    float var = sum(square) * per;
    // The differences are summed for few groups only: a deviation below 2^-15 of the mean is what its rounding may come to.  (For all
    // of them, beside the squares: 4096 rows of 10 groups of 100 values 18.9 us for 16.0, 16384 rows of 4096 82 for 77.)
    if (!(var > mean * mean * 0x1p-30f)) {
      mean += sum([&](float v) { return v - mean; }) * per;
      var = sum(square) * per;
    }
    const float rstd = 1.f / sqrtf(var + c.eps);
#pragma unroll
    for (int k = 0; k < NP; ++k)
      if (l + k * t.L < P) result<T, V>(c, r, g * D + (l + k * t.L) * V, x[k], row.gate[k], mean, rstd, w[k], b[k]);
    if (l == 0) {
      if (c.mean) c.mean[r * c.G + g] = mean;
      if (c.rstd) c.rstd[r * c.G + g] = rstd;
    }
  }
}

template <typename T, int V, int NP>
__global__ __launch_bounds__(kLanes) void teams_backward_kernel(GroupNormCall c, Teams t) {
  __shared__ float sums[2][kLanes * V];
  const int D = c.C / c.G, P = D / V, l = threadIdx.x % t.L, team = threadIdx.x / t.L;
  const int g = blockIdx.x * t.across + team % t.across, step = kLanes / (t.L * t.across), lane_row = team / t.across;
  const int64_t first = (int64_t)blockIdx.y * t.rows + lane_row, end = min(c.N, (int64_t)(blockIdx.y + 1) * t.rows);
  const bool mine = g < c.G && lane_row < step;
  const float per = 1.f / (float)D;
  float w[NP][V], b[NP][V], dw[NP][V], db[NP][V];
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int ch = min(g, c.G - 1) * D + min(l + k * t.L, P - 1) * V;
    params<V>(c.weight, ch, 1.f, w[k]);
    params<V>(c.bias, ch, 0.f, b[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) dw[k][i] = db[k][i] = 0.f;
  }
  // a row's operands, read while the row before it is worked on
  struct Row {
    Raw<T, V> x[NP], dy[NP], gate[NP];
    float mean, rstd;
  };
  auto read = [&](int64_t r, Row& row) {
    if (r >= end) return;
    row.mean = c.mean[r * c.G + g];
    row.rstd = c.rstd[r * c.G + g];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      const int ch = g * D + (l + k * t.L) * V;
      if (l + k * t.L >= P) continue;
      row.x[k] = *(const Raw<T, V>*)at<T>(c.x, r, ch);
      row.dy[k] = *(const Raw<T, V>*)at<T>(c.y, r, ch);
      if (c.gate.p) row.gate[k] = *(const Raw<T, V>*)at<T>(c.gate, r, ch);
    }
  };
  Row next;
  if (mine) {
    read(first, next);
    for (int64_t r = first; r < end; r += step) {
      const Row row = next;
      read(r + step, next);
      float xh[NP][V], dz[NP][V];
      const float mean = row.mean, rstd = row.rstd;
      float t1 = 0.f, t2 = 0.f;
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        const int ch = g * D + (l + k * t.L) * V;
        if (l + k * t.L >= P) continue;
        float dy[V], gate[V] = {};
        expand<T, V>(row.x[k], xh[k]);
        expand<T, V>(row.dy[k], dy);
        if (c.gate.p) expand<T, V>(row.gate[k], gate);
#pragma unroll
        for (int i = 0; i < V; ++i) xh[k][i] = (xh[k][i] - mean) * rstd;
        grad_z<T, V>(c, r, ch, xh[k], dy, gate, w[k], b[k], dz[k], true);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          dw[k][i] += dz[k][i] * xh[k][i];
          db[k][i] += dz[k][i];
          dz[k][i] *= w[k][i];
          t1 += dz[k][i];
          t2 += dz[k][i] * xh[k][i];
        }
      }
      t1 = team_sum(t1, t.L) * per;
      t2 = team_sum(t2, t.L) * per;
#pragma unroll
      for (int k = 0; k < NP; ++k) {
        if (l + k * t.L >= P) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) dz[k][i] = rstd * (dz[k][i] - t1 - xh[k][i] * t2);
        store<T, V>(at<T>(c.dx, r, g * D + (l + k * t.L) * V), dz[k]);
      }
    }
  }
  // over the rows of the workgroup, and out
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) {
      sums[0][threadIdx.x * V + i] = dw[k][i];
      sums[1][threadIdx.x * V + i] = db[k][i];
    }
    __syncthreads();
    if (mine && lane_row == 0 && l + k * t.L < P) {
      float* out = t.parts + (int64_t)blockIdx.y * 2 * c.C + g * D + (l + k * t.L) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float a = 0.f, s = 0.f;
        for (int row = 0; row < step; ++row) {
          a += sums[0][(threadIdx.x + row * t.L * t.across) * V + i];
          s += sums[1][(threadIdx.x + row * t.L * t.across) * V + i];
        }
        out[i] = a;
        out[c.C + i] = s;
      }
    }
  }
}

// dweight, dbias: sums over `shares` rows [2][C] of parts; 32 channels a workgroup, 8 lanes a channel
__device__ __forceinline__ void add_shares(const float* parts, int64_t shares, int C, int block, float* dweight, float* dbias,
                                           float (&red)[2][8][32]) {
  const int ch = block * 32 + (threadIdx.x & 31), lane = threadIdx.x >> 5;
  float a = 0.f, b = 0.f;
  if (ch < C)
#pragma unroll 4
    for (int64_t i = lane; i < shares; i += 8) {
      a += parts[i * 2 * C + ch];
      b += parts[i * 2 * C + C + ch];
    }
  red[0][lane][threadIdx.x & 31] = a;
  red[1][lane][threadIdx.x & 31] = b;
  __syncthreads();
  if (threadIdx.x < 64) {
    const int which = threadIdx.x >> 5, col = threadIdx.x & 31;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += red[which][i][col];
    float* out = which ? dbias : dweight;
    if (out && block * 32 + col < C) out[block * 32 + col] = s;
  }
}

__global__ __launch_bounds__(kLanes) void add_shares_kernel(const float* parts, int64_t shares, int C, float* dweight, float* dbias) {
  __shared__ float red[2][8][32];
  add_shares(parts, shares, C, blockIdx.x, dweight, dbias, red);
}

// ============================================================================================ slabs

struct Slabs {
  int groups;       // whole groups of a slab (1 where a group is several slabs)
  int per_group;    // slabs of a group
  int slabs;        // of a row
  int rows;         // positions of a share
  int shares;       // of an image
  void* stats;      // [n][group][share * per_group + slab of it]: Stat, backward Pair
  float* parts;     // backward: [n * shares + share][2][C]
  int last;         // workgroups of the images; those behind them add up parts
};

// the place of a workgroup's lane
struct SlabLane {
  int64_t n;
  int share, slab, sub, g0, groups;  // groups g0 .. g0 + groups, the sub-th part of them
  int across, down;                  // lanes along the channels and along the positions
  int c, r;                          // this one's; r >= down: idle
  int g, ch;                         // its group and first channel
  int64_t row0;                      // the share's first row
  int rows;                          // and its positions
};
template <int V>
__device__ __forceinline__ SlabLane place(const GroupNormCall& c, const Slabs& s, int block) {
  SlabLane p;
  p.slab = block % s.slabs;
  const int rest = block / s.slabs;
  p.share = rest % s.shares;
  p.n = rest / s.shares;
  const int D = c.C / c.G, P = D / V;
  p.sub = p.slab % s.per_group;
  p.g0 = p.slab / s.per_group * s.groups;
  p.groups = min(s.groups, c.G - p.g0);
  const int begin = p.sub * kLanes;
  p.across = s.per_group > 1 ? min(kLanes, P - begin) : p.groups * P;
  p.down = kLanes / p.across;
  p.c = threadIdx.x % p.across;
  p.r = threadIdx.x / p.across;
  p.g = p.g0 + (s.per_group > 1 ? 0 : p.c / P);
  p.ch = p.g0 * D + (begin + p.c) * V;
  const int64_t s0 = (int64_t)p.share * s.rows;
  p.row0 = p.n * c.S + s0;
  p.rows = (int)min(c.S - s0, (int64_t)s.rows);
  return p;
}

struct alignas(16) Stat {
  float n, mean, m2, none;
};
// Of two parts.  An empty one is passed over: merged, its mean of 0 would move the other's by the rounding of 1/n, and from
// 2^64 on square to infinity.
__device__ __forceinline__ Stat operator+(const Stat& a, const Stat& b) {
  if (b.n == 0.f) return a;
  if (a.n == 0.f) return b;
  const float n = a.n + b.n, d = b.mean - a.mean, f = b.n * __builtin_amdgcn_rcpf(n), df = d * f;
  return Stat{n, a.mean + df, a.m2 + b.m2 + df * d * a.n, 0.f};
}

// Combines val over the lanes of each group of a slab: positions first, then the group's pieces; the result is in the lane with
// r = 0 and the group's first piece.
template <typename X, typename F>
__device__ __forceinline__ X over_group(const SlabLane& p, int P, bool part, X val, X* lds, F add) {
  lds[threadIdx.x] = val;
  __syncthreads();
  int top = 1;
  while (top < p.down) top *= 2;
  for (int d = top / 2; d > 0; d /= 2) {
    if (p.r < d && p.r + d < p.down) lds[threadIdx.x] = add(lds[threadIdx.x], lds[threadIdx.x + d * p.across]);
    __syncthreads();
  }
  const int wide = part ? p.across : P, i = part ? p.c : p.c % P;
  for (int d = 1; d < wide; d *= 2) {
    if (p.r == 0 && i % (2 * d) == 0 && i + d < wide) lds[threadIdx.x] = add(lds[threadIdx.x], lds[threadIdx.x + d]);
    __syncthreads();
  }
  return lds[threadIdx.x];
}

// The sum of squares about the mean itself, from that about a mean off by a little: `taken` less, unless neither is a float.
__device__ __forceinline__ float about_mean(float squares, float taken) {
  const float rest = squares - taken;
  return rest > 0.f ? rest : taken < INFINITY ? 0.f : squares;
}

constexpr int kBatch = 4;  // positions whose loads are in flight together

template <typename T, int V>
__global__ __launch_bounds__(kLanes) void slabs_stats_kernel(GroupNormCall c, Slabs s) {
  __shared__ Stat lds[kLanes];
  const SlabLane p = place<V>(c, s, blockIdx.x);
  const int P = c.C / c.G / V;
  Stat mine{0.f, 0.f, 0.f, 0.f};
  if (p.r < p.down)
    for (int r0 = p.r; r0 < p.rows; r0 += kBatch * p.down) {
      float x[kBatch][V];
      const int n = min(kBatch, (p.rows - r0 + p.down - 1) / p.down);
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (u < n) load<T, V>(at<const T>(c.x, p.row0 + r0 + u * p.down, p.ch), x[u]);
      float sum = 0.f, off = 0.f, q = 0.f;
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (u < n)
#pragma unroll
          for (int i = 0; i < V; ++i) sum += x[u][i];
      const float count = (float)(n * V), near = sum / count;
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
        if (u < n)
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float d = x[u][i] - near;
            off += d;
            q += d * d;
          }
      const float more = off * __builtin_amdgcn_rcpf(count);
      mine = mine + Stat{count, near + more, about_mean(q, off * more), 0.f};
    }
  const Stat all = over_group(p, P, s.per_group > 1, mine, lds, [](const Stat& a, const Stat& b) { return a + b; });
  if (p.r == 0 && (s.per_group > 1 ? p.c == 0 : p.c % P == 0)) {
    ((Stat*)s.stats)[((p.n * c.G + p.g) * s.shares + p.share) * s.per_group + p.sub] = all;
  }
}

// The shares of the groups of a slab combined, in lds[group of the slab]: every group has kLanes / groups lanes, which take turns,
// eight shares of each on their way together.
template <typename X, typename F>
__device__ __forceinline__ void combine_shares(const GroupNormCall& c, const Slabs& s, const SlabLane& p, X zero, X* lds, F add) {
  const int K = s.shares * s.per_group, lanes = kLanes / p.groups, g = threadIdx.x % p.groups, lane = threadIdx.x / p.groups;
  X x = zero;
  if (lane < lanes) {
    const X* from = (const X*)s.stats + (p.n * c.G + p.g0 + g) * (int64_t)K;
    for (int k0 = lane; k0 < K; k0 += 8 * lanes) {
      X v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = from[min(k0 + u * lanes, K - 1)];
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (k0 + u * lanes < K) x = add(x, v[u]);
    }
  }
  lds[threadIdx.x] = x;
  __syncthreads();
  int top = 1;
  while (top < lanes) top *= 2;
  for (int d = top / 2; d > 0; d /= 2) {
    if (lane < d && lane + d < lanes) lds[threadIdx.x] = add(lds[threadIdx.x], lds[threadIdx.x + d * p.groups]);
    __syncthreads();
  }
}

template <typename T, int V>
__global__ __launch_bounds__(kLanes) void slabs_forward_kernel(GroupNormCall c, Slabs s) {
  __shared__ Stat lds[kLanes];
  const SlabLane p = place<V>(c, s, blockIdx.x);
  Raw<T, V> x_raw[kBatch], gate[kBatch];
  auto read = [&](int r0) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (r0 + u * p.down < p.rows) {
        x_raw[u] = *(const Raw<T, V>*)at<T>(c.x, p.row0 + r0 + u * p.down, p.ch);
        if (c.gate.p) gate[u] = *(const Raw<T, V>*)at<T>(c.gate, p.row0 + r0 + u * p.down, p.ch);
      }
  };
  if (p.r < p.down) read(p.r);  // (on its way while the statistics are combined)
  combine_shares(c, s, p, Stat{0.f, 0.f, 0.f, 0.f}, lds, [](const Stat& a, const Stat& b) { return a + b; });
  const Stat st = lds[p.g - p.g0];
  const float mean = st.mean, rstd = 1.f / sqrtf(st.m2 / st.n + c.eps);
  if (p.r >= p.down) return;
  const int P = c.C / c.G / V;
  if (p.share == 0 && p.r == 0 && p.sub == 0 && (s.per_group > 1 ? p.c == 0 : p.c % P == 0)) {
    if (c.mean) c.mean[p.n * c.G + p.g] = mean;
    if (c.rstd) c.rstd[p.n * c.G + p.g] = rstd;
  }
  float w[V], b[V];
  params<V>(c.weight, p.ch, 1.f, w);
  params<V>(c.bias, p.ch, 0.f, b);
  for (int r0 = p.r; r0 < p.rows; r0 += kBatch * p.down) {
    if (r0 != p.r) read(r0);
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (r0 + u * p.down < p.rows) {
        float x[V];
        expand<T, V>(x_raw[u], x);
        result<T, V>(c, p.row0 + r0 + u * p.down, p.ch, x, gate[u], mean, rstd, w, b);
      }
  }
}

struct alignas(8) Pair {
  float a, b;
};

constexpr int kBatchBack = 4;

// WRITE = false: sums over the positions of a share; true: the gradients
template <typename T, int V, bool WRITE>
__global__ __launch_bounds__(kLanes) void slabs_backward_kernel(GroupNormCall c, Slabs s) {
  __shared__ Pair lds[kLanes];
  __shared__ union {
    float sums[2][kLanes * V];
    float red[2][8][32];
  } u;
  if (WRITE && (int)blockIdx.x >= s.last) {
    add_shares(s.parts, c.N * s.shares, c.C, blockIdx.x - s.last, c.dweight, c.dbias, u.red);
    return;
  }
  const SlabLane p = place<V>(c, s, blockIdx.x);
  const int D = c.C / c.G, P = D / V;
  const auto add = [](const Pair& x, const Pair& y) { return Pair{x.a + y.a, x.b + y.b}; };
  float t1 = 0.f, t2 = 0.f;
  if (WRITE) {
    combine_shares(c, s, p, Pair{0.f, 0.f}, lds, add);
    const float per = 1.f / ((float)c.S * (float)D);
    t1 = lds[p.g - p.g0].a * per;
    t2 = lds[p.g - p.g0].b * per;
  }
  const float mean = c.mean[p.n * c.G + p.g], rstd = c.rstd[p.n * c.G + p.g];
  float w[V], b[V], dw[V], db[V];
  params<V>(c.weight, p.ch, 1.f, w);
  params<V>(c.bias, p.ch, 0.f, b);
#pragma unroll
  for (int i = 0; i < V; ++i) dw[i] = db[i] = 0.f;
  if (p.r < p.down)
    for (int r0 = p.r; r0 < p.rows; r0 += kBatchBack * p.down) {
      Raw<T, V> x_raw[kBatchBack], dy_raw[kBatchBack], gate_raw[kBatchBack];
      const int n = min(kBatchBack, (p.rows - r0 + p.down - 1) / p.down);
#pragma unroll
      for (int k = 0; k < kBatchBack; ++k)
        if (k < n) {
          const int64_t row = p.row0 + r0 + k * p.down;
          x_raw[k] = *(const Raw<T, V>*)at<T>(c.x, row, p.ch);
          dy_raw[k] = *(const Raw<T, V>*)at<T>(c.y, row, p.ch);
          if (c.gate.p) gate_raw[k] = *(const Raw<T, V>*)at<T>(c.gate, row, p.ch);
        }
#pragma unroll
      for (int k = 0; k < kBatchBack; ++k)
        if (k < n) {
          const int64_t row = p.row0 + r0 + k * p.down;
          float x[V], dy[V], gate[V] = {}, dz[V];
          expand<T, V>(x_raw[k], x);
          expand<T, V>(dy_raw[k], dy);
          if (c.gate.p) expand<T, V>(gate_raw[k], gate);
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] = (x[i] - mean) * rstd;
          grad_z<T, V>(c, row, p.ch, x, dy, gate, w, b, dz, WRITE);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            if (WRITE) {
              dz[i] = rstd * (dz[i] * w[i] - t1 - x[i] * t2);
            } else {
              dw[i] += dz[i] * x[i];
              db[i] += dz[i];
            }
          }
          if (WRITE) store<T, V>(at<T>(c.dx, row, p.ch), dz);
        }
    }
  if (WRITE) return;
  // over the positions of the share: each channel's sums ...
#pragma unroll
  for (int i = 0; i < V; ++i) {
    u.sums[0][threadIdx.x * V + i] = dw[i];
    u.sums[1][threadIdx.x * V + i] = db[i];
  }
  __syncthreads();
  int top = 1;
  while (top < p.down) top *= 2;
  for (int d = top / 2; d > 0; d /= 2) {
    if (p.r < d && p.r + d < p.down)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        u.sums[0][threadIdx.x * V + i] += u.sums[0][(threadIdx.x + d * p.across) * V + i];
        u.sums[1][threadIdx.x * V + i] += u.sums[1][(threadIdx.x + d * p.across) * V + i];
      }
    __syncthreads();
  }
  Pair group{0.f, 0.f};
  if (p.r == 0) {
    float* out = s.parts + (p.n * s.shares + p.share) * 2 * c.C + p.ch;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float a = u.sums[0][threadIdx.x * V + i], e = u.sums[1][threadIdx.x * V + i];
      out[i] = a;
      out[c.C + i] = e;
      group.a += e * w[i];
      group.b += a * w[i];
    }
  }
  // ... and those of the groups, weighted
  const Pair all = over_group(p, P, s.per_group > 1, group, lds, add);
  if (p.r == 0 && (s.per_group > 1 ? p.c == 0 : p.c % P == 0)) {
    ((Pair*)s.stats)[((p.n * c.G + p.g) * s.shares + p.share) * s.per_group + p.sub] = all;
  }
}

// ============================================================================================ rules

int bytes_of(const GroupNormCall& c) { return c.dtype == MDH_BF16 ? 2 : 4; }

// Channels of a lane's access for D channels a group: what divides them, of 16 bytes at most.  (No access of 8 bytes for bf16: groups
// of a multiple of 4 channels, but not of 8, take 4 bytes.  4096 rows of 16 groups of 100 channels 22 us, of 104 12.)
int widest(int D, int bytes) {
  for (int v : {8, 4, 2})
    if (v * bytes <= 16 && D % v == 0 && !(bytes == 2 && v == 4)) return v;
  return 1;
}
// and what the addresses allow
int width(const GroupNormCall& c, bool backward) {
  const int bytes = bytes_of(c);
  int v = widest(c.C / c.G, bytes);
  const RowView* all[5] = {&c.x, &c.gate, &c.y, &c.dx, &c.dgate};
  for (int i = 0; i < (backward ? 5 : 3); ++i)
    if (all[i]->p)
      while (v > 1 && ((uintptr_t)all[i]->p % (v * bytes) || all[i]->stride % v)) v = v == 8 && bytes == 2 ? 2 : v / 2;
  return v;
}

// Rows of wider groups go as images of one position, each with its own sums for the gradients of weight and bias: 16384 rows of 4096 as
// one group, bf16 with a gate, 259 us, trained 1180 with 541 MB of workspace.
bool use_teams(const GroupNormCall& c, int V) { return c.S == 1 && c.C / c.G / V <= 256; }

// pieces of a lane (four: the backward call has one wavefront a SIMD; trained, with a gate, 2048 rows of 4096 in 2 groups take 65 us,
// in 32 groups 42)
int pieces(const GroupNormCall& c, int V) {
  const int P = c.C / c.G / V;
  return P <= 64 ? 1 : P <= 128 ? 2 : 4;
}

Teams teams_of(const GroupNormCall& c, int V, bool backward) {
  Teams t{};
  const int P = c.C / c.G / V, NP = pieces(c, V);
  t.L = 1;
  while (t.L * NP < P) t.L *= 2;
  const int most = kLanes / t.L;
  t.across = c.G < most ? c.G : most;
  const int64_t slabs = cdiv(c.G, t.across), step = kLanes / (t.L * t.across);
  // Workgroups.  Forward: four goes each, within 1024 to 8192 (16384 rows of 4096 with a gate: 8192 79-81 us, 2048 88-90, 16384 86;
  // 2048 rows: 1024 12.9 us, 2048 13.9, 8192 14.7).  In the backward call each leaves a row of the workspace, which a launch
  // adds up: two a compute unit (256 / 512 / 1024 workgroups, the backward call, bf16 with a gate: 16384 rows of 4096 215 / 148 / 152 us
  // -- with the forward call before it 284 / 227 / 223 --, 4096 of 2048 33 / 30 / 39, 2048 of 4096 32 / 28 / 32).
  const int64_t goes = slabs * cdiv(c.N, step), most_wg = goes / 4 < 1024 ? 1024 : goes / 4 > 8192 ? 8192 : goes / 4;
  int64_t shares = (backward ? 512 : most_wg) / slabs;
  if (shares < 1) shares = 1;
  if (shares > cdiv(c.N, step)) shares = cdiv(c.N, step);
  t.rows = (int)(cdiv(cdiv(c.N, shares), step) * step);
  t.shares = (int)cdiv(c.N, t.rows);
  return t;
}

Slabs slabs_of(const GroupNormCall& c, int V) {
  Slabs s{};
  const int P = c.C / c.G / V;
  if (P > kLanes) {
    s.groups = 1;
    s.per_group = (int)cdiv(P, kLanes);
    s.slabs = c.G * s.per_group;
  } else {
    const int most = kLanes / P, n = (int)cdiv(c.G, most);
    s.groups = (int)cdiv(c.G, n);
    s.per_group = 1;
    s.slabs = (int)cdiv(c.G, s.groups);
  }
  // shares of an image: workgroups for the chip twice over, four times where there is enough to read
  const int across = s.per_group > 1 ? kLanes : s.groups * P, down = kLanes / across;
  const int64_t target = c.N * c.S * c.C * bytes_of(c) > ((int64_t)32 << 20) ? 1024 : 512;
  int64_t shares = cdiv(target, c.N * s.slabs);
  const int64_t most = cdiv(c.S, 4 * down);
  if (shares > most) shares = most;
  // (and no more than a group's lanes combine in two goes)
  const int at_once = 16 * (kLanes / s.groups) / s.per_group;
  if (shares > at_once) shares = at_once;
  if (shares < 1) shares = 1;
  // (A share's positions, and kBatch * kLanes more, are counted in 32 bits: images of 2^30 positions that fit the memory have fewer than
  // 256 channels, one slab, and so 16 shares at least.)
  s.rows = (int)cdiv(c.S, shares);
  s.shares = (int)cdiv(c.S, s.rows);
  return s;
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
size_t stats_bytes(const GroupNormCall& c, const Slabs& s) {
  return up16((size_t)c.N * c.G * s.shares * s.per_group * sizeof(Stat));
}

// f(T, V) with both as types
template <typename F>
void with_type(const GroupNormCall& c, int V, F f) {
  if (c.dtype == MDH_BF16) {
    if (V == 8)
      f(bf16{}, std::integral_constant<int, 8>{});
    else if (V == 2)
      f(bf16{}, std::integral_constant<int, 2>{});
    else
      f(bf16{}, std::integral_constant<int, 1>{});
  } else {
    if (V == 4)
      f(float{}, std::integral_constant<int, 4>{});
    else if (V == 2)
      f(float{}, std::integral_constant<int, 2>{});
    else
      f(float{}, std::integral_constant<int, 1>{});
  }
}
template <typename F>
void with_pieces(int n, F f) {
  if (n == 1)
    f(std::integral_constant<int, 1>{});
  else if (n == 2)
    f(std::integral_constant<int, 2>{});
  else
    f(std::integral_constant<int, 4>{});
}

mdh_status add_up(const GroupNormCall& c, const float* parts, int64_t shares, hipStream_t st) {
  if (!c.dweight && !c.dbias) return MDH_OK;
  add_shares_kernel<<<dim3((unsigned)cdiv(c.C, 32)), kLanes, 0, st>>>(parts, shares, c.C, c.dweight, c.dbias);
  return launch_status();
}

}  // namespace

// What any alignment of the operands may take: fewer channels a lane make more slabs and other shares.
size_t group_norm_workspace(const GroupNormCall& c, bool backward) {
  size_t most = 0;
  if (c.N == 0 || c.S == 0) return 0;
  for (int V = widest(c.C / c.G, bytes_of(c)); V >= 1; V = V == 8 && c.dtype == MDH_BF16 ? 2 : V / 2) {
    size_t n = 0;
    if (use_teams(c, V)) {
      if (backward) n = (size_t)teams_of(c, V, true).shares * 2 * c.C * sizeof(float);
    } else {
      const Slabs s = slabs_of(c, V);
      n = stats_bytes(c, s) + (backward ? (size_t)c.N * s.shares * 2 * c.C * sizeof(float) : 0);
    }
    if (n > most) most = n;
  }
  return up16(most);
}

mdh_status launch_group_norm(const GroupNormCall& c, hipStream_t st) {
  const int V = width(c, false);
  clear_stale_error();
  if (use_teams(c, V)) {
    const Teams t = teams_of(c, V, false);
    const dim3 grid((unsigned)cdiv(c.G, t.across), t.shares);
    with_type(c, V, [&](auto T_, auto V_) {
      with_pieces(pieces(c, V), [&](auto NP_) { teams_forward_kernel<decltype(T_), V_.value, NP_.value><<<grid, kLanes, 0, st>>>(c, t); });
    });
    return launch_status();
  }
  Slabs s = slabs_of(c, V);
  const int64_t blocks = c.N * s.shares * s.slabs;
  if (blocks >= 1 << 24) return MDH_ERR_SIZE;  // 2^32 lanes
  s.stats = c.ws;
  with_type(c, V, [&](auto T_, auto V_) {
    slabs_stats_kernel<decltype(T_), V_.value><<<dim3((unsigned)blocks), kLanes, 0, st>>>(c, s);
    slabs_forward_kernel<decltype(T_), V_.value><<<dim3((unsigned)blocks), kLanes, 0, st>>>(c, s);
  });
  return launch_status();
}

mdh_status launch_group_norm_backward(const GroupNormCall& c, hipStream_t st) {
  const int64_t more = cdiv(c.C, 32);      // workgroups that add up parts
  if (more >= 1 << 24) return MDH_ERR_SIZE;  // 2^32 lanes
  clear_stale_error();
  if (c.N == 0 || c.S == 0) return add_up(c, nullptr, 0, st);
  const int V = width(c, true);
  if (use_teams(c, V)) {
    Teams t = teams_of(c, V, true);
    t.parts = (float*)c.ws;
    const dim3 grid((unsigned)cdiv(c.G, t.across), t.shares);
    with_type(c, V, [&](auto T_, auto V_) {
      with_pieces(pieces(c, V), [&](auto NP_) { teams_backward_kernel<decltype(T_), V_.value, NP_.value><<<grid, kLanes, 0, st>>>(c, t); });
    });
    const mdh_status r = launch_status();
    return r != MDH_OK ? r : add_up(c, t.parts, t.shares, st);
  }
  Slabs s = slabs_of(c, V);
  const int64_t blocks = c.N * s.shares * s.slabs;
  if (blocks + more >= 1 << 24) return MDH_ERR_SIZE;
  s.stats = c.ws;
  s.parts = (float*)((char*)c.ws + stats_bytes(c, s));
  s.last = (int)blocks;
  with_type(c, V, [&](auto T_, auto V_) {
    slabs_backward_kernel<decltype(T_), V_.value, false><<<dim3((unsigned)blocks), kLanes, 0, st>>>(c, s);
    slabs_backward_kernel<decltype(T_), V_.value, true><<<dim3((unsigned)(blocks + more)), kLanes, 0, st>>>(c, s);
  });
  return launch_status();
}

}  // namespace mdh

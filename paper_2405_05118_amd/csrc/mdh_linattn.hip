// Linear attention with a decay for each head: md_hom(k v^T, (++, ++, prefix-sum)) over (b, h, t) whose prefix-sum operator
// combines matrices, S <- l^n S + S'.  One kernel evaluates a pass over the tokens (LinattnPass); the forward call is one
// pass, the backward call three, two of them from the last token to the first.
//
// A run of C positions is evaluated at once on the matrix cores (a, b, c: read, key and value of the pass; S: the state
// before the run; i, j positions in it):
//   out = scale_r ( l^(i+shift) a_i^T S + scale_u sum_{j<=i} l^(i-j) (a_i.b_j) c_j ),   S <- l^n S + scale_u sum_j l^(..) b_j c_j^T
// De-composition: (b, h), 64 or 128 columns of c and, with few of those, segments of the tokens go to workgroups; runs are
// walked in order, S in registers: a wavefront owns 16 columns of it, all rows.  Scores a_i.b_j are divided over
// the wavefronts and exchanged through LDS.  Segments: a pass that only sums up states (reads b and c), a prefix sum over
// the segments, then the pass itself, every segment from its state.
//
// Operands of the 16 x 16 x 32 block are read from LDS rows of a and b as they are, and through transposing reads of b and c
// (ds_read_b64_tr_b16: a lane gets one column of four rows).  Rows and columns of S are dealt out so that the lane that
// holds 4 rows of two blocks holds 8 consecutive ones: S is an operand of a_i^T S without leaving its registers.
//
// fp32 operands are three bf16 slices each (24 bits, cut off: exact), and products the six largest of nine (2^-23 of a
// product is lost).  bf16 operands are one slice; scores and S are rounded to one slice where they are operands (2^-9 of a
// term, as the output's own rounding), but what is added to S is not: c_j times its decay is three slices.
#include "mdh_internal.h"
#include "mdh_types.h"

namespace mdh {
namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) uint16_t Lds;
typedef __attribute__((address_space(3))) u4 LdsU4;
typedef __attribute__((address_space(3))) s4 LdsS4;

__device__ __forceinline__ int64_t slot_of(const LinattnCall& c, int64_t b) {
  if (!c.slots) return b;
  const int64_t s = c.slots[b];
  return s >= 0 && s < c.n_slots ? s : -1;
}
__device__ __forceinline__ int64_t length_of(const LinattnCall& c, int64_t b) {
  return c.lengths ? min(max((int64_t)c.lengths[b], (int64_t)0), c.T) : c.T;
}

// 8 values of a lane, in NS slices
template <int NS>
struct Frag {
  u4 s[NS];
};

// the upper halves of two words
__device__ __forceinline__ uint32_t upper(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

template <int NS, int N>
__device__ __forceinline__ void split(const float (&x)[N], uint32_t (&out)[NS][N / 2]) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    if constexpr (NS == 1) {
      out[0][i / 2] = pack_bf16(x[i], x[i + 1]);
    } else {
      float r0 = x[i], r1 = x[i + 1];
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        out[s][i / 2] = upper(__float_as_uint(r0), __float_as_uint(r1));
        if (s + 1 < NS) {
          r0 -= __uint_as_float(__float_as_uint(r0) & 0xffff0000u);
          r1 -= __uint_as_float(__float_as_uint(r1) & 0xffff0000u);
        }
      }
    }
  }
}

template <int NS>
__device__ __forceinline__ Frag<NS> frag_of(const float (&x)[8]) {
  uint32_t w[NS][4];
  split<NS, 8>(x, w);
  Frag<NS> f;
#pragma unroll
  for (int s = 0; s < NS; ++s) f.s[s] = (u4){w[s][0], w[s][1], w[s][2], w[s][3]};
  return f;
}

template <int NS>
__device__ __forceinline__ void floats_of(const Frag<NS>& f, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(f.s[0][e] << 16);
    x[2 * e + 1] = __uint_as_float(f.s[0][e] & 0xffff0000u);
#pragma unroll
    for (int s = 1; s < NS; ++s) {
      x[2 * e] += __uint_as_float(f.s[s][e] << 16);
      x[2 * e + 1] += __uint_as_float(f.s[s][e] & 0xffff0000u);
    }
  }
}

// acc + A B, smallest products first
template <int NA, int NB>
__device__ __forceinline__ f4 mma(const Frag<NA>& a, const Frag<NB>& b, f4 acc) {
  constexpr int N = NA > NB ? NA : NB;
#pragma unroll
  for (int o = N - 1; o >= 0; --o)
#pragma unroll
    for (int i = 0; i < NA; ++i)
      if (o - i >= 0 && o - i < NB)
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a.s[i]), __builtin_bit_cast(bf8, b.s[o - i]), acc, 0, 0, 0);
  return acc;
}

// 8 consecutive channels of a row as they come from memory.  load: through a descriptor whose loads past its 2^31 bytes give
// 0, at byte `at` + `step`; parts that are not there are asked for past the end.  load_each: element by element, any
// alignment and distance.
constexpr int kPast = (int)0x80000000;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffff, 0x00027000);
}
template <typename T>
struct Raw;
template <>
struct Raw<bf16> {
  u4 w;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, int at, int step, int col, int d, bool ok) {
    w = __builtin_amdgcn_raw_buffer_load_b128(from, ok && col < d ? at : kPast, step, 0);
  }
  __device__ __forceinline__ void load_each(const bf16* row, int col, int d, bool ok) {
    w = (u4){0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (ok && col + e < d) w[e / 2] |= (uint32_t)row[col + e].bits << (16 * (e & 1));
  }
};
template <>
struct Raw<float> {
  u4 w[2];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, int at, int step, int col, int d, bool ok) {
    w[0] = __builtin_amdgcn_raw_buffer_load_b128(from, ok && col < d ? at : kPast, step, 0);
    w[1] = __builtin_amdgcn_raw_buffer_load_b128(from, ok && col + 4 < d ? at + 16 : kPast, step, 0);
  }
  __device__ __forceinline__ void load_each(const float* row, int col, int d, bool ok) {
    w[0] = w[1] = (u4){0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (ok && col + e < d) w[e / 4][e & 3] = __float_as_uint(row[col + e]);
  }
};

// The rows of one operand that a run reads: lane i has channels col.. of rows row0, row0 + kStep, ..
template <typename T, int C, int WIDE, int THREADS>
struct Rows {
  static constexpr int kAcross = WIDE / 8, kStep = THREADS / kAcross, kPieces = C * kAcross, N = kPieces < THREADS ? 1 : kPieces / THREADS;
  Raw<T> r[N];
  static __device__ __forceinline__ int col() { return threadIdx.x % kAcross * 8; }
  static __device__ __forceinline__ int row(int j) { return threadIdx.x / kAcross + j * kStep; }
  // first: the run's lowest token; n of C rows are there, d channels of them
  __device__ __forceinline__ void load(const HeadView& v, const T* first, int n, int d) {
    if (v.vec) {
      const int pitch = (int)(v.st * sizeof(T));
      const __amdgpu_buffer_rsrc_t from = rsrc_of(first);
      const int at = row(0) * pitch + col() * (int)sizeof(T);
#pragma unroll
      for (int j = 0; j < N; ++j) r[j].load(from, at, j * kStep * pitch, col(), d, row(j) < n);
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) r[j].load_each(first + row(j) * v.st, col(), d, row(j) < n);
    }
  }
  // to rows of LDS, the last token first where rev is set
  template <int NS, int PITCH>
  __device__ __forceinline__ void store(uint16_t* to, int n, int rev) const {
    if (kPieces < THREADS && (int)threadIdx.x >= kPieces) return;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = row(j);
      uint16_t* at = to + (rev && i < n ? n - 1 - i : i) * PITCH + col();
      if constexpr (NS == 1) {
        *(u4*)at = r[j].w;
      } else {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(r[j].w[e / 4][e & 3]);
        const Frag<NS> f = frag_of<NS>(x);
#pragma unroll
        for (int s = 0; s < NS; ++s) *(u4*)(at + s * C * PITCH) = f.s[s];
      }
    }
  }
};

// The shape of a kernel: KP rows of the state (da padded), W wavefronts with 16 columns each
template <typename T, int KP_, int W_, bool STATE_>
struct Shape {
  static constexpr int NS = sizeof(T) == 2 ? 1 : 3;
  static constexpr int C = NS == 1 ? 64 : 32;  // positions of a run
  static constexpr int KP = KP_, W = W_, VT = 16 * W_;
  static constexpr bool STATE = STATE_;  // sums up the state only
  static constexpr int TB = C / 16, KS = KP / 32, CS = C / 32;
  // rows in LDS, in elements: 16 bytes past a multiple of 128 bytes, so that 16 rows at one column are all banks
  static constexpr int PA = KP + 8, PC = VT + 8, PP = C + 8;
  static constexpr int A = 0, B = A + (STATE ? 0 : NS * C * PA), CC = B + NS * C * PA, P = CC + NS * C * PC;
  static constexpr int kHalves = P + (STATE ? 0 : NS * C * PP);
  static constexpr int kBytes = kHalves * 2 + (C + 2 * (C + 4)) * 4;  // and the decays: l^(..) of an update, l^i
};

struct SegmentArgs {
  int n;           // segments
  int64_t len;     // positions of one, a multiple of C
  float* states;   // (B, H, n, dk, dv): the state that enters each
};

struct PassArgs {
  LinattnCall c;
  LinattnPass p[3];
  int tiles[3];     // column tiles of each pass, of 16 W columns
  int n;
  SegmentArgs seg[3];
  int seg_t[3];     // the states are (dc, da) of this pass
};

template <typename T, int KP, int W, bool STATE>
__global__ __launch_bounds__(64 * W, KP == 256 ? 2 : KP == 128 && W == 4 ? 3 : 4) void linattn_runs_kernel(PassArgs args) {
  using X = Shape<T, KP, W, STATE>;
  constexpr int C = X::C, NS = X::NS, TB = X::TB, KS = X::KS, CS = X::CS, TH = 64 * W;
  extern __shared__ __align__(16) uint16_t lds[];
  uint16_t* const As = lds + X::A;
  uint16_t* const Bs = lds + X::B;
  uint16_t* const Cs = lds + X::CC;
  uint16_t* const Ps = lds + X::P;
  float* const uw = (float*)(lds + X::kHalves);  // what position j of a run is multiplied with on its way into the state
  float* const pw = uw + C;                      // l^i, i <= C, as two floats
  float* const pl = pw + C + 4;

  const LinattnCall& call = args.c;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // (b, segment, h, pass, columns): neighbours share operands, and an XCD gets a run of neighbours
  int tiles = 0;
  for (int i = 0; i < args.n; ++i) tiles += args.tiles[i];
  const int id = xcd_order(blockIdx.x, gridDim.x);
  int tile = id % tiles, which = 0;
  const int rest = id / tiles;
  while (tile >= args.tiles[which]) tile -= args.tiles[which++];
  const LinattnPass& p = args.p[which];
  const SegmentArgs& sg = args.seg[which];
  const int h = rest % call.H;
  const int n_seg = STATE ? sg.n - 1 : sg.n;  // (the state after the last one is not asked for)
  const int seg = rest / call.H % n_seg, b = rest / call.H / n_seg;

  const int da = p.da, dc = p.dc, rev = p.rev;
  const int len = __builtin_amdgcn_readfirstlane((int)length_of(call, b));
  const int p0 = (int)min(seg * sg.len, (int64_t)len), pend = (int)min((int64_t)len, p0 + sg.len);
  const float log_decay = call.log_decay[h];
  const int64_t slot = slot_of(call, b);
  const int64_t elems = (int64_t)da * dc, at = (slot * call.H + h) * elems;
  const int64_t seg_at = (((int64_t)b * call.H + h) * sg.n + seg) * elems;
  const int tile0 = tile * X::VT, my_col = tile0 + 16 * wave + l16;  // of the state; of an output, a lane has rows of l16

  // S[ks][x][r]: row 32 ks + 8 g + 4 x + r, column my_col
  f4 S[KS][2];
  {
    const float* from = nullptr;
    int turned = 0;
    if (!STATE) {
      if (sg.n > 1) {
        if (seg > 0 || p.s_in) from = sg.states + seg_at;
        turned = args.seg_t[which];
      } else if (p.s_in && slot >= 0) {
        from = p.s_in + at;
        turned = p.s_in_t;
      }
    }
const int down = turned ? 4 : dc * 4, lane_at = 8 * g * down + my_col * (turned ? da * 4 : 4);
    const bool mine = from && my_col < dc;
    const int rows_here = da - 8 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 32 * ks + 4 * x + r;
          S[ks][x][r] = __uint_as_float(
              __builtin_amdgcn_raw_buffer_load_b32(rsrc_of(from), mine && row < rows_here ? lane_at : kPast, row * down, 0));
        }
  }

  // decays
  auto update_weights = [&](int n) {  // of a run of n positions
    if (tid < C) uw[tid] = tid < n ? p.scale_u * pw[n - tid - p.shift] : 0.f;
  };
  if (tid <= C) {
    const Decay d = decay_power(log_decay, tid);
    pw[tid] = d.hi;
    pl[tid] = d.lo;
  }
  __syncthreads();
  update_weights(C);
  // score blocks of a wavefront: 16 rows tb, 16 columns sb0 ..; the upper half of the blocks is of no use to anybody
  constexpr int BPW = TB * TB >= W ? TB * TB / W : 1;
  const int tb = wave * BPW / TB, sb0 = wave * BPW % TB;
  float near[BPW][4], far[TB];
  if (!STATE) {
#pragma unroll
    for (int i = 0; i < BPW; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = 16 * (tb - sb0 - i) + l16 - 4 * g - r;
        near[i][r] = d >= 0 && d <= C ? p.scale_r * p.scale_u * pw[d] : 0.f;
      }
#pragma unroll
    for (int i = 0; i < TB; ++i) far[i] = p.scale_r * pw[16 * i + l16 + p.shift];
  }

  // operands: the rows of the next run, in registers until this one is done
  Rows<T, C, KP, TH> ra, rb;
  Rows<T, C, X::VT, TH> rc;
  const T* const pa = (const T*)p.a.p + b * p.a.sb + (h / p.a.group) * p.a.sh;
  const T* const pb = (const T*)p.b.p + b * p.b.sb + (h / p.b.group) * p.b.sh;
  const T* const pc = (const T*)p.c.p + b * p.c.sb + (h / p.c.group) * p.c.sh + tile0;
  auto load = [&](int pos) {
    const int n = min(C, len - pos);
    const int64_t t = rev ? len - pos - n : pos;
    if (!STATE) ra.load(p.a, pa + t * p.a.st, n, da);
    rb.load(p.b, pb + t * p.b.st, n, da);
    rc.load(p.c, pc + t * p.c.st, n, dc - tile0);
  };
  // where a lane's operands are in LDS, but for constants: 8 consecutive columns of a row, or one column of 8 rows (of which
  // it supplies 4 columns of one)
  Lds* const rows_a = (Lds*)As + l16 * X::PA + 8 * g;
  Lds* const rows_b = (Lds*)Bs + l16 * X::PA + 8 * g;
  Lds* const rows_p = (Lds*)Ps + l16 * X::PP + 8 * g;
  Lds* const cols_b = (Lds*)Bs + (8 * g + (l16 >> 2)) * X::PA + 8 * (l16 & 3);
  Lds* const cols_c = (Lds*)Cs + (8 * g + (l16 >> 2)) * X::PC + 16 * wave + 4 * (l16 & 3);
  auto row_frag = [](Lds* at, int plane) {
    Frag<NS> f;
#pragma unroll
    for (int s = 0; s < NS; ++s) f.s[s] = *(LdsU4*)(at + s * plane);
    return f;
  };
  auto col_frag = [](Lds* at, int pitch) {
    Frag<NS> f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const u2 lo = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)(at + s * C * pitch)));
      const u2 hi = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsS4*)(at + (s * C + 4) * pitch)));
      f.s[s] = (u4){lo[0], lo[1], hi[0], hi[1]};
    }
    return f;
  };

  if (p0 < pend) load(p0);
  for (int pos = p0; pos < pend; pos += C) {
    const int n = min(C, len - pos);
    if (!STATE) ra.template store<NS, X::PA>(As, n, rev);
    rb.template store<NS, X::PA>(Bs, n, rev);
    rc.template store<NS, X::PC>(Cs, n, rev);
    if (n < C) update_weights(n);
    __syncthreads();
    if (pos + C < pend) load(pos + C);

    f4 out[STATE ? 1 : TB];
    if constexpr (!STATE) {
      // scores of the wavefront's blocks, decayed; zero where a position would see one behind it
      if (tb < TB)
#pragma unroll
        for (int i = 0; i < BPW; ++i) {
          const int sb = sb0 + i;
          if (sb > (tb | 1)) continue;
          f4 acc = {0.f, 0.f, 0.f, 0.f};
          if (sb <= tb)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
              acc = mma(row_frag(rows_b + 16 * sb * X::PA + 32 * ks, C * X::PA), row_frag(rows_a + 16 * tb * X::PA + 32 * ks, C * X::PA), acc);
          float x[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) x[r] = acc[r] * near[i][r];
          uint32_t w[NS][2];
          split<NS, 4>(x, w);
#pragma unroll
          for (int s = 0; s < NS; ++s) *(u2*)(Ps + s * C * X::PP + (16 * tb + l16) * X::PP + 16 * sb + 4 * g) = (u2){w[s][0], w[s][1]};
          __builtin_amdgcn_sched_barrier(0);
        }
      // what the state before the run gives
#pragma unroll
      for (int i = 0; i < TB; ++i) out[i] = (f4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const f4 lo = S[ks][0], hi = S[ks][1];
        const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        const Frag<NS> sf = frag_of<NS>(x);
#pragma unroll
        for (int i = 0; i < TB; ++i) out[i] = mma(sf, row_frag(rows_a + 16 * i * X::PA + 32 * ks, C * X::PA), out[i]);
        __builtin_amdgcn_sched_barrier(0);  // (moved up, the reads of all steps would take more registers than there are)
      }
#pragma unroll
      for (int i = 0; i < TB; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) out[i][r] *= far[i];
    }

    // the state after the run
    const Decay d{pw[n], pl[n]};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[ks][x][r] = d * S[ks][x][r];
#pragma unroll
    for (int ks2 = 0; ks2 < CS; ++ks2) {
      const f4 w0 = *(const f4*)(uw + 32 * ks2 + 8 * g), w1 = *(const f4*)(uw + 32 * ks2 + 8 * g + 4);
      float x[8];
      floats_of<NS>(col_frag(cols_c + 32 * ks2 * X::PC, X::PC), x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= e < 4 ? w0[e & 3] : w1[e & 3];
      const Frag<3> wc = frag_of<3>(x);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
        for (int y = 0; y < 2; ++y)
          S[ks][y] = mma(col_frag(cols_b + 32 * ks2 * X::PA + 32 * ks + 4 * y, X::PA), wc, S[ks][y]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();

    if constexpr (!STATE) {
      // what the run's own positions give
#pragma unroll
      for (int ks2 = 0; ks2 < CS; ++ks2) {
        const Frag<NS> cf = col_frag(cols_c + 32 * ks2 * X::PC, X::PC);
#pragma unroll
        for (int i = 2 * ks2; i < TB; ++i) out[i] = mma(cf, row_frag(rows_p + 16 * i * X::PP + 32 * ks2, C * X::PP), out[i]);
      }
      // a lane has 4 consecutive columns of one position of each block
      const int col = tile0 + 16 * wave + 4 * g;
      const int64_t first = b * p.out.sb + (h / p.out.group) * p.out.sh + col;
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        const int at_i = 16 * i + l16;
        if (at_i >= n) continue;
        const int64_t to = first + (int64_t)(rev ? len - 1 - pos - at_i : pos + at_i) * p.out.st;
        if (p.out_f32 || sizeof(T) == 4) {
          float* o = (float*)p.out.p + to;
          if (p.out.vec && col < dc)
            *(f4*)o = out[i];
          else
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (col + e < dc) o[e] = out[i][e];
        } else {
          uint16_t* o = (uint16_t*)p.out.p + to;
          const u2 w = {pack_bf16(out[i][0], out[i][1]), pack_bf16(out[i][2], out[i][3])};
          if (p.out.vec && col < dc)
            *(u2*)o = w;
          else
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (col + e < dc) o[e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
        }
      }
    }
    __syncthreads();
  }

  if constexpr (!STATE) {
    // tokens behind the last valid one
    const int64_t begin = max((int64_t)len, seg * sg.len), end = min(call.T, (seg + 1) * sg.len);
    const int cols = min(dc - tile0, X::VT);
    for (int64_t i = begin * cols + tid; i < end * cols; i += TH) {
      const int64_t to = b * p.out.sb + (h / p.out.group) * p.out.sh + i / cols * p.out.st + tile0 + i % cols;
      if (p.out_f32 || sizeof(T) == 4)
        ((float*)p.out.p)[to] = 0.f;
      else
        ((uint16_t*)p.out.p)[to] = 0;
    }
  }
  // the state: of the segment for the prefix sum (it enters the next one), or behind all of them
  float* const into = STATE ? sg.states + seg_at + elems : (p.s_out && slot >= 0 && seg == sg.n - 1 ? p.s_out + at : nullptr);
  if (into) {
    const int lane_at = 8 * g * dc * 4 + my_col * 4;
    int rows = da - 8 * g;
    asm volatile("" : "+v"(rows));  // (the conditions of the first loads of S are not to be kept until here)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int row = 32 * ks + 4 * x + r;
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[ks][x][r]), rsrc_of(into),
                                                my_col < dc && row < rows ? lane_at : kPast, row * dc * 4, 0);
        }
  }
}

// Prefix sum over the segments: what is in segment g's place is the sum of segment g - 1 alone; after it, the state that
// enters g.  One thread for each element of each (b, h).
struct CombineArgs {
  LinattnCall c;
  SegmentArgs seg;
  const float* s_in;
  int64_t elems;
};
__global__ __launch_bounds__(256) void linattn_segments_kernel(CombineArgs a) {
  const int64_t e = (int64_t)blockIdx.y * 256 + threadIdx.x;
  if (e >= a.elems) return;
  const int64_t bh = blockIdx.x, b = bh / a.c.H;
  const int h = (int)(bh % a.c.H);
  const int64_t len = length_of(a.c, b), slot = slot_of(a.c, b);
  const float log_decay = a.c.log_decay[h];
  const Decay full = decay_power(log_decay, a.seg.len);
  float* s = a.seg.states + bh * a.seg.n * a.elems + e;
  float run = a.s_in && slot >= 0 ? a.s_in[(slot * a.c.H + h) * a.elems + e] : 0.f;
  if (a.s_in) s[0] = run;
  constexpr int U = 8;
  for (int g0 = 1; g0 < a.seg.n; g0 += U) {
    float x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = g0 + u < a.seg.n ? s[(g0 + u) * a.elems] : 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g0 + u < a.seg.n) {
        const int64_t n = min(max(len - (g0 + u - 1) * a.seg.len, (int64_t)0), a.seg.len);  // positions of the segment before
        run = (n == a.seg.len ? full : decay_power(log_decay, n)) * run + x[u];
        s[(g0 + u) * a.elems] = run;
      }
  }
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

template <typename T, int KP, int W, bool STATE>
mdh_status run(const PassArgs& a, hipStream_t st) {
  using X = Shape<T, KP, W, STATE>;
  static int64_t done[kMaxDevices];
  int tiles = 0;
  for (int i = 0; i < a.n; ++i) tiles += a.tiles[i];
  const int64_t blocks = a.c.B * a.c.H * (STATE ? a.seg[0].n - 1 : a.seg[0].n) * tiles;
  if (blocks > 0x7fffffff) return MDH_ERR_SIZE;
  const void* kern = (const void*)linattn_runs_kernel<T, KP, W, STATE>;
  const mdh_status r = allow_dynamic_lds(kern, X::kBytes, done);
  if (r != MDH_OK) return r;
  clear_stale_error();
  linattn_runs_kernel<T, KP, W, STATE><<<dim3((unsigned)blocks), 64 * W, X::kBytes, st>>>(a);
  return launch_status();
}

template <typename T, int KP, bool STATE>
mdh_status run(const PassArgs& a, int W, hipStream_t st) {
  return W == 8 ? run<T, KP, 8, STATE>(a, st) : run<T, KP, 4, STATE>(a, st);
}

template <typename T, bool STATE>
mdh_status run(const PassArgs& a, int KP, int W, hipStream_t st) {
  return KP == 64 ? run<T, 64, STATE>(a, W, st) : KP == 128 ? run<T, 128, STATE>(a, W, st) : run<T, 256, STATE>(a, W, st);
}

template <bool STATE>
mdh_status run(const PassArgs& a, int dtype, int KP, int W, hipStream_t st) {
  return dtype == MDH_BF16 ? run<bf16, STATE>(a, KP, W, st) : run<float, STATE>(a, KP, W, st);
}

int padded(int da) { return da <= 64 ? 64 : da <= 128 ? 128 : 256; }
// wavefronts: of 16 columns each
int waves_of(int dc) { return dc > 64 ? 8 : 4; }

// Segments of T positions, of whole runs: enough that `work` workgroups for each fill the chip twice.
int segments_of(int64_t T, int C, int64_t work, int64_t* len) {
  const int64_t runs = cdiv(T, C);
  int64_t n = work > 0 ? 512 / work : 1;
  if (n > runs / 2) n = runs / 2;
  if (n < 1) n = 1;
  *len = cdiv(runs, n) * C;
  return T > 0 ? (int)cdiv(T, *len) : 1;
}
int run_length(int dtype) { return dtype == MDH_BF16 ? 64 : 32; }
int64_t tiles_of(int dc) { return cdiv(dc, 16 * waves_of(dc)); }

}  // namespace

// bytes for the states of the segments: one set for the forward call, two for the backward call
size_t linattn_segment_bytes(int64_t B, int64_t T, int H, int dk, int dv, int dtype, bool backward) {
  int64_t len;
  const int n = linattn_segments(B, T, H, dk, dv, dtype, backward, &len);
  return n > 1 ? (size_t)B * H * n * dk * dv * sizeof(float) * (backward ? 2 : 1) : 0;
}

int linattn_segments(int64_t B, int64_t T, int H, int dk, int dv, int dtype, bool backward, int64_t* len) {
  const int64_t work = B * H * (backward ? tiles_of(dk) * 2 + tiles_of(dv) : tiles_of(dv));
  return segments_of(T, run_length(dtype), work, len);
}

// The state entering each of n segments: `p` gives the operands (da x dc = dk x dv).
mdh_status launch_linattn_segments(const LinattnCall& c, const LinattnPass* p, int np, int n, int64_t len, float* const* states,
                                   int dtype, hipStream_t st) {
  PassArgs a{};
  a.c = c;
  a.n = np;
  const int KP = padded(p[0].da), W = waves_of(p[0].dc);
  for (int i = 0; i < np; ++i) {
    a.p[i] = p[i];
    a.tiles[i] = (int)cdiv(p[i].dc, 16 * W);
    a.seg[i] = SegmentArgs{n, len, states[i]};
  }
  mdh_status r = run<true>(a, dtype, KP, W, st);
  for (int i = 0; i < np && r == MDH_OK; ++i) {
    const CombineArgs k{c, a.seg[i], p[i].s_in, (int64_t)p[i].da * p[i].dc};
    clear_stale_error();
    linattn_segments_kernel<<<dim3((unsigned)(c.B * c.H), (unsigned)cdiv(k.elems, 256)), 256, 0, st>>>(k);
    r = launch_status();
  }
  return r;
}

mdh_status launch_linattn_pass(const LinattnCall& c, const LinattnPass* passes, int np, int n, int64_t len, float* const* states,
                               const int* turned, int dtype, hipStream_t st) {
  // passes of one kernel go in one launch
  bool gone[3] = {};
  for (int i = 0; i < np; ++i) {
    if (gone[i]) continue;
    const int KP = padded(passes[i].da), W = waves_of(passes[i].dc);
    PassArgs a{};
    a.c = c;
    for (int j = i; j < np; ++j) {
      if (gone[j] || padded(passes[j].da) != KP || waves_of(passes[j].dc) != W) continue;
      gone[j] = true;
      a.p[a.n] = passes[j];
      a.tiles[a.n] = (int)cdiv(passes[j].dc, 16 * W);
      a.seg[a.n] = SegmentArgs{n, len, states[j]};
      a.seg_t[a.n] = turned[j];
      ++a.n;
    }
    const mdh_status r = run<false>(a, dtype, KP, W, st);
    if (r != MDH_OK) return r;
  }
  return MDH_OK;
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

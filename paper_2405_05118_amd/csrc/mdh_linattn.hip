// Linear attention with a decay for each head: md_hom(k v^T, (++, ++, prefix-sum)) over (b, h, t) whose prefix-sum operator
// combines matrices, S <- l^n S + S'.  One kernel evaluates a pass over the tokens (LinattnPass); the forward call is one
// pass, the backward call three, two of them from the last token to the first.
//
// A run of C positions is evaluated at once on the matrix cores (a, b, c: read, key and value of the pass; S: the state
// before the run; i, j positions in it):
//   out = scale_r ( l^(i+shift) a_i^T S + scale_u sum_{j<=i} l^(i-j) (a_i.b_j) c_j ),   S <- l^n S + scale_u sum_j l^(..) b_j c_j^T
// De-composition: (b, h), 64 or 128 columns of c and, with few of those, segments of the tokens go to workgroups; runs are
// walked in order, S in registers: a wavefront owns 16 or 32 columns of it, all rows.  Scores a_i.b_j are divided over
// the wavefronts and exchanged through LDS.  Segments: a pass that only sums up states (reads b and c), a prefix sum over
// the segments, then the pass itself, every segment from its state.
//
// Operands of the 16 x 16 x 32 block are read from LDS rows of a and b as they are, and through transposing reads of b and c
// (ds_read_b64_tr_b16: a lane gets one column of four rows).  S is an operand of a_i^T S without leaving its registers: of
// 32 rows a lane has 4 of each 16, and reads the same channels of a, which lie side by side in LDS for that.
//
// fp32 operands are three bf16 slices each (24 bits, cut off), and products the six largest of nine (2^-23 of a product is
// lost).  bf16 operands are one slice; scores and S are rounded to one slice where they are operands (2^-9 of a
// term, as the output's own rounding), but what is added to S is not: c_j times its decay is three slices.
//
// Bound by memory where the sequence is long: 65536 x 16 heads of 128 x 128, bf16, 390 us a call; in a kernel trace, whose sums
// are up to a tenth more, 142 for the states of 32 segments (3.8 TB/s; its arithmetic taken out, 122 of 131 were left), 15 for
// their prefix sum and 271 for the pass (4.0 TB/s, 253 TFLOP/s).  2048 x 32 heads: 48 us, 15 + 8 + 29, the last for four runs
// of a workgroup one after the other.  Trained, 8 x 4096 x 16 heads: 590 us, 64 + 10 + 127 for the forward call and 407 for
// the three passes of the backward call, which read nine tensors and write three.
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
typedef __attribute__((address_space(3))) u2 LdsU2;
typedef __attribute__((address_space(3))) float LdsF;
typedef __attribute__((address_space(3))) f4 LdsF4;
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

// Two values in NS bf16 slices: one is rounded to nearest, three are cut off and hold all 24 bits.
template <int NS, int N>
__device__ __forceinline__ void split(const float (&x)[N], uint32_t (&out)[NS][N / 2]) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    if constexpr (NS == 1) {
      out[0][i / 2] = pack_bf16(x[i], x[i + 1]);
    } else {
      uint32_t r0 = __float_as_uint(x[i]), r1 = __float_as_uint(x[i + 1]);
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        out[s][i / 2] = __builtin_amdgcn_perm(r1, r0, 0x07060302u);  // the upper halves
        if (s + 1 < NS) {
          r0 = __float_as_uint(__uint_as_float(r0) - __uint_as_float(r0 & 0xffff0000u));
          r1 = __float_as_uint(__uint_as_float(r1) - __uint_as_float(r1 & 0xffff0000u));
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

constexpr int kWaves = 4, kThreads = 64 * kWaves;

// How rows are read and written (one kernel for each: what the general ones keep in registers would cost the first its speed).
//   kVec   16 bytes at a time: bases, strides and rows are multiples of 16 bytes
//   kAny   16 bytes at a time at any address; the row's last ones are read as the 16 bytes that end with it and moved down
//          (rows have 16 bytes at least).  The bf16 passes keep 52 to 72 bytes a lane in scratch: 4 x 2048 x 16 heads of 100 x 90,
//          93 us, trained 302, where 104 x 96 aligned take 70 and 196.
//   kEach  element by element: shorter rows
enum Access { kVec = 0, kAny = 1, kEach = 2 };

// Loads go through a descriptor whose loads past its 2^31 bytes give 0: what is not there is asked for past the end.
constexpr int kPast = (int)0x80000000;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7fffffff, 0x00027000);
}

// The rows of one operand that a run reads: the lane has channels col.. of positions row, row + kStep, .. of it
template <typename T, int C, int WIDE, int ACCESS>
struct Rows {
  static constexpr int kAcross = WIDE / 8, kStep = kThreads / kAcross, N = C / kStep;
  static constexpr int kLoads = sizeof(T) / 2, kPer = 16 / sizeof(T);  // 16-byte loads of 8 channels, channels of one
  static_assert(C % kStep == 0 && N >= 1, "every lane has whole rows");
  u4 w[N][kLoads];
  int at[kLoads], pitch, rev;
  int down[ACCESS == kAny ? kLoads : 1];  // channels that a load's are moved down by
  const T* base;  // position 0's row would be here, were all runs full
  int64_t st;
  static __device__ __forceinline__ int col() { return threadIdx.x % kAcross * 8; }
  static __device__ __forceinline__ int row() { return threadIdx.x / kAcross; }
  __device__ __forceinline__ void init(const HeadView& v, int64_t offset, int col0, int d, int rev_) {  // channels from col0 on, of rows of d
    base = (const T*)v.p + offset;
    st = v.st;
    pitch = (int)(v.st * sizeof(T));
    rev = rev_;
    const int first = (rev ? C - 1 - row() - (N - 1) * kStep : row()) * pitch;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int c = col0 + col() + i * kPer;
      at[i] = ACCESS == kEach || c < d ? first + c * (int)sizeof(T) : kPast;
      if (ACCESS == kAny) {
        down[i] = c < d && c + kPer > d ? c + kPer - d : 0;
        at[i] -= down[i] * (int)sizeof(T);
      }
    }
  }
  // the run of n positions whose first is pos, of len (the loads of a sequence's last run, which may be shorter, are checked)
  __device__ __forceinline__ void load(int pos, int n, int len, int d) {
    const __amdgpu_buffer_rsrc_t from = rsrc_of(base + (int64_t)(rev ? len - pos - C : pos) * st);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int step = (rev ? N - 1 - j : j) * kStep * pitch;
      const bool there = row() + j * kStep < n;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        if constexpr (ACCESS == kEach) {
          const int left = there ? d - col() - i * kPer : 0;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if constexpr (sizeof(T) == 4) {
              w[j][i][e] = __builtin_amdgcn_raw_buffer_load_b32(from, e < left ? at[i] + 4 * e : kPast, step, 0);
            } else {
              const uint32_t lo = __builtin_amdgcn_raw_buffer_load_b16(from, 2 * e < left ? at[i] + 4 * e : kPast, step, 0);
              const uint32_t hi = __builtin_amdgcn_raw_buffer_load_b16(from, 2 * e + 1 < left ? at[i] + 4 * e + 2 : kPast, step, 0);
              w[j][i][e] = (lo & 0xffffu) | hi << 16;
            }
        } else if (n == C) {
          w[j][i] = __builtin_amdgcn_raw_buffer_load_b128(from, at[i], step, 0);
        } else {
          w[j][i] = __builtin_amdgcn_raw_buffer_load_b128(from, there ? at[i] : kPast, step, 0);
        }
      }
    }
  }
  // what load j has left of its channels, moved down to where they belong
  __device__ __forceinline__ u4 placed(int j, int i) const {
    u4 v = w[j][i];
    if constexpr (ACCESS == kAny) {
      const int words = sizeof(T) == 4 ? down[i] : down[i] >> 1;
      if (words & 2) v = (u4){v[2], v[3], 0, 0};
      if (words & 1) v = (u4){v[1], v[2], v[3], 0};
      if (sizeof(T) == 2 && (down[i] & 1)) v = (u4){v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    }
    return v;
  }
  // PAIRED: of 32 channels, 4g.. and 16 + 4g.. side by side
  template <int NS, int PITCH, bool PAIRED = false>
  __device__ __forceinline__ void store(Lds* to) const {
    const int c = PAIRED ? (col() & ~31) + ((col() & 8) << 1) + ((col() & 16) >> 2) : col();
    Lds* const first = to + row() * PITCH + c;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      Frag<NS> f;
      if constexpr (NS == 1) {
        f.s[0] = placed(j, 0);
      } else {
        const u4 lo = placed(j, 0), hi = placed(j, kLoads - 1);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(e < 4 ? lo[e & 3] : hi[e & 3]);
        f = frag_of<NS>(x);
      }
#pragma unroll
      for (int s = 0; s < NS; ++s) {
        Lds* const to_s = first + (s * C + j * kStep) * PITCH;
        if constexpr (PAIRED) {
          *(LdsU2*)to_s = (u2){f.s[s][0], f.s[s][1]};
          *(LdsU2*)(to_s + 8) = (u2){f.s[s][2], f.s[s][3]};
        } else {
          *(LdsU4*)to_s = f.s[s];
        }
      }
    }
  }
};

// The shape of a kernel: KP rows of the state (da padded), four wavefronts with NB blocks of 16 columns each.  Two blocks where
// they can be: what a wavefront reads of a, b and the scores serves both, and LDS is what the passes are short of (32 x 4096
// x 16 x 128 x 128, forward: 495 us; one block each for eight wavefronts 579).
template <typename T, int KP_, int NB_, bool STATE_>
struct Shape {
  static constexpr int NS = sizeof(T) == 2 ? 1 : 3;
  static constexpr int C = NS == 1 ? 64 : 32;  // positions of a run
  static constexpr int KP = KP_, NB = NB_, VT = 16 * NB_ * kWaves;
  static constexpr bool STATE = STATE_;  // sums up the state only
  static constexpr int TB = C / 16, KS = KP / 32, CS = C / 32;
  // Rows in LDS, in elements, without bank conflicts.  a and scores are read 16 rows at a time at one column: 16 bytes past a
  // multiple of 128 bytes.  A transposing read of b, or of c for two blocks, takes from 4 rows every other 8 bytes of 64:
  // 64 bytes past a multiple of 256 (or short of it), so that the rows lie beside one another.
  static constexpr int PA = KP + 8, PB = KP + 32, PC = NB == 2 ? VT + 32 : VT + 16, PP = C + 8;
  static constexpr int A = 0, B = A + (STATE ? 0 : NS * C * PA), CC = B + NS * C * PB, P = CC + NS * C * PC;
  static constexpr int kHalves = P + (STATE ? 0 : NS * C * PP);
  static constexpr int kBytes = kHalves * 2 + (5 * C + 4) * 4;  // and the decays (below)
};

struct SegmentArgs {
  int n;           // segments
  int64_t len;     // positions of one, a multiple of C
  float* states;   // (B, H, n, dk, dv): the state that enters each
};

struct PassArgs {
  LinattnCall c;
  LinattnPass p[3];
  int tiles[3];     // column tiles of each pass, of 64 NB columns
  int n;
  SegmentArgs seg[3];
  int seg_t[3];     // the states are (dc, da) of this pass
};

template <typename T, int KP, int NB, bool STATE, int ACCESS>
__global__ __launch_bounds__(kThreads, ACCESS == kEach ? 2 : KP == 64 && NB == 1 ? 4 : KP == 128 && NB == 1 ? 3 : 2) void linattn_runs_kernel(PassArgs args) {
  using X = Shape<T, KP, NB, STATE>;
  constexpr int C = X::C, NS = X::NS, TB = X::TB, KS = X::KS, CS = X::CS;
  extern __shared__ __align__(16) uint16_t lds[];
  Lds* const As = (Lds*)lds + X::A;
  Lds* const Bs = (Lds*)lds + X::B;
  Lds* const Cs = (Lds*)lds + X::CC;
  Lds* const Ps = (Lds*)lds + X::P;
  LdsF* const uw = (LdsF*)((Lds*)lds + X::kHalves);  // what position j of a run is multiplied with on its way into the state,
  LdsF* const fw = uw + C;                           // what position i reads of the state before the run,
  LdsF* const nw = fw + 2 * C;                       // what position i reads of position i - d, 0 for d < 0
  LdsF* const pw = nw + C;                           // and l^i, i <= C

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
  const int tile0 = tile * X::VT, wave0 = 16 * NB * wave;  // first column of the tile, and in it of the wavefront
  // the column of lane m in block nb: with two blocks every other four, so that an output's lane has 8 side by side
  auto col_of = [&](int m, int nb) { return tile0 + wave0 + (NB == 2 ? 8 * (m >> 2) + 4 * nb + (m & 3) : m); };

  // S[ks][x][nb][r]: row 32 ks + 16 x + 4 g + r, column col_of(l16, nb)
  f4 S[KS][2][NB];
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
    const int down = turned ? 4 : dc * 4, across = turned ? da * 4 : 4, rows_here = da - 4 * g;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int col = col_of(l16, nb), lane_at = 4 * g * down + col * across;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int row = 32 * ks + 16 * x + r;
            S[ks][x][nb][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
                rsrc_of(from), from && col < dc && row < rows_here ? lane_at : kPast, row * down, 0));
          }
        }
  }

  // decays
  auto update_weights = [&](int n) {  // of a run of n positions
    if (tid < C) uw[tid] = tid < n ? p.scale_u * pw[n - tid - p.shift] : 0.f;
  };
  if (tid <= C) pw[tid] = decay_power(log_decay, tid).hi;
  __syncthreads();
  update_weights(C);
  if (tid < C) {
    fw[tid] = p.scale_r * pw[tid + p.shift];
    nw[tid] = p.scale_r * p.scale_u * pw[tid];
    nw[tid - C] = 0.f;
  }
  // The state is multiplied with l^C run after run, by one float for each: the relative error that the roundings so far have
  // left (`off`) is taken back by the next one.  Without that, 2^-25 a run adds up over a long memory.
  const double run_decay = log_decay == 0.f ? 1.0 : exp((double)log_decay * C), per = run_decay > 0.0 ? 1.0 / run_decay : 0.0;
  double off = 0.0;
  // score blocks of a wavefront: 16 rows wave_tb, 16 columns sb0 ..; the upper half of the blocks is of no use to anybody
  constexpr int BPW = TB * TB / kWaves;
  const int wave_tb = wave * BPW / TB, sb0 = wave * BPW % TB;

  // operands: the rows of the next run, in registers until this one is done
  Rows<T, C, KP, ACCESS> ra, rb;
  Rows<T, C, X::VT, ACCESS> rc;
  if (!STATE) ra.init(p.a, b * p.a.sb + (h / p.a.group) * p.a.sh, 0, da, rev);
  rb.init(p.b, b * p.b.sb + (h / p.b.group) * p.b.sh, 0, da, rev);
  rc.init(p.c, b * p.c.sb + (h / p.c.group) * p.c.sh, tile0, dc, rev);
  auto load = [&](int pos) {
    if (pos < p0 || pos >= pend) return;
    const int n = min(C, len - pos);
    if (!STATE) ra.load(pos, n, len, da);
    rb.load(pos, n, len, da);
    rc.load(pos, n, len, dc - tile0);
  };
  auto store = [&](int pos) {
    if (pos < p0 || pos >= pend) return;
    if (!STATE) ra.template store<NS, X::PA, true>(As);
    rb.template store<NS, X::PB, true>(Bs);
    rc.template store<NS, X::PC>(Cs);
    if (!STATE && len - pos < C) update_weights(len - pos);
  };
  // outputs: a lane has 4 NB consecutive columns of position l16 of each block of 16
  const int out_bytes = p.out_f32 ? 4 : (int)sizeof(T), out_pitch = (int)(p.out.st * out_bytes);
  const int out_col = tile0 + wave0 + 4 * NB * g, out_at = (rev ? 15 - l16 : l16) * out_pitch + out_col * out_bytes;
  char* const out_base = (char*)p.out.p + (b * p.out.sb + (h / p.out.group) * p.out.sh) * out_bytes;

  // where a lane's operands are in LDS, but for constants: 8 consecutive columns of a row, or one column of 8 rows (of which
  // it supplies 4 columns of one)
  Lds* const rows_a = As + l16 * X::PA + 8 * g;
  Lds* const rows_b = Bs + l16 * X::PB + 8 * g;
  Lds* const rows_p = Ps + l16 * X::PP + 8 * g;
  Lds* const cols_b = Bs + (8 * g + (l16 >> 2)) * X::PB + 8 * (l16 & 3);
  Lds* const cols_c = Cs + (8 * g + (l16 >> 2)) * X::PC + wave0 + 4 * NB * (l16 & 3);
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

  // A sum of states is made from the last run to the first, each times the decay of those behind it: the runs that are read
  // first by the pass afterwards are the ones that the chip's cache has seen last.
  const int runs = (pend - p0 + C - 1) / C, first = STATE ? p0 + (runs - 1) * C : p0, next = STATE ? -C : C;
  double behind = 1.0;  // STATE: the decay of the runs behind this one
  load(first);
  store(first);
  load(first + next);
  if (STATE && runs > 0 && pend - first < C) update_weights(pend - first);
  __syncthreads();
  for (int i_run = 0, pos = first; i_run < runs; ++i_run, pos += next) {
    const int n = min(C, len - pos);
    f4 out[STATE ? 1 : TB][NB];
    if constexpr (!STATE) {
      // scores of the wavefront's blocks, decayed; zero where a position would see one behind it
      // (the places of the block in LDS are worked out for every run: kept, they took registers that are not there, and a
      // reload from memory waits for the loads of the next run)
      int tb = wave_tb;
      asm volatile("" : "+s"(tb));
      f4 score[BPW];
#pragma unroll
      for (int i = 0; i < BPW; ++i) score[i] = (f4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const Frag<NS> q = row_frag(rows_a + 16 * tb * X::PA + 32 * ks, C * X::PA);
#pragma unroll
        for (int i = 0; i < BPW; ++i) score[i] = mma(row_frag(rows_b + 16 * (sb0 + i) * X::PB + 32 * ks, C * X::PB), q, score[i]);
      }
#pragma unroll
      for (int i = 0; i < BPW; ++i) {
        const int sb = sb0 + i;
        float x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = score[i][r] * nw[max(16 * (tb - sb) + l16 - 4 * g - r, -1)];
        uint32_t w[NS][2];
        split<NS, 4>(x, w);
#pragma unroll
        for (int s = 0; s < NS; ++s) *(LdsU2*)(Ps + s * C * X::PP + (16 * tb + l16) * X::PP + 16 * sb + 4 * g) = (u2){w[s][0], w[s][1]};
      }
      __builtin_amdgcn_sched_barrier(0);  // (reads of LDS moved further up would take registers that are not there)
      // what the state before the run gives
#pragma unroll
      for (int i = 0; i < TB; ++i)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) out[i][nb] = (f4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        Frag<NS> sf[NB];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const f4 lo = S[ks][0][nb], hi = S[ks][1][nb];
          const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
          sf[nb] = frag_of<NS>(x);
        }
#pragma unroll
        for (int i = 0; i < TB; ++i) {
          const Frag<NS> q = row_frag(rows_a + 16 * i * X::PA + 32 * ks, C * X::PA);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) out[i][nb] = mma(sf[nb], q, out[i][nb]);
        }
      }
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        const float far = fw[16 * i + l16];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int r = 0; r < 4; ++r) out[i][nb][r] *= far;
      }
    }

    __builtin_amdgcn_sched_barrier(0);
    // the state after the run
    const float times = (float)behind;
    if constexpr (STATE) {
      if (times == 0.f) break;  // (for everybody alike; nothing further back is left of)
      behind *= n == C ? run_decay : (double)pw[n];
    } else {
      const double want = run_decay - run_decay * off;
      const float d = n == C ? (float)want : pw[n];
      off = ((double)(float)want - want) * per;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[ks][x][nb][r] = d * S[ks][x][nb][r];
    }
#pragma unroll
    for (int ks2 = 0; ks2 < CS; ++ks2) {
      Frag<3> wc[NB];
      f4 w0 = *(LdsF4*)(uw + 32 * ks2 + 8 * g), w1 = *(LdsF4*)(uw + 32 * ks2 + 8 * g + 4);
      if (STATE)
#pragma unroll
        for (int e = 0; e < 4; ++e) w0[e] *= times, w1[e] *= times;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float x[8];
        floats_of<NS>(col_frag(cols_c + 32 * ks2 * X::PC + 4 * nb, X::PC), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= e < 4 ? w0[e & 3] : w1[e & 3];
        wc[nb] = frag_of<3>(x);
      }
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const Frag<NS> kt = col_frag(cols_b + 32 * ks2 * X::PB + 32 * ks + 4 * y, X::PB);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) S[ks][y][nb] = mma(kt, wc[nb], S[ks][y][nb]);
        }
      if (!STATE) __builtin_amdgcn_sched_barrier(0);
    }
    Frag<NS> cf[CS][NB];
    if constexpr (!STATE)
#pragma unroll
      for (int ks2 = 0; ks2 < CS; ++ks2)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) cf[ks2][nb] = col_frag(cols_c + 32 * ks2 * X::PC + 4 * nb, X::PC);
    __syncthreads();

    // the next run's operands take the place of this one's, of which only the scores are still asked for
    store(pos + next);
    if (STATE && n < C) update_weights(C);
    load((int)((uint32_t)pos + 2u * (uint32_t)next));  // (past 2^31: negative, and nothing to load)
    if constexpr (!STATE) {
      // what the run's own positions give
#pragma unroll
      for (int ks2 = 0; ks2 < CS; ++ks2)
#pragma unroll
        for (int i = 2 * ks2; i < TB; ++i) {
          const Frag<NS> pf = row_frag(rows_p + 16 * i * X::PP + 32 * ks2, C * X::PP);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) out[i][nb] = mma(cf[ks2][nb], pf, out[i][nb]);
        }
      const __amdgpu_buffer_rsrc_t to = rsrc_of(out_base + (int64_t)(rev ? len - pos - C : pos) * out_pitch);
#pragma unroll
      for (int i = 0; i < TB; ++i) {
        // The whole distance is in the vector register: with a scalar offset beside it, a 16-byte store was seen to take its first
        // words from after the next write to their registers (lanes 12 to 15 of 16, with the chip loaded), which the compiler
        // guards against without one only.
        const int out_i = out_at + (rev ? TB - 1 - i : i) * 16 * out_pitch;
        const bool there = 16 * i + l16 < n;
        if (p.out_f32 || sizeof(T) == 4) {
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const int c = out_col + 4 * nb, to_c = out_i + 16 * nb;
            const bool whole = ACCESS == kVec ? c < dc : c + 4 <= dc;  // (rows of fp32 partial sums: their own multiple of 4)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, out[i][nb]), to, there && whole ? to_c : kPast, 0, 0);
            if (ACCESS != kVec)
#pragma unroll
              for (int e = 0; e < 3; ++e)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(out[i][nb][e]), to,
                                                      there && !whole && c + e < dc ? to_c + 4 * e : kPast, 0, 0);
          }
        } else {
          uint32_t w[2 * NB];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            w[2 * nb] = pack_bf16(out[i][nb][0], out[i][nb][1]);
            w[2 * nb + 1] = pack_bf16(out[i][nb][2], out[i][nb][3]);
          }
          const bool whole = ACCESS == kVec ? out_col < dc : out_col + 4 * NB <= dc;
          if constexpr (NB == 2)
            __builtin_amdgcn_raw_buffer_store_b128((u4){w[0], w[1], w[2], w[3]}, to, there && whole ? out_i : kPast, 0, 0);
          else
            __builtin_amdgcn_raw_buffer_store_b64((u2){w[0], w[1]}, to, there && whole ? out_i : kPast, 0, 0);
          if (ACCESS != kVec)
#pragma unroll
            for (int e = 0; e < 4 * NB - 1; ++e)
              __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(w[e / 2] >> (16 * (e & 1))), to,
                                                    there && !whole && out_col + e < dc ? out_i + 2 * e : kPast, 0, 0);
        }
      }
    }
    __syncthreads();
  }

  if constexpr (!STATE) {
    // tokens behind the last valid one
    const int64_t begin = max((int64_t)len, seg * sg.len), end = min(call.T, (seg + 1) * sg.len);
    const int cols = min(dc - tile0, X::VT);
    for (int64_t i = begin * cols + tid; i < end * cols; i += kThreads) {
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
    int rows = da - 4 * g;
    asm volatile("" : "+v"(rows));  // (the conditions of the first loads of S are not to be kept until here)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int col = col_of(l16, nb), lane_at = 4 * g * dc * 4 + col * 4;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int row = 32 * ks + 16 * x + r;
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[ks][x][nb][r]), rsrc_of(into),
                                                  col < dc && row < rows ? lane_at : kPast, row * dc * 4, 0);
          }
        }
  }
}

// Prefix sum over the segments: what is in segment g's place is the sum of segment g - 1 alone; after it, the state that
// enters g.  One thread for V elements of each (b, h): bound by the states' way to memory and back.
struct CombineArgs {
  LinattnCall c;
  SegmentArgs seg;
  const float* s_in;
  int64_t elems;
};
template <int V>
__global__ __launch_bounds__(256) void linattn_segments_kernel(CombineArgs a) {
  typedef float fv __attribute__((ext_vector_type(V)));
  const int64_t e = ((int64_t)blockIdx.y * 256 + threadIdx.x) * V;
  if (e >= a.elems) return;
  const int64_t bh = blockIdx.x, b = bh / a.c.H;
  const int h = (int)(bh % a.c.H);
  const int64_t len = length_of(a.c, b), slot = slot_of(a.c, b);
  const float log_decay = a.c.log_decay[h];
  const Decay full = decay_power(log_decay, a.seg.len);
  float* s = a.seg.states + bh * a.seg.n * a.elems + e;
  fv run = {};
  if (a.s_in && slot >= 0) run = *(const fv*)(a.s_in + (slot * a.c.H + h) * a.elems + e);
  if (a.s_in) *(fv*)s = run;
  constexpr int U = 8;
  for (int g0 = 1; g0 < a.seg.n; g0 += U) {
    fv x[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g0 + u < a.seg.n) x[u] = *(const fv*)(s + (g0 + u) * a.elems);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (g0 + u < a.seg.n) {
        const int64_t n = min(max(len - (g0 + u - 1) * a.seg.len, (int64_t)0), a.seg.len);  // positions of the segment before
        const Decay d = n == a.seg.len ? full : decay_power(log_decay, n);
#pragma unroll
        for (int i = 0; i < V; ++i) run[i] = d * run[i] + x[u][i];
        *(fv*)(s + (g0 + u) * a.elems) = run;
      }
  }
}

// Gradients of shared heads: a workgroup for each token (more tokens than a grid has: for some), a lane for the channels that
// are 256 apart.
constexpr int64_t kShareGrid = 1 << 20;
template <typename T>
__global__ __launch_bounds__(256) void linattn_share_kernel(const float* __restrict__ src, HeadView dst, int64_t tokens, int T_, int H,
                                                            int heads, int d) {
  const int g = H / heads;
  for (int64_t bt = blockIdx.x; bt < tokens; bt += kShareGrid) {
    const float* from = src + bt * H * d;
    T* to = (T*)dst.p + bt / T_ * dst.sb + bt % T_ * dst.st;
    for (int e = threadIdx.x; e < heads * d; e += 256) {
      const int hs = e / d, ch = e % d;
      float sum = 0.f;
      for (int j = 0; j < g; ++j) sum += from[(int64_t)(hs * g + j) * d + ch];
      to[hs * dst.sh + ch] = from_float<T>(sum);
    }
  }
}

template <typename T, int KP, int NB, bool STATE, int ACCESS>
mdh_status run(const PassArgs& a, hipStream_t st) {
  using X = Shape<T, KP, NB, STATE>;
  static int64_t done[kMaxDevices];
  int tiles = 0;
  for (int i = 0; i < a.n; ++i) tiles += a.tiles[i];
  const int64_t blocks = a.c.B * a.c.H * (STATE ? a.seg[0].n - 1 : a.seg[0].n) * tiles;
  if (blocks >= 1 << 24) return MDH_ERR_SIZE;  // 2^32 lanes
  const void* kern = (const void*)linattn_runs_kernel<T, KP, NB, STATE, ACCESS>;
  const mdh_status r = allow_dynamic_lds(kern, X::kBytes, done);
  if (r != MDH_OK) return r;
  clear_stale_error();
  linattn_runs_kernel<T, KP, NB, STATE, ACCESS><<<dim3((unsigned)blocks), kThreads, X::kBytes, st>>>(a);
  return launch_status();
}

template <typename T, bool STATE, int ACCESS>
mdh_status run_one(const PassArgs& a, int KP, hipStream_t st) {
  return KP == 64 ? run<T, 64, 1, STATE, ACCESS>(a, st)
                  : KP == 128 ? run<T, 128, 1, STATE, ACCESS>(a, st) : run<T, 256, 1, STATE, ACCESS>(a, st);
}

template <typename T, bool STATE>
mdh_status run(const PassArgs& a, int KP, int NB, int access, hipStream_t st) {
  if (access == kAny) return run_one<T, STATE, kAny>(a, KP, st);
  if (access == kEach) return run_one<T, STATE, kEach>(a, KP, st);
  if (NB == 1) return run_one<T, STATE, kVec>(a, KP, st);
  return KP == 128 ? run<T, 128, 2, STATE, kVec>(a, st) : run<T, 64, 2, STATE, kVec>(a, st);
}

// Launches of one workgroup a compute unit at most with two blocks a wavefront take one: twice the workgroups, each half the
// columns, unless the last tile would be mostly empty.  T = 2048, 32 heads of 128 x 128, 8 segments: 48.8 us against 51.8;
// 512, 16 heads, 4 segments: 23.9 against 26.9; 6 x 1021, 12 heads of 80 x 96: 54.8 against 48.7 (half a tile empty).  With
// more workgroups the operands that both halves read cost more: 8 x 4096, 16 heads, trained: 710 against 608.
template <bool STATE>
mdh_status run(PassArgs& a, int dtype, int KP, int NB, int access, hipStream_t st) {
  if (NB == 2) {
    int64_t blocks = 0;
    bool full = true;
    for (int i = 0; i < a.n; ++i) {
      blocks += a.c.B * a.c.H * (STATE ? a.seg[i].n - 1 : a.seg[i].n) * a.tiles[i];
      full = full && (a.p[i].dc - 1) % 64 >= 48;
    }
    if (blocks <= 256 && full) {
      NB = 1;
      for (int i = 0; i < a.n; ++i) a.tiles[i] = (int)cdiv(a.p[i].dc, 64);
    }
  }
  return dtype == MDH_BF16 ? run<bf16, STATE>(a, KP, NB, access, st) : run<float, STATE>(a, KP, NB, access, st);
}

// The kernel for a pass's operands and output.
int access_of(const LinattnPass& p, int dtype, bool output) {
  if (p.a.vec && p.b.vec && p.c.vec && (!output || p.out.vec)) return kVec;
  const int row = dtype == MDH_BF16 ? 8 : 4;
  return p.da >= row && p.dc >= row ? kAny : kEach;
}

int padded(int da) { return da <= 64 ? 64 : da <= 128 ? 128 : 256; }
// column blocks of a wavefront: two where there are columns for them and the registers hold the state
int blocks_of(int KP, int dc, int access) { return access == kVec && KP <= 128 && dc > 64 ? 2 : 1; }

int run_length(int dtype) { return dtype == MDH_BF16 ? 64 : 32; }
int64_t tiles_of(int da, int dc) { return cdiv(dc, 64 * blocks_of(padded(da), dc, kVec)); }

}  // namespace

// bytes for the states of the segments: one set for the forward call, two for the backward call
size_t linattn_segment_bytes(int64_t B, int64_t T, int H, int dk, int dv, int dtype, bool backward) {
  int64_t len;
  const int n = linattn_segments(B, T, H, dk, dv, dtype, backward, &len);
  return n > 1 ? (size_t)B * H * n * dk * dv * sizeof(float) * (backward ? 2 : 1) : 0;
}

// Segments are whole runs.  Their number is that of the least estimated time, in microseconds: a run takes 3.6 where the
// chip's compute units have a workgroup each, 6 where they have two (more wait for those); with more than one segment
// their states are summed up first, in 0.6 of that, and each goes through memory four times at 4.5 TB/s.  Sweeps of 1 to 32
// segments over fifteen sizes: the choice is within some 12 % of the best of them; work to fill the chip twice in every
// case was up to 17 % off (1 x 2048 x 32 x 128 x 128: 8 segments 52.6 us, 16 60.5; one segment 120).
int linattn_segments(int64_t B, int64_t T, int H, int dk, int dv, int dtype, bool backward, int64_t* len) {
  const int C = run_length(dtype);
  const int64_t runs = cdiv(T, C);
  // workgroups of the largest launch, for one segment: the passes of d_q and d_k are alike, d_v's may be another kernel
  const int64_t forward = tiles_of(dk, dv), back = 2 * tiles_of(dv, dk);
  const bool alike = padded(dk) == padded(dv) && blocks_of(padded(dk), dv, kVec) == blocks_of(padded(dv), dk, kVec);
  const int64_t work = B * H * (!backward ? forward : alike ? back + forward : back > forward ? back : forward);
  const double run = (dk > 64 || dv > 64 ? 1.0 : 0.65), state = 4.0 * 4.0 * B * H * dk * dv * (backward ? 2 : 1) / 4.5e6;
  double best = 0.0;
  int best_n = 1;
  *len = (runs < 1 ? 1 : runs) * C;
  for (int n : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128}) {
    if (n > 1 && n > runs / 2) break;
    int64_t each = cdiv(runs, n);
    // an odd number: segments a power of two apart ask for the same memory channels in step (65536 x 16 x 128 x 128: 452 us
    // with 32 runs each, 433 with 33)
    if (n > 1 && each >= 16) each |= 1;
    const int64_t segs = runs > 0 ? cdiv(runs, each) : 1, groups = work * segs;
    double t = (double)each * run * (groups <= 256 ? 3.6 : groups <= 512 ? 3.6 + 2.4 * (double)(groups - 256) / 256.0 : 6.0 * (double)groups / 512.0);
    if (segs > 1) t = 1.6 * t + (double)segs * state + 8.0;
    if (n == 1 || t < best) best = t, best_n = (int)segs, *len = each * C;
    if (groups > 1024) break;
  }
  return best_n;
}

// The state entering each of n segments: `p` gives the operands (da x dc = dk x dv).
mdh_status launch_linattn_segments(const LinattnCall& c, const LinattnPass* p, int np, int n, int64_t len, float* const* states,
                                   int dtype, hipStream_t st) {
  PassArgs a{};
  a.c = c;
  a.n = np;
  int access = kVec;
  for (int i = 0; i < np; ++i) access = access_of(p[i], dtype, false) > access ? access_of(p[i], dtype, false) : access;
  const int KP = padded(p[0].da), NB = blocks_of(KP, p[0].dc, access);
  for (int i = 0; i < np; ++i) {
    a.p[i] = p[i];
    a.tiles[i] = (int)cdiv(p[i].dc, 64 * NB);
    a.seg[i] = SegmentArgs{n, len, states[i]};
  }
  mdh_status r = run<true>(a, dtype, KP, NB, access, st);
  for (int i = 0; i < np && r == MDH_OK; ++i) {
    const CombineArgs k{c, a.seg[i], p[i].s_in, (int64_t)p[i].da * p[i].dc};
    clear_stale_error();
    const unsigned states_n = (unsigned)(c.B * c.H);
    if (k.elems % 4 == 0)  // (the states are 16-byte aligned)
      linattn_segments_kernel<4><<<dim3(states_n, (unsigned)cdiv(k.elems, 1024)), 256, 0, st>>>(k);
    else
      linattn_segments_kernel<1><<<dim3(states_n, (unsigned)cdiv(k.elems, 256)), 256, 0, st>>>(k);
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
    const int access = access_of(passes[i], dtype, true), KP = padded(passes[i].da), NB = blocks_of(KP, passes[i].dc, access);
    PassArgs a{};
    a.c = c;
    for (int j = i; j < np; ++j) {
      if (gone[j] || access_of(passes[j], dtype, true) != access || padded(passes[j].da) != KP || blocks_of(KP, passes[j].dc, access) != NB)
        continue;
      gone[j] = true;
      a.p[a.n] = passes[j];
      a.tiles[a.n] = (int)cdiv(passes[j].dc, 64 * NB);
      a.seg[a.n] = SegmentArgs{n, len, states[j]};
      a.seg_t[a.n] = turned[j];
      ++a.n;
    }
    const mdh_status r = run<false>(a, dtype, KP, NB, access, st);
    if (r != MDH_OK) return r;
  }
  return MDH_OK;
}

mdh_status launch_linattn_share(const LinattnCall& c, const float* src, int d, const HeadView& dst, int heads, int dtype,
                                hipStream_t st) {
  const int64_t tokens = c.B * c.T;
  if (tokens == 0) return MDH_OK;
  const dim3 grid((unsigned)(tokens < kShareGrid ? tokens : kShareGrid));
  clear_stale_error();
  if (dtype == MDH_BF16)
    linattn_share_kernel<bf16><<<grid, 256, 0, st>>>(src, dst, tokens, (int)c.T, c.H, heads, d);
  else
    linattn_share_kernel<float><<<grid, 256, 0, st>>>(src, dst, tokens, (int)c.T, c.H, heads, d);
  return launch_status();
}

}  // namespace mdh

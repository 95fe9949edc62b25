// Device entry points of the sequence layers (include/mdh.h): argument checks, views, the passes of a call.
#include "mdh_internal.h"

using namespace mdh;

namespace {

struct LinattnSizes {
  int64_t B, T;
  int H, Hq, Hk, Hv, dk, dv;
};

// T is 1 and absent from the sizes of a single token
mdh_status linattn_sizes(const int64_t* sizes, bool step, LinattnSizes* z) {
  if (!sizes) return MDH_ERR_NULL;
  z->B = sizes[0];
  z->T = step ? 1 : sizes[1];
  const int64_t* heads = sizes + (step ? 1 : 2);
  if (z->B < 0 || z->T < 0 || z->B > 0x7fffffff || z->T > 0x7fffffff - 64) return MDH_ERR_SIZE;
  for (int i = 0; i < 6; ++i)
    if (heads[i] < 1 || heads[i] > 0x7fffffff) return MDH_ERR_SIZE;
  if (z->B * heads[0] > 0x7fffffff) return MDH_ERR_SIZE;
  for (int i = 1; i < 4; ++i)
    if (heads[0] % heads[i]) return MDH_ERR_SIZE;
  if (heads[4] > 256 || heads[5] > 256) return MDH_ERR_UNSUPPORTED;
  z->H = (int)heads[0], z->Hq = (int)heads[1], z->Hk = (int)heads[2], z->Hv = (int)heads[3];
  z->dk = (int)heads[4], z->dv = (int)heads[5];
  return MDH_OK;
}

// The view of (B, T, heads, d) elements of `bytes` bytes; strides: (batch, token, head), or null: dense.  Strides of an
// extent of 1 are not used.
HeadView view_of(const void* p, const int64_t* strides, const LinattnSizes& z, int heads, int d, int bytes) {
  HeadView v{p, 0, 0, 0, z.H / heads, 0};
  if (strides) {
    v.sb = strides[0], v.st = strides[1], v.sh = strides[2];
  } else {
    v.sh = d, v.st = (int64_t)heads * d, v.sb = z.T * v.st;
  }
  if (z.B == 1) v.sb = 0;
  if (z.T == 1) v.st = 0;
  if (heads == 1) v.sh = 0;
  const int unit = 16 / bytes;
  v.vec = (uintptr_t)p % 16 == 0 && v.sb % unit == 0 && v.st % unit == 0 && v.sh % unit == 0 && d % unit == 0;
  return v;
}

// the rows of 64 consecutive tokens are addressed with 31 bits
bool out_of_reach(const HeadView& v, int bytes) { return v.st < 0 || v.st > (((int64_t)1 << 31) - 4096) / 64 / bytes; }

// an output whose elements share a place has no value
bool overlaps(const HeadView& v, const LinattnSizes& z, int heads) {
  return (z.B > 1 && z.T > 0 && v.sb == 0) || (z.T > 1 && v.st == 0) || (heads > 1 && z.T > 0 && v.sh == 0);
}

int bytes_of(mdh_dtype t) { return t == MDH_BF16 ? 2 : t == MDH_F32 ? 4 : 0; }
size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
bool misaligned(const void* p, size_t to) { return (uintptr_t)p % to != 0; }

// gradients of shared heads: fp32 of every head first, summed afterwards
size_t share_bytes(const LinattnSizes& z, int heads, int d) {
  return heads == z.H ? 0 : up16((size_t)z.B * (size_t)z.T * (size_t)z.H * (size_t)d * sizeof(float));
}

size_t segment_bytes(const LinattnSizes& z, mdh_dtype dtype, bool backward) {
  return up16(linattn_segment_bytes(z.B, z.T, z.H, z.dk, z.dv, dtype, backward));
}
size_t linattn_need(const LinattnSizes& z, mdh_dtype dtype, bool backward) {
  const size_t forward = segment_bytes(z, dtype, false);
  if (!backward) return forward;
  const size_t n = segment_bytes(z, dtype, true) + share_bytes(z, z.Hq, z.dk) + share_bytes(z, z.Hk, z.dk) + share_bytes(z, z.Hv, z.dv);
  return n > forward ? n : forward;  // one workspace for both calls of a training step
}

LinattnCall call_of(const LinattnSizes& z, const float* log_decay, const int32_t* lengths, const int32_t* slots, int64_t n_slots) {
  return LinattnCall{z.B, z.T, z.H, log_decay, lengths, slots, n_slots};
}

}  // namespace

extern "C" {

size_t mdh_linattn_workspace_size(const int64_t* sizes, mdh_dtype dtype, int32_t backward) {
  LinattnSizes z;
  if (!bytes_of(dtype) || linattn_sizes(sizes, false, &z) != MDH_OK) return 0;
  return linattn_need(z, dtype, backward != 0);
}

mdh_status mdh_linattn(const int64_t* sizes, mdh_dtype dtype, const void* q, const void* k, const void* v,
                       const int64_t* strides, const float* log_decay, float scale, const int32_t* lengths,
                       const float* initial_state, float* final_state, const int32_t* slots, int64_t n_slots, void* o,
                       void* workspace, size_t workspace_bytes, void* stream) {
  LinattnSizes z;
  const mdh_status st = linattn_sizes(sizes, false, &z);
  if (st != MDH_OK) return st;
  const int e = bytes_of(dtype);
  if (!e) return MDH_ERR_UNSUPPORTED;
  if (slots && n_slots < 0) return MDH_ERR_SIZE;
  if (z.B == 0 || (z.T == 0 && !final_state)) return MDH_OK;
  if (!log_decay || (z.T > 0 && (!q || !k || !v || !o))) return MDH_ERR_NULL;
  if (misaligned(initial_state, 16) || misaligned(final_state, 16) || misaligned(q, e) || misaligned(k, e) || misaligned(v, e) ||
      misaligned(o, e))
    return MDH_ERR_UNSUPPORTED;
  const size_t need = linattn_need(z, dtype, false);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return MDH_ERR_WORKSPACE;
  auto sub = [&](int i) { return strides ? strides + 3 * i : nullptr; };
  LinattnPass p{};
  p.a = view_of(q, sub(0), z, z.Hq, z.dk, e);
  p.b = view_of(k, sub(1), z, z.Hk, z.dk, e);
  p.c = view_of(v, sub(2), z, z.Hv, z.dv, e);
  p.out = view_of(o, sub(3), z, z.H, z.dv, e);
  if (overlaps(p.out, z, z.H)) return MDH_ERR_SIZE;
  if (out_of_reach(p.a, e) || out_of_reach(p.b, e) || out_of_reach(p.c, e) || out_of_reach(p.out, e)) return MDH_ERR_SIZE;
  p.da = z.dk, p.dc = z.dv;
  p.scale_r = scale, p.scale_u = 1.f;
  p.rev = 0, p.shift = 1;
  p.s_in = initial_state, p.s_out = final_state;
  const LinattnCall c = call_of(z, log_decay, lengths, slots, n_slots);
  int64_t len;
  const int n = linattn_segments(z.B, z.T, z.H, z.dk, z.dv, dtype, false, &len);
  float* const states[1] = {(float*)workspace};
  const int turned[1] = {0};
  if (n > 1) {
    const mdh_status r = launch_linattn_segments(c, &p, 1, n, len, states, dtype, (hipStream_t)stream);
    if (r != MDH_OK) return r;
  }
  return launch_linattn_pass(c, &p, 1, n, len, states, turned, dtype, (hipStream_t)stream);
}

mdh_status mdh_linattn_backward(const int64_t* sizes, mdh_dtype dtype, const void* q, const void* k, const void* v,
                                const void* d_o, const int64_t* strides, const float* log_decay, float scale,
                                const int32_t* lengths, const float* initial_state, const float* d_final_state, void* d_q,
                                void* d_k, void* d_v, float* d_initial_state, void* workspace, size_t workspace_bytes,
                                void* stream) {
  LinattnSizes z;
  mdh_status st = linattn_sizes(sizes, false, &z);
  if (st != MDH_OK) return st;
  const int e = bytes_of(dtype);
  if (!e) return MDH_ERR_UNSUPPORTED;
  if (z.B == 0 || (z.T == 0 && !d_initial_state)) return MDH_OK;
  if (!log_decay || (z.T > 0 && (!q || !k || !v || !d_o || !d_q || !d_k || !d_v))) return MDH_ERR_NULL;
  if (misaligned(initial_state, 16) || misaligned(d_final_state, 16) || misaligned(d_initial_state, 16) ||
      (d_initial_state && d_initial_state == d_final_state))
    return MDH_ERR_UNSUPPORTED;
  const void* all[7] = {q, k, v, d_o, d_q, d_k, d_v};
  for (const void* p : all)
    if (misaligned(p, e)) return MDH_ERR_UNSUPPORTED;
  const size_t need = linattn_need(z, dtype, true);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return MDH_ERR_WORKSPACE;
  auto view = [&](int i, int heads, int d) { return view_of(all[i], strides ? strides + 3 * i : nullptr, z, heads, d, e); };
  const HeadView vq = view(0, z.Hq, z.dk), vk = view(1, z.Hk, z.dk), vv = view(2, z.Hv, z.dv), vo = view(3, z.H, z.dv);
  const HeadView grad[3] = {view(4, z.Hq, z.dk), view(5, z.Hk, z.dk), view(6, z.Hv, z.dv)};
  const int heads[3] = {z.Hq, z.Hk, z.Hv};
  for (int i = 0; i < 3; ++i)
    if (overlaps(grad[i], z, heads[i]) || out_of_reach(grad[i], e)) return MDH_ERR_SIZE;
  if (out_of_reach(vq, e) || out_of_reach(vk, e) || out_of_reach(vv, e) || out_of_reach(vo, e)) return MDH_ERR_SIZE;
  const LinattnCall c = call_of(z, log_decay, lengths, nullptr, 0);
  LinattnPass p[3] = {};
  p[0].a = vo, p[0].b = vv, p[0].c = vk;  // d_q: the forward state, from its other side
  p[0].da = z.dv, p[0].dc = z.dk;
  p[0].scale_r = scale, p[0].scale_u = 1.f, p[0].shift = 1;
  p[0].s_in = initial_state, p[0].s_in_t = 1;
  p[1].a = vv, p[1].b = vo, p[1].c = vq;  // d_k
  p[1].da = z.dv, p[1].dc = z.dk;
  p[1].scale_r = 1.f, p[1].scale_u = scale, p[1].rev = 1;
  p[1].s_in = d_final_state, p[1].s_in_t = 1;
  p[2].a = vk, p[2].b = vq, p[2].c = vo;  // d_v
  p[2].da = z.dk, p[2].dc = z.dv;
  p[2].scale_r = 1.f, p[2].scale_u = scale, p[2].rev = 1;
  p[2].s_in = d_final_state, p[2].s_out = d_initial_state;
  char* ws = (char*)workspace + segment_bytes(z, dtype, true);
  for (int i = 0; i < 3; ++i) {
    p[i].out = grad[i];
    if (heads[i] == z.H) continue;
    p[i].out = view_of(ws, nullptr, z, z.H, p[i].dc, sizeof(float));
    p[i].out_f32 = 1;
    if (out_of_reach(p[i].out, sizeof(float))) return MDH_ERR_SIZE;
    ws += share_bytes(z, heads[i], p[i].dc);
  }
  int64_t len;
  const int n = linattn_segments(z.B, z.T, z.H, z.dk, z.dv, dtype, true, &len);
  // the states of the segments, as dk x dv: forward in time for d_q, backward for d_k and d_v
  float* const two[2] = {(float*)workspace, (float*)workspace + (size_t)z.B * z.H * n * z.dk * z.dv};
  float* const states[3] = {two[0], two[1], two[1]};
  const int turned[3] = {1, 1, 0};
  if (n > 1) {
    LinattnPass sums[2] = {};
    sums[0].b = vk, sums[0].c = vv, sums[0].scale_u = 1.f, sums[0].shift = 1, sums[0].s_in = initial_state;
    sums[1].b = vq, sums[1].c = vo, sums[1].scale_u = scale, sums[1].rev = 1, sums[1].s_in = d_final_state;
    for (LinattnPass& s : sums) s.a = s.b, s.da = z.dk, s.dc = z.dv;
    st = launch_linattn_segments(c, sums, 2, n, len, two, dtype, (hipStream_t)stream);
    if (st != MDH_OK) return st;
  }
  st = launch_linattn_pass(c, p, 3, n, len, states, turned, dtype, (hipStream_t)stream);
  for (int i = 0; i < 3 && st == MDH_OK; ++i)
    if (p[i].out_f32) st = launch_linattn_share(c, (const float*)p[i].out.p, p[i].dc, grad[i], heads[i], dtype, (hipStream_t)stream);
  return st;
}

mdh_status mdh_linattn_step(const int64_t* sizes, mdh_dtype dtype, const void* q, const void* k, const void* v,
                            const int64_t* strides, const float* log_decay, float scale, float* state,
                            const int32_t* slots, int64_t n_slots, void* o, void* stream) {
  LinattnSizes z;
  const mdh_status st = linattn_sizes(sizes, true, &z);
  if (st != MDH_OK) return st;
  const int e = bytes_of(dtype);
  if (!e) return MDH_ERR_UNSUPPORTED;
  if (slots && n_slots < 0) return MDH_ERR_SIZE;
  if (z.B == 0) return MDH_OK;
  if (!q || !k || !v || !o || !log_decay || !state) return MDH_ERR_NULL;
  if (misaligned(state, 4) || misaligned(q, e) || misaligned(k, e) || misaligned(v, e) || misaligned(o, e)) return MDH_ERR_UNSUPPORTED;
  auto view = [&](int i, const void* p, int heads, int d) {
    if (!strides) return view_of(p, nullptr, z, heads, d, e);
    const int64_t s[3] = {strides[2 * i], 0, strides[2 * i + 1]};
    return view_of(p, s, z, heads, d, e);
  };
  const HeadView out = view(3, o, z.H, z.dv);
  if (overlaps(out, z, z.H)) return MDH_ERR_SIZE;
  return launch_linattn_step(call_of(z, log_decay, nullptr, slots, n_slots), view(0, q, z.Hq, z.dk), view(1, k, z.Hk, z.dk),
                             view(2, v, z.Hv, z.dv), out, z.dk, z.dv, scale, state, dtype, (hipStream_t)stream);
}

// ------------------------------------------------------------------------------ group norm

namespace {
mdh_status group_norm_sizes(const int64_t* sizes, mdh_dtype dtype, int32_t act, GroupNormCall* c) {
  if (!sizes) return MDH_ERR_NULL;
  for (int i = 0; i < 4; ++i)
    if (sizes[i] < (i < 2 ? 0 : 1) || sizes[i] > 0x7fffffff) return MDH_ERR_SIZE;
  if (sizes[2] % sizes[3]) return MDH_ERR_SIZE;
  if (sizes[0] && (sizes[0] * sizes[3] > 0x7fffffff || sizes[0] * sizes[1] > 0x7fffffff)) return MDH_ERR_SIZE;
  if (!bytes_of(dtype) || act < MDH_ACT_NONE || act > MDH_ACT_GELU) return MDH_ERR_UNSUPPORTED;
  *c = GroupNormCall{};
  c->N = sizes[0], c->S = sizes[1], c->C = (int)sizes[2], c->G = (int)sizes[3];
  c->dtype = dtype, c->act = act;
  return MDH_OK;
}
RowView rows_of(const void* p, const int64_t* strides, int i, const GroupNormCall& c) {
  RowView v{p, strides ? strides[i] : (int64_t)c.C};
  if (c.N * c.S == 1) v.stride = 0;
  return v;
}
}  // namespace

size_t mdh_group_norm_workspace_size(const int64_t* sizes, mdh_dtype dtype, int32_t backward) {
  GroupNormCall c;
  if (group_norm_sizes(sizes, dtype, MDH_ACT_NONE, &c) != MDH_OK) return 0;
  return group_norm_workspace(c, backward != 0);
}

mdh_status mdh_group_norm(const int64_t* sizes, mdh_dtype dtype, const void* x, const void* gate, const int64_t* row_strides,
                          const float* weight, const float* bias, float eps, int32_t act, void* y, float* mean, float* rstd,
                          void* workspace, size_t workspace_bytes, void* stream) {
  GroupNormCall c;
  const mdh_status st = group_norm_sizes(sizes, dtype, act, &c);
  if (st != MDH_OK) return st;
  if (c.N == 0 || c.S == 0) return MDH_OK;
  if (!x || !y) return MDH_ERR_NULL;
  const int e = bytes_of(dtype);
  if (misaligned(x, e) || misaligned(y, e) || misaligned(gate, e)) return MDH_ERR_UNSUPPORTED;
  const size_t need = group_norm_workspace(c, false);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return MDH_ERR_WORKSPACE;
  c.x = rows_of(x, row_strides, 0, c), c.gate = rows_of(gate, row_strides, 1, c), c.y = rows_of(y, row_strides, 2, c);
  if (c.N * c.S > 1 && c.y.stride < c.C) return MDH_ERR_SIZE;
  c.weight = weight, c.bias = bias, c.eps = eps, c.mean = mean, c.rstd = rstd, c.ws = workspace;
  return launch_group_norm(c, (hipStream_t)stream);
}

mdh_status mdh_group_norm_backward(const int64_t* sizes, mdh_dtype dtype, const void* x, const void* gate,
                                   const void* d_y, const int64_t* row_strides, const float* weight, const float* bias,
                                   const float* mean, const float* rstd, int32_t act, void* d_x, void* d_gate,
                                   float* d_weight, float* d_bias, void* workspace, size_t workspace_bytes, void* stream) {
  GroupNormCall c;
  const mdh_status st = group_norm_sizes(sizes, dtype, act, &c);
  if (st != MDH_OK) return st;
  const bool empty = c.N == 0 || c.S == 0;
  if (!empty && (!x || !d_y || !mean || !rstd || !d_x || (gate && !d_gate))) return MDH_ERR_NULL;
  const int e = bytes_of(dtype);
  if (misaligned(x, e) || misaligned(gate, e) || misaligned(d_y, e) || misaligned(d_x, e) || misaligned(d_gate, e))
    return MDH_ERR_UNSUPPORTED;
  const size_t need = group_norm_workspace(c, true);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, 16))) return MDH_ERR_WORKSPACE;
  c.x = rows_of(x, row_strides, 0, c), c.gate = rows_of(gate, row_strides, 1, c), c.y = rows_of(d_y, row_strides, 2, c);
  c.dx = rows_of(d_x, row_strides, 3, c), c.dgate = rows_of(gate ? d_gate : nullptr, row_strides, 4, c);
  if (c.N * c.S > 1 && (c.dx.stride < c.C || (gate && c.dgate.stride < c.C))) return MDH_ERR_SIZE;
  c.weight = weight, c.bias = bias, c.mean = (float*)mean, c.rstd = (float*)rstd, c.ws = workspace;
  c.dweight = d_weight, c.dbias = d_bias;
  return launch_group_norm_backward(c, (hipStream_t)stream);
}

}  // extern "C"

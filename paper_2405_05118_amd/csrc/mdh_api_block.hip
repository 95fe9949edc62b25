// Device entry points of a selective state space block (include/mdh.h): argument checks and views.
#include "mdh_internal.h"

using namespace mdh;

namespace {

constexpr int64_t kMax = 0x7fffffff, kChannels = 1 << 24;

int bytes_of(mdh_dtype t) { return t == MDH_BF16 ? 2 : t == MDH_F32 ? 4 : 0; }
bool misaligned(const void* p, size_t to) { return (uintptr_t)p % to != 0; }
template <typename... P>
bool any_misaligned(size_t to, P... p) {
  return (misaligned(p, to) || ...);
}
bool short_of(const void* p, size_t bytes, size_t need) { return need && (!p || bytes < need || misaligned(p, 16)); }

bool tokens_fit(int64_t B, int64_t T) { return B >= 0 && T >= 0 && B <= kMax && T <= kMax - 64 && B * T <= kMax; }

// strides of an extent of 1 are not used
TokenView tokens(const void* p, const int64_t* strides, int64_t B, int64_t T, int64_t C) {
  TokenView v{p, strides ? strides[0] : T * C, strides ? strides[1] : C};
  if (B == 1) v.sb = 0;
  if (T == 1) v.st = 0;
  return v;
}
SharedView shared(const void* p, const int64_t* strides, const ScanCall& c) {
  SharedView v{p, strides ? strides[0] : c.T * c.G * c.N, strides ? strides[1] : (int64_t)c.G * c.N, strides ? strides[2] : c.N};
  if (c.B == 1) v.sb = 0;
  if (c.T == 1) v.st = 0;
  if (c.G == 1) v.sg = 0;
  return v;
}
// an output whose elements share a place has no value: rows of n elements closer than that
bool closer(int64_t extent, int64_t stride, int64_t n) { return extent > 1 && (stride < 0 ? -stride : stride) < n; }
bool overlaps(const TokenView& v, int64_t B, int64_t T, int64_t C) { return T > 0 && (closer(B, v.sb, C) || closer(T, v.st, C)); }
bool overlaps(const SharedView& v, const ScanCall& c) {
  return c.T > 0 && (closer(c.B, v.sb, c.N) || closer(c.T, v.st, c.N) || closer(c.G, v.sg, c.N));
}

// (B, T, C, W), without T for one token
mdh_status conv_sizes(const int64_t* sizes, mdh_dtype dtype, int32_t act, bool step, ConvCall* c) {
  if (!sizes) return MDH_ERR_NULL;
  const int64_t B = sizes[0], T = step ? 1 : sizes[1], C = sizes[step ? 1 : 2], W = sizes[step ? 2 : 3];
  if (!tokens_fit(B, T) || C < 1 || C >= kChannels || W < 1) return MDH_ERR_SIZE;
  if (W > 8 || !bytes_of(dtype) || act < MDH_ACT_NONE || act > MDH_ACT_GELU) return MDH_ERR_UNSUPPORTED;
  *c = ConvCall{};
  c->B = B, c->T = T, c->C = (int)C, c->W = (int)W, c->dtype = dtype, c->act = act;
  return MDH_OK;
}
// (B, T, D, N, G), without T for one token
mdh_status scan_sizes(const int64_t* sizes, mdh_dtype dtype, bool step, ScanCall* c) {
  if (!sizes) return MDH_ERR_NULL;
  const int64_t B = sizes[0], T = step ? 1 : sizes[1], *rest = sizes + (step ? 1 : 2), D = rest[0], N = rest[1], G = rest[2];
  if (!tokens_fit(B, T) || D < 1 || D >= kChannels || N < 1 || G < 1 || D % G) return MDH_ERR_SIZE;
  if (N > 64 || !bytes_of(dtype)) return MDH_ERR_UNSUPPORTED;
  if (B * T * G >= ((int64_t)1 << 32) / N) return MDH_ERR_SIZE;
  *c = ScanCall{};
  c->B = B, c->T = T, c->tiles = cdiv(T, kScanTile), c->D = (int)D, c->N = (int)N, c->G = (int)G, c->E = (int)(D / G), c->dtype = dtype;
  return MDH_OK;
}
size_t checkpoint_bytes(const ScanCall& c) { return (size_t)c.B * c.tiles * c.D * c.N * sizeof(float); }
mdh_status norm_sizes(const int64_t* sizes, mdh_dtype dtype, LayerNormCall* c) {
  if (!sizes) return MDH_ERR_NULL;
  if (sizes[0] < 0 || sizes[0] > kMax || sizes[1] < 1 || sizes[1] >= kChannels) return MDH_ERR_SIZE;
  if (!bytes_of(dtype)) return MDH_ERR_UNSUPPORTED;
  *c = LayerNormCall{};
  c->rows = sizes[0], c->C = (int)sizes[1], c->dtype = dtype;
  return MDH_OK;
}
RowView rows_of(const void* p, const int64_t* strides, int i, const LayerNormCall& c) {
  return RowView{p, c.rows == 1 ? 0 : strides ? strides[i] : (int64_t)c.C};
}
size_t more(size_t a, size_t b) { return a > b ? a : b; }

}  // namespace

extern "C" {

// ------------------------------------------------------------------------------ causal convolution

mdh_status mdh_causal_conv(const int64_t* sizes, mdh_dtype dtype, const void* x, const int64_t* strides, const float* weight,
                           const float* bias, int32_t act, const int32_t* lengths, const void* initial_window,
                           void* final_window, const int32_t* slots, int64_t n_slots, void* y, void* stream) {
  ConvCall c;
  const mdh_status st = conv_sizes(sizes, dtype, act, false, &c);
  if (st != MDH_OK) return st;
  if (slots && n_slots < 0) return MDH_ERR_SIZE;
  if (c.B == 0 || (c.T == 0 && !final_window)) return MDH_OK;
  if (!weight || (c.T > 0 && (!x || !y))) return MDH_ERR_NULL;
  if (any_misaligned(bytes_of(dtype), x, y, initial_window, final_window) || any_misaligned(4, weight, bias)) return MDH_ERR_UNSUPPORTED;
  c.x = tokens(x, strides, c.B, c.T, c.C), c.y = tokens(y, strides ? strides + 2 : nullptr, c.B, c.T, c.C);
  if (overlaps(c.y, c.B, c.T, c.C)) return MDH_ERR_SIZE;
  c.weight = weight, c.bias = bias, c.lengths = lengths, c.slots = slots, c.n_slots = n_slots;
  c.s_in = initial_window, c.s_out = final_window;
  return launch_conv(c, (hipStream_t)stream);
}

size_t mdh_causal_conv_workspace_size(const int64_t* sizes, mdh_dtype dtype) {
  ConvCall c;
  return conv_sizes(sizes, dtype, MDH_ACT_NONE, false, &c) == MDH_OK ? conv_workspace(c) : 0;
}

mdh_status mdh_causal_conv_backward(const int64_t* sizes, mdh_dtype dtype, const void* x, const void* d_y, const int64_t* strides,
                                    const float* weight, const float* bias, int32_t act, const int32_t* lengths,
                                    const void* initial_window, const void* d_final_window, void* d_x, void* d_initial_window,
                                    float* d_weight, float* d_bias, void* workspace, size_t workspace_bytes, void* stream) {
  ConvCall c;
  const mdh_status st = conv_sizes(sizes, dtype, act, false, &c);
  if (st != MDH_OK) return st;
  if (c.B > 0 && (!weight || (c.T > 0 && (!x || !d_y || !d_x)))) return MDH_ERR_NULL;
  if (any_misaligned(bytes_of(dtype), x, d_y, d_x, initial_window, d_final_window, d_initial_window) ||
      any_misaligned(4, weight, bias, d_weight, d_bias) || (d_initial_window && d_initial_window == d_final_window))
    return MDH_ERR_UNSUPPORTED;
  if (short_of(workspace, workspace_bytes, conv_workspace(c))) return MDH_ERR_WORKSPACE;
  auto view = [&](const void* p, int i) { return tokens(p, strides ? strides + 2 * i : nullptr, c.B, c.T, c.C); };
  c.x = view(x, 0), c.y = view(d_y, 1), c.dx = view(d_x, 2);
  if (overlaps(c.dx, c.B, c.T, c.C)) return MDH_ERR_SIZE;
  c.weight = weight, c.bias = bias, c.lengths = lengths, c.s_in = initial_window, c.d_out = d_final_window, c.d_in = d_initial_window;
  c.part = (float*)workspace, c.dweight = d_weight, c.dbias = d_bias;
  return launch_conv_backward(c, (hipStream_t)stream);
}

mdh_status mdh_causal_conv_step(const int64_t* sizes, mdh_dtype dtype, const void* x, const int64_t* strides, const float* weight,
                                const float* bias, int32_t act, void* window, const int32_t* slots, int64_t n_slots, void* y,
                                void* stream) {
  ConvCall c;
  const mdh_status st = conv_sizes(sizes, dtype, act, true, &c);
  if (st != MDH_OK) return st;
  if (slots && n_slots < 0) return MDH_ERR_SIZE;
  if (c.B == 0) return MDH_OK;
  if (!x || !y || !weight || (!window && c.W > 1)) return MDH_ERR_NULL;
  if (any_misaligned(bytes_of(dtype), x, y, window) || any_misaligned(4, weight, bias)) return MDH_ERR_UNSUPPORTED;
  const int64_t sx[2] = {strides ? strides[0] : c.C, 0}, sy[2] = {strides ? strides[1] : c.C, 0};
  c.x = tokens(x, sx, c.B, 1, c.C), c.y = tokens(y, sy, c.B, 1, c.C);
  if (overlaps(c.y, c.B, 1, c.C)) return MDH_ERR_SIZE;
  c.weight = weight, c.bias = bias, c.slots = slots, c.n_slots = n_slots, c.s_out = window;
  return launch_conv_step(c, (hipStream_t)stream);
}

// ------------------------------------------------------------------------------ selective scan

size_t mdh_selective_scan_workspace_size(const int64_t* sizes, mdh_dtype dtype, int32_t backward) {
  ScanCall c;
  if (scan_sizes(sizes, dtype, false, &c) != MDH_OK) return 0;
  return backward ? more(scan_workspace(c), scan_backward_workspace(c)) : scan_workspace(c);
}
size_t mdh_selective_scan_checkpoints_size(const int64_t* sizes) {
  ScanCall c;
  return scan_sizes(sizes, MDH_F32, false, &c) == MDH_OK ? checkpoint_bytes(c) : 0;
}

mdh_status mdh_selective_scan(const int64_t* sizes, mdh_dtype dtype, const void* x, const void* dt, const void* gate, const void* b,
                              const void* c_, const int64_t* strides, const float* A, const float* skip, const float* dt_bias,
                              int32_t softplus, const int32_t* lengths, const float* initial_state, float* final_state,
                              const int32_t* slots, int64_t n_slots, void* y, void* checkpoints, size_t checkpoints_bytes,
                              void* workspace, size_t workspace_bytes, void* stream) {
  ScanCall c;
  const mdh_status st = scan_sizes(sizes, dtype, false, &c);
  if (st != MDH_OK) return st;
  if (slots && n_slots < 0) return MDH_ERR_SIZE;
  if (c.B == 0 || (c.T == 0 && !final_state)) return MDH_OK;
  if (!A || (c.T > 0 && (!x || !dt || !b || !c_ || !y))) return MDH_ERR_NULL;
  if (any_misaligned(bytes_of(dtype), x, dt, gate, b, c_, y) || any_misaligned(4, A, skip, dt_bias, initial_state, final_state))
    return MDH_ERR_UNSUPPORTED;
  if (short_of(workspace, workspace_bytes, scan_workspace(c))) return MDH_ERR_WORKSPACE;
  if (checkpoints && short_of(checkpoints, checkpoints_bytes, checkpoint_bytes(c))) return MDH_ERR_WORKSPACE;
  auto view = [&](const void* p, int i) { return tokens(p, strides ? strides + 2 * i : nullptr, c.B, c.T, c.D); };
  c.in[0] = view(x, 0), c.in[1] = view(dt, 1), c.in[2] = view(gate, 2), c.out[0] = view(y, 3);
  c.bc[0] = shared(b, strides ? strides + 8 : nullptr, c), c.bc[1] = shared(c_, strides ? strides + 11 : nullptr, c);
  if (overlaps(c.out[0], c.B, c.T, c.D)) return MDH_ERR_SIZE;
  c.A = A, c.skip = skip, c.dt_bias = dt_bias, c.softplus = softplus != 0, c.lengths = lengths, c.slots = slots, c.n_slots = n_slots;
  c.s_in = initial_state, c.s_out = final_state, c.checkpoints = (float*)checkpoints, c.ws = workspace;
  return launch_scan_forward(c, (hipStream_t)stream);
}

mdh_status mdh_selective_scan_backward(const int64_t* sizes, mdh_dtype dtype, const void* x, const void* dt, const void* gate,
                                       const void* b, const void* c_, const void* d_y, const int64_t* strides, const float* A,
                                       const float* skip, const float* dt_bias, int32_t softplus, const int32_t* lengths,
                                       const float* d_final_state, const void* checkpoints, size_t checkpoints_bytes, void* d_x,
                                       void* d_dt, void* d_gate, void* d_b, void* d_c, float* d_A, float* d_skip, float* d_dt_bias,
                                       float* d_initial_state, void* workspace, size_t workspace_bytes, void* stream) {
  ScanCall c;
  const mdh_status st = scan_sizes(sizes, dtype, false, &c);
  if (st != MDH_OK) return st;
  if (c.B > 0 && (!A || (c.T > 0 && (!x || !dt || !b || !c_ || !d_y || !d_x || !d_dt || !d_b || !d_c || (gate && !d_gate)))))
    return MDH_ERR_NULL;
  if (any_misaligned(bytes_of(dtype), x, dt, gate, b, c_, d_y, d_x, d_dt, d_gate, d_b, d_c) ||
      any_misaligned(4, A, skip, dt_bias, d_final_state, d_A, d_skip, d_dt_bias, d_initial_state) ||
      (d_initial_state && d_initial_state == d_final_state))
    return MDH_ERR_UNSUPPORTED;
  if (short_of(workspace, workspace_bytes, scan_backward_workspace(c)) || short_of(checkpoints, checkpoints_bytes, checkpoint_bytes(c)))
    return MDH_ERR_WORKSPACE;
  auto view = [&](const void* p, int i) { return tokens(p, strides ? strides + 2 * i : nullptr, c.B, c.T, c.D); };
  auto view2 = [&](const void* p, int i) { return shared(p, strides ? strides + 14 + 3 * i : nullptr, c); };
  c.in[0] = view(x, 0), c.in[1] = view(dt, 1), c.in[2] = view(gate, 2), c.in[3] = view(d_y, 3);
  c.out[0] = view(d_x, 4), c.out[1] = view(d_dt, 5), c.out[2] = view(gate ? d_gate : nullptr, 6);
  c.bc[0] = view2(b, 0), c.bc[1] = view2(c_, 1), c.dbc[0] = view2(d_b, 2), c.dbc[1] = view2(d_c, 3);
  for (int i = 0; i < (gate ? 3 : 2); ++i)
    if (overlaps(c.out[i], c.B, c.T, c.D)) return MDH_ERR_SIZE;
  if (overlaps(c.dbc[0], c) || overlaps(c.dbc[1], c)) return MDH_ERR_SIZE;
  c.A = A, c.skip = skip, c.dt_bias = dt_bias, c.softplus = softplus != 0, c.lengths = lengths;
  c.s_in = d_final_state, c.s_out = d_initial_state, c.checkpoints = (float*)checkpoints, c.ws = workspace;
  c.dA = d_A, c.dskip = d_skip, c.ddt_bias = d_dt_bias;
  return launch_scan_backward(c, (hipStream_t)stream);
}

mdh_status mdh_selective_scan_step(const int64_t* sizes, mdh_dtype dtype, const void* x, const void* dt, const void* gate,
                                   const void* b, const void* c_, const int64_t* strides, const float* A, const float* skip,
                                   const float* dt_bias, int32_t softplus, float* state, const int32_t* slots, int64_t n_slots,
                                   void* y, void* stream) {
  ScanCall c;
  const mdh_status st = scan_sizes(sizes, dtype, true, &c);
  if (st != MDH_OK) return st;
  if (slots && n_slots < 0) return MDH_ERR_SIZE;
  if (c.B == 0) return MDH_OK;
  if (!x || !dt || !b || !c_ || !A || !state || !y) return MDH_ERR_NULL;
  if (any_misaligned(bytes_of(dtype), x, dt, gate, b, c_, y) || any_misaligned(4, A, skip, dt_bias, state)) return MDH_ERR_UNSUPPORTED;
  auto view = [&](const void* p, int i) {
    const int64_t s[2] = {strides ? strides[i] : c.D, 0};
    return tokens(p, s, c.B, 1, c.D);
  };
  auto view2 = [&](const void* p, int i) {
    const int64_t s[3] = {strides ? strides[4 + 2 * i] : (int64_t)c.G * c.N, 0, strides ? strides[5 + 2 * i] : c.N};
    return shared(p, s, c);
  };
  c.in[0] = view(x, 0), c.in[1] = view(dt, 1), c.in[2] = view(gate, 2), c.out[0] = view(y, 3);
  c.bc[0] = view2(b, 0), c.bc[1] = view2(c_, 1);
  if (overlaps(c.out[0], c.B, 1, c.D)) return MDH_ERR_SIZE;
  c.A = A, c.skip = skip, c.dt_bias = dt_bias, c.softplus = softplus != 0, c.slots = slots, c.n_slots = n_slots, c.s_out = state;
  return launch_scan_step(c, (hipStream_t)stream);
}

// ------------------------------------------------------------------------------ layer norm

mdh_status mdh_layer_norm(const int64_t* sizes, mdh_dtype dtype, const void* x, const void* residual, const int64_t* row_strides,
                          const float* weight, const float* bias, float eps, void* total, void* y, float* mean, float* rstd,
                          void* stream) {
  LayerNormCall c;
  const mdh_status st = norm_sizes(sizes, dtype, &c);
  if (st != MDH_OK) return st;
  if (c.rows == 0) return MDH_OK;
  if (!x || !y || (residual && !total)) return MDH_ERR_NULL;
  if (any_misaligned(bytes_of(dtype), x, residual, total, y) || any_misaligned(4, weight, bias, mean, rstd)) return MDH_ERR_UNSUPPORTED;
  c.x = rows_of(x, row_strides, 0, c), c.residual = rows_of(residual, row_strides, 1, c);
  c.total = rows_of(residual ? total : nullptr, row_strides, 2, c), c.y = rows_of(y, row_strides, 3, c);
  if (c.rows > 1 && (c.y.stride < c.C || (residual && c.total.stride < c.C))) return MDH_ERR_SIZE;
  c.weight = weight, c.bias = bias, c.eps = eps, c.mean = mean, c.rstd = rstd;
  return launch_layer_norm(c, (hipStream_t)stream);
}

size_t mdh_layer_norm_workspace_size(const int64_t* sizes, mdh_dtype dtype) {
  LayerNormCall c;
  return norm_sizes(sizes, dtype, &c) == MDH_OK ? layer_norm_workspace(c) : 0;
}

mdh_status mdh_layer_norm_backward(const int64_t* sizes, mdh_dtype dtype, const void* s, const void* d_y, const void* d_total,
                                   const int64_t* row_strides, const float* weight, const float* mean, const float* rstd, void* d_s,
                                   float* d_weight, float* d_bias, void* workspace, size_t workspace_bytes, void* stream) {
  LayerNormCall c;
  const mdh_status st = norm_sizes(sizes, dtype, &c);
  if (st != MDH_OK) return st;
  if (c.rows > 0 && (!s || !d_y || !mean || !rstd || !d_s)) return MDH_ERR_NULL;
  if (any_misaligned(bytes_of(dtype), s, d_y, d_total, d_s) || any_misaligned(4, weight, mean, rstd, d_weight, d_bias))
    return MDH_ERR_UNSUPPORTED;
  if (short_of(workspace, workspace_bytes, layer_norm_workspace(c))) return MDH_ERR_WORKSPACE;
  c.x = rows_of(s, row_strides, 0, c), c.y = rows_of(d_y, row_strides, 1, c), c.dtotal = rows_of(d_total, row_strides, 2, c);
  c.dx = rows_of(d_s, row_strides, 3, c);
  if (c.rows > 1 && c.dx.stride < c.C) return MDH_ERR_SIZE;
  c.weight = weight, c.mean = (float*)mean, c.rstd = (float*)rstd, c.ws = workspace, c.dweight = d_weight, c.dbias = d_bias;
  return launch_layer_norm_backward(c, (hipStream_t)stream);
}

}  // extern "C"

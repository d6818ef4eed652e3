// C ABI of the operators around the attention (norm with rotation, short convolution, selective scan): argument validation,
// scratch and dispatch.  Declarations and the contract of every entry point are in include/kata.h.
#include <cmath>

#include "kata_common.cuh"

namespace kata {
namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
constexpr int kMaxTokens = 1 << 30;     // of a sequence: token numbers rounded up to whole tiles stay ints
inline long long elem_bytes(int dtype) { return dtype == KATA_F32 ? 4 : 2; }

// A view that the kernels read 16 bytes at a time: pointer and strides of whole 16-byte units.  Axes of one entry have no stride.
struct Checked {
  View v;
  int status;
};
Checked rows(const void* p, const int64_t* stride, int axes, int n0, int n1, int n2, int dtype, bool output) {
  View v{static_cast<char*>(const_cast<void*>(p)), n0 > 1 ? stride[0] : 0, n1 > 1 ? stride[1] : 0, axes > 2 && n2 > 1 ? stride[2] : 0};
  if (p == nullptr) return {v, KATA_ERR_INVALID_ARG};
  if (v.s0 < 0 || v.s1 < 0 || v.s2 < 0) return {v, KATA_ERR_INVALID_ARG};
  if (output && ((n0 > 1 && v.s0 == 0) || (n1 > 1 && v.s1 == 0) || (axes > 2 && n2 > 1 && v.s2 == 0))) return {v, KATA_ERR_INVALID_ARG};
  const long long e = elem_bytes(dtype);
  if ((reinterpret_cast<uintptr_t>(p) & 15u) != 0 || (v.s0 * e) % 16 != 0 || (v.s1 * e) % 16 != 0 || (v.s2 * e) % 16 != 0)
    return {v, KATA_ERR_ALIGNMENT};
  return {v, KATA_OK};
}

int check_workspace(const CallOpts& o, size_t need) {
  if (need == 0) return KATA_OK;
  if (o.workspace == nullptr || o.workspace_bytes < need) return KATA_ERR_WORKSPACE_TOO_SMALL;
  return (reinterpret_cast<uintptr_t>(o.workspace) & (kAlign - 1)) != 0 ? KATA_ERR_ALIGNMENT : KATA_OK;
}

bool rope_width(int d) { return d == 16 || d == 32 || d == 64 || d == 128; }

#define KATA_TRY(x)                      \
  do {                                   \
    const int st_ = (x);                 \
    if (st_ != KATA_OK) return st_;      \
  } while (0)

int norm_rope(const kata_norm_rope_args* a, const kata_opts* opts, bool backward) {
  CallOpts o;
  KATA_TRY(read_call_opts(opts, o));
  if (a == nullptr || a->struct_size != sizeof(kata_norm_rope_args)) return KATA_ERR_INVALID_ARG;
  if (a->B < 1 || a->T < 1 || a->H_q < 1 || a->H_k < 0 || a->d < 1 || a->rotary_dim < 0) return KATA_ERR_INVALID_ARG;
  if (!rope_width(a->d) || a->rotary_dim > a->d || a->rotary_dim % 16 != 0) return KATA_ERR_UNSUPPORTED_SHAPE;
  // (tokens are numbered in 32 bits, heads of q and k together in 16)
  if (a->H_q > 32767 || a->H_k > 32767 || (long long)a->B * a->T > (1LL << 31) - 1024) return KATA_ERR_UNSUPPORTED_SHAPE;
  if (o.impl == KATA_IMPL_TENSOR) return KATA_ERR_UNSUPPORTED_SHAPE;
  if (!(a->eps >= 0.0) || !std::isfinite(a->eps) || (a->rotary_dim > 0 && a->inv_freq == nullptr)) return KATA_ERR_INVALID_ARG;
  NormRope r = {};
  r.B = a->B; r.T = a->T; r.Hq = a->H_q; r.Hk = a->H_k; r.d = a->d; r.rot = a->rotary_dim; r.dtype = o.dtype;
  r.interleaved = a->interleaved != 0;
  r.eps = (float)a->eps;
  r.positions = reinterpret_cast<const long long*>(a->positions);
  r.ps0 = a->pos_stride[0]; r.ps1 = a->pos_stride[1]; r.pos_offset = a->pos_offset;
  if ((reinterpret_cast<uintptr_t>(a->positions) & 7u) != 0) return KATA_ERR_ALIGNMENT;
  if (a->positions != nullptr && (r.ps0 < 0 || r.ps1 < 0)) return KATA_ERR_INVALID_ARG;
  for (int i = 0; i < a->rotary_dim / 2; ++i) {
    if (!std::isfinite(a->inv_freq[i])) return KATA_ERR_INVALID_ARG;
    // turns a position: a fraction of 2^64 (whole turns do not count), to the 64 bits of a long double
    long double turn = (long double)a->inv_freq[i] * (1.0L / 6.283185307179586476925286766559005768L);
    if (!(turn >= 0.0L && turn < 1.0L)) turn -= floorl(turn);
    const long double scaled = turn * 18446744073709551616.0L + 0.5L;
    r.turns[i] = scaled >= 18446744073709551616.0L ? 0ull : (unsigned long long)scaled;
  }
  struct Tensor { View* to; const void* p; const int64_t* stride; int heads; bool output; };
  const Tensor all[] = {{&r.q, a->q, a->q_stride, a->H_q, false}, {&r.q_out, a->q_out, a->q_out_stride, a->H_q, !backward},
                        {&r.dq, a->dq, a->dq_stride, a->H_q, true}, {&r.k, a->k, a->k_stride, a->H_k, false},
                        {&r.k_out, a->k_out, a->k_out_stride, a->H_k, !backward}, {&r.dk, a->dk, a->dk_stride, a->H_k, true}};
  for (const Tensor& t : all) {
    if (t.heads == 0 || (!backward && (t.to == &r.dq || t.to == &r.dk))) continue;
    const Checked c = rows(t.p, t.stride, 3, a->B, t.heads, a->T, o.dtype, t.output);
    KATA_TRY(c.status);
    *t.to = c.v;
  }
  r.q_weight = a->q_weight;
  r.k_weight = a->k_weight;
  const uintptr_t entry = (uintptr_t)elem_bytes(o.dtype) - 1;
  if ((reinterpret_cast<uintptr_t>(a->q_weight) & entry) != 0 || (reinterpret_cast<uintptr_t>(a->k_weight) & entry) != 0) return KATA_ERR_ALIGNMENT;
  size_t need = 0;
  if (backward) {
    r.dq_weight = a->dq_weight;
    r.dk_weight = a->dk_weight;
    if ((r.dq_weight != nullptr && r.q_weight == nullptr) || (r.dk_weight != nullptr && (r.k_weight == nullptr || a->H_k == 0))) return KATA_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(r.dq_weight) & 3u) != 0 || (reinterpret_cast<uintptr_t>(r.dk_weight) & 3u) != 0) return KATA_ERR_ALIGNMENT;
    if (r.dq_weight != nullptr || r.dk_weight != nullptr)
      need = align_up(norm_rope_bwd_workspace_elems(a->B, a->T, a->H_q + a->H_k, a->d) * sizeof(float));
    KATA_TRY(check_workspace(o, need));
  }
  KATA_TRY(check_device());
  LaunchCtx ctx{o.stream, 0, KATA_OK};
  if (backward) norm_rope_bwd(r, static_cast<float*>(o.workspace), ctx);
  else norm_rope_fwd(r, ctx);
  return finish_call(ctx, KATA_IMPL_SIMT);
}

enum ConvCall { kConvForward, kConvStep, kConvBackward };

int short_conv(const kata_short_conv_args* a, const kata_opts* opts, ConvCall call) {
  CallOpts o;
  KATA_TRY(read_call_opts(opts, o));
  if (a == nullptr || a->struct_size != sizeof(kata_short_conv_args)) return KATA_ERR_INVALID_ARG;
  const int T = call == kConvStep ? 1 : a->T;
  if (a->B < 1 || T < 1 || a->D < 1 || a->width < 1) return KATA_ERR_INVALID_ARG;
  if (a->width < 2 || a->width > 4) return KATA_ERR_UNSUPPORTED_SHAPE;
  // (at most 2^31 blocks over tokens x channels)
  if (T > kMaxTokens || a->D > (1 << 24) || (double)a->B * T * a->D > 1e11) return KATA_ERR_UNSUPPORTED_SHAPE;
  if (o.impl == KATA_IMPL_TENSOR) return KATA_ERR_UNSUPPORTED_SHAPE;
  if (a->weight == nullptr) return KATA_ERR_INVALID_ARG;
  if (call == kConvStep && (a->s_init == nullptr || a->s_final == nullptr || a->lengths != nullptr)) return KATA_ERR_INVALID_ARG;
  if (call == kConvBackward && (a->s_init != nullptr || a->s_final != nullptr)) return KATA_ERR_INVALID_ARG;
  if (call == kConvBackward && a->dbias != nullptr && a->bias == nullptr) return KATA_ERR_INVALID_ARG;
  ShortConv r = {};
  r.B = a->B; r.T = T; r.D = a->D; r.W = a->width; r.dtype = o.dtype; r.silu = a->silu != 0;
  r.weight = a->weight; r.bias = a->bias;
  r.s_init = a->s_init; r.s_final = a->s_final; r.lengths = a->lengths;
  struct Tensor { View* to; const void* p; const int64_t* stride; bool output, used; };
  const Tensor all[] = {{&r.x, a->x, a->x_stride, false, true}, {&r.out, a->out, a->out_stride, true, call != kConvBackward},
                        {&r.dout, a->dout, a->dout_stride, false, call == kConvBackward}, {&r.dx, a->dx, a->dx_stride, true, call == kConvBackward}};
  const uintptr_t entry = (uintptr_t)elem_bytes(o.dtype) - 1;
  for (const Tensor& t : all) {
    if (!t.used) continue;
    const Checked c = rows(t.p, t.stride, 2, a->B, T, 1, o.dtype, t.output);
    if (c.status == KATA_ERR_INVALID_ARG) return c.status;          // (rows of any alignment are taken)
    if ((reinterpret_cast<uintptr_t>(t.p) & entry) != 0) return KATA_ERR_ALIGNMENT;
    *t.to = c.v;
  }
  for (const void* p : {a->weight, a->bias, a->s_init, (const void*)a->s_final})
    if ((reinterpret_cast<uintptr_t>(p) & entry) != 0) return KATA_ERR_ALIGNMENT;
  if ((reinterpret_cast<uintptr_t>(a->lengths) & 3u) != 0) return KATA_ERR_ALIGNMENT;
  if (call == kConvBackward) {
    r.dweight = a->dweight;
    r.dbias = a->dbias;
    if ((reinterpret_cast<uintptr_t>(r.dweight) & 3u) != 0 || (reinterpret_cast<uintptr_t>(r.dbias) & 3u) != 0) return KATA_ERR_ALIGNMENT;
    if (r.dweight != nullptr || r.dbias != nullptr)
      KATA_TRY(check_workspace(o, align_up(short_conv_bwd_workspace_elems(a->B, T, a->D, a->width) * sizeof(float))));
  }
  KATA_TRY(check_device());
  LaunchCtx ctx{o.stream, 0, KATA_OK};
  if (call == kConvBackward) short_conv_bwd(r, static_cast<float*>(o.workspace), ctx);
  else short_conv_fwd(r, ctx);
  return finish_call(ctx, KATA_IMPL_SIMT);
}

int ssm_shape(int B, int H, int T, int n, int d) {
  if (B < 1 || H < 1 || T < 1 || n < 1 || d < 1) return KATA_ERR_INVALID_ARG;
  if ((long long)B * H > 65535 || T > kMaxTokens) return KATA_ERR_UNSUPPORTED_SHAPE;
  if ((n != 16 && n != 32 && n != 64 && n != 128) || (d != 16 && d != 32 && d != 64)) return KATA_ERR_UNSUPPORTED_SHAPE;
  return KATA_OK;
}

// A tile of the tensor cores is 128 tokens, and a final state takes a pass and a launch more: short sequences go token by token.
// Measured, us, tensor cores / token by token (n = 64), with a final state: 2048 heads, T = 16: 222 / 29, 64: 225 / 93; 64 heads, T = 64:
// 14.4 / 11.9; 16 heads, T = 100: 12.3 / 18.8; without: 2048 heads, T = 16: 81 / 27, 32: 81 / 48, 64: 81 / 91; 64 heads, T = 32: 6.2 / 6.8.
bool ssm_tensor(const CallOpts& o, int n, int d, int T, bool final_state) {
  if (o.impl == KATA_IMPL_SIMT || !tc_ssm_supported(o.dtype, n, d)) return false;
  return o.impl == KATA_IMPL_TENSOR || T > (final_state ? 64 : 32);
}

// Slots of states in the scratch (see SsmPlan).
int ssm_slots(const SsmPlan& plan, bool tensor, bool final_state) {
  const int more = tensor && final_state ? 1 : 0;
  return plan.segments + more > 1 ? plan.segments + more : 0;
}

int ssm(const kata_ssm_args* a, const kata_opts* opts, bool step) {
  CallOpts o;
  KATA_TRY(read_call_opts(opts, o));
  if (a == nullptr || a->struct_size != sizeof(kata_ssm_args)) return KATA_ERR_INVALID_ARG;
  const int T = step ? 1 : a->T;
  KATA_TRY(ssm_shape(a->B, a->H, T, a->n, a->d_v));
  if (a->G < 1 || a->H % a->G != 0) return KATA_ERR_INVALID_ARG;
  bool tensor = !step && ssm_tensor(o, a->n, a->d_v, T, a->s_final != nullptr);
  if (o.impl == KATA_IMPL_TENSOR && !tensor) return KATA_ERR_UNSUPPORTED_SHAPE;
  if (a->A == nullptr || a->dt == nullptr) return KATA_ERR_INVALID_ARG;
  if (step && (a->s_init == nullptr || a->s_final != a->s_init || a->lengths != nullptr)) return KATA_ERR_INVALID_ARG;
  Ssm r = {};
  r.B = a->B; r.T = T; r.H = a->H; r.G = a->G; r.n = a->n; r.d = a->d_v; r.dtype = o.dtype; r.softplus = a->dt_softplus != 0;
  r.A = a->A; r.D = a->D; r.dt_bias = a->dt_bias; r.s_init = a->s_init; r.s_final = a->s_final; r.lengths = a->lengths;
  struct Tensor { View* to; const void* p; const int64_t* stride; int heads; bool output; };
  const Tensor all[] = {{&r.q, a->q, a->q_stride, a->G, false}, {&r.k, a->k, a->k_stride, a->G, false},
                        {&r.v, a->v, a->v_stride, a->H, false}, {&r.out, a->out, a->out_stride, a->H, true}};
  for (const Tensor& t : all) {
    const Checked c = rows(t.p, t.stride, 3, a->B, t.heads, T, o.dtype, t.output);
    KATA_TRY(c.status);
    *t.to = c.v;
  }
  const Checked c = rows(a->dt, a->dt_stride, 3, a->B, a->H, T, o.dtype, false);
  if (c.status == KATA_ERR_INVALID_ARG) return c.status;
  r.dt = c.v;
  const uintptr_t entry = (uintptr_t)elem_bytes(o.dtype) - 1;
  if ((reinterpret_cast<uintptr_t>(a->dt) & entry) != 0) return KATA_ERR_ALIGNMENT;
  for (const void* p : {(const void*)a->A, (const void*)a->D, (const void*)a->dt_bias, (const void*)a->lengths})
    if ((reinterpret_cast<uintptr_t>(p) & 3u) != 0) return KATA_ERR_ALIGNMENT;
  if ((reinterpret_cast<uintptr_t>(a->s_init) & 15u) != 0 || (reinterpret_cast<uintptr_t>(a->s_final) & 15u) != 0) return KATA_ERR_ALIGNMENT;
  const SsmPlan plan = step ? SsmPlan{1, 1} : ssm_plan(a->B * a->H, T, a->n, a->d_v, tensor, r.s_final != nullptr);
  if (tensor && T > 1 && (r.q.s2 == 0 || r.k.s2 == 0 || r.v.s2 == 0)) {      // (one row for all tokens has no tensor map)
    if (o.impl == KATA_IMPL_TENSOR) return KATA_ERR_UNSUPPORTED_SHAPE;
    tensor = false;
  }
  const int slots = ssm_slots(plan, tensor, r.s_final != nullptr);
  KATA_TRY(check_workspace(o, align_up(ssm_workspace_bytes(a->B * a->H, a->n, a->d_v, slots))));
  KATA_TRY(check_device());
  LaunchCtx ctx{o.stream, 0, KATA_OK};
  float* ws = static_cast<float*>(o.workspace);
  if (step) ssm_step(r, ctx);
  else if (tensor) tc_ssm(r, plan, ws, o.device_status, ctx);
  else simt_ssm(r, plan, ws, ctx);
  return finish_call(ctx, tensor ? KATA_IMPL_TENSOR : KATA_IMPL_SIMT);
}

}  // namespace

size_t mixer_workspace_bytes(int fn, int B, int H, int T, int d_k, int d_v, const kata_opts* opts) {
  CallOpts o;
  if (read_call_opts(opts, o) != KATA_OK || B < 1 || H < 1 || T < 1) return 0;
  if (fn == KATA_FN_BWD_NORM_ROPE && (H > 65534 || (long long)B * T > (1LL << 31) - 1024)) return 0;
  if (fn == KATA_FN_BWD_NORM_ROPE) return rope_width(d_k) ? align_up(norm_rope_bwd_workspace_elems(B, T, H, d_k) * sizeof(float)) : 0;
  if (fn == KATA_FN_BWD_SHORT_CONV)
    return d_k >= 2 && d_k <= 4 && T <= kMaxTokens && H <= (1 << 24) && (double)B * T * H <= 1e11 ? align_up(short_conv_bwd_workspace_elems(B, T, H, d_k) * sizeof(float)) : 0;
  if (ssm_shape(B, H, T, d_k, d_v) != KATA_OK) return 0;
  // (what a call with or without a final state takes)
  int slots = 0;
  for (const bool last : {false, true}) {
    const bool tensor = ssm_tensor(o, d_k, d_v, T, last);
    const int n = ssm_slots(ssm_plan(B * H, T, d_k, d_v, tensor, last), tensor, last);
    if (n > slots) slots = n;
  }
  return align_up(ssm_workspace_bytes(B * H, d_k, d_v, slots));
}

}  // namespace kata

using namespace kata;

extern "C" {

int kata_fwd_norm_rope(const kata_norm_rope_args* a, const kata_opts* opts) { return norm_rope(a, opts, false); }
int kata_bwd_norm_rope(const kata_norm_rope_args* a, const kata_opts* opts) { return norm_rope(a, opts, true); }
int kata_fwd_short_conv(const kata_short_conv_args* a, const kata_opts* opts) { return short_conv(a, opts, kConvForward); }
int kata_decode_short_conv(const kata_short_conv_args* a, const kata_opts* opts) { return short_conv(a, opts, kConvStep); }
int kata_bwd_short_conv(const kata_short_conv_args* a, const kata_opts* opts) { return short_conv(a, opts, kConvBackward); }
int kata_fwd_ssm_scan(const kata_ssm_args* a, const kata_opts* opts) { return ssm(a, opts, false); }
int kata_decode_ssm_step(const kata_ssm_args* a, const kata_opts* opts) { return ssm(a, opts, true); }

}  // extern "C"

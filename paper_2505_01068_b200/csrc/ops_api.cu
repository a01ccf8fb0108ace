// C ABI of the training operators (gsit_ops.h): argument checks and launches.
#include <math.h>

#include "gsit_ops.h"
#include "ops.cuh"
#include "scored.cuh"

namespace gsit {
namespace {

gsit_status status_of(cudaError_t e) {
  if (e == cudaSuccess) return GSIT_OK;
  return e == cudaErrorNotSupported ? GSIT_ERR_UNSUPPORTED : GSIT_ERR_CUDA;
}
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
int element_size(int32_t dtype) { return dtype == GSIT_BF16 ? 2 : 4; }

// Geometry of a call on the padded layout, with the device's status word.
gsit_status padded_geometry(const gsit_shape* shape, Geometry* g) {
  const gsit_status st = basic_geometry(shape, g);
  if (st != GSIT_OK) return st;
  return g->row_start == nullptr ? GSIT_OK : GSIT_ERR_UNSUPPORTED;
}

// The shape of a call that reads no block pattern: what stands in its fields is not looked at.
gsit_shape any_phase(gsit_shape s) {
  s.phase = GSIT_PHASE_INTRA;
  s.custom_mask = 0;
  return s;
}

gsit_status rotary(const gsit_shape* shape, const gsit_rotary* r, const void* q, int64_t ldq, const void* k, int64_t ldk, void* q_out, int64_t ldqo,
                   void* k_out, int64_t ldko, bool backward, gsit_stream stream) {
  if (shape == nullptr) return GSIT_ERR_INVALID_ARG;
  const gsit_shape rows = any_phase(*shape);
  Geometry g;
  const gsit_status st = padded_geometry(&rows, &g);
  if (st != GSIT_OK) return st;
  if (r == nullptr || r->positions == nullptr || q == nullptr || q_out == nullptr || (k == nullptr) != (k_out == nullptr)) return GSIT_ERR_INVALID_ARG;
  int64_t pairs = 0;
  for (int n : r->sections) {
    if (n < 0) return GSIT_ERR_INVALID_ARG;
    pairs += n;
  }
  const int kv_heads = r->kv_heads == 0 ? g.heads : r->kv_heads;
  if (pairs < 1 || 2 * pairs > g.hd || kv_heads < 1 || !(r->base > 0.0) || r->axis_stride < 0 || r->batch_stride < 0) return GSIT_ERR_INVALID_ARG;
  if (pairs > MAX_ROTARY_PAIRS || (int64_t)(g.heads + kv_heads) * g.hd > 65536) return GSIT_ERR_UNSUPPORTED;
  const int64_t dq = g.d, dk = (int64_t)kv_heads * g.hd;
  if (ldq < dq || ldqo < dq || (k != nullptr && (ldk < dk || ldko < dk))) return GSIT_ERR_INVALID_ARG;
  const size_t es = element_size(shape->dtype);
  if (!aligned(q, es) || !aligned(k, es) || !aligned(q_out, es) || !aligned(k_out, es) || !aligned(r->positions, 4)) return GSIT_ERR_INVALID_ARG;
  if (status_of(device_status_word(&g.status)) != GSIT_OK) return GSIT_ERR_CUDA;
  const RotaryCall c = {{q, k}, {q_out, k_out}, {ldq, ldk}, {ldqo, ldko}, {g.heads, k == nullptr ? 0 : kv_heads}, r->positions, r->axis_stride,
                        r->batch_stride, {r->sections[0], r->sections[1], r->sections[2]}, r->interleaved != 0, backward, r->base};
  return status_of(launch_rotary(g, shape->dtype, c, static_cast<cudaStream_t>(stream)));
}

// Norms of heads with the rotation, or (dq != nullptr) their gradients: the checks of both.
struct HeadRows {
  const void* p;
  int64_t ld;
};
gsit_status head_norm(const gsit_shape* shape, const gsit_rotary* r, float eps, const HeadRows (&x)[2], const float* const (&gamma)[2], const HeadRows* dy,
                      const HeadRows (&out)[2], float* const (&dgamma)[2], void* workspace, size_t workspace_bytes, gsit_stream stream) {
  if (shape == nullptr) return GSIT_ERR_INVALID_ARG;
  const gsit_shape rows = any_phase(*shape);
  Geometry g;
  const gsit_status st = padded_geometry(&rows, &g);
  if (st != GSIT_OK) return st;
  if (r == nullptr || x[0].p == nullptr || (eps > 0.f && !isfinite(eps)) || eps != eps) return GSIT_ERR_INVALID_ARG;
  const bool has_k = x[1].p != nullptr;
  HeadNormCall c = {};
  int64_t pairs = 0;
  for (int i = 0; i < 3; ++i) {
    if (r->sections[i] < 0) return GSIT_ERR_INVALID_ARG;
    pairs += c.sections[i] = r->sections[i];
  }
  const int kv_heads = r->kv_heads == 0 ? g.heads : r->kv_heads;
  if (2 * pairs > g.hd || kv_heads < 1) return GSIT_ERR_INVALID_ARG;
  if (pairs > 0 && (r->positions == nullptr || !aligned(r->positions, 4) || !(r->base > 0.0) || r->axis_stride < 0 || r->batch_stride < 0)) return GSIT_ERR_INVALID_ARG;
  if (pairs > MAX_ROTARY_PAIRS || g.hd > MAX_NORM_HEAD || (int64_t)(g.heads + kv_heads) * g.hd > 65536) return GSIT_ERR_UNSUPPORTED;
  const size_t es = element_size(shape->dtype);
  for (int i = 0; i < 2; ++i) {
    const bool here = i == 0 || has_k;
    for (const HeadRows* m : {&x[i], dy == nullptr ? &x[i] : &dy[i], &out[i]})
      if (here ? m->p == nullptr || m->ld < (int64_t)(i == 0 ? g.heads : kv_heads) * g.hd || !aligned(m->p, es) : m->p != nullptr) return GSIT_ERR_INVALID_ARG;
    if (!aligned(gamma[i], 4) || !aligned(dgamma[i], 4) || (!here && dgamma[i] != nullptr)) return GSIT_ERR_INVALID_ARG;
    c.heads[i] = !here ? 0 : i == 0 ? g.heads : kv_heads;
    c.x[i] = x[i].p; c.ldx[i] = x[i].ld;
    if (dy != nullptr) { c.dy[i] = dy[i].p; c.lddy[i] = dy[i].ld; }
    c.out[i] = const_cast<void*>(out[i].p); c.ldo[i] = out[i].ld;
    c.gamma[i] = gamma[i];
    c.dgamma[i] = dgamma[i];
  }
  if (has_k && (dgamma[0] == nullptr) != (dgamma[1] == nullptr)) return GSIT_ERR_INVALID_ARG;
  if (dgamma[0] != nullptr) {
    if (workspace == nullptr || workspace_bytes < head_norm_scratch(g)) return GSIT_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return GSIT_ERR_INVALID_ARG;
    c.partial = static_cast<float*>(workspace);
  }
  if (status_of(device_status_word(&g.status)) != GSIT_OK) return GSIT_ERR_CUDA;
  c.positions = r->positions;
  c.axis_stride = r->axis_stride;
  c.batch_stride = r->batch_stride;
  c.interleaved = r->interleaved != 0;
  c.backward = dy != nullptr;
  c.base = r->base;
  c.eps = eps > 0.f ? eps : 1e-6f;
  return status_of(launch_head_norm(g, shape->dtype, c, static_cast<cudaStream_t>(stream)));
}

bool norm_type(int32_t t) { return t == GSIT_F32 || t == GSIT_BF16; }
gsit_status norm_geometry(const gsit_shape* shape, Geometry* g) {
  if (shape == nullptr) return GSIT_ERR_INVALID_ARG;
  gsit_shape rows = any_phase(*shape);   // rows of d_model features: neither heads nor the type are read
  rows.heads = 1;
  rows.dtype = GSIT_F32;
  const gsit_status st = padded_geometry(&rows, g);
  if (st != GSIT_OK) return st;
  return g->d <= MAX_NORM_WIDTH ? GSIT_OK : GSIT_ERR_UNSUPPORTED;
}

// Geometry and rule of an attention call, checked; the tensors are filled in by the caller.
gsit_status scored_args(const gsit_shape* shape, const gsit_score_rule* r, Geometry* g, ScoredArgs* a) {
  const gsit_status st = padded_geometry(shape, g);
  if (st != GSIT_OK) return st;
  if (r == nullptr) return GSIT_ERR_INVALID_ARG;
  *a = {};
  a->kv_heads = r->kv_heads == 0 ? g->heads : r->kv_heads;
  if (a->kv_heads < 1 || g->heads % a->kv_heads != 0 || r->softcap != r->softcap) return GSIT_ERR_INVALID_ARG;
  a->group = g->heads / a->kv_heads;
  if (g->batch > 65535 || g->heads > 65535) return GSIT_ERR_UNSUPPORTED;
  if (shape->dtype == GSIT_BF16 ? (g->hd != 8 && g->hd != 16 && g->hd != 32 && g->hd != 64) : g->hd > 128) return GSIT_ERR_UNSUPPORTED;
  if (!aligned(r->slopes, 4) || !aligned(r->times, 4) || !aligned(r->documents, 4) || !aligned(r->prefix, 4)) return GSIT_ERR_INVALID_ARG;
  a->tail = r->tail != 0;
  for (int s = 0; s < 3; ++s) {
    a->q_len[s] = a->tail ? r->q_len[s] : g->seg_len[s];
    if (a->q_len[s] < 0 || a->q_len[s] > g->seg_len[s]) return GSIT_ERR_INVALID_ARG;
    a->q_off[s] = a->Lq;
    a->Lq += a->q_len[s];
  }
  if (a->Lq < 1) return GSIT_ERR_INVALID_ARG;
  a->scale = shape->scale > 0.f ? shape->scale : 1.0f / sqrtf((float)g->hd);
  a->softcap = r->softcap > 0.f ? r->softcap : 0.f;
  a->inner = a->softcap > 0.f ? a->scale / a->softcap : a->scale * LOG2E;
  a->outer = a->softcap * LOG2E;
  if (!isfinite(a->inner) || !isfinite(a->outer)) return GSIT_ERR_INVALID_ARG;
  if (a->softcap > 0.f) {
    // tanh(y) / y and 1 - tanh(y)^2 as quadratics of y^2: least squares fits of the relative error over |y| <= 1/4, refined towards equal
    // error (4.2e-7 and 2.8e-6)
    static const double P[3] = {0.999999604, -0.333219082, 0.128416126}, B[3] = {0.999997213, -0.999202503, 0.632425479};
    const double in = (double)a->inner, out = (double)a->outer;
    a->near_dot = in < 1e6 ? (float)(0.25 / in) : -1.f;   // beyond, the coefficients leave the range of float: never
    double even = 1.0;   // in^(2 i)
    for (int i = 0; i < 3; ++i) {
      a->near_p[i] = (float)(P[i] * out * even * in);
      a->near_b[i] = (float)(B[i] * even);
      even *= in * in;
    }
  }
  a->causal = r->causal != 0;
  a->slopes = r->slopes;
  a->times = r->times;
  a->documents = r->documents;
  a->prefix = a->causal ? r->prefix : nullptr;
  return GSIT_OK;
}

// Which kernels serve a call, and the scratch they need (forward: none, running sums and joins stay on the SMs).
cudaError_t launch_scored_fwd(const Geometry& g, int dtype, const ScoredArgs& a, cudaStream_t st) {
  if (scored_tail_supported(g, dtype, a)) return launch_scored_tail(g, dtype, a, st);
  if (dtype == GSIT_BF16) return scored_tc_preferred(g, a.q_len) ? launch_scored_fwd_tc(g, a, st) : launch_scored_fwd_bf16(g, a, st);
  return g.hd <= 64 ? launch_scored_fwd_f32(g, a, st) : launch_scored_rows_fwd(g, a, st);
}
size_t scored_bwd_scratch(const Geometry& g, int, const ScoredArgs&) { return sizeof(float2) * (size_t)g.batch * g.heads * g.L; }
cudaError_t launch_scored_bwd(const Geometry& g, int dtype, const ScoredArgs& a, cudaStream_t st) {
  if (dtype == GSIT_BF16) return scored_tc_preferred(g, g.seg_len) ? launch_scored_bwd_tc(g, a, st) : launch_scored_bwd_bf16(g, a, st);
  return g.hd <= 64 ? launch_scored_bwd_f32(g, a, st) : launch_scored_rows_bwd(g, a, st);
}

// A matrix of `cols` columns whose rows the kernels may load: 16-byte pieces for bf16, elements for float.
bool rows_ok(const void* p, int64_t ld, int64_t cols, int32_t dtype) {
  if (p == nullptr || ld < cols) return false;
  return dtype == GSIT_BF16 ? aligned(p, 16) && ld % 8 == 0 : aligned(p, 4);
}

}  // namespace
}  // namespace gsit

using namespace gsit;

extern "C" {

gsit_status gsit_rotary_fwd(const gsit_shape* shape, const gsit_rotary* rotary_, const void* q, int64_t q_row_stride, const void* k,
                            int64_t k_row_stride, void* q_out, int64_t q_out_row_stride, void* k_out, int64_t k_out_row_stride,
                            gsit_stream stream) {
  return rotary(shape, rotary_, q, q_row_stride, k, k_row_stride, q_out, q_out_row_stride, k_out, k_out_row_stride, false, stream);
}

gsit_status gsit_rotary_bwd(const gsit_shape* shape, const gsit_rotary* rotary_, const void* dq, int64_t dq_row_stride, const void* dk,
                            int64_t dk_row_stride, void* dq_out, int64_t dq_out_row_stride, void* dk_out, int64_t dk_out_row_stride,
                            gsit_stream stream) {
  return rotary(shape, rotary_, dq, dq_row_stride, dk, dk_row_stride, dq_out, dq_out_row_stride, dk_out, dk_out_row_stride, true, stream);
}

gsit_status gsit_head_norm_rotary_fwd(const gsit_shape* shape, const gsit_rotary* rotary_, float eps, const void* q, int64_t q_row_stride,
                                      const float* q_gamma, const void* k, int64_t k_row_stride, const float* k_gamma, void* q_out,
                                      int64_t q_out_row_stride, void* k_out, int64_t k_out_row_stride, gsit_stream stream) {
  return head_norm(shape, rotary_, eps, {{q, q_row_stride}, {k, k_row_stride}}, {q_gamma, k_gamma}, nullptr, {{q_out, q_out_row_stride}, {k_out, k_out_row_stride}},
                   {nullptr, nullptr}, nullptr, 0, stream);
}

size_t gsit_head_norm_rotary_bwd_workspace(const gsit_shape* shape) {
  if (shape == nullptr) return (size_t)-1;
  const gsit_shape rows = any_phase(*shape);
  Geometry g;
  return padded_geometry(&rows, &g) == GSIT_OK && g.hd <= MAX_NORM_HEAD ? head_norm_scratch(g) : (size_t)-1;
}

gsit_status gsit_head_norm_rotary_bwd(const gsit_shape* shape, const gsit_rotary* rotary_, float eps, const void* q, int64_t q_row_stride,
                                      const float* q_gamma, const void* k, int64_t k_row_stride, const float* k_gamma, const void* dq,
                                      int64_t dq_row_stride, const void* dk, int64_t dk_row_stride, void* dq_out, int64_t dq_out_row_stride,
                                      void* dk_out, int64_t dk_out_row_stride, float* dq_gamma, float* dk_gamma, void* workspace,
                                      size_t workspace_bytes, gsit_stream stream) {
  const HeadRows dy[2] = {{dq, dq_row_stride}, {dk, dk_row_stride}};
  return head_norm(shape, rotary_, eps, {{q, q_row_stride}, {k, k_row_stride}}, {q_gamma, k_gamma}, dy, {{dq_out, dq_out_row_stride}, {dk_out, dk_out_row_stride}},
                   {dq_gamma, dk_gamma}, workspace, workspace_bytes, stream);
}

gsit_status gsit_layer_norm_fwd(const gsit_shape* shape, int32_t x_dtype, const void* x, int64_t x_row_stride, const float* gamma,
                                const float* beta, float eps, int32_t y_dtype, void* y, int64_t y_row_stride, float* mean, float* rstd,
                                gsit_stream stream) {
  Geometry g;
  const gsit_status st = norm_geometry(shape, &g);
  if (st != GSIT_OK) return st;
  if (!norm_type(x_dtype) || !norm_type(y_dtype) || x == nullptr || y == nullptr || x_row_stride < g.d || y_row_stride < g.d) return GSIT_ERR_INVALID_ARG;
  if ((mean == nullptr) != (rstd == nullptr)) return GSIT_ERR_INVALID_ARG;
  if (!aligned(x, element_size(x_dtype)) || !aligned(y, element_size(y_dtype)) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4))
    return GSIT_ERR_INVALID_ARG;
  if (status_of(device_status_word(&g.status)) != GSIT_OK) return GSIT_ERR_CUDA;
  NormCall c = {};
  c.x = x; c.ldx = x_row_stride; c.x_dtype = x_dtype;
  c.gamma = gamma; c.beta = beta;
  c.eps = eps > 0.f ? eps : 1e-5f;
  c.y = y; c.ldy = y_row_stride; c.y_dtype = y_dtype;
  c.mean = mean; c.rstd = rstd;
  return status_of(launch_layer_norm_fwd(g, c, static_cast<cudaStream_t>(stream)));
}

size_t gsit_layer_norm_bwd_workspace(const gsit_shape* shape) {
  Geometry g;
  return norm_geometry(shape, &g) == GSIT_OK ? layer_norm_bwd_scratch(g) : (size_t)-1;
}

gsit_status gsit_layer_norm_bwd(const gsit_shape* shape, int32_t y_dtype, const void* dy, int64_t dy_row_stride, int32_t x_dtype,
                                const void* x, int64_t x_row_stride, const float* mean, const float* rstd, const float* gamma,
                                const void* residual, int64_t residual_row_stride, void* dx, int64_t dx_row_stride, float* dgamma,
                                float* dbeta, void* workspace, size_t workspace_bytes, gsit_stream stream) {
  Geometry g;
  const gsit_status st = norm_geometry(shape, &g);
  if (st != GSIT_OK) return st;
  if (!norm_type(x_dtype) || !norm_type(y_dtype) || x == nullptr || dy == nullptr || mean == nullptr || rstd == nullptr || dx == nullptr)
    return GSIT_ERR_INVALID_ARG;
  if (x_row_stride < g.d || dy_row_stride < g.d || dx_row_stride < g.d || (residual != nullptr && residual_row_stride < g.d)) return GSIT_ERR_INVALID_ARG;
  if ((dgamma == nullptr) != (dbeta == nullptr)) return GSIT_ERR_INVALID_ARG;
  const size_t ex = element_size(x_dtype), ey = element_size(y_dtype);
  if (!aligned(x, ex) || !aligned(residual, ex) || !aligned(dx, ex) || !aligned(dy, ey) || !aligned(gamma, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
    return GSIT_ERR_INVALID_ARG;
  if (dgamma != nullptr) {
    if (workspace == nullptr || workspace_bytes < layer_norm_bwd_scratch(g)) return GSIT_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return GSIT_ERR_INVALID_ARG;
  }
  if (status_of(device_status_word(&g.status)) != GSIT_OK) return GSIT_ERR_CUDA;
  NormCall c = {};
  c.x = x; c.ldx = x_row_stride; c.x_dtype = x_dtype;
  c.gamma = gamma;
  c.y_dtype = y_dtype;
  c.mean = const_cast<float*>(mean); c.rstd = const_cast<float*>(rstd);
  c.dy = dy; c.lddy = dy_row_stride;
  c.residual = residual; c.ldres = residual_row_stride;
  c.dx = dx; c.lddx = dx_row_stride;
  c.dgamma = dgamma; c.dbeta = dbeta;
  c.partial = dgamma != nullptr ? static_cast<float*>(workspace) : nullptr;
  return status_of(launch_layer_norm_bwd(g, c, static_cast<cudaStream_t>(stream)));
}

size_t gsit_scored_attention_fwd_workspace(const gsit_shape* shape, const gsit_score_rule* rule) {
  Geometry g;
  ScoredArgs a;
  return scored_args(shape, rule, &g, &a) == GSIT_OK ? 0 : (size_t)-1;
}

gsit_status gsit_im_scored_attention_fwd(const gsit_shape* shape, const gsit_score_rule* rule, const void* q, int64_t q_row_stride,
                                         const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride, void* out, float* lse,
                                         void*, size_t, gsit_stream stream) {
  Geometry g;
  ScoredArgs a;
  const gsit_status st = scored_args(shape, rule, &g, &a);
  if (st != GSIT_OK) return st;
  const int64_t dk = (int64_t)a.kv_heads * g.hd;
  const int32_t t = shape->dtype;
  if (!rows_ok(q, q_row_stride, g.d, t) || !rows_ok(k, k_row_stride, dk, t) || !rows_ok(v, v_row_stride, dk, t) || !rows_ok(out, g.d, g.d, t) ||
      !aligned(lse, 4))
    return GSIT_ERR_INVALID_ARG;
  if (status_of(device_status_word(&g.status)) != GSIT_OK) return GSIT_ERR_CUDA;
  a.q = q; a.ldq = q_row_stride;
  a.k = k; a.ldk = k_row_stride;
  a.v = v; a.ldv = v_row_stride;
  a.out = out; a.ldo = g.d;
  a.lse = lse;
  return status_of(launch_scored_fwd(g, t, a, static_cast<cudaStream_t>(stream)));
}

size_t gsit_scored_attention_bwd_workspace(const gsit_shape* shape, const gsit_score_rule* rule) {
  Geometry g;
  ScoredArgs a;
  return scored_args(shape, rule, &g, &a) == GSIT_OK && !a.tail ? scored_bwd_scratch(g, shape->dtype, a) : (size_t)-1;
}

gsit_status gsit_im_scored_attention_bwd(const gsit_shape* shape, const gsit_score_rule* rule, const void* q, int64_t q_row_stride,
                                         const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride, const void* out,
                                         int64_t out_row_stride, const float* lse, const void* dout, int64_t dout_row_stride, void* dq,
                                         int64_t dq_row_stride, void* dk, int64_t dk_row_stride, void* dv, int64_t dv_row_stride,
                                         void* workspace, size_t workspace_bytes, gsit_stream stream) {
  Geometry g;
  ScoredArgs a;
  const gsit_status st = scored_args(shape, rule, &g, &a);
  if (st != GSIT_OK) return st;
  if (a.tail) return GSIT_ERR_UNSUPPORTED;
  const int64_t cols = (int64_t)a.kv_heads * g.hd;
  const int32_t t = shape->dtype;
  if (!rows_ok(q, q_row_stride, g.d, t) || !rows_ok(k, k_row_stride, cols, t) || !rows_ok(v, v_row_stride, cols, t) ||
      !rows_ok(out, out_row_stride, g.d, t) || !rows_ok(dout, dout_row_stride, g.d, t) || !rows_ok(dq, dq_row_stride, g.d, t) ||
      !rows_ok(dk, dk_row_stride, cols, t) || !rows_ok(dv, dv_row_stride, cols, t) || lse == nullptr || !aligned(lse, 4))
    return GSIT_ERR_INVALID_ARG;
  if (workspace == nullptr || workspace_bytes < scored_bwd_scratch(g, t, a)) return GSIT_ERR_WORKSPACE;
  if (!aligned(workspace, 16)) return GSIT_ERR_INVALID_ARG;
  if (status_of(device_status_word(&g.status)) != GSIT_OK) return GSIT_ERR_CUDA;
  a.q = q; a.ldq = q_row_stride;
  a.k = k; a.ldk = k_row_stride;
  a.v = v; a.ldv = v_row_stride;
  a.out = const_cast<void*>(out); a.ldo = out_row_stride;
  a.lse = const_cast<float*>(lse);
  a.dout = dout; a.lddo = dout_row_stride;
  a.dq = dq; a.lddq = dq_row_stride;
  a.dk = dk; a.lddk = dk_row_stride;
  a.dv = dv; a.lddv = dv_row_stride;
  a.row_stats = static_cast<float2*>(workspace);
  return status_of(launch_scored_bwd(g, t, a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

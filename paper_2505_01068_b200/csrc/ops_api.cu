// C ABI of the training operators (gsit_ops.h): argument checks and launches.
#include "gsit_ops.h"
#include "ops.cuh"

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

gsit_status rotary(const gsit_shape* shape, const gsit_rotary* r, const void* q, int64_t ldq, const void* k, int64_t ldk, void* q_out, int64_t ldqo,
                   void* k_out, int64_t ldko, bool backward, gsit_stream stream) {
  Geometry g;
  const gsit_status st = padded_geometry(shape, &g);
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
  if (!aligned(q, es) || !aligned(k, es) || !aligned(q_out, es) || !aligned(k_out, es)) return GSIT_ERR_INVALID_ARG;
  if (status_of(device_status_word(&g.status)) != GSIT_OK) return GSIT_ERR_CUDA;
  const RotaryCall c = {{q, k}, {q_out, k_out}, {ldq, ldk}, {ldqo, ldko}, {g.heads, k == nullptr ? 0 : kv_heads}, r->positions, r->axis_stride,
                        r->batch_stride, {r->sections[0], r->sections[1], r->sections[2]}, r->interleaved != 0, backward, r->base};
  return status_of(launch_rotary(g, shape->dtype, c, static_cast<cudaStream_t>(stream)));
}

bool norm_type(int32_t t) { return t == GSIT_F32 || t == GSIT_BF16; }
gsit_status norm_geometry(const gsit_shape* shape, Geometry* g) {
  const gsit_status st = padded_geometry(shape, g);
  if (st != GSIT_OK) return st;
  return g->d <= MAX_NORM_WIDTH ? GSIT_OK : GSIT_ERR_UNSUPPORTED;
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

}  // extern "C"

// C ABI of the streaming calls (gsit_stream.h): argument checks and launches.
#include <math.h>

#include "cache.cuh"

namespace gsit {
namespace {

gsit_status status_of(cudaError_t e) {
  if (e == cudaSuccess) return GSIT_OK;
  return e == cudaErrorNotSupported ? GSIT_ERR_UNSUPPORTED : GSIT_ERR_CUDA;
}
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// Geometry of a step: rows only, in the padded layout.
gsit_status step_geometry(const gsit_shape* shape, Geometry* g) {
  if (shape == nullptr) return GSIT_ERR_INVALID_ARG;
  gsit_shape rows = *shape;   // neither widths nor the block pattern are read
  rows.phase = GSIT_PHASE_INTRA;
  rows.custom_mask = 0;
  rows.d_model = rows.heads = 1;
  rows.dtype = GSIT_F32;
  const gsit_status st = basic_geometry(&rows, g);
  if (st != GSIT_OK) return st;
  return g->row_start == nullptr ? GSIT_OK : GSIT_ERR_UNSUPPORTED;
}

// What every call reads of a cache, and the rest of it where rows are moved.
gsit_status tables_of(const gsit_cache* c, const Geometry& g, Cache* out) {
  if (c == nullptr || c->batch != g.batch || c->pages < 1 || c->blocks < 1 || c->tables == nullptr || c->lengths == nullptr) return GSIT_ERR_INVALID_ARG;
  if (!aligned(c->tables, 4) || !aligned(c->lengths, 4)) return GSIT_ERR_INVALID_ARG;
  if (c->pages >= 1 << 26 || c->blocks >= 1 << 22 || g.batch > 65535) return GSIT_ERR_UNSUPPORTED;   // slots and positions are 32-bit
  *out = {c->kind, c->batch, c->kv_heads, c->head_dim, c->pages, c->blocks, static_cast<uint8_t*>(c->keys), static_cast<uint8_t*>(c->values), c->key_scale,
          c->value_scale, c->times, c->open_keys, c->open_values, c->tables, c->lengths, c->free_list, c->n_free};
  return GSIT_OK;
}
gsit_status cache_of(const gsit_cache* c, const Geometry& g, Cache* out) {
  const gsit_status st = tables_of(c, g, out);
  if (st != GSIT_OK) return st;
  if ((c->kind != GSIT_CACHE_INT8 && c->kind != GSIT_CACHE_E4M3) || (c->dtype != GSIT_F32 && c->dtype != GSIT_BF16) || c->kv_heads < 1) return GSIT_ERR_INVALID_ARG;
  if ((c->head_dim != 8 && c->head_dim != 16 && c->head_dim != 32 && c->head_dim != 64) || c->kv_heads > 65535) return GSIT_ERR_UNSUPPORTED;
  for (const void* p : {(const void*)c->keys, (const void*)c->values, (const void*)c->open_keys, (const void*)c->open_values})
    if (p == nullptr || !aligned(p, 16)) return GSIT_ERR_INVALID_ARG;
  if (c->key_scale == nullptr || c->value_scale == nullptr || !aligned(c->key_scale, 4) || !aligned(c->value_scale, 4) || !aligned(c->times, 16))
    return GSIT_ERR_INVALID_ARG;
  return GSIT_OK;
}
// Rows that the kernels load 16 bytes at a time.
bool rows_ok(const void* p, int64_t ld, int64_t cols, int32_t dtype) {
  return p != nullptr && aligned(p, 16) && ld >= cols && ld % (dtype == GSIT_BF16 ? 8 : 4) == 0;
}

gsit_status attention_args(const gsit_shape* shape, const gsit_score_rule* r, const gsit_cache* cache, const RowTimes& times, Geometry* g, CachedArgs* a) {
  gsit_status st = basic_geometry(shape, g);
  if (st != GSIT_OK) return st;
  if (g->row_start != nullptr) return GSIT_ERR_UNSUPPORTED;
  *a = {};
  st = cache_of(cache, *g, &a->c);
  if (st != GSIT_OK) return st;
  if (r == nullptr || shape->dtype != cache->dtype || g->hd != cache->head_dim || (r->kv_heads != 0 && r->kv_heads != cache->kv_heads)) return GSIT_ERR_INVALID_ARG;
  if (g->heads % cache->kv_heads != 0 || r->softcap != r->softcap || !aligned(r->slopes, 4) || !aligned(times.p, 4)) return GSIT_ERR_INVALID_ARG;
  if (r->times != nullptr || r->documents != nullptr || (r->causal && r->prefix != nullptr) || r->tail) return GSIT_ERR_UNSUPPORTED;
  a->group = g->heads / cache->kv_heads;
  if ((int64_t)g->L * a->group > 1 << 20) return GSIT_ERR_UNSUPPORTED;
  a->rows = g->L * a->group;
  a->causal = r->causal != 0;
  a->slopes = r->slopes;
  a->times = times;
  if ((a->causal || a->slopes != nullptr) && (times.p != nullptr) != (cache->times != nullptr)) return GSIT_ERR_INVALID_ARG;
  // indices are compared and subtracted as floats, which are whole numbers up to 2^24
  if ((a->causal || a->slopes != nullptr) && cache->times == nullptr && cache->blocks > (1 << 24) / CACHE_BLOCK) return GSIT_ERR_UNSUPPORTED;
  const float scale = shape->scale > 0.f ? shape->scale : 1.0f / sqrtf((float)g->hd);
  constexpr float LOG2E = 1.4426950408889634f;
  a->softcap = r->softcap > 0.f ? r->softcap : 0.f;
  // bf16 rows' tanh by 1 - 2 / (e^2y + 1) is off by 2^-22 of 1, however small it is: by 2^-22 of the cap in the score, 2^-16 at FAST_CAP
  constexpr float FAST_CAP = 64.f;
  a->fast_cap = shape->dtype == GSIT_BF16 && a->softcap <= FAST_CAP;
  a->inner = a->softcap > 0.f ? scale / a->softcap * (a->fast_cap ? 2.f * LOG2E : 1.f) : scale * LOG2E;
  a->outer = a->softcap * LOG2E;
  return isfinite(a->inner) && isfinite(a->outer) ? GSIT_OK : GSIT_ERR_INVALID_ARG;
}

cudaError_t launch_attention(const Geometry& g, int32_t dtype, CachedArgs& a, cudaStream_t st, size_t* scratch) {
  return dtype == GSIT_BF16 ? launch_cached_bf16(g, a, st, scratch) : launch_cached_f32(g, a, st, scratch);
}

// The calls' checks; what is left behind them is ready() and to launch.
gsit_status ready(Geometry* g) { return status_of(device_status_word(&g->status)) == GSIT_OK ? GSIT_OK : GSIT_ERR_CUDA; }
struct Rows {
  const void* p;
  int64_t ld;
};
gsit_status plan_call(const gsit_shape* shape, const gsit_cache* cache, const int32_t* held, const int32_t* ended, const int32_t* slots, Geometry* g, Cache* c) {
  gsit_status st = step_geometry(shape, g);
  if (st == GSIT_OK) st = tables_of(cache, *g, c);
  if (st != GSIT_OK) return st;
  for (const void* p : {(const void*)c->free_list, (const void*)c->n_free, (const void*)slots})
    if (p == nullptr || !aligned(p, 4)) return GSIT_ERR_INVALID_ARG;
  if (!aligned(held, 4) || !aligned(ended, 4)) return GSIT_ERR_INVALID_ARG;
  return GSIT_OK;
}
gsit_status append_call(const gsit_shape* shape, const gsit_cache* cache, const Rows& k, const Rows& v, const int32_t* slots, const float* times, Geometry* g, Cache* c) {
  gsit_status st = step_geometry(shape, g);
  if (st == GSIT_OK) st = cache_of(cache, *g, c);
  if (st != GSIT_OK) return st;
  const int64_t cols = (int64_t)c->kv_heads * c->hd;
  if (!rows_ok(k.p, k.ld, cols, cache->dtype) || !rows_ok(v.p, v.ld, cols, cache->dtype) || slots == nullptr || !aligned(slots, 4) || !aligned(times, 4) ||
      (c->times != nullptr && times == nullptr))
    return GSIT_ERR_INVALID_ARG;
  return GSIT_OK;
}
gsit_status attention_call(const gsit_shape* shape, const gsit_score_rule* rule, const gsit_cache* cache, const Rows& q, const RowTimes& times, void* out, float* lse,
                           void* workspace, size_t workspace_bytes, Geometry* g, CachedArgs* a) {
  const gsit_status st = attention_args(shape, rule, cache, times, g, a);
  if (st != GSIT_OK) return st;
  if (!rows_ok(q.p, q.ld, g->d, cache->dtype) || out == nullptr || !aligned(out, cache->dtype == GSIT_BF16 ? 2 : 4) || !aligned(lse, 4)) return GSIT_ERR_INVALID_ARG;
  size_t need = 0;
  const cudaError_t e = launch_attention(*g, cache->dtype, *a, nullptr, &need);
  if (e != cudaSuccess) return status_of(e);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return GSIT_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 16)) return GSIT_ERR_INVALID_ARG;
  a->q = q.p;
  a->ldq = q.ld;
  a->out = out;
  a->lse = lse;
  a->parts = static_cast<float*>(workspace);
  return GSIT_OK;
}

}  // namespace
}  // namespace gsit

using namespace gsit;

extern "C" {

gsit_status gsit_cache_plan(const gsit_shape* shape, const gsit_cache* cache, const int32_t* held, const int32_t* ended, int32_t* slots, gsit_stream stream) {
  Geometry g;
  Cache c;
  gsit_status st = plan_call(shape, cache, held, ended, slots, &g, &c);
  if (st == GSIT_OK) st = ready(&g);
  return st != GSIT_OK ? st : status_of(launch_cache_plan(g, c, held, ended, slots, static_cast<cudaStream_t>(stream)));
}

gsit_status gsit_cache_append(const gsit_shape* shape, const gsit_cache* cache, const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride,
                              const int32_t* slots, const float* times, int64_t times_batch_stride, int64_t times_row_stride, gsit_stream stream) {
  Geometry g;
  Cache c;
  gsit_status st = append_call(shape, cache, {k, k_row_stride}, {v, v_row_stride}, slots, times, &g, &c);
  if (st == GSIT_OK) st = ready(&g);
  if (st != GSIT_OK) return st;
  return status_of(launch_cache_append(g, cache->dtype, c, k, k_row_stride, v, v_row_stride, slots, {times, times_batch_stride, times_row_stride}, static_cast<cudaStream_t>(stream)));
}

gsit_status gsit_cache_read(const gsit_shape* shape, const gsit_cache* cache, void* k, int64_t k_row_stride, void* v, int64_t v_row_stride, gsit_stream stream) {
  Geometry g;
  Cache c;
  gsit_status st = step_geometry(shape, &g);
  if (st == GSIT_OK) st = cache_of(cache, g, &c);
  if (st != GSIT_OK) return st;
  const int64_t cols = (int64_t)c.kv_heads * c.hd;
  if (!rows_ok(k, k_row_stride, cols, cache->dtype) || !rows_ok(v, v_row_stride, cols, cache->dtype)) return GSIT_ERR_INVALID_ARG;
  if (status_of(device_status_word(&g.status)) != GSIT_OK) return GSIT_ERR_CUDA;
  return status_of(launch_cache_read(g, cache->dtype, c, k, k_row_stride, v, v_row_stride, static_cast<cudaStream_t>(stream)));
}

size_t gsit_cached_attention_workspace(const gsit_shape* shape, const gsit_score_rule* rule, const gsit_cache* cache) {
  Geometry g;
  CachedArgs a;
  if (cache == nullptr || attention_args(shape, rule, cache, {cache->times, 0, 0}, &g, &a) != GSIT_OK) return (size_t)-1;
  size_t need = 0;
  return launch_attention(g, cache->dtype, a, nullptr, &need) == cudaSuccess ? need : (size_t)-1;
}

gsit_status gsit_im_cached_attention_fwd(const gsit_shape* shape, const gsit_score_rule* rule, const gsit_cache* cache, const void* q, int64_t q_row_stride,
                                         const float* times, int64_t times_batch_stride, int64_t times_row_stride, void* out, float* lse, void* workspace,
                                         size_t workspace_bytes, gsit_stream stream) {
  Geometry g;
  CachedArgs a;
  gsit_status st = attention_call(shape, rule, cache, {q, q_row_stride}, {times, times_batch_stride, times_row_stride}, out, lse, workspace, workspace_bytes, &g, &a);
  if (st == GSIT_OK) st = ready(&g);
  return st != GSIT_OK ? st : status_of(launch_attention(g, cache->dtype, a, static_cast<cudaStream_t>(stream), nullptr));
}

gsit_status gsit_cache_step(const gsit_shape* shape, const gsit_score_rule* rule, const gsit_cache* cache, const int32_t* held, const int32_t* ended,
                            int32_t* slots, const void* q, int64_t q_row_stride, const void* k, int64_t k_row_stride, const void* v, int64_t v_row_stride,
                            const float* times, int64_t times_batch_stride, int64_t times_row_stride, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, gsit_stream stream) {
  const RowTimes moments = {times, times_batch_stride, times_row_stride};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  Geometry gp = {}, ga = {}, gq = {};
  Cache tables, c;
  CachedArgs a;
  // all checks, then all launches
  gsit_status st = plan_call(shape, cache, held, ended, slots, &gp, &tables);
  if (st == GSIT_OK) st = append_call(shape, cache, {k, k_row_stride}, {v, v_row_stride}, slots, times, &ga, &c);
  if (st == GSIT_OK) st = attention_call(shape, rule, cache, {q, q_row_stride}, moments, out, lse, workspace, workspace_bytes, &gq, &a);
  if (st == GSIT_OK) st = ready(&gp);
  ga.status = gq.status = gp.status;
  if (st == GSIT_OK) st = status_of(launch_cache_plan(gp, tables, held, ended, slots, s));
  if (st == GSIT_OK) st = status_of(launch_cache_append(ga, cache->dtype, c, k, k_row_stride, v, v_row_stride, slots, moments, s));
  if (st == GSIT_OK) st = status_of(launch_attention(gq, cache->dtype, a, s, nullptr));
  return st;
}

}  // extern "C"

// Attention with a rule on its scores (gsit_ops.h): what its kernels share -- the arguments, which pairs are open, the score function,
// and the row-wise path, which takes one row at a time and touches open pairs only.
#pragma once
#include <math.h>

#include "ops.cuh"

namespace gsit {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct ScoredArgs {
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv;                  // elements between rows
  void* out; int64_t ldo;                 // forward: written; backward: read
  float* lse;                             // natural logarithm, [B, H, Lq]
  float scale, softcap;
  int causal, kv_heads, group;            // group = heads / kv_heads
  const float *slopes, *times, *prefix;
  const int32_t* documents;
  int tail, q_len[3], q_off[3], Lq;       // queries per segment and their offsets in q
  // what the scores are computed with, in base 2: x = outer * tanh(inner * dot) with a cap, x = inner * dot without
  float inner, outer;
  // backward
  const void* dout; int64_t lddo;
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
  float2* row_stats;                      // [B, H, L]: (lse in base 2, +inf for a row without open keys; dO . O)
  float* partial;                         // scratch of kernels that split a row's keys
  int splits;
};

inline bool rule_masks(const ScoredArgs& a) { return a.causal != 0 || a.documents != nullptr; }

// Queries of segment s of sample b: rows [lo, hi) of the segment's q_len rows are real, row i is position i + shift of the segment.
struct QueryRows {
  int lo, hi, shift;
};
__device__ __forceinline__ QueryRows query_rows(const Geometry& g, const ScoredArgs& a, int b, int s) {
  const int n = valid_rows(g, b, s);
  if (!a.tail) return {0, n, 0};
  return {max(0, a.q_len[s] - n), a.q_len[s], n - a.q_len[s]};
}

// Moment and document of position `pos` of segment s.
__device__ __forceinline__ float time_of(const Geometry& g, const ScoredArgs& a, int b, int s, int pos) {
  return a.times != nullptr ? a.times[(int64_t)b * g.L + g.off(s) + pos] : (float)pos;
}
__device__ __forceinline__ int document_of(const Geometry& g, const ScoredArgs& a, int b, int s, int pos) {
  return a.documents != nullptr ? a.documents[(int64_t)b * g.L + g.off(s) + pos] : 0;
}
// The latest moment a query at `time` sees: its own, or the last one before the prefix ends.  key time <= limit is the causal rule.
__device__ __forceinline__ float latest_seen(const ScoredArgs& a, int b, float time) {
  if (!a.causal) return INFINITY;
  return a.prefix != nullptr ? fmaxf(time, nextafterf(a.prefix[b], -INFINITY)) : time;
}

// tanh by an odd polynomial of degree 9 (least squares fit of the relative error over |y| <= 3/4, refined towards equal error: 5.7e-7)
// and, beyond, by 1 - 2 / (e^2y + 1), where nothing cancels any more.
constexpr float TANH_RANGE = 0.75f;
constexpr float TANH_C0 = 0.99999943f, TANH_C1 = -0.33328251f, TANH_C2 = 0.13258982f, TANH_C3 = -0.05005628f, TANH_C4 = 0.01292961f;
__device__ __forceinline__ float2 tanh_near2(float2 y) {   // |y| <= 3/4
  const float2 z = __fmul2_rn(y, y);
  float2 p = __ffma2_rn(z, make_float2(TANH_C4, TANH_C4), make_float2(TANH_C3, TANH_C3));
  p = __ffma2_rn(p, z, make_float2(TANH_C2, TANH_C2));
  p = __ffma2_rn(p, z, make_float2(TANH_C1, TANH_C1));
  p = __ffma2_rn(p, z, make_float2(TANH_C0, TANH_C0));
  return __fmul2_rn(p, y);
}
__device__ __forceinline__ float tanh_far(float y) {       // |y| > 3/4
  const float e = ptx::ex2(2.0f * LOG2E * fabsf(y));
  return copysignf(1.0f - __fdividef(2.0f, e + 1.0f), y);
}
__device__ __forceinline__ float2 tanh_any2(float2 y) {
  const float2 t = tanh_near2(y);
  return make_float2(fabsf(y.x) > TANH_RANGE ? tanh_far(y.x) : t.x, fabsf(y.y) > TANH_RANGE ? tanh_far(y.y) : t.y);
}

// ---- the row-wise path: a warp takes one row, its lanes every 32nd partner; closed pairs are skipped, so that nothing in them counts.
// It serves the rows whose matrix products came out non-finite because a closed partner holds NaN or Inf (0 * NaN), whatever the type.
template <typename T, int HD> __device__ __forceinline__ void load_row(const T* p, int hd, float (&f)[HD]) {
#pragma unroll
  for (int e = 0; e < HD; ++e) f[e] = e < hd ? to_float(p[e]) : 0.f;
}
template <typename T, int HD> __device__ __forceinline__ float dot_row(const T* p, int hd, const float (&f)[HD]) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < HD; ++e)
    if (e < hd) s += to_float(p[e]) * f[e];
  return s;
}
// Score of one pair in base 2, and the derivative of the cap.
__device__ __forceinline__ float score_of(const ScoredArgs& a, float dot, float slope2, float distance, float* bend) {
  float x = dot * a.inner;
  *bend = 1.f;
  if (a.softcap > 0.f) {
    const float t = tanh_any2(make_float2(x, x)).x;
    *bend = 1.f - t * t;
    x = t * a.outer;
  }
  return x - slope2 * distance;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Row i (of segment s's queries), head h: out and lse.
template <typename T, int HD>
__device__ __noinline__ void attend_row(const Geometry& g, const ScoredArgs& a, int b, int h, int s, int i) {
  const int lane = threadIdx.x & 31, hk = h / a.group;
  const QueryRows rows = query_rows(g, a, b, s);
  const int64_t row = (int64_t)b * a.Lq + a.q_off[s] + i;
  float m = -INFINITY, l = 0.f, q[HD], acc[HD];
  load_row<T, HD>(static_cast<const T*>(a.q) + row * a.ldq + (int64_t)h * g.hd, g.hd, q);
#pragma unroll
  for (int e = 0; e < HD; ++e) acc[e] = 0.f;
  if (i >= rows.lo && i < rows.hi) {
    const float t = time_of(g, a, b, s, i + rows.shift), limit = latest_seen(a, b, t), slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
    const int doc = document_of(g, a, b, s, i + rows.shift);
    for (int r = 0; r < 3; ++r) {
      const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
      for (int j = lane; j < n; j += 32) {
        const float tj = time_of(g, a, b, r, j);
        if (tj > limit || document_of(g, a, b, r, j) != doc) continue;
        const int64_t key = (int64_t)b * g.L + g.off(r) + j;
        float bend;
        const float x = score_of(a, dot_row<T, HD>(static_cast<const T*>(a.k) + key * a.ldk + (int64_t)hk * g.hd, g.hd, q), slope2, fabsf(t - tj), &bend);
        if (x > m) {
          const float f = ptx::ex2(m - x);
          l *= f;
#pragma unroll
          for (int e = 0; e < HD; ++e) acc[e] *= f;
          m = x;
        }
        const float p = x == -INFINITY ? 0.f : ptx::ex2(x - m);
        const T* v = static_cast<const T*>(a.v) + key * a.ldv + (int64_t)hk * g.hd;
        l += p;
#pragma unroll
        for (int e = 0; e < HD; ++e)
          if (e < g.hd) acc[e] += p * to_float(v[e]);
      }
    }
  }
  __syncwarp();
  const float top = warp_max(m), f = m == -INFINITY ? 0.f : ptx::ex2(m - top);
  l = warp_sum(l * f);
  const float inv = l != 0.f ? 1.f / l : 0.f;   // NaN stays
  T* out = static_cast<T*>(a.out) + row * a.ldo + (int64_t)h * g.hd;
#pragma unroll
  for (int e = 0; e < HD; ++e)
    if (e < g.hd) {
      const float o = warp_sum(f == 0.f ? 0.f : acc[e] * f) * inv;
      if (lane == 0) store_as(out + e, o);
    }
  if (lane == 0 && a.lse != nullptr) a.lse[((int64_t)b * g.heads + h) * a.Lq + a.q_off[s] + i] = l != 0.f ? (top + log2f(l)) * LN2 : -INFINITY;
}

// Gradient of query row i of segment s, head h; also writes the row's statistics.
template <typename T, int HD>
__device__ __noinline__ void dq_row(const Geometry& g, const ScoredArgs& a, int b, int h, int s, int i) {
  const int lane = threadIdx.x & 31, hk = h / a.group;
  const int n_q = valid_rows(g, b, s);
  const int64_t row = (int64_t)b * g.L + g.off(s) + i, at = ((int64_t)b * g.heads + h) * g.L + g.off(s) + i;
  const float lse = i < n_q ? a.lse[at] : -INFINITY;
  float q[HD], go[HD], acc[HD], lse2 = INFINITY, delta = 0.f;
#pragma unroll
  for (int e = 0; e < HD; ++e) acc[e] = 0.f;
  if (lse != -INFINITY) {
    load_row<T, HD>(static_cast<const T*>(a.q) + row * a.ldq + (int64_t)h * g.hd, g.hd, q);
    load_row<T, HD>(static_cast<const T*>(a.dout) + row * a.lddo + (int64_t)h * g.hd, g.hd, go);
    delta = dot_row<T, HD>(static_cast<const T*>(a.out) + row * a.ldo + (int64_t)h * g.hd, g.hd, go);
    lse2 = lse * LOG2E;
    const float t = time_of(g, a, b, s, i), limit = latest_seen(a, b, t), slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
    const int doc = document_of(g, a, b, s, i);
    for (int r = 0; r < 3; ++r) {
      const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
      for (int j = lane; j < n; j += 32) {
        const float tj = time_of(g, a, b, r, j);
        if (tj > limit || document_of(g, a, b, r, j) != doc) continue;
        const int64_t key = (int64_t)b * g.L + g.off(r) + j;
        const T* k = static_cast<const T*>(a.k) + key * a.ldk + (int64_t)hk * g.hd;
        float bend;
        const float p = ptx::ex2(score_of(a, dot_row<T, HD>(k, g.hd, q), slope2, fabsf(t - tj), &bend) - lse2);
        const float ds = p * (dot_row<T, HD>(static_cast<const T*>(a.v) + key * a.ldv + (int64_t)hk * g.hd, g.hd, go) - delta) * bend;
#pragma unroll
        for (int e = 0; e < HD; ++e)
          if (e < g.hd) acc[e] += ds * to_float(k[e]);
      }
    }
  }
  __syncwarp();
  T* dq = static_cast<T*>(a.dq) + row * a.lddq + (int64_t)h * g.hd;
#pragma unroll
  for (int e = 0; e < HD; ++e)
    if (e < g.hd) {
      const float d = warp_sum(acc[e]) * a.scale;
      if (lane == 0) store_as(dq + e, lse2 == INFINITY ? 0.f : d);
    }
  if (lane == 0) a.row_stats[at] = make_float2(lse2, delta);
}

// Gradients of key and value row j of segment r, key head hk: over the query heads that share it and all their open rows.
template <typename T, int HD>
__device__ __noinline__ void dkv_row(const Geometry& g, const ScoredArgs& a, int b, int hk, int r, int j) {
  const int lane = threadIdx.x & 31;
  const int64_t key = (int64_t)b * g.L + g.off(r) + j;
  float k[HD], v[HD], dk[HD], dv[HD];
#pragma unroll
  for (int e = 0; e < HD; ++e) dk[e] = dv[e] = 0.f;
  if (j < valid_rows(g, b, r)) {
    load_row<T, HD>(static_cast<const T*>(a.k) + key * a.ldk + (int64_t)hk * g.hd, g.hd, k);
    load_row<T, HD>(static_cast<const T*>(a.v) + key * a.ldv + (int64_t)hk * g.hd, g.hd, v);
    const float tj = time_of(g, a, b, r, j);
    const int doc = document_of(g, a, b, r, j);
    for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
      const float slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
      for (int s = 0; s < 3; ++s) {
        const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, s) : 0;
        for (int i = lane; i < n; i += 32) {
          const float t = time_of(g, a, b, s, i);
          const float2 stats = a.row_stats[((int64_t)b * g.heads + h) * g.L + g.off(s) + i];
          if (tj > latest_seen(a, b, t) || document_of(g, a, b, s, i) != doc || stats.x == INFINITY) continue;
          const int64_t row = (int64_t)b * g.L + g.off(s) + i;
          const T* q = static_cast<const T*>(a.q) + row * a.ldq + (int64_t)h * g.hd;
          const T* go = static_cast<const T*>(a.dout) + row * a.lddo + (int64_t)h * g.hd;
          float bend;
          const float p = ptx::ex2(score_of(a, dot_row<T, HD>(q, g.hd, k), slope2, fabsf(t - tj), &bend) - stats.x);
          const float ds = p * (dot_row<T, HD>(go, g.hd, v) - stats.y) * bend;
#pragma unroll
          for (int e = 0; e < HD; ++e)
            if (e < g.hd) {
              dk[e] += ds * to_float(q[e]);
              dv[e] += p * to_float(go[e]);
            }
        }
      }
    }
  }
  __syncwarp();
  T* pk = static_cast<T*>(a.dk) + key * a.lddk + (int64_t)hk * g.hd;
  T* pv = static_cast<T*>(a.dv) + key * a.lddv + (int64_t)hk * g.hd;
#pragma unroll
  for (int e = 0; e < HD; ++e)
    if (e < g.hd) {
      const float x = warp_sum(dk[e]) * a.scale, y = warp_sum(dv[e]);
      if (lane == 0) {
        store_as(pk + e, x);
        store_as(pv + e, y);
      }
    }
}

// ---- launch entry points ----
cudaError_t launch_scored_rows_fwd(const Geometry& g, int dtype, const ScoredArgs& a, cudaStream_t st);   // scored_rows.cu
cudaError_t launch_scored_rows_bwd(const Geometry& g, int dtype, const ScoredArgs& a, cudaStream_t st);
cudaError_t launch_scored_fwd_bf16(const Geometry& g, const ScoredArgs& a, cudaStream_t st);              // scored_fwd.cu
cudaError_t launch_scored_bwd_bf16(const Geometry& g, const ScoredArgs& a, cudaStream_t st);              // scored_bwd.cu

}  // namespace gsit

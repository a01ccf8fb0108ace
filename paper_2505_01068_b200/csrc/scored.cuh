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
  // ... and, for dots of at most near_dot (|tanh's argument| <= 1/4), as polynomials of the dot d:  x = d (p0 + p1 d^2 + p2 d^4),
  // derivative of the cap = b0 + b1 d^2 + b2 d^4
  float near_dot, near_p[3], near_b[3];
  // backward
  const void* dout; int64_t lddo;
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
  float2* row_stats;                      // [B, H, L]: (lse in base 2, +inf for a row without open keys; sum over P dP)
};

__host__ __device__ __forceinline__ bool rule_masks(const ScoredArgs& a) { return a.causal != 0 || a.documents != nullptr; }

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

// tanh where operands are bf16: by an odd polynomial of degree 7 (least squares fit of the relative error over |y| <= 1/2, refined towards
// equal error: 5.5e-7) and, beyond, by 1 - 2 / (e^2y + 1), where little cancels any more: some 2^-21 of the score, next to dots whose
// operands were rounded at 2^-9.  The float kernels and the row-wise path call tanhf, which keeps float's own rounding (a capped score 5.4e-8 off,
// root mean square, where this fit leaves 3.5e-7): 8 x (50, 500, 500), 8 heads of 8, float, forward and gradients 55 + 136 us, with the fit 52 + 131.
constexpr float TANH_RANGE = 0.5f;
constexpr float TANH_C0 = 0.999999456f, TANH_C1 = -0.333263179f, TANH_C2 = 0.131902962f, TANH_C3 = -0.0444022147f;
__device__ __forceinline__ float2 tanh_near2(float2 y) {   // |y| <= 1/2
  const float2 z = __fmul2_rn(y, y);
  float2 p = __ffma2_rn(z, make_float2(TANH_C3, TANH_C3), make_float2(TANH_C2, TANH_C2));
  p = __ffma2_rn(p, z, make_float2(TANH_C1, TANH_C1));
  p = __ffma2_rn(p, z, make_float2(TANH_C0, TANH_C0));
  return __fmul2_rn(p, y);
}
__device__ __forceinline__ float tanh_far(float y) {       // |y| > 1/2
  const float e = ptx::ex2(2.0f * LOG2E * fabsf(y));
  return copysignf(1.0f - __fdividef(2.0f, e + 1.0f), y);
}
__device__ __forceinline__ float2 tanh_any2(float2 y) {
  const float2 t = tanh_near2(y);
  return make_float2(fabsf(y.x) > TANH_RANGE ? tanh_far(y.x) : t.x, fabsf(y.y) > TANH_RANGE ? tanh_far(y.y) : t.y);
}

// Score of one pair in base 2, and the derivative of the cap.
__device__ __forceinline__ float score_of(const ScoredArgs& a, float dot, float slope2, float distance, float* bend) {
  float x = dot * a.inner;
  *bend = 1.f;
  if (a.softcap > 0.f) {
    const float t = tanhf(x);
    *bend = 1.f - t * t;
    x = t * a.outer;
  }
  return x - slope2 * distance;
}

// ---- the row-wise path: a warp takes one row, its lanes the features (at most four each), one partner after the other; closed pairs
// are skipped, so that nothing in them counts.  It serves the rows whose matrix products came out non-finite because a closed partner
// holds NaN or Inf (0 * NaN), and the widest float heads.  Few registers, so that it costs the kernels that call it none.
struct LaneRow {
  float f[4];
};
template <typename T> __device__ __forceinline__ LaneRow lane_row(const void* base, int64_t at, int hd) {
  LaneRow r;
  const T* p = static_cast<const T*>(base) + at;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = (threadIdx.x & 31) + 32 * e;
    r.f[e] = c < hd ? to_float(p[c]) : 0.f;
  }
  return r;
}
template <typename T> __device__ __forceinline__ void store_lane_row(void* base, int64_t at, int hd, const LaneRow& r, float scale) {
  T* p = static_cast<T*>(base) + at;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int c = (threadIdx.x & 31) + 32 * e;
    if (c < hd) store_as(p + c, r.f[e] * scale);
  }
}
__device__ __forceinline__ float lane_dot(const LaneRow& x, const LaneRow& y) {
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) s += x.f[e] * y.f[e];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}
__device__ __forceinline__ void lane_add(LaneRow& x, float w, const LaneRow& y) {
#pragma unroll
  for (int e = 0; e < 4; ++e) x.f[e] += w * y.f[e];
}

// Row i (of segment s's queries), head h: out and lse.
template <typename T>
__device__ __noinline__ void attend_row(const Geometry& g, const ScoredArgs& a, int b, int h, int s, int i) {
  const QueryRows rows = query_rows(g, a, b, s);
  const int64_t row = (int64_t)b * a.Lq + a.q_off[s] + i, head = (int64_t)h * g.hd, key_head = (int64_t)(h / a.group) * g.hd;
  float m = -INFINITY, l = 0.f;
  LaneRow acc = {};
  if (i >= rows.lo && i < rows.hi) {
    const LaneRow q = lane_row<T>(a.q, row * a.ldq + head, g.hd);
    const float t = time_of(g, a, b, s, i + rows.shift), limit = latest_seen(a, b, t), slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
    const int doc = document_of(g, a, b, s, i + rows.shift);
    for (int r = 0; r < 3; ++r) {
      const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
      for (int j = 0; j < n; ++j) {
        const float tj = time_of(g, a, b, r, j);
        if (tj > limit || document_of(g, a, b, r, j) != doc) continue;
        const int64_t key = (int64_t)b * g.L + g.off(r) + j;
        float bend;
        const float x = score_of(a, lane_dot(lane_row<T>(a.k, key * a.ldk + key_head, g.hd), q), slope2, fabsf(t - tj), &bend);
        if (x > m) {
          const float f = ptx::ex2(m - x);
          l *= f;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc.f[e] *= f;
          m = x;
        }
        const float p = x == -INFINITY ? 0.f : ptx::ex2(x - m);
        l += p;
        lane_add(acc, p, lane_row<T>(a.v, key * a.ldv + key_head, g.hd));
      }
    }
  }
  __syncwarp();
  store_lane_row<T>(a.out, row * a.ldo + head, g.hd, acc, l != 0.f ? 1.f / l : 0.f);   // a sum of NaN stays
  if ((threadIdx.x & 31) == 0 && a.lse != nullptr)
    a.lse[((int64_t)b * g.heads + h) * a.Lq + a.q_off[s] + i] = l != 0.f ? (m + log2f(l)) * LN2 : -INFINITY;
}

// Gradient of query row i of segment s, head h; also writes the row's statistics.
template <typename T>
__device__ __noinline__ void dq_row(const Geometry& g, const ScoredArgs& a, int b, int h, int s, int i) {
  const int64_t row = (int64_t)b * g.L + g.off(s) + i, at = ((int64_t)b * g.heads + h) * g.L + g.off(s) + i;
  const int64_t head = (int64_t)h * g.hd, key_head = (int64_t)(h / a.group) * g.hd;
  const float lse = i < valid_rows(g, b, s) ? a.lse[at] : -INFINITY;
  float lse2 = INFINITY, delta = 0.f, more = 0.f;   // more, along: see scored_bwd.cu
  LaneRow acc = {}, along = {};
  if (lse != -INFINITY) {
    const LaneRow q = lane_row<T>(a.q, row * a.ldq + head, g.hd), go = lane_row<T>(a.dout, row * a.lddo + head, g.hd);
    delta = lane_dot(lane_row<T>(a.out, row * a.ldo + head, g.hd), go);
    lse2 = lse * LOG2E;
    const float t = time_of(g, a, b, s, i), limit = latest_seen(a, b, t), slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
    const int doc = document_of(g, a, b, s, i);
    for (int r = 0; r < 3; ++r) {
      const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
      for (int j = 0; j < n; ++j) {
        const float tj = time_of(g, a, b, r, j);
        if (tj > limit || document_of(g, a, b, r, j) != doc) continue;
        const int64_t key = (int64_t)b * g.L + g.off(r) + j;
        const LaneRow k = lane_row<T>(a.k, key * a.ldk + key_head, g.hd);
        float bend;
        const float p = ptx::ex2(score_of(a, lane_dot(k, q), slope2, fabsf(t - tj), &bend) - lse2);
        const float d = lane_dot(lane_row<T>(a.v, key * a.ldv + key_head, g.hd), go) - delta;
        more += p * d;
        lane_add(acc, p * d * bend, k);
        lane_add(along, p * bend, k);
      }
    }
  }
  lane_add(acc, -more, along);
  __syncwarp();
  store_lane_row<T>(a.dq, row * a.lddq + head, g.hd, acc, a.scale);
  if ((threadIdx.x & 31) == 0) a.row_stats[at] = make_float2(lse2, delta + more);
}

// Gradients of key and value row j of segment r, key head hk: over the query heads that share it and all their open rows.
template <typename T>
__device__ __noinline__ void dkv_row(const Geometry& g, const ScoredArgs& a, int b, int hk, int r, int j) {
  const int64_t key = (int64_t)b * g.L + g.off(r) + j, key_head = (int64_t)hk * g.hd;
  LaneRow dk = {}, dv = {};
  if (j < valid_rows(g, b, r)) {
    const LaneRow k = lane_row<T>(a.k, key * a.ldk + key_head, g.hd), v = lane_row<T>(a.v, key * a.ldv + key_head, g.hd);
    const float tj = time_of(g, a, b, r, j);
    const int doc = document_of(g, a, b, r, j);
    for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
      const float slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
      const int64_t head = (int64_t)h * g.hd;
      for (int s = 0; s < 3; ++s) {
        const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, s) : 0;
        for (int i = 0; i < n; ++i) {
          const float t = time_of(g, a, b, s, i);
          const float2 stats = a.row_stats[((int64_t)b * g.heads + h) * g.L + g.off(s) + i];
          if (tj > latest_seen(a, b, t) || document_of(g, a, b, s, i) != doc || stats.x == INFINITY) continue;
          const int64_t row = (int64_t)b * g.L + g.off(s) + i;
          const LaneRow q = lane_row<T>(a.q, row * a.ldq + head, g.hd), go = lane_row<T>(a.dout, row * a.lddo + head, g.hd);
          float bend;
          const float p = ptx::ex2(score_of(a, lane_dot(q, k), slope2, fabsf(t - tj), &bend) - stats.x);
          lane_add(dk, p * (lane_dot(go, v) - stats.y) * bend, q);
          lane_add(dv, p, go);
        }
      }
    }
  }
  __syncwarp();
  store_lane_row<T>(a.dk, key * a.lddk + key_head, g.hd, dk, a.scale);
  store_lane_row<T>(a.dv, key * a.lddv + key_head, g.hd, dv, 1.f);
}

// Query tiles (or key tiles) of the three segments, in the order they are handed out: longest walks first, over all samples, so that the
// short ones fill the places that are left at the end.  Sample by sample instead: MOSEI step 96 + 104 + 109 us for 84 + 101 + 95 (forward,
// dq, dk and dv), packed causal rows 50 + 44 + 42 for 43 + 30 + 35.
struct Tiles {
  int count[3];
  int order;         // segments, two bits each
};
struct Place {
  int tile, segment, sample, head;
};
// CTA x of tiles * batch * heads (the latter in rounds, where a CTA takes several)
__device__ __forceinline__ Place find_place(const Tiles& tiles, int batch, int heads) {
  const int x = blockIdx.x, per_tile = batch * heads;
  Place p;
  p.tile = x / per_tile;
  const int y = x - p.tile * per_tile;
  p.sample = y / heads;
  p.head = y - p.sample * heads;
  p.segment = tiles.order & 3;
  if (p.tile >= tiles.count[p.segment]) {
    p.tile -= tiles.count[p.segment];
    p.segment = (tiles.order >> 2) & 3;
    if (p.tile >= tiles.count[p.segment]) {
      p.tile -= tiles.count[p.segment];
      p.segment = tiles.order >> 4;
    }
  }
  p.tile = tiles.count[p.segment] - 1 - p.tile;   // from the back: under the causal rule the later rows walk further
  return p;
}
// ---- which pairs of a block are open ----
constexpr int BLOCK = 64;   // partners that are classified together
__device__ __forceinline__ int ordered(float f) {   // floats as integers of the same order; both zeros are 0, as comparisons have them
  const int i = __float_as_int(f + 0.f);
  return i ^ ((i >> 31) & 0x7fffffff);
}
struct Range {   // over real rows: moments (as ordered integers) and documents
  int t_lo, t_hi, d_lo, d_hi;
};
__device__ __forceinline__ Range warp_range(int t_lo, int t_hi, int d_lo, int d_hi) {
  return {__reduce_min_sync(0xffffffffu, t_lo), __reduce_max_sync(0xffffffffu, t_hi), __reduce_min_sync(0xffffffffu, d_lo), __reduce_max_sync(0xffffffffu, d_hi)};
}
constexpr Range NO_ROWS = {0x7fffffff, (int)0x80000000, 0x7fffffff, (int)0x80000000};
// Queries have their latest moment seen in t, keys their own moment.
enum Openness { SHUT, SOME, ALL };
__device__ __forceinline__ Openness openness(const Range& queries, const Range& keys) {
  if (queries.d_hi < keys.d_lo || keys.d_hi < queries.d_lo || keys.t_lo > queries.t_hi) return SHUT;
  return queries.d_lo == queries.d_hi && keys.d_lo == keys.d_hi && keys.t_hi <= queries.t_lo ? ALL : SOME;
}

// Moments and documents of a block of 64 partners as a range; `t` holds what openness() compares.
__device__ __forceinline__ Range block_range(const float* t, const int* d, int j0, int rem, int lane) {
  Range r = NO_ROWS;
#pragma unroll
  for (int i = 0; i < BLOCK; i += 32)
    if (j0 + i + lane < rem) {
      const int o = ordered(t[j0 + i + lane]), e = d[j0 + i + lane];
      r = {min(r.t_lo, o), max(r.t_hi, o), min(r.d_lo, e), max(r.d_hi, e)};
    }
  return warp_range(r.t_lo, r.t_hi, r.d_lo, r.d_hi);
}
// The segments that are walked, in order, in chunks: `pos` is moved on by the caller, settle() goes to the next segment that has rows.
struct Walk {
  int n[3];          // rows to walk per segment, 0 where shut
  int seg, pos;      // where it stands; seg 3: over
  __device__ __forceinline__ int rows(int s) const { return s == 0 ? n[0] : s == 1 ? n[1] : n[2]; }
  __device__ __forceinline__ void settle() {   // over segments that hold nothing more
    if (seg == 0 && pos >= n[0]) { seg = 1; pos = 0; }
    if (seg == 1 && pos >= n[1]) { seg = 2; pos = 0; }
    if (seg == 2 && pos >= n[2]) { seg = 3; pos = 0; }
  }
  __device__ __forceinline__ bool over() const { return seg == 3; }
  __device__ __forceinline__ int left() const { return rows(seg) - pos; }
};

// Tiles of `rows` rows of segments of these lengths; returns their number.
inline int64_t make_tiles(Tiles* t, const int (&len)[3], int rows) {
  int64_t n = 0;
  for (int s = 0; s < 3; ++s) n += t->count[s] = (len[s] + rows - 1) / rows;
  return n;
}
// The block pattern seen from the keys: bit (3 r + s) is open where query segment s attends key segment r.
inline uint32_t transposed(uint32_t allowed) {
  uint32_t t = 0;
  for (int s = 0; s < 3; ++s)
    for (int r = 0; r < 3; ++r)
      if ((allowed >> (3 * s + r)) & 1u) t |= 1u << (3 * r + s);
  return t;
}

// ---- launch entry points ----
cudaError_t launch_scored_rows_fwd(const Geometry& g, const ScoredArgs& a, cudaStream_t st);              // scored_rows.cu, float
cudaError_t launch_scored_rows_bwd(const Geometry& g, const ScoredArgs& a, cudaStream_t st);
cudaError_t launch_scored_fwd_f32(const Geometry& g, const ScoredArgs& a, cudaStream_t st);               // scored_f32.cu, head_dim <= 64
cudaError_t launch_scored_bwd_f32(const Geometry& g, const ScoredArgs& a, cudaStream_t st);
bool scored_tc_preferred(const Geometry& g, const int (&rows)[3]);                                        // scored_tc.cu, head_dim 64
cudaError_t launch_scored_fwd_tc(const Geometry& g, const ScoredArgs& a, cudaStream_t st);
cudaError_t launch_scored_bwd_tc(const Geometry& g, const ScoredArgs& a, cudaStream_t st);
bool scored_tail_supported(const Geometry& g, int dtype, const ScoredArgs& a);                            // scored_tail.cu
cudaError_t launch_scored_tail(const Geometry& g, int dtype, const ScoredArgs& a, cudaStream_t st);
cudaError_t launch_scored_fwd_bf16(const Geometry& g, const ScoredArgs& a, cudaStream_t st);              // scored_fwd.cu
cudaError_t launch_scored_bwd_bf16(const Geometry& g, const ScoredArgs& a, cudaStream_t st);              // scored_bwd.cu

}  // namespace gsit

// Scored attention in single precision, forward and backward, on the FMA pipe (head_dim <= 64).
//
// A CTA of 256 threads takes 64 rows (queries in the forward pass and for dq, keys for dk and dv) and walks its partners in tiles of
// 64.  Two kinds of product, both from row-major tiles in shared memory whose rows are HD + 4 floats apart (any eight lanes that load
// 16 bytes of neighbouring rows then meet eight different bank groups):
//   over features  a thread owns rows 4 ty .. and partners tx + 16 j of the 64 x 64 tile: per four features 8 loads of 16 bytes feed 32
//                  packed multiply-adds, whose halves are the even and the odd features
//   over partners  the 64 x HD result is owned in pieces of 4 x 4; where that takes fewer than 256 threads the partners of a tile are
//                  split over groups of them, which are added up once at the end
// Between the two the weights go through shared memory, partner-major.  With 2 HD (forward), 3 HD (dq) and 4 HD (dk, dv) multiply-adds
// a pair the FMA pipe is the bound: 128 a clock and SM.
#include "scored.cuh"

namespace gsit {
namespace {

constexpr int THREADS = 256, TILE = 64, PITCH_W = TILE + 4;

template <int HD> struct Sizes {
  static constexpr int PITCH = HD + 4, ROWS = TILE * PITCH;      // floats of a staged tile of rows
  static constexpr int WEIGHTS = TILE * PITCH_W;                 // floats of a tile of weights, partner-major
  static constexpr int OWNERS = 4 * HD, GROUPS = THREADS / OWNERS, SHARE = TILE / GROUPS;   // of the 64 x HD result
};

// Rows [row0, row0 + TILE) of a [.., ld] matrix (this head's features) into shared memory; zeros from row `n` on and from feature hd on.
template <int HD> __device__ __forceinline__ void stage_rows(float* dst, const float* src, int64_t ld, int n, int hd) {
  constexpr int P = Sizes<HD>::PITCH;
  if (hd == HD && ld % 4 == 0 && (reinterpret_cast<uintptr_t>(src) & 15u) == 0) {
    for (int i = threadIdx.x; i < TILE * HD / 4; i += THREADS) {
      const int r = i / (HD / 4), c = i % (HD / 4) * 4;
      *reinterpret_cast<float4*>(dst + r * P + c) = r < n ? *reinterpret_cast<const float4*>(src + r * ld + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  } else {
    for (int i = threadIdx.x; i < TILE * HD; i += THREADS) {
      const int r = i / HD, c = i % HD;
      dst[r * P + c] = r < n && c < hd ? src[r * ld + c] : 0.f;
    }
  }
}

// x[i][j] = own row 4 ty + i . partner tx + 16 j
template <int HD> __device__ __forceinline__ void product_over_features(float (&x)[4][4], const float* own, const float* partner, int tx, int ty) {
  constexpr int P = Sizes<HD>::PITCH;
  float2 s[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) s[i][j] = make_float2(0.f, 0.f);
#pragma unroll(HD <= 16 ? HD / 4 : 4)
  for (int f = 0; f < HD; f += 4) {
    float4 q[4], k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const float4*>(own + (4 * ty + i) * P + f);
#pragma unroll
    for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4*>(partner + (tx + 16 * j) * P + f);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[i][j] = __ffma2_rn(make_float2(q[i].x, q[i].y), make_float2(k[j].x, k[j].y), s[i][j]);
        s[i][j] = __ffma2_rn(make_float2(q[i].z, q[i].w), make_float2(k[j].z, k[j].w), s[i][j]);
      }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) x[i][j] = s[i][j].x + s[i][j].y;
}

// w[partner][row] = x
__device__ __forceinline__ void put_weights(float* w, const float (&x)[4][4], int tx, int ty) {
#pragma unroll
  for (int j = 0; j < 4; ++j) *reinterpret_cast<float4*>(w + (tx + 16 * j) * PITCH_W + 4 * ty) = make_float4(x[0][j], x[1][j], x[2][j], x[3][j]);
}

// This thread's piece of a 64 x HD result: rows 4 rt .., features 4 ct .., and its group's share of the partners.
template <int HD> struct Piece {
  int rt, ct, group;
  __device__ __forceinline__ Piece() {
    const int t = threadIdx.x % Sizes<HD>::OWNERS;
    ct = t % (HD / 4);
    rt = t / (HD / 4);
    group = threadIdx.x / Sizes<HD>::OWNERS;
  }
};
template <int HD> __device__ __forceinline__ void product_over_partners(float2 (&o)[4][2], const float* w, const float* rows, const Piece<HD>& p) {
  constexpr int SHARE = Sizes<HD>::SHARE;
#pragma unroll 4
  for (int k = p.group * SHARE; k < (p.group + 1) * SHARE; ++k) {
    const float4 a = *reinterpret_cast<const float4*>(w + k * PITCH_W + 4 * p.rt), v = *reinterpret_cast<const float4*>(rows + k * Sizes<HD>::PITCH + 4 * p.ct);
    const float f[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i][0] = __ffma2_rn(make_float2(f[i], f[i]), make_float2(v.x, v.y), o[i][0]);
      o[i][1] = __ffma2_rn(make_float2(f[i], f[i]), make_float2(v.z, v.w), o[i][1]);
    }
  }
}
// Adds the groups' results up in order; the sums end in group 0.  `room`: (GROUPS - 1) * 64 * HD floats, free.
template <int HD> __device__ __forceinline__ void join_groups(float2 (&o)[4][2], float* room, const Piece<HD>& p) {
  constexpr int G = Sizes<HD>::GROUPS;
  if constexpr (G > 1) {
    __syncthreads();
    if (p.group > 0)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(room + ((p.group - 1) * TILE + 4 * p.rt + i) * HD + 4 * p.ct) = make_float4(o[i][0].x, o[i][0].y, o[i][1].x, o[i][1].y);
    __syncthreads();
    if (p.group == 0)
      for (int k = 0; k < G - 1; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 v = *reinterpret_cast<const float4*>(room + (k * TILE + 4 * p.rt + i) * HD + 4 * p.ct);
          o[i][0].x += v.x; o[i][0].y += v.y; o[i][1].x += v.z; o[i][1].y += v.w;
        }
  }
}
// Row `i` of the piece to memory (group 0); returns whether all of it is finite.
__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
template <int HD> __device__ __forceinline__ bool put_row(float* dst, int hd, const float2 (&o)[2], float scale, bool real, int ct) {
  const float f[4] = {o[0].x * scale, o[0].y * scale, o[1].x * scale, o[1].y * scale};
  bool ok = true;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (4 * ct + e < hd) {
      dst[4 * ct + e] = real ? f[e] : 0.f;
      ok = ok && finite(f[e]);
    }
  return ok || !real;
}

struct Times {   // moments, documents and limits of 64 rows
  float time[TILE], limit[TILE];
  int doc[TILE];
};
__device__ __forceinline__ void stage_times(Times& t, const Geometry& g, const ScoredArgs& a, int b, int s, int pos0, int n) {
  const int i = threadIdx.x;
  if (i < TILE) {
    const bool in = i >= 0 && i < n && pos0 + i >= 0;
    t.time[i] = in ? time_of(g, a, b, s, pos0 + i) : 0.f;
    t.limit[i] = in ? latest_seen(a, b, t.time[i]) : -INFINITY;
    t.doc[i] = in ? document_of(g, a, b, s, pos0 + i) : 0;
  }
}

// Dots of the tile -> scores in base 2, -inf where closed; `bend` times the cap's derivative.  queries_are_rows tells which side is which.
template <bool BEND>
__device__ __forceinline__ void scores(float (&x)[4][4], float (&bend)[BEND ? 4 : 1][4], const ScoredArgs& a, float slope2, const Times& own, const Times& partner,
                                       int partners, bool rule, bool queries_are_rows, int tx, int ty) {
  const float2 f = make_float2(a.inner, a.inner);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      float2 y = __fmul2_rn(make_float2(x[i][j], x[i][j + 1]), f);
      if (BEND) bend[i][j] = bend[i][j + 1] = 1.f;
      if (a.softcap > 0.f) {
        const float2 t = tanh_any2(y);
        y = __fmul2_rn(t, make_float2(a.outer, a.outer));
        if (BEND) {
          bend[i][j] = 1.f - t.x * t.x;
          bend[i][j + 1] = 1.f - t.y * t.y;
        }
      }
      x[i][j] = y.x;
      x[i][j + 1] = y.y;
    }
  if (rule) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = tx + 16 * j;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * ty + i;
        const float limit = queries_are_rows ? own.limit[r] : partner.limit[c], key = queries_are_rows ? partner.time[c] : own.time[r];
        x[i][j] -= slope2 * fabsf(own.time[r] - partner.time[c]);
        if (key > limit || own.doc[r] != partner.doc[c]) x[i][j] = -INFINITY;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (tx + 16 * j >= partners)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i][j] = -INFINITY;
}

// Over the 16 threads that share rows 4 ty ..
__device__ __forceinline__ float row_max(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

template <int HD>
__global__ void __launch_bounds__(THREADS)
scored_fwd_f32_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  using S = Sizes<HD>;
  extern __shared__ __align__(16) float smem[];
  float *s_q = smem, *s_k = s_q + S::ROWS, *s_v = s_k + S::ROWS, *s_w = s_v + S::ROWS;
  __shared__ Times own, partner;
  __shared__ __align__(16) float s_row[TILE];   // what the accumulators are scaled by, per row
  __shared__ int s_any;
  const Place at = find_place(tiles, g.batch, g.heads);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, h = at.head, b = at.sample, hk = h / a.group, s = at.segment;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int q0 = at.tile * TILE, q_end = min(q0 + TILE, a.q_len[s]);
  const QueryRows rows = query_rows(g, a, b, s);
  const bool rule = rule_masks(a) || a.slopes != nullptr, work = max(q0, rows.lo) < min(q_end, rows.hi);
  const int64_t row0 = (int64_t)b * a.Lq + a.q_off[s] + q0;
  const float slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
  const Piece<HD> piece;
  float2 o[4][2] = {};
  float ref[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, l[4] = {0.f, 0.f, 0.f, 0.f};
  if (work) {
    // rows that are padding are staged as zeros where they come last; in front (tail form) they are real memory, and not stored
    stage_rows<HD>(s_q, static_cast<const float*>(a.q) + row0 * a.ldq + (int64_t)h * g.hd, a.ldq, min(q_end, rows.hi) - q0, g.hd);
    if (rule) stage_times(own, g, a, b, s, q0 + rows.shift, min(q_end, rows.hi) - q0);
    for (int r = 0; r < 3; ++r) {
      const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
      for (int j0 = 0; j0 < n; j0 += TILE) {
        const int64_t key0 = (int64_t)b * g.L + g.off(r) + j0;
        __syncthreads();   // the tiles before have been read
        stage_rows<HD>(s_k, static_cast<const float*>(a.k) + key0 * a.ldk + (int64_t)hk * g.hd, a.ldk, n - j0, g.hd);
        stage_rows<HD>(s_v, static_cast<const float*>(a.v) + key0 * a.ldv + (int64_t)hk * g.hd, a.ldv, n - j0, g.hd);
        if (rule) stage_times(partner, g, a, b, r, j0, n - j0);
        __syncthreads();
        float x[4][4], unused[1][4];
        product_over_features<HD>(x, s_q, s_k, tx, ty);
        scores<false>(x, unused, a, slope2, own, partner, n - j0, rule, true, tx, ty);
        float scale[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float top = fmaxf(ref[i], row_max(fmaxf(fmaxf(x[i][0], x[i][1]), fmaxf(x[i][2], x[i][3]))));
          const float base = top == -INFINITY ? 0.f : top;   // no open key so far: weights of zero
          scale[i] = ptx::ex2(ref[i] - base);
          ref[i] = top;
          float t = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) t += x[i][j] = ptx::ex2(x[i][j] - base);
          l[i] = l[i] * scale[i] + row_sum(t);
        }
        put_weights(s_w, x, tx, ty);
        if (tx == 0) *reinterpret_cast<float4*>(s_row + 4 * ty) = make_float4(scale[0], scale[1], scale[2], scale[3]);
        __syncthreads();
        const float4 f = *reinterpret_cast<const float4*>(s_row + 4 * piece.rt);
        const float fs[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          o[i][0] = __fmul2_rn(o[i][0], make_float2(fs[i], fs[i]));
          o[i][1] = __fmul2_rn(o[i][1], make_float2(fs[i], fs[i]));
        }
        product_over_partners<HD>(o, s_w, s_v, piece);
      }
    }
    __syncthreads();
    join_groups<HD>(o, smem, piece);
  }
  if (tid == 0) s_any = 0;
  if (tx == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = q0 + 4 * ty + i;
      const bool real = row >= rows.lo && row < min(q_end, rows.hi) && l[i] != 0.f;
      s_row[4 * ty + i] = real ? 1.f / l[i] : 0.f;
      if (row < q_end && a.lse != nullptr) a.lse[((int64_t)b * g.heads + h) * a.Lq + a.q_off[s] + row] = real ? (ref[i] + log2f(l[i])) * LN2 : -INFINITY;
    }
  __syncthreads();
  bool ok = true;
  if (piece.group == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * piece.rt + i;
      const float inv = s_row[row];
      if (q0 + row < q_end) ok = put_row<HD>(static_cast<float*>(a.out) + (row0 + row) * a.ldo + (int64_t)h * g.hd, g.hd, o[i], inv, inv != 0.f, piece.ct) && ok;
    }
  if (!rule_masks(a)) return;
  // zero times NaN or Inf of a closed key: the tile's rows once more, pair by pair
  if (!ok) s_any = 1;
  __syncthreads();
  if (s_any != 0)
    for (int row = max(q0, rows.lo) + (tid >> 5); row < min(q_end, rows.hi); row += THREADS / 32) attend_row<float>(g, a, b, h, s, row);
}

template <int HD>
__global__ void __launch_bounds__(THREADS)
scored_dq_f32_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  using S = Sizes<HD>;
  extern __shared__ __align__(16) float smem[];
  float *s_q = smem, *s_g = s_q + S::ROWS, *s_k = s_g + S::ROWS, *s_v = s_k + S::ROWS, *s_w = s_v + S::ROWS;
  __shared__ Times own, partner;
  __shared__ float2 s_stats[TILE];
  __shared__ int s_any;
  const Place at = find_place(tiles, g.batch, g.heads);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, h = at.head, b = at.sample, hk = h / a.group, s = at.segment;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int q0 = at.tile * TILE, q_end = min(q0 + TILE, g.len(s)), n_q = valid_rows(g, b, s);
  const bool rule = rule_masks(a) || a.slopes != nullptr;
  const int64_t row0 = (int64_t)b * g.L + g.off(s) + q0, stat0 = ((int64_t)b * g.heads + h) * g.L + g.off(s) + q0;
  const float slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
  const Piece<HD> piece;
  float2 dq[4][2] = {};
  const int n_rows = min(q_end, n_q) - q0;   // of this tile
  bool ok = true;
  if (n_rows > 0) {
    stage_rows<HD>(s_q, static_cast<const float*>(a.q) + row0 * a.ldq + (int64_t)h * g.hd, a.ldq, n_rows, g.hd);
    stage_rows<HD>(s_g, static_cast<const float*>(a.dout) + row0 * a.lddo + (int64_t)h * g.hd, a.lddo, n_rows, g.hd);
    if (rule) stage_times(own, g, a, b, s, q0, n_rows);
    __syncthreads();
    if (tid < TILE) {   // (lse in base 2, delta); a row without an open key takes no part
      float2 st = make_float2(INFINITY, 0.f);
      if (tid < n_rows) {
        const float lse = a.lse[stat0 + tid];
        if (lse != -INFINITY) {
          st.x = lse * LOG2E;
          const float* out = static_cast<const float*>(a.out) + (row0 + tid) * a.ldo + (int64_t)h * g.hd;
          for (int f = 0; f < g.hd; ++f) st.y += out[f] * s_g[tid * S::PITCH + f];
        }
      }
      s_stats[tid] = st;
      ok = finite(st.y);
    }
    __syncthreads();
    float2 st[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) st[i] = s_stats[4 * ty + i];
    for (int r = 0; r < 3; ++r) {
      const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
      for (int j0 = 0; j0 < n; j0 += TILE) {
        const int64_t key0 = (int64_t)b * g.L + g.off(r) + j0;
        __syncthreads();
        stage_rows<HD>(s_k, static_cast<const float*>(a.k) + key0 * a.ldk + (int64_t)hk * g.hd, a.ldk, n - j0, g.hd);
        stage_rows<HD>(s_v, static_cast<const float*>(a.v) + key0 * a.ldv + (int64_t)hk * g.hd, a.ldv, n - j0, g.hd);
        if (rule) stage_times(partner, g, a, b, r, j0, n - j0);
        __syncthreads();
        float x[4][4], dp[4][4], bend[4][4];
        product_over_features<HD>(x, s_q, s_k, tx, ty);
        scores<true>(x, bend, a, slope2, own, partner, n - j0, rule, true, tx, ty);
        product_over_features<HD>(dp, s_g, s_v, tx, ty);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = ptx::ex2(x[i][j] - st[i].x) * (dp[i][j] - st[i].y) * bend[i][j];
        put_weights(s_w, x, tx, ty);
        __syncthreads();
        product_over_partners<HD>(dq, s_w, s_k, piece);
      }
    }
    __syncthreads();
    join_groups<HD>(dq, smem + 2 * S::ROWS, piece);
  }
  if (tid == 0) s_any = 0;
  if (tid < TILE && q0 + tid < q_end) a.row_stats[stat0 + tid] = n_rows > 0 ? s_stats[tid] : make_float2(INFINITY, 0.f);
  __syncthreads();
  if (piece.group == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * piece.rt + i;
      if (q0 + row < q_end)
        ok = put_row<HD>(static_cast<float*>(a.dq) + (row0 + row) * a.lddq + (int64_t)h * g.hd, g.hd, dq[i], a.scale, n_rows > 0 && s_stats[row].x != INFINITY, piece.ct) && ok;
    }
  if (!rule_masks(a)) return;
  if (!ok) s_any = 1;
  __syncthreads();
  if (s_any != 0)
    for (int row = q0 + (tid >> 5); row < q0 + n_rows; row += THREADS / 32) dq_row<float>(g, a, b, h, s, row);
}

template <int HD>
__global__ void __launch_bounds__(THREADS)
scored_dkv_f32_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  using S = Sizes<HD>;
  extern __shared__ __align__(16) float smem[];
  float *s_k = smem, *s_v = s_k + S::ROWS, *s_q = s_v + S::ROWS, *s_g = s_q + S::ROWS, *s_p = s_g + S::ROWS, *s_w = s_p + S::WEIGHTS;
  __shared__ Times own, partner;
  __shared__ float2 s_stats[TILE];
  __shared__ int s_any;
  const Place at = find_place(tiles, g.batch, a.kv_heads);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, hk = at.head, b = at.sample, r = at.segment;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int k0 = at.tile * TILE, k_end = min(k0 + TILE, g.len(r)), n_k = valid_rows(g, b, r), n_rows = min(k_end, n_k) - k0;
  const bool rule = rule_masks(a) || a.slopes != nullptr;
  const int64_t key0 = (int64_t)b * g.L + g.off(r) + k0;
  const Piece<HD> piece;
  float2 dk[4][2] = {}, dv[4][2] = {};
  if (n_rows > 0) {
    stage_rows<HD>(s_k, static_cast<const float*>(a.k) + key0 * a.ldk + (int64_t)hk * g.hd, a.ldk, n_rows, g.hd);
    stage_rows<HD>(s_v, static_cast<const float*>(a.v) + key0 * a.ldv + (int64_t)hk * g.hd, a.ldv, n_rows, g.hd);
    if (rule) stage_times(own, g, a, b, r, k0, n_rows);
    for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
      const float slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
      for (int s = 0; s < 3; ++s) {
        const int n = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, s) : 0;
        for (int i0 = 0; i0 < n; i0 += TILE) {
          const int64_t row0 = (int64_t)b * g.L + g.off(s) + i0;
          __syncthreads();
          stage_rows<HD>(s_q, static_cast<const float*>(a.q) + row0 * a.ldq + (int64_t)h * g.hd, a.ldq, n - i0, g.hd);
          stage_rows<HD>(s_g, static_cast<const float*>(a.dout) + row0 * a.lddo + (int64_t)h * g.hd, a.lddo, n - i0, g.hd);
          if (rule) stage_times(partner, g, a, b, s, i0, n - i0);
          if (tid < TILE) s_stats[tid] = tid < n - i0 ? a.row_stats[((int64_t)b * g.heads + h) * g.L + g.off(s) + i0 + tid] : make_float2(INFINITY, 0.f);
          __syncthreads();
          float x[4][4], dp[4][4], bend[4][4];
          product_over_features<HD>(x, s_k, s_q, tx, ty);
          scores<true>(x, bend, a, slope2, own, partner, n - i0, rule, false, tx, ty);
          product_over_features<HD>(dp, s_v, s_g, tx, ty);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 st = s_stats[tx + 16 * j];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              x[i][j] = ptx::ex2(x[i][j] - st.x);
              dp[i][j] = x[i][j] * (dp[i][j] - st.y) * bend[i][j];
            }
          }
          put_weights(s_p, x, tx, ty);
          put_weights(s_w, dp, tx, ty);
          __syncthreads();
          product_over_partners<HD>(dv, s_p, s_g, piece);
          product_over_partners<HD>(dk, s_w, s_q, piece);
        }
      }
    }
    __syncthreads();
    join_groups<HD>(dk, smem, piece);
    join_groups<HD>(dv, smem, piece);
  }
  if (tid == 0) s_any = 0;
  __syncthreads();
  bool ok = true;
  if (piece.group == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 4 * piece.rt + i;
      if (k0 + row < k_end) {
        ok = put_row<HD>(static_cast<float*>(a.dk) + (key0 + row) * a.lddk + (int64_t)hk * g.hd, g.hd, dk[i], a.scale, row < n_rows, piece.ct) && ok;
        ok = put_row<HD>(static_cast<float*>(a.dv) + (key0 + row) * a.lddv + (int64_t)hk * g.hd, g.hd, dv[i], 1.f, row < n_rows, piece.ct) && ok;
      }
    }
  if (!rule_masks(a)) return;
  if (!ok) s_any = 1;
  __syncthreads();
  if (s_any != 0)
    for (int row = k0 + (tid >> 5); row < k0 + n_rows; row += THREADS / 32) dkv_row<float>(g, a, b, hk, r, row);
}

enum Pass { FWD, DQ, DKV };
template <int HD> constexpr int smem_bytes(int pass) {
  using S = Sizes<HD>;
  return 4 * (pass == FWD ? 3 * S::ROWS + S::WEIGHTS : pass == DQ ? 4 * S::ROWS + S::WEIGHTS : 4 * S::ROWS + 2 * S::WEIGHTS);
}
// join_groups() puts (GROUPS - 1) * 64 * HD floats over the tiles (behind the first two for dq)
static_assert(4 * 7 * 64 * 8 <= smem_bytes<8>(FWD) && 4 * (2 * Sizes<8>::ROWS + 7 * 64 * 8) <= smem_bytes<8>(DQ), "room to join the groups");
static_assert(4 * 3 * 64 * 16 <= smem_bytes<16>(FWD) && 4 * (2 * Sizes<16>::ROWS + 3 * 64 * 16) <= smem_bytes<16>(DQ), "room to join the groups");

template <int PASS, int HD>
cudaError_t launch(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  const int heads = PASS == DKV ? a.kv_heads : g.heads;
  Tiles t = {};
  t.order = segment_order(g, PASS == DKV ? transposed(g.allowed) : g.allowed);
  const int64_t n = make_tiles(&t, PASS == FWD ? a.q_len : g.seg_len, TILE) * heads * g.batch;
  if (n > 0x7fffffffLL) return cudaErrorNotSupported;
  const auto kernel = PASS == FWD ? scored_fwd_f32_kernel<HD> : PASS == DQ ? scored_dq_f32_kernel<HD> : scored_dkv_f32_kernel<HD>;
  constexpr int bytes = smem_bytes<HD>(PASS);
  const cudaError_t e = sm_count_and_smem_once(reinterpret_cast<const void*>(kernel), bytes, nullptr);
  if (e != cudaSuccess) return e;
  return launch_overlapped(kernel, dim3((unsigned)n), dim3(THREADS), bytes, st, g, a, t);
}
template <int PASS>
cudaError_t launch_width(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  if (g.hd <= 8) return launch<PASS, 8>(g, a, st);
  if (g.hd <= 16) return launch<PASS, 16>(g, a, st);
  if (g.hd <= 32) return launch<PASS, 32>(g, a, st);
  return launch<PASS, 64>(g, a, st);
}

}  // namespace

cudaError_t launch_scored_fwd_f32(const Geometry& g, const ScoredArgs& a, cudaStream_t st) { return launch_width<FWD>(g, a, st); }

cudaError_t launch_scored_bwd_f32(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  const cudaError_t e = launch_width<DQ>(g, a, st);
  return e != cudaSuccess ? e : launch_width<DKV>(g, a, st);
}

}  // namespace gsit

// Scored attention in single precision, forward and backward, on the FMA pipe (head_dim <= 64).
//
// A CTA of 256 threads takes 64 rows (queries in the forward pass and for dq, keys for dk and dv), a warp eight of them, and walks the
// partners in tiles of 64, which cp.async brings into two buffers.  Two kinds of product, both from row-major tiles in shared memory
// whose rows are HD + 4 floats apart (any eight lanes that load 16 bytes of neighbouring rows then meet eight different bank groups):
//   over features  a lane owns rows 4 ty .. and partners tx + 16 j of the warp's 8 x 64 pairs: per four features 8 loads of 16 bytes feed
//                  32 packed multiply-adds, whose halves are the even and the odd features
//   over partners  the warp's 8 x HD result is owned in pieces of 4 x 4; where that takes fewer than 32 lanes the partners of a tile are
//                  dealt out to groups of lanes, whose sums shuffles bring together at the end
// Between the two the weights go through shared memory, partner-major; a warp reads only what its own lanes wrote, so that a tile costs
// one barrier.  With 2 HD (forward), 3 HD (dq) and 4 HD (dk, dv) multiply-adds a pair the FMA pipe is the bound: 128 a clock and SM.
// Measured: MIntRec's unmasked graph (8 samples of (30, 480, 230), half of the rows padding, 8 heads of 16, forward and gradients) 305 - 349 us by
// the lengths drawn, of which the multiply-adds are 54; 30% of the FMA pipe's time, half of the issue slots (sums over halves, bias, addresses), the rest shared
// memory's latency and the last of two and a fraction waves of CTAs.  One CTA an SM (more registers, nothing spilled) 350 us; weights
// exchanged by the whole CTA, which takes two more barriers a tile, 555 us.  Warps without a real row only fetch, and tiles without an open
// pair are passed over (341 -> 323 us; 86 x (5, 12, 131), causal, 335 -> 288).
#include "scored.cuh"

namespace gsit {
namespace {

constexpr int THREADS = 256, TILE = 64, WARP_ROWS = 8, WARP_WEIGHTS = TILE * WARP_ROWS;

template <int HD> struct Sizes {
  static constexpr int PITCH = HD + 4, ROWS = TILE * PITCH;   // floats of a staged tile of rows
  static constexpr int OWNERS = HD / 2, GROUPS = 32 / OWNERS; // of a warp's 8 x HD result, in pieces of 4 x 4
};

__device__ __forceinline__ void cp_row(float* dst, const float* src, bool real) {    // 16 bytes, zeros where the row is not real
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_float(float* dst, const float* src, bool real) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(real ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

// Rows [0, TILE) behind `src`, a [.., ld] matrix (this head's features), into shared memory; zeros from row `n` >= 1 on and from feature hd on.
template <int HD> __device__ __forceinline__ void stage_rows(float* dst, const float* src, int64_t ld, int n, int hd) {
  constexpr int P = Sizes<HD>::PITCH;
  if (hd == HD && ld % 4 == 0 && (reinterpret_cast<uintptr_t>(src) & 15u) == 0) {
    for (int i = threadIdx.x; i < TILE * HD / 4; i += THREADS) {
      const int r = i / (HD / 4), c = i % (HD / 4) * 4;
      cp_row(dst + r * P + c, src + (r < n ? r * ld + c : 0), r < n);
    }
  } else {
    for (int i = threadIdx.x; i < TILE * HD; i += THREADS) {
      const int r = i / HD, c = i % HD;
      const bool in = r < n && c < hd;
      cp_float(dst + r * P + c, src + (in ? r * ld + c : 0), in);
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

// The warp's weights: w[partner][row of the warp] = x
__device__ __forceinline__ void put_weights(float* w, const float (&x)[4][4], int tx, int ty) {
#pragma unroll
  for (int j = 0; j < 4; ++j) *reinterpret_cast<float4*>(w + (tx + 16 * j) * WARP_ROWS + 4 * (ty & 1)) = make_float4(x[0][j], x[1][j], x[2][j], x[3][j]);
}

// This lane's piece of a warp's 8 x HD result: rows 4 rt .., features 4 ct .., over partners group, group + GROUPS, ...
template <int HD> struct Piece {
  int rt, ct, group;
  __device__ __forceinline__ Piece() {
    const int lane = threadIdx.x & 31, t = lane % Sizes<HD>::OWNERS;
    ct = t % (HD / 4);
    rt = t / (HD / 4);
    group = lane / Sizes<HD>::OWNERS;
  }
};
template <int HD> __device__ __forceinline__ void product_over_partners(float2 (&o)[4][2], const float* w, const float* rows, const Piece<HD>& p, int partners) {
  w += p.group * WARP_ROWS + 4 * p.rt;
  rows += p.group * Sizes<HD>::PITCH + 4 * p.ct;
#pragma unroll 4
  for (int k = 0; k < min(TILE, partners); k += Sizes<HD>::GROUPS) {   // weights past the last partner are zero, and so are its rows
    const float4 a = *reinterpret_cast<const float4*>(w + k * WARP_ROWS), v = *reinterpret_cast<const float4*>(rows + k * Sizes<HD>::PITCH);
    const float f[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i][0] = __ffma2_rn(make_float2(f[i], f[i]), make_float2(v.x, v.y), o[i][0]);
      o[i][1] = __ffma2_rn(make_float2(f[i], f[i]), make_float2(v.z, v.w), o[i][1]);
    }
  }
}
// Adds the groups' results up; every group has the sums.
template <int HD> __device__ __forceinline__ void join_groups(float2 (&o)[4][2]) {
#pragma unroll
  for (int d = Sizes<HD>::OWNERS; d < 32; d *= 2)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        o[i][e].x += __shfl_xor_sync(0xffffffffu, o[i][e].x, d);
        o[i][e].y += __shfl_xor_sync(0xffffffffu, o[i][e].y, d);
      }
}
// Row `i` of the piece to memory (group 0); returns whether all of it is finite.
__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ bool put_row(float* dst, int hd, const float2 (&o)[2], float scale, bool real, int ct) {
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
    const bool in = i < n && pos0 + i >= 0;
    t.time[i] = in ? time_of(g, a, b, s, pos0 + i) : 0.f;
    t.limit[i] = in ? latest_seen(a, b, t.time[i]) : -INFINITY;
    t.doc[i] = in ? document_of(g, a, b, s, pos0 + i) : 0;
  }
}

// Dots -> scores in base 2, -inf where closed; d *= the cap's derivative.  queries_are_rows tells which side is which.
template <bool BEND>
__device__ __forceinline__ void scores(float (&x)[4][4], float (&d)[4][4], const ScoredArgs& a, float slope2, const Times& own, const Times& partner,
                                       int partners, bool queries_are_rows, int tx, int ty) {
  const float2 f = make_float2(a.inner, a.inner);
  const bool cap = a.softcap > 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      float2 y = __fmul2_rn(make_float2(x[i][j], x[i][j + 1]), f);
      if (cap) {
        const float2 t = make_float2(tanhf(y.x), tanhf(y.y));
        y = __fmul2_rn(t, make_float2(a.outer, a.outer));
        if (BEND) {
          d[i][j] *= 1.f - t.x * t.x;
          d[i][j + 1] *= 1.f - t.y * t.y;
        }
      }
      x[i][j] = y.x;
      x[i][j + 1] = y.y;
    }
  if (a.slopes != nullptr) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float t = partner.time[tx + 16 * j];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i][j] -= slope2 * fabsf(own.time[4 * ty + i] - t);
    }
  }
  if (rule_masks(a)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = tx + 16 * j;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * ty + i;
        const float limit = queries_are_rows ? own.limit[r] : partner.limit[c], key = queries_are_rows ? partner.time[c] : own.time[r];
        if (key > limit || own.doc[r] != partner.doc[c]) x[i][j] = -INFINITY;
      }
    }
  }
  if (partners < TILE) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (tx + 16 * j >= partners)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i][j] = -INFINITY;
  }
}

// Moments (or limits) and documents of a warp's rows [row, row + 8) of a segment, as far as they lie in [lo, hi).
__device__ __forceinline__ Range rows_range(const Geometry& g, const ScoredArgs& a, int b, int s, int row, int lo, int hi, int shift, bool limits) {
  const int i = row + (threadIdx.x & 7);
  Range r = NO_ROWS;
  if (i >= lo && i < hi) {
    const float t = time_of(g, a, b, s, i + shift);
    r.t_lo = r.t_hi = ordered(limits ? latest_seen(a, b, t) : t);
    r.d_lo = r.d_hi = document_of(g, a, b, s, i + shift);
  }
  __syncwarp();
  return warp_range(r.t_lo, r.t_hi, r.d_lo, r.d_hi);
}

// CTAs an SM that registers are kept for: what a warp waits for (shared memory, exponentials) another one's products hide.
template <int HD> constexpr int MIN_CTAS = HD <= 32 ? 2 : 1;

template <int HD>
__global__ void __launch_bounds__(THREADS, MIN_CTAS<HD>)
scored_fwd_f32_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  using S = Sizes<HD>;
  extern __shared__ __align__(16) float smem[];
  float *s_q = smem, *s_k = s_q + S::ROWS, *s_v = s_k + 2 * S::ROWS;
  __shared__ Times own, partner[2];
  __shared__ int s_any;
  const Place at = find_place(tiles, g.batch, g.heads);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, h = at.head, b = at.sample, hk = h / a.group, s = at.segment;
  float* const s_w = s_v + 2 * S::ROWS + (tid >> 5) * WARP_WEIGHTS;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  const int q0 = at.tile * TILE, q_end = min(q0 + TILE, a.q_len[s]);
  const QueryRows rows = query_rows(g, a, b, s);
  const bool rule = rule_masks(a) || a.slopes != nullptr;
  const int64_t row0 = (int64_t)b * a.Lq + a.q_off[s] + q0, sample0 = (int64_t)b * g.L;
  const float slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
  const Piece<HD> piece;
  float2 o[4][2] = {};
  float ref[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, l[4] = {0.f, 0.f, 0.f, 0.f};   // l: this lane's part of the sums
  Walk next = {};
#pragma unroll
  for (int r = 0; r < 3; ++r) next.n[r] = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
  if (max(q0, rows.lo) >= min(q_end, rows.hi)) next.seg = 3;
  next.settle();
  auto stage = [&](const Walk& w, int buf) {
    const int64_t key0 = sample0 + g.off(w.seg) + w.pos;
    stage_rows<HD>(s_k + buf * S::ROWS, static_cast<const float*>(a.k) + key0 * a.ldk + (int64_t)hk * g.hd, a.ldk, w.left(), g.hd);
    stage_rows<HD>(s_v + buf * S::ROWS, static_cast<const float*>(a.v) + key0 * a.ldv + (int64_t)hk * g.hd, a.ldv, w.left(), g.hd);
    cp_commit();
    if (rule) stage_times(partner[buf], g, a, b, w.seg, w.pos, w.left());
  };
  if (!next.over()) {
    // rows that are padding are staged as zeros where they come last; in front (tail form) they are real memory, and not stored
    stage_rows<HD>(s_q, static_cast<const float*>(a.q) + row0 * a.ldq + (int64_t)h * g.hd, a.ldq, min(q_end, rows.hi) - q0, g.hd);
    if (rule) stage_times(own, g, a, b, s, q0 + rows.shift, min(q_end, rows.hi) - q0);
    stage(next, 0);
  }
  const int w0 = q0 + (tid >> 5) * WARP_ROWS;   // the warp's rows; one without a real row only fetches, and tiles without an open pair are passed
  const bool working = w0 < min(q_end, rows.hi) && w0 + WARP_ROWS > rows.lo, masks = rule_masks(a);
  const Range mine = masks ? rows_range(g, a, b, s, w0, rows.lo, min(q_end, rows.hi), rows.shift, true) : NO_ROWS;
  for (int buf = 0; !next.over(); buf ^= 1) {
    const int rem = next.left();
    cp_wait();
    __syncthreads();   // the tile is there, and nobody reads the other buffer any more
    next.pos += TILE;
    next.settle();
    if (!next.over()) stage(next, buf ^ 1);
    if (!working || (masks && openness(mine, block_range(partner[buf].time, partner[buf].doc, 0, rem, tid & 31)) == SHUT)) continue;
    float x[4][4], unused[4][4], top[4];
    product_over_features<HD>(x, s_q, s_k + buf * S::ROWS, tx, ty);
    scores<false>(x, unused, a, slope2, own, partner[buf], rem, true, tx, ty);
    // a row's reference follows its maximum when a score exceeds it by more than 8 (weights stay below 256)
    bool outgrown = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      top[i] = fmaxf(fmaxf(x[i][0], x[i][1]), fmaxf(x[i][2], x[i][3]));
      outgrown = outgrown || top[i] > ref[i] + 8.f;
    }
    if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float t = top[i], f = 1.f;
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));   // over the 16 lanes that share the row
        if (t > ref[i] + 8.f) {
          f = ptx::ex2(ref[i] - t);
          l[i] *= f;
          ref[i] = t;
        }
        f = __shfl_sync(0xffffffffu, f, 16 * piece.rt);
        o[i][0] = __fmul2_rn(o[i][0], make_float2(f, f));
        o[i][1] = __fmul2_rn(o[i][1], make_float2(f, f));
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float base = ref[i] == -INFINITY ? 0.f : ref[i];   // no open key so far: weights of zero
#pragma unroll
      for (int j = 0; j < 4; ++j) l[i] += x[i][j] = ptx::ex2(x[i][j] - base);
    }
    put_weights(s_w, x, tx, ty);
    __syncwarp();
    product_over_partners<HD>(o, s_w, s_v + buf * S::ROWS, piece, rem);
    __syncwarp();
  }
  ptx::grid_dep_launch();   // only now: see scored_tile.cuh
  join_groups<HD>(o);
  if (tid == 0) s_any = 0;
  float inv[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
    const int row = q0 + 4 * ty + i;
    const bool real = row >= rows.lo && row < min(q_end, rows.hi) && l[i] != 0.f;
    if (tx == 0 && row < q_end && a.lse != nullptr) a.lse[((int64_t)b * g.heads + h) * a.Lq + a.q_off[s] + row] = real ? (ref[i] + log2f(l[i])) * LN2 : -INFINITY;
    inv[i] = __shfl_sync(0xffffffffu, real ? 1.f / l[i] : 0.f, 16 * piece.rt);
  }
  bool ok = true;
  if (piece.group == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (tid >> 5) * WARP_ROWS + 4 * piece.rt + i;
      if (q0 + row < q_end) ok = put_row(static_cast<float*>(a.out) + (row0 + row) * a.ldo + (int64_t)h * g.hd, g.hd, o[i], inv[i], inv[i] != 0.f, piece.ct) && ok;
    }
  if (!rule_masks(a)) return;
  // zero times NaN or Inf of a closed key: the tile's rows once more, pair by pair
  __syncthreads();
  if (!ok) s_any = 1;
  __syncthreads();
  if (s_any != 0)
    for (int row = max(q0, rows.lo) + (tid >> 5); row < min(q_end, rows.hi); row += THREADS / 32) attend_row<float>(g, a, b, h, s, row);
}

template <int HD>
__global__ void __launch_bounds__(THREADS, MIN_CTAS<HD>)
scored_dq_f32_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  using S = Sizes<HD>;
  extern __shared__ __align__(16) float smem[];
  float *s_q = smem, *s_g = s_q + S::ROWS, *s_k = s_g + S::ROWS, *s_v = s_k + 2 * S::ROWS;
  __shared__ Times own, partner[2];
  __shared__ float2 s_stats[TILE];
  __shared__ int s_any;
  const Place at = find_place(tiles, g.batch, g.heads);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, h = at.head, b = at.sample, hk = h / a.group, s = at.segment;
  float* const s_w = s_v + 2 * S::ROWS + (tid >> 5) * WARP_WEIGHTS;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  const int q0 = at.tile * TILE, q_end = min(q0 + TILE, g.len(s)), n_rows = min(q_end, valid_rows(g, b, s)) - q0;   // real rows of this tile
  const bool rule = rule_masks(a) || a.slopes != nullptr;
  const int64_t sample0 = (int64_t)b * g.L, row0 = sample0 + g.off(s) + q0, stat0 = ((int64_t)b * g.heads + h) * g.L + g.off(s) + q0;
  const float slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
  const Piece<HD> piece;
  float2 dq[4][2] = {};
  Walk next = {};
#pragma unroll
  for (int r = 0; r < 3; ++r) next.n[r] = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
  if (n_rows <= 0) next.seg = 3;
  next.settle();
  auto stage = [&](const Walk& w, int buf) {
    const int64_t key0 = sample0 + g.off(w.seg) + w.pos;
    stage_rows<HD>(s_k + buf * S::ROWS, static_cast<const float*>(a.k) + key0 * a.ldk + (int64_t)hk * g.hd, a.ldk, w.left(), g.hd);
    stage_rows<HD>(s_v + buf * S::ROWS, static_cast<const float*>(a.v) + key0 * a.ldv + (int64_t)hk * g.hd, a.ldv, w.left(), g.hd);
    cp_commit();
    if (rule) stage_times(partner[buf], g, a, b, w.seg, w.pos, w.left());
  };
  if (!next.over()) {
    stage_rows<HD>(s_q, static_cast<const float*>(a.q) + row0 * a.ldq + (int64_t)h * g.hd, a.ldq, n_rows, g.hd);
    stage_rows<HD>(s_g, static_cast<const float*>(a.dout) + row0 * a.lddo + (int64_t)h * g.hd, a.lddo, n_rows, g.hd);
    if (rule) stage_times(own, g, a, b, s, q0, n_rows);
    stage(next, 0);
  }
  bool ok = true;
  {   // (lse in base 2, delta) of the warp's rows, four lanes to a row; a row without an open key takes no part
    const int row = tid >> 2, part = tid & 3;
    const float lse = row < n_rows ? a.lse[stat0 + row] : -INFINITY;
    float delta = 0.f;
    if (lse != -INFINITY) {
      const float *out = static_cast<const float*>(a.out) + (row0 + row) * a.ldo + (int64_t)h * g.hd, *grad = static_cast<const float*>(a.dout) + (row0 + row) * a.lddo + (int64_t)h * g.hd;
#pragma unroll 4
      for (int f = part; f < g.hd; f += 4) delta += out[f] * grad[f];
    }
    __syncwarp();
    delta += __shfl_xor_sync(0xffffffffu, delta, 1);
    delta += __shfl_xor_sync(0xffffffffu, delta, 2);
    ok = finite(delta);
    if (part == 0) {
      s_stats[row] = make_float2(lse == -INFINITY ? INFINITY : lse * LOG2E, delta);
      if (q0 + row < q_end) a.row_stats[stat0 + row] = s_stats[row];
    }
    __syncwarp();
  }
  float2 st[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) st[i] = s_stats[4 * ty + i];
  const int w0 = (tid >> 5) * WARP_ROWS;
  const bool working = w0 < n_rows, masks = rule_masks(a);
  const Range mine = masks ? rows_range(g, a, b, s, q0 + w0, 0, q0 + n_rows, 0, true) : NO_ROWS;
  for (int buf = 0; !next.over(); buf ^= 1) {
    const int rem = next.left();
    cp_wait();
    __syncthreads();   // the tile is there, and nobody reads the other buffer any more
    next.pos += TILE;
    next.settle();
    if (!next.over()) stage(next, buf ^ 1);
    if (!working || (masks && openness(mine, block_range(partner[buf].time, partner[buf].doc, 0, rem, tid & 31)) == SHUT)) continue;
    float x[4][4], d[4][4];
    product_over_features<HD>(d, s_g, s_v + buf * S::ROWS, tx, ty);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) d[i][j] -= st[i].y;
    product_over_features<HD>(x, s_q, s_k + buf * S::ROWS, tx, ty);
    scores<true>(x, d, a, slope2, own, partner[buf], rem, true, tx, ty);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i][j] = ptx::ex2(x[i][j] - st[i].x) * d[i][j];
    put_weights(s_w, x, tx, ty);
    __syncwarp();
    product_over_partners<HD>(dq, s_w, s_k + buf * S::ROWS, piece, rem);
    __syncwarp();
  }
  ptx::grid_dep_launch();   // only now: see scored_tile.cuh
  join_groups<HD>(dq);
  if (tid == 0) s_any = 0;
  if (piece.group == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (tid >> 5) * WARP_ROWS + 4 * piece.rt + i;
      if (q0 + row < q_end)
        ok = put_row(static_cast<float*>(a.dq) + (row0 + row) * a.lddq + (int64_t)h * g.hd, g.hd, dq[i], a.scale, s_stats[row].x != INFINITY, piece.ct) && ok;
    }
  if (!rule_masks(a)) return;
  __syncthreads();
  if (!ok) s_any = 1;
  __syncthreads();
  if (s_any != 0)
    for (int row = q0 + (tid >> 5); row < q0 + n_rows; row += THREADS / 32) dq_row<float>(g, a, b, h, s, row);
}

template <int HD>
__global__ void __launch_bounds__(THREADS, MIN_CTAS<HD>)
scored_dkv_f32_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  using S = Sizes<HD>;
  extern __shared__ __align__(16) float smem[];
  float *s_k = smem, *s_v = s_k + S::ROWS, *s_q = s_v + S::ROWS, *s_g = s_q + 2 * S::ROWS;
  __shared__ Times own, partner[2];
  __shared__ float2 s_stats[2][TILE];
  __shared__ int s_any;
  const Place at = find_place(tiles, g.batch, a.kv_heads);
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, hk = at.head, b = at.sample, r = at.segment;
  float* const s_w = s_g + 2 * S::ROWS + (tid >> 5) * WARP_WEIGHTS;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  const int k0 = at.tile * TILE, k_end = min(k0 + TILE, g.len(r)), n_rows = min(k_end, valid_rows(g, b, r)) - k0;
  const bool rule = rule_masks(a) || a.slopes != nullptr;
  const int64_t sample0 = (int64_t)b * g.L, key0 = sample0 + g.off(r) + k0;
  const Piece<HD> piece;
  float2 dk[4][2] = {}, dv[4][2] = {};
  Walk next = {};
#pragma unroll
  for (int s = 0; s < 3; ++s) next.n[s] = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, s) : 0;
  if (n_rows <= 0) next.seg = 3;
  next.settle();
  const Walk first = next;
  int h = hk * a.group;   // the head whose queries come next
  const int last_head = h + a.group - 1;
  auto stage = [&](const Walk& w, int head, int buf) {
    const int64_t at_row = sample0 + g.off(w.seg) + w.pos;
    stage_rows<HD>(s_q + buf * S::ROWS, static_cast<const float*>(a.q) + at_row * a.ldq + (int64_t)head * g.hd, a.ldq, w.left(), g.hd);
    stage_rows<HD>(s_g + buf * S::ROWS, static_cast<const float*>(a.dout) + at_row * a.lddo + (int64_t)head * g.hd, a.lddo, w.left(), g.hd);
    cp_commit();
    if (rule) stage_times(partner[buf], g, a, b, w.seg, w.pos, w.left());
    if (tid < TILE)   // no weight for rows past the last
      s_stats[buf][tid] = tid < w.left() ? a.row_stats[((int64_t)b * g.heads + head) * g.L + g.off(w.seg) + w.pos + tid] : make_float2(INFINITY, 0.f);
  };
  if (!next.over()) {
    stage_rows<HD>(s_k, static_cast<const float*>(a.k) + key0 * a.ldk + (int64_t)hk * g.hd, a.ldk, n_rows, g.hd);
    stage_rows<HD>(s_v, static_cast<const float*>(a.v) + key0 * a.ldv + (int64_t)hk * g.hd, a.ldv, n_rows, g.hd);
    if (rule) stage_times(own, g, a, b, r, k0, n_rows);
    stage(next, h, 0);
  }
  const int w0 = (tid >> 5) * WARP_ROWS;
  const bool working = w0 < n_rows, masks = rule_masks(a);
  const Range mine = masks ? rows_range(g, a, b, r, k0 + w0, 0, k0 + n_rows, 0, false) : NO_ROWS;
  for (int buf = 0; !next.over(); buf ^= 1) {
    const int rem = next.left();
    const float slope2 = a.slopes != nullptr ? a.slopes[h] * LOG2E : 0.f;
    cp_wait();
    __syncthreads();   // the tile is there, and nobody reads the other buffer any more
    next.pos += TILE;
    next.settle();
    if (next.over() && h < last_head) {
      next = first;
      ++h;
    }
    if (!next.over()) stage(next, h, buf ^ 1);
    if (!working || (masks && openness(block_range(partner[buf].limit, partner[buf].doc, 0, rem, tid & 31), mine) == SHUT)) continue;
    float x[4][4], d[4][4];
    product_over_features<HD>(d, s_v, s_g + buf * S::ROWS, tx, ty);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float delta = s_stats[buf][tx + 16 * j].y;
#pragma unroll
      for (int i = 0; i < 4; ++i) d[i][j] -= delta;
    }
    product_over_features<HD>(x, s_k, s_q + buf * S::ROWS, tx, ty);
    scores<true>(x, d, a, slope2, own, partner[buf], rem, false, tx, ty);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float lse2 = s_stats[buf][tx + 16 * j].x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i][j] = ptx::ex2(x[i][j] - lse2);
        d[i][j] *= x[i][j];
      }
    }
    put_weights(s_w, x, tx, ty);
    __syncwarp();
    product_over_partners<HD>(dv, s_w, s_g + buf * S::ROWS, piece, rem);
    __syncwarp();
    put_weights(s_w, d, tx, ty);
    __syncwarp();
    product_over_partners<HD>(dk, s_w, s_q + buf * S::ROWS, piece, rem);
    __syncwarp();
  }
  ptx::grid_dep_launch();   // only now: see scored_tile.cuh
  join_groups<HD>(dk);
  join_groups<HD>(dv);
  if (tid == 0) s_any = 0;
  bool ok = true;
  if (piece.group == 0)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (tid >> 5) * WARP_ROWS + 4 * piece.rt + i;
      if (k0 + row < k_end) {
        ok = put_row(static_cast<float*>(a.dk) + (key0 + row) * a.lddk + (int64_t)hk * g.hd, g.hd, dk[i], a.scale, row < n_rows, piece.ct) && ok;
        ok = put_row(static_cast<float*>(a.dv) + (key0 + row) * a.lddv + (int64_t)hk * g.hd, g.hd, dv[i], 1.f, row < n_rows, piece.ct) && ok;
      }
    }
  if (!rule_masks(a)) return;
  __syncthreads();
  if (!ok) s_any = 1;
  __syncthreads();
  if (s_any != 0)
    for (int row = k0 + (tid >> 5); row < k0 + n_rows; row += THREADS / 32) dkv_row<float>(g, a, b, hk, r, row);
}

enum Pass { FWD, DQ, DKV };
template <int HD> constexpr int smem_bytes(int pass) { return 4 * ((pass == FWD ? 5 : 6) * Sizes<HD>::ROWS + THREADS / 32 * WARP_WEIGHTS); }

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

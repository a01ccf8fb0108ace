// Scored attention, backward, bf16, on mma.sync (see scored_tile.cuh).
//
// With P = exp(x - lse), dP = dO V^T and delta = rowsum(dO o O):  dX = P o (dP - delta),  dS = dX o (derivative of the cap),
// dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.  Two kernels, each of which owns the rows it adds up and recomputes the scores:
// no atomics, no partial sums in memory, the same bits every time.
//   dq    a warp owns 16 * MT query rows and walks keys (as the forward kernel does); it also writes each row's (lse in base 2, delta), delta as
//         the sum over P dP that it makes on its way
//   dkv   a warp owns 16 * MT key rows and walks the queries of all heads that share them, products transposed: x^T = K Q^T
// delta enters as the start of the accumulators of dP.
// What is rounded to fewer bits: P and dS, to bf16, as operands of the second products (any product on these units rounds its operands; sums are
// held in 32 bits), which makes as large an error as rounding the gradients does: together 2^-8.7 of their norm, where the latter alone is 2^-9.2.
// Two more errors of that size are taken out, in dq:
//   the O that comes in was rounded, so dO . O is not the sum over P dP, and where rows see a handful of keys dq and dk had 2^-8.1 to 2^-8.6 from
//   that.  With r = sum over P (dP - dO . O), summed up in 32 bits, dq takes off r times sum over P o bend K (`along`, one product more)
//   and dk and dv get delta = dO . O + r.
//   heads of 8: the terms of dq cancel (2^-8.65 of its norm with one rounded operand), so dS goes into the product as two bf16 terms.
// Gradients of MOSEI's step 187 us, 169 without either (dq 108 for 89 under the profiler); 64 x (39, 55, 400), 8 heads of 16 65 us for 63.
// What bounds them is what bounds the forward kernel, with more instructions to a pair of scores: 71 M (dq) and 63 M (dk and dv) for 58 M.
#include "scored_tile.cuh"

namespace gsit {
namespace {

constexpr int W = 4;                      // warps of a CTA
constexpr int MT = 1, OWN = 16 * MT * W;  // row tiles of a warp (two: dq 107 us for 104, dk and dv 119 for 109), rows of a CTA

template <int HD, int CTAS, bool CAP, bool BIAS, bool MASK>
__global__ void __launch_bounds__(32 * W, CTAS)
scored_dq_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  constexpr int KC = CHUNK_ROWS<HD>, CH = HD / 8, NT = HD == 8 || (HD == 16 && CTAS < 7) ? 4 : 2;
  constexpr bool REST = HD == 8;   // dS as two terms
  constexpr bool TIMES = BIAS || MASK;
  __shared__ __align__(128) uint8_t s_k[2][KC * HD * 2], s_v[2][KC * HD * 2];
  __shared__ __align__(16) float s_time[2][TIMES ? KC : 4];
  __shared__ int s_doc[2][MASK ? KC : 1];
  const int tid = threadIdx.x, warp = ptx::uniform(tid >> 5), lane = tid & 31;
  const Place at = find_place(tiles, g.batch, g.heads);
  const int b = at.sample, s = at.segment, h = at.head, hk = h / a.group;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();

  const int q0 = at.tile * OWN, n_q = valid_rows(g, b, s), q_end = min(q0 + OWN, g.len(s));
  Walk next = {};
#pragma unroll
  for (int r = 0; r < 3; ++r) next.n[r] = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
  if (q0 >= n_q) next.seg = 3;
  next.settle();

  const int64_t sample0 = (int64_t)b * g.L;
  const bf16* const k0 = static_cast<const bf16*>(a.k) + sample0 * a.ldk + (int64_t)hk * HD;
  const bf16* const v0 = static_cast<const bf16*>(a.v) + sample0 * a.ldv + (int64_t)hk * HD;
  auto stage = [&](const Walk& w, int buf) {
    const int row0 = g.off(w.seg) + w.pos, rem = w.left();
    stage_pair<HD, KC, W>(smem_u32(s_k[buf]), smem_u32(s_v[buf]), k0 + (int64_t)row0 * a.ldk, a.ldk, v0 + (int64_t)row0 * a.ldv, a.ldv, rem, tid);
    if (TIMES)
      for (int i = tid; i < min(KC, (rem + BLOCK - 1) / BLOCK * BLOCK); i += 32 * W) {
        s_time[buf][i] = i >= rem ? 0.f : a.times != nullptr ? a.times[sample0 + row0 + i] : (float)(w.pos + i);
        if (MASK) s_doc[buf][i] = i < rem && a.documents != nullptr ? a.documents[sample0 + row0 + i] : 0;
      }
  };
  if (!next.over()) stage(next, 0);

  // ---- the warp's rows: q, dO, statistics ----
  const int w0 = q0 + warp * 16 * MT;
  const int64_t row0 = sample0 + g.off(s), stat0 = ((int64_t)b * g.heads + h) * g.L + g.off(s);
  uint32_t qf[MT][(HD + 15) / 16][4], gf[MT][(HD + 15) / 16][4];
  float own_time[MT][2], limit[MT][2], lse2[MT][2], delta[MT][2];
  int own_doc[MT][2];
  bool real[MT][2];
  Range mine = NO_ROWS;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const bf16 *pq[2], *pg[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = w0 + 16 * m + 8 * i + (lane >> 2);
      const float lse = row < min(q_end, n_q) ? a.lse[stat0 + row] : -INFINITY;
      real[m][i] = lse != -INFINITY;   // a row without an open key has no gradient
      pq[i] = real[m][i] ? static_cast<const bf16*>(a.q) + (row0 + row) * a.ldq + (int64_t)h * HD : nullptr;
      pg[i] = real[m][i] ? static_cast<const bf16*>(a.dout) + (row0 + row) * a.lddo + (int64_t)h * HD : nullptr;
      lse2[m][i] = real[m][i] ? lse * LOG2E : INFINITY;
      own_time[m][i] = 0.f;
      limit[m][i] = INFINITY;
      own_doc[m][i] = 0;
      if (TIMES && real[m][i]) own_time[m][i] = time_of(g, a, b, s, row);
      if (MASK && real[m][i]) {
        limit[m][i] = latest_seen(a, b, own_time[m][i]);
        own_doc[m][i] = document_of(g, a, b, s, row);
        mine = {min(mine.t_lo, ordered(limit[m][i])), max(mine.t_hi, ordered(limit[m][i])), min(mine.d_lo, own_doc[m][i]), max(mine.d_hi, own_doc[m][i])};
      }
    }
    own_rows<HD>(pq[0], pq[1], lane, qf[m]);
    own_rows<HD>(pg[0], pg[1], lane, gf[m]);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = w0 + 16 * m + 8 * i + (lane >> 2);
      float d = 0.f;
      if (real[m][i]) {   // the same features of O as this lane holds of dO
        const bf16* po = static_cast<const bf16*>(a.out) + (row0 + row) * a.ldo + (int64_t)h * HD + 2 * (lane & 3);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          float ox, oy, gx, gy;
          unpack_bf16(*reinterpret_cast<const uint32_t*>(po + 8 * c), ox, oy);
          unpack_bf16(gf[m][c / 2][2 * (c & 1) + i], gx, gy);
          d += ox * gx + oy * gy;
        }
      }
      d += __shfl_xor_sync(0xffffffffu, d, 1);
      d += __shfl_xor_sync(0xffffffffu, d, 2);
      delta[m][i] = d;
    }
  }
  if (MASK) mine = warp_range(mine.t_lo, mine.t_hi, mine.d_lo, mine.d_hi);
  const bool working = w0 < min(q_end, n_q);
  const float slope2 = BIAS ? a.slopes[h] * LOG2E : 0.f;

  const LaneAt<HD> at_kn = lane_as_n<HD>(smem_u32(s_k[0]), lane), at_kk = lane_as_k<HD>(smem_u32(s_k[0]), lane);
  const LaneAt<HD> at_v = lane_as_n<HD>(smem_u32(s_v[0]), lane);

  float dq[MT][CH][4], along[MT][CH][4];
  float2 missed[MT][2] = {};   // sums over P (dP - dO . O)
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) dq[m][c][e] = along[m][c][e] = 0.f;

  auto step = [&](auto some_tag, int buf, int j, int rem) {
    constexpr bool SOME_SHUT = decltype(some_tag)::value;
    float x[MT][NT][4], dp[MT][NT][4];
    const uint32_t from = (buf * KC + j) * HD * 2;
    product_over_features<HD, MT, NT>(x, qf, at_kn, from, from_zero);
    product_over_features<HD, MT, NT>(dp, gf, at_v, from, [&](int m, int, float (&z)[4]) {
      z[0] = z[1] = -delta[m][0];
      z[2] = z[3] = -delta[m][1];
    });
    uint32_t w[MT][NT][2], wb[MT][NT][2], rest[MT][REST ? NT : 2][2];
    in_form<CAP, MT, NT>(x, a, [&](auto near) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float2 times = make_float2(0.f, 0.f);
          if constexpr (BIAS) times = *reinterpret_cast<const float2*>(&s_time[buf][j + 8 * n + 2 * (lane & 3)]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float2 d = make_float2(dp[m][n][2 * i], dp[m][n][2 * i + 1]);
            float2 bend, y = score_pair<CAP, true, decltype(near)::value != 0>(make_float2(x[m][n][2 * i], x[m][n][2 * i + 1]), make_float2(lse2[m][i], lse2[m][i]), bend, a);
            if constexpr (BIAS) y = bias_pair(y, times, own_time[m][i], slope2);
            if constexpr (SOME_SHUT) {
              auto shut = [&](int col) { return col >= rem || (MASK && (s_time[buf][col] > limit[m][i] || s_doc[buf][col] != own_doc[m][i])); };
              const int col = j + 8 * n + 2 * (lane & 3);
              y = make_float2(shut(col) ? -INFINITY : y.x, shut(col + 1) ? -INFINITY : y.y);
            }
            const float2 p = make_float2(ptx::ex2(y.x), ptx::ex2(y.y)), pb = times_bend<CAP>(p, bend), ds = __fmul2_rn(pb, d);
            missed[m][i] = CAP ? __ffma2_rn(p, d, missed[m][i]) : __fadd2_rn(missed[m][i], ds);
            w[m][n][i] = ptx::pack_bf16(ds.x, ds.y);
            if constexpr (REST) rest[m][n][i] = pack_rest(ds, w[m][n][i]);
            wb[m][n][i] = ptx::pack_bf16(pb.x, pb.y);
          }
        }
    });
    __syncwarp();   // lanes may have taken different ways; matrix instructions need the whole warp
    for_partner_rows<HD, NT>(at_kk, from, [&](int first, int c, const uint32_t (&f)[4]) {
      add_product<HD>(dq, w, first, c, f);
      if constexpr (REST) add_product<HD>(dq, rest, first, c, f);
      add_product<HD>(along, wb, first, c, f);
    });
  };

  for (int buf = 0; !next.over(); buf ^= 1) {
    const int rem = min(KC, next.left());
    cp_wait();
    __syncthreads();   // the chunk is there, and nobody reads the other buffer any more
    next.pos += KC;
    next.settle();
    if (!next.over()) stage(next, buf ^ 1);
    if (!working) continue;
    int j = 0;
    if constexpr (!MASK) {
#pragma unroll 1
      for (; j + 8 * NT <= rem; j += 8 * NT) step(IntTag<0>{}, buf, j, rem);
      if (j < rem) step(IntTag<1>{}, buf, j, rem);
    } else {
#pragma unroll 1
      while (j < rem) {
        const Openness open = openness(mine, block_range(s_time[buf], s_doc[buf], j, rem, lane));
        const int end = min(j + BLOCK, rem);
        if (open == ALL && end - j == BLOCK)
#pragma unroll 1
          for (; j < end; j += 8 * NT) step(IntTag<0>{}, buf, j, rem);
        else if (open != SHUT)
#pragma unroll 1
          for (; j < end; j += 8 * NT) step(IntTag<1>{}, buf, j, rem);
        j = end;
      }
    }
  }

  ptx::grid_dep_launch();   // see scored_tile.cuh
  bool broken = false;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = w0 + 16 * m + 8 * i + (lane >> 2);
      float more = missed[m][i].x + missed[m][i].y;
      more += __shfl_xor_sync(0xffffffffu, more, 1);
      more += __shfl_xor_sync(0xffffffffu, more, 2);
      if (!real[m][i]) more = 0.f;
      if (row < q_end && (lane & 3) == 0) a.row_stats[stat0 + row] = make_float2(lse2[m][i], delta[m][i] + more);
#pragma unroll
      for (int q = 0; q < CH; ++q)
#pragma unroll
        for (int e = 0; e < 2; ++e) dq[m][q][2 * i + e] -= more * along[m][q][2 * i + e];
      if (MASK && real[m][i]) {
        broken = broken || !finite(delta[m][i] + more);
#pragma unroll
        for (int q = 0; q < CH; ++q) broken = broken || !finite(dq[m][q][2 * i]) || !finite(dq[m][q][2 * i + 1]);
      }
      if (row < q_end) {
        bf16* dst = static_cast<bf16*>(a.dq) + (row0 + row) * a.lddq + (int64_t)h * HD + 2 * (lane & 3);
#pragma unroll
        for (int q = 0; q < CH; ++q)
          *reinterpret_cast<uint32_t*>(dst + 8 * q) = real[m][i] ? ptx::pack_bf16(dq[m][q][2 * i] * a.scale, dq[m][q][2 * i + 1] * a.scale) : 0u;
      }
    }
  if (MASK && __any_sync(0xffffffffu, broken))
    for (int row = w0; row < min(w0 + 16 * MT, min(q_end, n_q)); ++row) dq_row<bf16>(g, a, b, h, s, row);
}

template <int HD, int CTAS, bool CAP, bool BIAS, bool MASK>
__global__ void __launch_bounds__(32 * W, CTAS)
scored_dkv_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  constexpr int QC = CHUNK_ROWS<HD>, CH = HD / 8, NT = HD <= 16 ? 4 : 2;
  constexpr bool TIMES = BIAS || MASK;
  __shared__ __align__(128) uint8_t s_q[2][QC * HD * 2], s_g[2][QC * HD * 2];
  __shared__ __align__(16) float2 s_stats[2][QC];
  __shared__ __align__(16) float s_time[2][TIMES ? QC : 4], s_limit[2][MASK ? QC : 4];
  __shared__ int s_doc[2][MASK ? QC : 1];
  const int tid = threadIdx.x, warp = ptx::uniform(tid >> 5), lane = tid & 31;
  const Place at = find_place(tiles, g.batch, a.kv_heads);
  const int b = at.sample, r = at.segment, hk = at.head;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();

  const int k0 = at.tile * OWN, n_k = valid_rows(g, b, r), k_end = min(k0 + OWN, g.len(r));
  Walk next = {};
#pragma unroll
  for (int s = 0; s < 3; ++s) next.n[s] = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, s) : 0;
  if (k0 >= n_k) next.seg = 3;
  next.settle();
  const Walk first = next;
  int h = hk * a.group;   // the head whose queries come next
  const int last_head = h + a.group - 1;

  const int64_t sample0 = (int64_t)b * g.L;
  auto stage = [&](const Walk& w, int head, int buf) {
    const int row0 = g.off(w.seg) + w.pos, rem = w.left();
    stage_pair<HD, QC, W>(smem_u32(s_q[buf]), smem_u32(s_g[buf]), static_cast<const bf16*>(a.q) + (sample0 + row0) * a.ldq + (int64_t)head * HD, a.ldq,
                          static_cast<const bf16*>(a.dout) + (sample0 + row0) * a.lddo + (int64_t)head * HD, a.lddo, rem, tid);
    const float2* stats = a.row_stats + ((int64_t)b * g.heads + head) * g.L + row0;
    for (int i = tid; i < min(QC, (rem + BLOCK - 1) / BLOCK * BLOCK); i += 32 * W) {
      s_stats[buf][i] = i < rem ? stats[i] : make_float2(INFINITY, 0.f);   // no weight for rows past the last
      if (TIMES) {
        const float t = i >= rem ? 0.f : a.times != nullptr ? a.times[sample0 + row0 + i] : (float)(w.pos + i);
        s_time[buf][i] = t;
        if (MASK) {
          s_limit[buf][i] = latest_seen(a, b, t);
          s_doc[buf][i] = i < rem && a.documents != nullptr ? a.documents[sample0 + row0 + i] : 0;
        }
      }
    }
  };
  if (!next.over()) stage(next, h, 0);

  const int w0 = k0 + warp * 16 * MT;
  const int64_t key0 = sample0 + g.off(r);
  uint32_t kf[MT][(HD + 15) / 16][4], vf[MT][(HD + 15) / 16][4];
  float own_time[MT][2];
  int own_doc[MT][2];
  bool real[MT][2];
  Range mine = NO_ROWS;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const bf16 *pk[2], *pv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = w0 + 16 * m + 8 * i + (lane >> 2);
      real[m][i] = row < min(k_end, n_k);
      pk[i] = real[m][i] ? static_cast<const bf16*>(a.k) + (key0 + row) * a.ldk + (int64_t)hk * HD : nullptr;
      pv[i] = real[m][i] ? static_cast<const bf16*>(a.v) + (key0 + row) * a.ldv + (int64_t)hk * HD : nullptr;
      own_time[m][i] = 0.f;
      own_doc[m][i] = 0;
      if (TIMES && real[m][i]) own_time[m][i] = time_of(g, a, b, r, row);
      if (MASK && real[m][i]) {
        own_doc[m][i] = document_of(g, a, b, r, row);
        mine = {min(mine.t_lo, ordered(own_time[m][i])), max(mine.t_hi, ordered(own_time[m][i])), min(mine.d_lo, own_doc[m][i]), max(mine.d_hi, own_doc[m][i])};
      }
    }
    own_rows<HD>(pk[0], pk[1], lane, kf[m]);
    own_rows<HD>(pv[0], pv[1], lane, vf[m]);
  }
  if (MASK) mine = warp_range(mine.t_lo, mine.t_hi, mine.d_lo, mine.d_hi);
  const bool working = w0 < min(k_end, n_k);

  const LaneAt<HD> at_qn = lane_as_n<HD>(smem_u32(s_q[0]), lane), at_qk = lane_as_k<HD>(smem_u32(s_q[0]), lane);
  const LaneAt<HD> at_gn = lane_as_n<HD>(smem_u32(s_g[0]), lane), at_gk = lane_as_k<HD>(smem_u32(s_g[0]), lane);

  float dk[MT][CH][4], dv[MT][CH][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) dk[m][c][e] = dv[m][c][e] = 0.f;

  auto step = [&](auto some_tag, int buf, int j, float slope2) {
    constexpr bool SOME_SHUT = decltype(some_tag)::value;
    float x[MT][NT][4], dp[MT][NT][4];
    float2 lse2[NT], delta[NT];   // of this lane's two columns of every tile
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float4 t = *reinterpret_cast<const float4*>(&s_stats[buf][j + 8 * n + 2 * (lane & 3)]);
      lse2[n] = make_float2(t.x, t.z);
      delta[n] = make_float2(-t.y, -t.w);
    }
    const uint32_t from = (buf * QC + j) * HD * 2;
    product_over_features<HD, MT, NT>(x, kf, at_qn, from, from_zero);
    product_over_features<HD, MT, NT>(dp, vf, at_gn, from, [&](int, int n, float (&z)[4]) {
      z[0] = z[2] = delta[n].x;
      z[1] = z[3] = delta[n].y;
    });
    uint32_t wp[MT][NT][2], ws[MT][NT][2];
    in_form<CAP, MT, NT>(x, a, [&](auto near) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float2 times = make_float2(0.f, 0.f);
          if constexpr (BIAS) times = *reinterpret_cast<const float2*>(&s_time[buf][j + 8 * n + 2 * (lane & 3)]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float2 d = make_float2(dp[m][n][2 * i], dp[m][n][2 * i + 1]);
            float2 bend, y = score_pair<CAP, true, decltype(near)::value != 0>(make_float2(x[m][n][2 * i], x[m][n][2 * i + 1]), lse2[n], bend, a);
            if constexpr (BIAS) y = bias_pair(y, times, own_time[m][i], slope2);
            if constexpr (SOME_SHUT) {   // columns past the last row have an lse of +inf: no weight
              auto shut = [&](int col) { return own_time[m][i] > s_limit[buf][col] || s_doc[buf][col] != own_doc[m][i]; };
              const int col = j + 8 * n + 2 * (lane & 3);
              y = make_float2(shut(col) ? -INFINITY : y.x, shut(col + 1) ? -INFINITY : y.y);
            }
            const float2 p = make_float2(ptx::ex2(y.x), ptx::ex2(y.y)), ds = __fmul2_rn(p, times_bend<CAP>(d, bend));
            wp[m][n][i] = ptx::pack_bf16(p.x, p.y);
            ws[m][n][i] = ptx::pack_bf16(ds.x, ds.y);
          }
        }
    });
    __syncwarp();   // lanes may have taken different ways; matrix instructions need the whole warp
    product_over_partners<HD, MT, NT>(dv, wp, at_gk, from);
    product_over_partners<HD, MT, NT>(dk, ws, at_qk, from);
  };

  for (int buf = 0; !next.over(); buf ^= 1) {
    const int rem = min(QC, next.left()), head = h;
    cp_wait();
    __syncthreads();
    next.pos += QC;
    next.settle();
    if (next.over() && h < last_head) {
      next = first;
      ++h;
    }
    if (!next.over()) stage(next, h, buf ^ 1);
    if (!working) continue;
    const float slope2 = BIAS ? a.slopes[head] * LOG2E : 0.f;
    int j = 0;
    if constexpr (!MASK) {
#pragma unroll 1
      for (; j < rem; j += 8 * NT) step(IntTag<0>{}, buf, j, slope2);
    } else {
#pragma unroll 1
      while (j < rem) {
        const Openness open = openness(block_range(s_limit[buf], s_doc[buf], j, rem, lane), mine);
        const int end = min(j + BLOCK, rem);
        if (open == ALL)
#pragma unroll 1
          for (; j < end; j += 8 * NT) step(IntTag<0>{}, buf, j, slope2);
        else if (open != SHUT)
#pragma unroll 1
          for (; j < end; j += 8 * NT) step(IntTag<1>{}, buf, j, slope2);
        j = end;
      }
    }
  }

  ptx::grid_dep_launch();   // see scored_tile.cuh
  bool broken = false;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = w0 + 16 * m + 8 * i + (lane >> 2);
      if (row < k_end) {
        bf16* pk = static_cast<bf16*>(a.dk) + (key0 + row) * a.lddk + (int64_t)hk * HD + 2 * (lane & 3);
        bf16* pv = static_cast<bf16*>(a.dv) + (key0 + row) * a.lddv + (int64_t)hk * HD + 2 * (lane & 3);
#pragma unroll
        for (int q = 0; q < CH; ++q) {
          const float2 k2 = make_float2(dk[m][q][2 * i] * a.scale, dk[m][q][2 * i + 1] * a.scale), v2 = make_float2(dv[m][q][2 * i], dv[m][q][2 * i + 1]);
          if (MASK && real[m][i]) broken = broken || !finite(k2.x) || !finite(k2.y) || !finite(v2.x) || !finite(v2.y);
          *reinterpret_cast<uint32_t*>(pk + 8 * q) = real[m][i] ? ptx::pack_bf16(k2.x, k2.y) : 0u;
          *reinterpret_cast<uint32_t*>(pv + 8 * q) = real[m][i] ? ptx::pack_bf16(v2.x, v2.y) : 0u;
        }
      }
    }
  if (MASK && __any_sync(0xffffffffu, broken))
    for (int row = w0; row < min(w0 + 16 * MT, min(k_end, n_k)); ++row) dkv_row<bf16>(g, a, b, hk, r, row);
}

// Which of the two kernels, by a type.
struct Dq {
  static constexpr int MANY = 7;
  template <int HD, int CTAS, bool CAP, bool BIAS, bool MASK> static constexpr auto kernel = scored_dq_kernel<HD, CTAS, CAP, BIAS, MASK>;
};
struct Dkv {
  static constexpr int MANY = 6;
  template <int HD, int CTAS, bool CAP, bool BIAS, bool MASK> static constexpr auto kernel = scored_dkv_kernel<HD, CTAS, CAP, BIAS, MASK>;
};

template <typename K, int HD, int CTAS, bool CAP, bool BIAS>
cudaError_t launch_masked(const Geometry& g, const ScoredArgs& a, const Tiles& t, dim3 grid, cudaStream_t st) {
  return rule_masks(a) ? launch_overlapped(K::template kernel<HD, CTAS, CAP, BIAS, true>, grid, dim3(32 * W), 0, st, g, a, t)
                       : launch_overlapped(K::template kernel<HD, CTAS, CAP, BIAS, false>, grid, dim3(32 * W), 0, st, g, a, t);
}
template <typename K, int HD, int CTAS>
cudaError_t launch_rule(const Geometry& g, const ScoredArgs& a, const Tiles& t, dim3 grid, cudaStream_t st) {
  const bool cap = a.softcap > 0.f, bias = a.slopes != nullptr;
  return cap ? (bias ? launch_masked<K, HD, CTAS, true, true>(g, a, t, grid, st) : launch_masked<K, HD, CTAS, true, false>(g, a, t, grid, st))
             : (bias ? launch_masked<K, HD, CTAS, false, true>(g, a, t, grid, st) : launch_masked<K, HD, CTAS, false, false>(g, a, t, grid, st));
}
template <typename K, int HD>
cudaError_t launch_pass(const Geometry& g, const ScoredArgs& a, int heads, uint32_t walks, int n_sm, cudaStream_t st) {
  Tiles t = {};
  t.order = segment_order(g, walks);
  const int64_t n = make_tiles(&t, g.seg_len, OWN) * heads * g.batch;
  if (n > 0x7fffffffLL) return cudaErrorNotSupported;
  const dim3 grid((unsigned)n);
  // as in the forward pass (these hold more: dq 7, dk and dv 6 for 8); both kernels, more / fewer CTAs an SM, us, 8 heads of 16: 2 x (50, 500, 500)
  // 22.7 / 18.5, 8 x 46 / 40, 64 x (20, 20, 20) 14.4 / 16.7, 64 x (39, 55, 400) 65 / 74, 512 x (50, 50, 50) 141 / 169; dq with 8 CTAs an SM 73 us for
  // 70 (64 x (39, 55, 400)), with steps of 32 keys in place of 16 70 for 65
  if constexpr (HD <= 16)
    if (n > 8LL * n_sm) return launch_rule<K, HD, K::MANY>(g, a, t, grid, st);
  return launch_rule<K, HD, HD == 64 ? 3 : 4>(g, a, t, grid, st);
}
template <int HD>
cudaError_t launch_width(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  int n_sm = 0;
  cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  e = launch_pass<Dq, HD>(g, a, g.heads, g.allowed, n_sm, st);
  return e != cudaSuccess ? e : launch_pass<Dkv, HD>(g, a, a.kv_heads, transposed(g.allowed), n_sm, st);
}

}  // namespace

cudaError_t launch_scored_bwd_bf16(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  switch (g.hd) {
    case 8: return launch_width<8>(g, a, st);
    case 16: return launch_width<16>(g, a, st);
    case 32: return launch_width<32>(g, a, st);
    case 64: return launch_width<64>(g, a, st);
    default: return cudaErrorNotSupported;
  }
}

}  // namespace gsit

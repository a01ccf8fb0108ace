// Scored attention, forward, bf16, on mma.sync (see scored_tile.cuh).
//
// One pass over the keys: scores x = outer tanh(inner q.k) - slope |time difference| in base 2 stay in registers, weights 2^(x - ref) go into the
// second product as they lie there, and a running reference and sum make the softmax.  Weights are rounded to bf16 for that product
// (their sum is not): the result's error against 64 bits is 2^-8.6 of its norm, where its own rounding to bf16 is 2^-9.2.
// What bounds it: a pair of scores costs 4 packed multiply-adds (2 clocks each), 2 exponentials (16 a clock and SM), a conversion and what
// mask and bias add, and products of 8 or 16 features none of the time; for MOSEI's step (64 samples of (50, 500, 500), half of the rows
// padding, 8 heads of 8, cap and bias: 82 million pairs) that is 18 us of exponentials, measured 76 us.  The rest is a warp's prologue
// (some 400 instructions for 16 rows that walk 250 keys on average), staging, and the latency of a step's chain.
#include "scored_tile.cuh"

namespace gsit {
namespace {

constexpr int W = 4;   // warps of a CTA

// Row tiles of a warp (two share the fragments of K and V, but cost the warps that hide latency: MOSEI's step 103 us for 96) and rows of a CTA
// (128: 512 x (50, 50, 50), 8 heads of 8 72 us for 50, 128 x (50, 500, 500) 165 for 162)
constexpr int MT = 1, TQ = 16 * MT * W;

// CTAS: CTAs of an SM that registers are kept for
template <int HD, int CTAS, bool CAP, bool BIAS, bool MASK>
__global__ void __launch_bounds__(32 * W, CTAS)
scored_fwd_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  constexpr int KC = CHUNK_ROWS<HD>, CH = HD / 8, NT = 4, NS = HD == 8 ? 4 : 2;   // tiles of 8 keys in a step, and where some pairs are shut
  constexpr bool TIMES = BIAS || MASK;
  __shared__ __align__(128) uint8_t s_k[2][KC * HD * 2], s_v[2][KC * HD * 2];
  __shared__ __align__(16) float s_time[2][TIMES ? KC : 4];
  __shared__ int s_doc[2][MASK ? KC : 1];
  const int tid = threadIdx.x, warp = ptx::uniform(tid >> 5), lane = tid & 31;
  const Place at = find_place(tiles, g.batch, g.heads);
  const int b = at.sample, s = at.segment, h = at.head, hk = h / a.group;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();

  const int q0 = at.tile * TQ, q_end = min(q0 + TQ, a.q_len[s]);
  const QueryRows rows = query_rows(g, a, b, s);
  Walk next = {};
#pragma unroll
  for (int r = 0; r < 3; ++r) next.n[r] = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
  if (max(q0, rows.lo) >= min(q_end, rows.hi)) next.seg = 3;
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

  // ---- the warp's rows ----
  const int w0 = q0 + warp * 16 * MT;
  const int64_t q_row0 = (int64_t)b * a.Lq + a.q_off[s];
  uint32_t qf[MT][(HD + 15) / 16][4];
  float own_time[MT][2], limit[MT][2];
  int own_doc[MT][2];
  bool real[MT][2];
  Range mine = NO_ROWS;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const bf16* p[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = w0 + 16 * m + 8 * i + (lane >> 2);
      real[m][i] = row >= rows.lo && row < min(q_end, rows.hi);
      p[i] = real[m][i] ? static_cast<const bf16*>(a.q) + (q_row0 + row) * a.ldq + (int64_t)h * HD : nullptr;
      own_time[m][i] = 0.f;
      limit[m][i] = INFINITY;
      own_doc[m][i] = 0;
      if (TIMES && real[m][i]) own_time[m][i] = time_of(g, a, b, s, row + rows.shift);
      if (MASK && real[m][i]) {
        limit[m][i] = latest_seen(a, b, own_time[m][i]);
        own_doc[m][i] = document_of(g, a, b, s, row + rows.shift);
        mine = {min(mine.t_lo, ordered(limit[m][i])), max(mine.t_hi, ordered(limit[m][i])), min(mine.d_lo, own_doc[m][i]), max(mine.d_hi, own_doc[m][i])};
      }
    }
    own_rows<HD>(p[0], p[1], lane, qf[m]);
  }
  if (MASK) mine = warp_range(mine.t_lo, mine.t_hi, mine.d_lo, mine.d_hi);
  const bool working = w0 < min(q_end, rows.hi) && w0 + 16 * MT > rows.lo;
  const float slope2 = BIAS ? a.slopes[h] * LOG2E : 0.f;
  const LaneAt<HD> at_k = lane_as_n<HD>(smem_u32(s_k[0]), lane), at_v = lane_as_k<HD>(smem_u32(s_v[0]), lane);

  // ref: what a row's weights are relative to (base 2); it follows the row's maximum when a score exceeds it by more than `room` (2^8, so
  // that weights stay below 256; any score as long as the row has seen no open key)
  float o[MT][CH][4], ref[MT][2], room[MT][2];
  float2 sum[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[m][c][e] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ref[m][i] = 0.f;
      room[m][i] = -INFINITY;
      sum[m][i] = make_float2(0.f, 0.f);
    }
  }

  // One step: 8 N keys from column j of the chunk on; `some`: pairs of it may be closed, or it reaches past the last key.
  auto step = [&](auto n_tag, auto some_tag, int buf, int j, int rem) {
    constexpr int N = decltype(n_tag)::value;
    constexpr bool SOME_SHUT = decltype(some_tag)::value;
    float x[MT][N][4];
    const uint32_t from = (buf * KC + j) * HD * 2;
    product_over_features<HD, MT, N>(x, qf, at_k, from, from_zero);
    uint32_t w[MT][N][2];
    float top[MT][2];
    float2 added[MT][2] = {};
    bool outgrown = false;
    in_form<CAP, MT, N>(x, a, [&](auto near) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        top[m][0] = top[m][1] = -INFINITY;
#pragma unroll
        for (int n = 0; n < N; ++n) {
          float2 times = make_float2(0.f, 0.f), none;
          if constexpr (BIAS) times = *reinterpret_cast<const float2*>(&s_time[buf][j + 8 * n + 2 * (lane & 3)]);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float2 y = score_pair<CAP, false, decltype(near)::value != 0>(make_float2(x[m][n][2 * i], x[m][n][2 * i + 1]), make_float2(ref[m][i], ref[m][i]), none, a);
            if constexpr (BIAS) y = bias_pair(y, times, own_time[m][i], slope2);
            if constexpr (SOME_SHUT) {
              auto shut = [&](int col) { return col >= rem || (MASK && (s_time[buf][col] > limit[m][i] || s_doc[buf][col] != own_doc[m][i])); };
              const int col = j + 8 * n + 2 * (lane & 3);
              y = make_float2(shut(col) ? -INFINITY : y.x, shut(col + 1) ? -INFINITY : y.y);
            }
            top[m][i] = ptx::fmax3(top[m][i], y.x, y.y);
            x[m][n][2 * i] = y.x;
            x[m][n][2 * i + 1] = y.y;
            const float2 p = make_float2(ptx::ex2(y.x), ptx::ex2(y.y));
            added[m][i] = __fadd2_rn(added[m][i], p);
            w[m][n][i] = ptx::pack_bf16(p.x, p.y);
          }
        }
        outgrown = outgrown || top[m][0] > room[m][0] || top[m][1] > room[m][1];
      }
    });
    // rare: a score has outgrown its row's reference (as long as no lane's own have, the lanes of a row need not be brought together);
    // the weights once more, relative to a new one
    if (__any_sync(0xffffffffu, outgrown)) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float t = fmaxf(top[m][i], __shfl_xor_sync(0xffffffffu, top[m][i], 1));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
          if (t > room[m][i]) {
            // nothing to scale down before the first open key.  The first reference is a maximum in any case: a weight of 1 is exact in
            // bf16, and with it the output of a row that sees one key
            const float f = room[m][i] == -INFINITY ? 1.f : ptx::ex2(-t);
            room[m][i] = 8.f;
            sum[m][i] = __fmul2_rn(sum[m][i], make_float2(f, f));
#pragma unroll
            for (int q = 0; q < CH; ++q) {
              o[m][q][2 * i] *= f;
              o[m][q][2 * i + 1] *= f;
            }
            ref[m][i] += t;
            added[m][i] = make_float2(0.f, 0.f);
#pragma unroll
            for (int n = 0; n < N; ++n) {
              const float2 p = make_float2(ptx::ex2(x[m][n][2 * i] - t), ptx::ex2(x[m][n][2 * i + 1] - t));
              added[m][i] = __fadd2_rn(added[m][i], p);
              w[m][n][i] = ptx::pack_bf16(p.x, p.y);
            }
          }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int i = 0; i < 2; ++i) sum[m][i] = __fadd2_rn(sum[m][i], added[m][i]);
    __syncwarp();   // lanes may have taken different ways; matrix instructions need the whole warp
    product_over_partners<HD, MT, N>(o, w, at_v, from);
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
      for (; j + 8 * NT <= rem; j += 8 * NT) step(IntTag<NT>{}, IntTag<0>{}, buf, j, rem);
#pragma unroll 1
      for (; j < rem; j += 8 * NS) step(IntTag<NS>{}, IntTag<1>{}, buf, j, rem);
    } else {
#pragma unroll 1
      while (j < rem) {
        const Openness open = openness(mine, block_range(s_time[buf], s_doc[buf], j, rem, lane));
        const int end = min(j + BLOCK, rem);
        if (open == ALL && end - j == BLOCK)
#pragma unroll 1
          for (; j < end; j += 8 * NT) step(IntTag<NT>{}, IntTag<0>{}, buf, j, rem);
        else if (open != SHUT)
#pragma unroll 1
          for (; j < end; j += 8 * NS) step(IntTag<NS>{}, IntTag<1>{}, buf, j, rem);
        j = end;
      }
    }
  }

  ptx::grid_dep_launch();   // see scored_tile.cuh
  // ---- results ----
  bool broken = false;
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float l = sum[m][i].x + sum[m][i].y;
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      const int row = w0 + 16 * m + 8 * i + (lane >> 2);
      const float inv = real[m][i] && l != 0.f ? 1.f / l : 0.f;
      if (MASK && real[m][i]) {
        broken = broken || !finite(l);
#pragma unroll
        for (int q = 0; q < CH; ++q) broken = broken || !finite(o[m][q][2 * i]) || !finite(o[m][q][2 * i + 1]);
      }
      if (row < q_end) {
        bf16* dst = static_cast<bf16*>(a.out) + (q_row0 + row) * a.ldo + (int64_t)h * HD + 2 * (lane & 3);
#pragma unroll
        for (int q = 0; q < CH; ++q)
          *reinterpret_cast<uint32_t*>(dst + 8 * q) = inv == 0.f ? 0u : ptx::pack_bf16(o[m][q][2 * i] * inv, o[m][q][2 * i + 1] * inv);
        if (a.lse != nullptr && (lane & 3) == 0)
          a.lse[((int64_t)b * g.heads + h) * a.Lq + a.q_off[s] + row] = real[m][i] && l != 0.f ? (ref[m][i] + log2f(l)) * LN2 : -INFINITY;
      }
    }
  // zero times NaN or Inf of a closed key: those rows once more, pair by pair
  if (MASK && __any_sync(0xffffffffu, broken))
    for (int row = max(w0, rows.lo); row < min(w0 + 16 * MT, min(q_end, rows.hi)); ++row) attend_row<bf16>(g, a, b, h, s, row);
}

template <int HD, int CTAS, bool CAP, bool BIAS>
cudaError_t launch_masked(const Geometry& g, const ScoredArgs& a, const Tiles& t, dim3 grid, cudaStream_t st) {
  return rule_masks(a) ? launch_overlapped(scored_fwd_kernel<HD, CTAS, CAP, BIAS, true>, grid, dim3(32 * W), 0, st, g, a, t)
                       : launch_overlapped(scored_fwd_kernel<HD, CTAS, CAP, BIAS, false>, grid, dim3(32 * W), 0, st, g, a, t);
}
template <int HD, int CTAS>
cudaError_t launch_rule(const Geometry& g, const ScoredArgs& a, const Tiles& t, dim3 grid, cudaStream_t st) {
  const bool cap = a.softcap > 0.f, bias = a.slopes != nullptr;
  return cap ? (bias ? launch_masked<HD, CTAS, true, true>(g, a, t, grid, st) : launch_masked<HD, CTAS, true, false>(g, a, t, grid, st))
             : (bias ? launch_masked<HD, CTAS, false, true>(g, a, t, grid, st) : launch_masked<HD, CTAS, false, false>(g, a, t, grid, st));
}
template <int HD>
cudaError_t launch_width(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  int n_sm = 0;
  const cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  Tiles t = {};
  t.order = segment_order(g, g.allowed);
  const int64_t n = make_tiles(&t, a.q_len, TQ) * g.heads * g.batch;
  if (n > 0x7fffffffLL) return cudaErrorNotSupported;
  const dim3 grid((unsigned)n);
  // Narrow heads: in a grid of more than a wave twice the warps with half the registers, which hide a step's latency; in a smaller one, where there
  // are no more warps, all registers.  8 / 4 CTAs an SM, us, 8 heads of 16: 2 x (50, 500, 500) 9.3 / 8.6, 8 x 17.6 / 15.8, 64 x (20, 20, 20) 6.9 /
  // 8.0, 64 x (39, 55, 400) 25.9 / 27.8, 512 x (50, 50, 50) 59 / 65.
  if constexpr (HD <= 16)
    if (n > 8LL * n_sm) return launch_rule<HD, 8>(g, a, t, grid, st);
  return launch_rule<HD, 4>(g, a, t, grid, st);
}

}  // namespace

cudaError_t launch_scored_fwd_bf16(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  switch (g.hd) {
    case 8: return launch_width<8>(g, a, st);
    case 16: return launch_width<16>(g, a, st);
    case 32: return launch_width<32>(g, a, st);
    case 64: return launch_width<64>(g, a, st);
    default: return cudaErrorNotSupported;
  }
}

}  // namespace gsit

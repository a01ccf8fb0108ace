// Scored attention at head_dim 64 on the 5th-generation tensor cores (tcgen05) with accumulators in tensor memory: forward, dq, and dk
// with dv, as one kernel of three kinds.
//
// A CTA owns 128 rows of one head -- queries (FWD, DQ) or keys (DKV) -- and walks its partners in tiles of 64:
//   x  = own0 partner0^T                       (Q K^T, Q K^T, K Q^T)
//   dp =                own1 partner1^T        (        dO V^T, V dO^T)
//   a thread per own row (= lane of tensor memory) turns them into weights p = exp2(score - reference or log-sum-exp) and, backward,
//   ds = p (dp - delta) bend, packed to bf16 back into tensor memory
//   acc0 += p partner1 (FWD)  or  ds partner0 (DQ, DKV);   acc1 += p partner1 (DKV)  or  p bend partner0 (DQ, what dq is corrected along: scored_bwd.cu)
// with weights from tensor memory as the A operand and the partner tile, as TMA wrote it, as an MN-major B operand: nothing is
// transposed, no score leaves the SM.  A CTA has 256 columns of tensor memory, so two CTAs share an SM.  What one tile after the
// other would take is mostly latency (products -> barrier -> scores -> barrier -> products: 4600 clocks a tile of the forward kind,
// against 212 of products and 512 of exponentials), so the next tile's first products are issued as early as the columns allow:
//   FWD  x twice (the weights take the columns of the x they come from): x of tile t + 1 beside the scores of tile t
//   DQ, DKV  x, dp and two accumulators; p and ds take the columns of dp: x of tile t + 1 as soon as that of tile t is in registers, dp
//        once the products with p and ds are over
// Weights and ds are rounded to bf16 for the second products, as in scored_fwd.cu and scored_bwd.cu.
// Measured: 32 samples of (128, 1024, 1024), a quarter of the rows padding, 8 heads of 64, cap (272 million pairs): 184 us (FWD) and 514 (DQ and DKV,
// half each), 350 TFLOP/s; 463 without what dq is corrected along, where ds had columns of its own and dp of the next tile came early, too.  The
// products alone are 143 us at the measured cuBLAS rate, the exponentials 117 us of the special function units, which are 38%, 24% and 25% busy:
// two computing warps a scheduler do not hide the trips through tensor memory and barriers of every tile.  attn_tc.cu, which keeps weights in
// columns of their own and sets up once for many items, takes 116 us for the forward pass of the same pairs without a cap (162 here).
// With documents and causality a quarter of the pairs are open, in 45% of the tiles, and nothing is gained: 211 + 568 us; the fetching warp looks
// at tiles one after the other, closed ones, too, and a partly open one costs two loads and two comparisons for four columns.
// Two threads a row, so four warps a scheduler: 793 us for 706.  Three CTAs an SM in the forward kind, with 128 columns of
// tensor memory and x only once, so that a CTA's products and scores take turns: 193 us for 189, and 23 for 17 where a grid is small.
// Warps: 0 fetches (own tiles once, a ring of three partner stages with what the scores need beside them, and which tiles are open at
// all), 1 issues every product, 2 .. 5 compute.  All waits are bounded.
#include <cuda.h>

#include "scored_tile.cuh"
#include "tensor_map.cuh"
#include "tmem_ldst.cuh"

namespace gsit {
namespace {

using namespace ptx;

enum Kind { FWD, DQ, DKV };
constexpr int HD = 64, OWN = 128, PARTNER = 64, STAGES = 3, THREADS = 192;
constexpr int OWN_BYTES = OWN * 128, TILE_BYTES = PARTNER * 128;
// A stage's record and what its partners bring to the scores
struct Meta {
  float time[PARTNER], limit[PARTNER], lse[PARTNER], delta[PARTNER];
  int doc[PARTNER];
  int rem;      // real partners of the tile (64 or more: whole); < 0: the walk is over
  int some;     // pairs of the tile may be closed
  float slope2;
  int pad;
};
template <int KIND> struct Map {   // shared memory, relative to a 1024-byte aligned base
  static constexpr int OWN_TILES = KIND == FWD ? 1 : 2;
  static constexpr int TILES = OWN_TILES * OWN_BYTES, META = TILES + STAGES * 2 * TILE_BYTES, BARS = META + STAGES * (int)sizeof(Meta);
  static constexpr int BYTES = BARS + 128 + 1024;
  static constexpr int TMEM = 256, CTAS = 2;
  // columns of tensor memory: x (FWD: twice, and weights there), dp (and weights and ds there), accumulators
  static constexpr int X = 0, DP = 64, ACC = 128;
};
constexpr int BAR_OWN = 0, BAR_FULL = 8, BAR_EMPTY = BAR_FULL + 8 * STAGES, BAR_X = BAR_EMPTY + 8 * STAGES, BAR_W = BAR_X + 16, BAR_DP = BAR_W + 16,
              BAR_READ = BAR_DP + 8, BAR_ACC = BAR_READ + 8, SLOT_TMEM = BAR_ACC + 8, SLOT_GAVE_UP = SLOT_TMEM + 4;

template <bool V> struct BoolTag { static constexpr bool value = V; };

struct Maps {
  CUtensorMap own0, own1, partner0, partner1;
};

// The largest argument of a row's dots.
template <int N> __device__ __forceinline__ float largest(const float (&x)[N]) {
  float top[4] = {};
#pragma unroll
  for (int c = 0; c < N; c += 2) top[c / 2 % 4] = fmax3(top[c / 2 % 4], fabsf(x[c]), fabsf(x[c + 1]));
  return fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
}

__device__ __forceinline__ float sum_of(const float2 (&part)[4]) {
  const float2 s = __fadd2_rn(__fadd2_rn(part[0], part[1]), __fadd2_rn(part[2], part[3]));
  return s.x + s.y;
}

template <int KIND, bool CAP, bool BIAS, bool MASK>
__global__ void __launch_bounds__(THREADS, Map<KIND>::CTAS)
scored_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  using M = Map<KIND>;
  constexpr bool TIMES = BIAS || MASK, BWD = KIND != FWD;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u, bars = base + M::BARS;
  Meta* const metas = reinterpret_cast<Meta*>(smem_raw + (base - smem_u32(smem_raw)) + M::META);
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  const WaitCtx wc{g.status, bars + SLOT_GAVE_UP};
  if (tid == 0) {
    map_early(maps.own0);
    map_early(maps.partner0);
    map_early(maps.partner1);
    asm volatile("st.shared.u32 [%0], %1;" ::"r"(bars + SLOT_GAVE_UP), "r"(0u) : "memory");
    mbar_init(bars + BAR_OWN, 1);
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(bars + BAR_FULL + 8 * i, 1);
      mbar_init(bars + BAR_EMPTY + 8 * i, 5);   // the products' commit, four computing warps
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mbar_init(bars + BAR_X + 8 * i, 1);     // x is there (FWD: buffer i; backward: i = 0)
      mbar_init(bars + BAR_W + 8 * i, 128);   // the weights of tile i, i + 2, .. are there
    }
    mbar_init(bars + BAR_DP, 1);              // backward: dp is there
    mbar_init(bars + BAR_READ, 128);          // ... and x is in registers
    mbar_init(bars + BAR_ACC, 1);             // a tile's second products are over
    mbar_init_fence();
  }
  if (warp == 1) tmem_alloc(bars + SLOT_TMEM, M::TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  uint32_t tmem;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(bars + SLOT_TMEM) : "memory");
  load_params_early(g, a, tiles);
  grid_dep_wait();

  // ---- the CTA's rows: [o0, o_end) of segment s of sample b, of which [lo, hi) are real; position = row + shift ----
  const Place at = find_place(tiles, g.batch, KIND == DKV ? a.kv_heads : g.heads);
  const int h = at.head, b = at.sample, s = at.segment, o0 = at.tile * OWN;
  const QueryRows rows = KIND == FWD ? query_rows(g, a, b, s) : QueryRows{0, valid_rows(g, b, s), 0};
  const int own_len = KIND == FWD ? a.q_len[s] : g.len(s), o_end = min(o0 + OWN, own_len), lo = max(o0, rows.lo), hi = min(o_end, rows.hi);
  const int64_t own_row0 = KIND == FWD ? (int64_t)b * a.Lq + a.q_off[s] : (int64_t)b * g.L + g.off(s);
  int n[3];
#pragma unroll
  for (int r = 0; r < 3; ++r) n[r] = lo < hi && ((g.allowed >> (KIND == DKV ? 3 * r + s : 3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
  const bool any = n[0] + n[1] + n[2] > 0;

  if (warp == 0) {
    // ================================ fetching ================================
    if (any) {
      Range mine = NO_ROWS;
      if (MASK) {
        for (int i = lo + lane; i < hi; i += 32) {
          const float t = time_of(g, a, b, s, i + rows.shift);
          const int o = ordered(KIND == DKV ? t : latest_seen(a, b, t)), d = document_of(g, a, b, s, i + rows.shift);
          mine = {min(mine.t_lo, o), max(mine.t_hi, o), min(mine.d_lo, d), max(mine.d_hi, d)};
        }
        mine = warp_range(mine.t_lo, mine.t_hi, mine.d_lo, mine.d_hi);
      }
      if (elect_one()) {
        mbar_expect_tx(bars + BAR_OWN, M::OWN_TILES * OWN_BYTES);
        tma_load_2d(base, &maps.own0, h * HD, (int)own_row0 + o0, bars + BAR_OWN);
        if (BWD) tma_load_2d(base + OWN_BYTES, &maps.own1, h * HD, (int)own_row0 + o0, bars + BAR_OWN);
      }
      __syncwarp();
      int t = 0;   // tiles requested
      for (int k = 0; k < (KIND == DKV ? a.group : 1); ++k) {
        const int partner_head = KIND == DKV ? h * a.group + k : h / a.group, score_head = KIND == DKV ? partner_head : h;
#pragma unroll 1
        for (int r = 0; r < 3; ++r)
#pragma unroll 1
          for (int p0 = 0; p0 < n[r]; p0 += PARTNER) {
            const int rem = n[r] - p0, row0 = b * g.L + g.off(r) + p0;
            float time[2], limit[2];
            int doc[2];
            float2 stats[2];
            Range theirs = NO_ROWS;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int at = lane + 32 * i;
              const bool in = at < rem;
              time[i] = limit[i] = 0.f;
              doc[i] = 0;
              if (TIMES) time[i] = !in ? 0.f : a.times != nullptr ? a.times[(int64_t)row0 + at] : (float)(p0 + at);
              if (MASK) {
                limit[i] = KIND == DKV ? latest_seen(a, b, time[i]) : time[i];
                doc[i] = in && a.documents != nullptr ? a.documents[(int64_t)row0 + at] : 0;
                if (in) theirs = {min(theirs.t_lo, ordered(limit[i])), max(theirs.t_hi, ordered(limit[i])), min(theirs.d_lo, doc[i]), max(theirs.d_hi, doc[i])};
              }
              if (KIND == DKV) stats[i] = in ? a.row_stats[((int64_t)b * g.heads + partner_head) * g.L + g.off(r) + p0 + at] : make_float2(INFINITY, 0.f);
            }
            Openness open = ALL;
            if (MASK) {
              theirs = warp_range(theirs.t_lo, theirs.t_hi, theirs.d_lo, theirs.d_hi);
              open = KIND == DKV ? openness(theirs, mine) : openness(mine, theirs);
              if (open == SHUT) continue;
            }
            const int st = t % STAGES, use = t / STAGES;
            if (use > 0) mbar_wait_warp(wc, bars + BAR_EMPTY + 8 * st, (use - 1) & 1);
            Meta& m = metas[st];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int at = lane + 32 * i;
              if (TIMES) m.time[at] = time[i];
              if (MASK) {
                m.limit[at] = limit[i];
                m.doc[at] = doc[i];
              }
              if (KIND == DKV) {
                m.lse[at] = stats[i].x;
                m.delta[at] = stats[i].y;
              }
            }
            if (lane == 0) {
              m.rem = rem;
              m.some = open == SOME;
              m.slope2 = BIAS ? a.slopes[score_head] * LOG2E : 0.f;
            }
            __syncwarp();
            if (elect_one()) {
              const uint32_t tile = base + M::TILES + st * 2 * TILE_BYTES;
              mbar_expect_tx(bars + BAR_FULL + 8 * st, 2 * TILE_BYTES);
              tma_load_2d(tile, &maps.partner0, partner_head * HD, row0, bars + BAR_FULL + 8 * st);
              tma_load_2d(tile + TILE_BYTES, &maps.partner1, partner_head * HD, row0, bars + BAR_FULL + 8 * st);
            }
            __syncwarp();
            ++t;
          }
      }
      const int st = t % STAGES, use = t / STAGES;
      if (use > 0) mbar_wait_warp(wc, bars + BAR_EMPTY + 8 * st, (use - 1) & 1);
      if (lane == 0) {
        metas[st].rem = -1;
        mbar_arrive(bars + BAR_FULL + 8 * st);
      }
    }
  } else if (warp == 1) {
    // ================================ products ================================
    if (any) {
      constexpr uint32_t TO_X = idesc_bf16(PARTNER, false), TO_ACC = idesc_bf16(HD, true);
      auto tile_of = [&](int t) { return base + M::TILES + (t % STAGES) * 2 * TILE_BYTES; };
      auto more = [&](int t) {   // is there a tile t?
        const bool ok = mbar_wait_warp(wc, bars + BAR_FULL + 8 * (t % STAGES), (t / STAGES) & 1);
        return ok && uniform(metas[t % STAGES].rem) >= 0;
      };
      auto to_x = [&](int t) {
        const uint32_t tile = tile_of(t);
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
          umma_ss(tmem + M::X + (KIND == FWD ? 64 * (t & 1) : 0), smem_desc_sw128(base + 32 * k), smem_desc_sw128(tile + 32 * k), TO_X, k > 0);
      };
      auto to_dp = [&](int t) {
        const uint32_t tile = tile_of(t) + TILE_BYTES;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
          umma_ss(tmem + M::DP, smem_desc_sw128(base + OWN_BYTES + 32 * k), smem_desc_sw128(tile + 32 * k), TO_X, k > 0);
      };
      mbar_wait_warp(wc, bars + BAR_OWN, 0);
      bool go = more(0);
      tc_fence_after();
      if (go && elect_one()) {
        to_x(0);
        umma_commit(bars + BAR_X);
        if (BWD) {
          to_dp(0);
          umma_commit(bars + BAR_DP);
        }
      }
      __syncwarp();
#pragma unroll 1
      for (int t = 0; go; ++t) {
        go = more(t + 1);
        if (go) {
          if (KIND == FWD && t > 0) mbar_wait_warp(wc, bars + BAR_ACC, (t - 1) & 1);   // the weights of tile t - 1 lie where x of t + 1 goes
          if (KIND != FWD) mbar_wait_warp(wc, bars + BAR_READ, t & 1);
          tc_fence_after();
          if (elect_one()) {
            to_x(t + 1);
            umma_commit(bars + BAR_X + (KIND == FWD ? 8 * ((t + 1) & 1) : 0));
          }
          __syncwarp();
        }
        mbar_wait_warp(wc, bars + BAR_W + 8 * (t & 1), (t >> 1) & 1);
        tc_fence_after();
        const uint32_t tile = tile_of(t);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < PARTNER / 16; ++k) {   // 16 partners: 8 columns of weights, 2048 bytes of a tile
            const uint32_t acc = (t > 0 || k > 0) ? 1u : 0u;
            if (KIND == FWD) umma_ts(tmem + M::ACC, tmem + M::X + 64 * (t & 1) + 8 * k, smem_desc_sw128(tile + TILE_BYTES + 2048 * k), TO_ACC, acc);
            if (BWD) {   // each half of dp's columns: p, then ds
              umma_ts(tmem + M::ACC + 64, tmem + M::DP + 32 * (k / 2) + 8 * (k % 2), smem_desc_sw128(tile + (KIND == DKV ? TILE_BYTES : 0) + 2048 * k), TO_ACC, acc);
              umma_ts(tmem + M::ACC, tmem + M::DP + 32 * (k / 2) + 16 + 8 * (k % 2), smem_desc_sw128(tile + 2048 * k), TO_ACC, acc);
            }
          }
          umma_commit(bars + BAR_EMPTY + 8 * (t % STAGES));
          umma_commit(bars + BAR_ACC);
        }
        __syncwarp();
        if (BWD && go) {
          mbar_wait_warp(wc, bars + BAR_ACC, t & 1);
          tc_fence_after();
          if (elect_one()) {
            to_dp(t + 1);
            umma_commit(bars + BAR_DP);
          }
          __syncwarp();
        }
      }
    }
  } else {
    // ================================ scores and weights, one thread per own row ================================
    const int r = ((warp & 3) << 5) + lane, row = o0 + r;
    const uint32_t tl = tmem + ((uint32_t)((warp & 3) << 5) << 16);
    const bool real = row >= lo && row < hi;
    const int64_t stat = ((int64_t)b * g.heads + h) * g.L + g.off(s) + row;   // DQ: this row's statistics
    float own_time = 0.f, limit = INFINITY, lse2 = INFINITY, delta = 0.f;
    int own_doc = 0;
    if (TIMES && real) own_time = time_of(g, a, b, s, row + rows.shift);
    if (MASK && real) {
      limit = KIND == DKV ? own_time : latest_seen(a, b, own_time);
      own_doc = document_of(g, a, b, s, row + rows.shift);
    }
    if (KIND == DQ) {
      const float lse = real ? a.lse[stat] : -INFINITY;
      if (lse != -INFINITY) {
        lse2 = lse * LOG2E;
        const bf16* po = static_cast<const bf16*>(a.out) + (own_row0 + row) * a.ldo + h * HD;
        const bf16* pg = static_cast<const bf16*>(a.dout) + (own_row0 + row) * a.lddo + h * HD;
#pragma unroll
        for (int c = 0; c < HD; c += 8) {
          float o8[8], g8[8];
          load_n(po + c, o8);
          load_n(pg + c, g8);
#pragma unroll
          for (int e = 0; e < 8; ++e) delta += o8[e] * g8[e];
        }
      }
    }
    float2 missed = make_float2(0.f, 0.f);   // DQ: see scored_bwd.cu
    float ref = 0.f, room = -INFINITY, sum = 0.f;   // FWD: see scored_fwd.cu
    int t = 0;
#pragma unroll 1
    for (; any; ++t) {
      const int st = t % STAGES;
      const bool ok = mbar_wait_warp(wc, bars + BAR_FULL + 8 * st, (t / STAGES) & 1);
      const Meta& m = metas[st];
      const int rem = uniform(m.rem);
      if (!ok || rem < 0) break;
      const bool some = uniform(m.some) != 0 || rem < PARTNER;
      const float slope2 = BIAS ? m.slope2 : 0.f;
      // which columns of [c, c + 4) are closed to this row
      auto shut = [&](int c, bool (&is)[4]) {
        const float4 l = *reinterpret_cast<const float4*>(m.limit + c);
        const int4 d = *reinterpret_cast<const int4*>(m.doc + c);
        const float lim[4] = {l.x, l.y, l.z, l.w};
        const int dc[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) is[e] = c + e >= rem || (MASK && ((KIND == DKV ? limit > lim[e] : lim[e] > limit) || dc[e] != own_doc));
      };
      auto bias = [&](int c, float2& x0, float2& x1) {
        const float4 tm = *reinterpret_cast<const float4*>(m.time + c);
        const float2 f = make_float2(-slope2, -slope2), d0 = __fadd2_rn(make_float2(tm.x, tm.y), make_float2(-own_time, -own_time)),
                     d1 = __fadd2_rn(make_float2(tm.z, tm.w), make_float2(-own_time, -own_time));
        x0 = __ffma2_rn(make_float2(fabsf(d0.x), fabsf(d0.y)), f, x0);
        x1 = __ffma2_rn(make_float2(fabsf(d1.x), fabsf(d1.y)), f, x1);
      };
      // Which form the tile's scores take: one decision for the warp, ahead of everything, so that the multiply-adds of some columns and the
      // exponentials of others are one stream of instructions.  Only real rows and columns take part: what padding holds must not
      // change the others' bits.
      auto in_form = [&](bool far, auto body) {
        if (CAP && __any_sync(0xffffffffu, real && far)) body(BoolTag<false>{}, BoolTag<true>{});
        else if (some) body(BoolTag<true>{}, BoolTag<true>{});
        else body(BoolTag<true>{}, BoolTag<false>{});
        __syncwarp();   // lanes may have taken different ways; accesses of tensor memory need the whole warp
      };
      const uint32_t x_at = tl + M::X + (KIND == FWD ? 64 * (t & 1) : 0);
      if (KIND == FWD) mbar_wait_warp(wc, bars + BAR_X + 8 * (t & 1), (t >> 1) & 1);
      else mbar_wait_warp(wc, bars + BAR_X, t & 1);
      tc_fence_after();
      if constexpr (KIND == FWD) {
        uint32_t xr[2][32];
        tmem_ld32(x_at, xr[0]);
        tmem_ld32(x_at + 32, xr[1]);
        tmem_wait_ld(xr[0], xr[1]);
        float x[PARTNER];
#pragma unroll
        for (int c = 0; c < PARTNER; ++c) x[c] = __uint_as_float(xr[c / 32][c % 32]);
        if (CAP && rem < PARTNER)
#pragma unroll
          for (int c = 0; c < PARTNER; ++c)
            if (c >= rem) x[c] = 0.f;
        uint32_t w[32];
        float top = -INFINITY, added = 0.f;
        in_form(CAP && largest(x) > a.near_dot, [&](auto near, auto some_shut) {
          float2 part[4] = {};
          float top4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < PARTNER; c += 4) {
            float2 none, y[2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
              y[e] = score_pair<CAP, false, decltype(near)::value>(make_float2(x[c + 2 * e], x[c + 2 * e + 1]), make_float2(ref, ref), none, a);
            if constexpr (BIAS) bias(c, y[0], y[1]);
            if constexpr (decltype(some_shut)::value) {
              bool is[4];
              shut(c, is);
#pragma unroll
              for (int e = 0; e < 2; ++e) y[e] = make_float2(is[2 * e] ? -INFINITY : y[e].x, is[2 * e + 1] ? -INFINITY : y[e].y);
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              top4[(c / 2 + e) % 4] = fmax3(top4[(c / 2 + e) % 4], y[e].x, y[e].y);
              x[c + 2 * e] = y[e].x;
              x[c + 2 * e + 1] = y[e].y;
              const float2 p = make_float2(ex2(y[e].x), ex2(y[e].y));
              part[(c / 2 + e) % 4] = __fadd2_rn(part[(c / 2 + e) % 4], p);
              w[c / 2 + e] = pack_bf16(p.x, p.y);
            }
          }
          added = sum_of(part);
          top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3]));
        });
        const bool grow = real && top > room;
        if (__any_sync(0xffffffffu, grow)) {   // rare: the weights once more, relative to a new reference, added up in the same order
          const float f = grow && room != -INFINITY ? ex2(-top) : 1.f;
          if (t > 0) {   // once the accumulator holds all earlier tiles
            mbar_wait_warp(wc, bars + BAR_ACC, (t - 1) & 1);
            tc_fence_after();
            sum *= f;
#pragma unroll
            for (int c = 0; c < HD; c += 16) {
              uint32_t o[16];
              tmem_ld16(tl + M::ACC + c, o);
              tmem_wait_ld(o);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
              tmem_st16(tl + M::ACC + c, o);
            }
          }
          const float shift = grow ? top : 0.f;
          if (grow) {
            ref += top;
            room = 8.f;
          }
          float2 part[4] = {};
#pragma unroll
          for (int c = 0; c < PARTNER; c += 2) {
            const float2 p = make_float2(ex2(x[c] - shift), ex2(x[c + 1] - shift));
            part[c / 2 % 4] = __fadd2_rn(part[c / 2 % 4], p);
            w[c / 2] = pack_bf16(p.x, p.y);
          }
          added = sum_of(part);
          __syncwarp();
        }
        sum += added;
        tmem_st32(x_at, w);
        // every warp sees every phase of this barrier: x of the next tile is there before this tile's products with weights are, so a warp
        // that is ahead of the others could else meet, in the end, the parity of two phases before the one it waits for
        if (t > 0) mbar_wait_warp(wc, bars + BAR_ACC, (t - 1) & 1);
      } else {
        uint32_t xr[2][32];   // x leaves its columns at once
        tmem_ld32(x_at, xr[0]);
        tmem_ld32(x_at + 32, xr[1]);
        tmem_wait_ld(xr[0], xr[1]);
        tc_fence_before();
        mbar_arrive(bars + BAR_READ);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          constexpr int N = 32;
          uint32_t dr[32];
          if (half == 0) {
            mbar_wait_warp(wc, bars + BAR_DP, t & 1);
            tc_fence_after();
          }
          tmem_ld32(tl + M::DP + N * half, dr);
          tmem_wait_ld(dr);
          float x[N];
#pragma unroll
          for (int c = 0; c < N; ++c) x[c] = __uint_as_float(xr[half][c]);
          if (CAP && rem < PARTNER)
#pragma unroll
            for (int c = 0; c < N; ++c)
              if (N * half + c >= rem) x[c] = 0.f;
          uint32_t wp[16], ws[16];
          in_form(CAP && largest(x) > a.near_dot, [&](auto near, auto some_shut) {
#pragma unroll
            for (int c = 0; c < N; c += 4) {
              float4 dl = make_float4(delta, delta, delta, delta), ls = make_float4(lse2, lse2, lse2, lse2);
              if (KIND == DKV) {
                dl = *reinterpret_cast<const float4*>(m.delta + N * half + c);
                ls = *reinterpret_cast<const float4*>(m.lse + N * half + c);
              }
              float2 d[2] = {__fadd2_rn(make_float2(__uint_as_float(dr[c]), __uint_as_float(dr[c + 1])), make_float2(-dl.x, -dl.y)),
                             __fadd2_rn(make_float2(__uint_as_float(dr[c + 2]), __uint_as_float(dr[c + 3])), make_float2(-dl.z, -dl.w))};
              float2 bend[2], y[2] = {score_pair<CAP, true, decltype(near)::value>(make_float2(x[c], x[c + 1]), make_float2(ls.x, ls.y), bend[0], a),
                                      score_pair<CAP, true, decltype(near)::value>(make_float2(x[c + 2], x[c + 3]), make_float2(ls.z, ls.w), bend[1], a)};
              if constexpr (BIAS) bias(N * half + c, y[0], y[1]);
              if constexpr (decltype(some_shut)::value) {   // rows past the last hold whatever follows in memory: neither factor may be NaN
                bool is[4];
                shut(N * half + c, is);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  y[e] = make_float2(is[2 * e] ? -INFINITY : y[e].x, is[2 * e + 1] ? -INFINITY : y[e].y);
                  d[e] = make_float2(is[2 * e] ? 0.f : d[e].x, is[2 * e + 1] ? 0.f : d[e].y);
                }
              }
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float2 p = make_float2(ex2(y[e].x), ex2(y[e].y)), pb = KIND == DQ ? times_bend<CAP>(p, bend[e]) : p;
                const float2 ds = KIND == DQ ? __fmul2_rn(pb, d[e]) : __fmul2_rn(p, times_bend<CAP>(d[e], bend[e]));
                if (KIND == DQ) missed = CAP ? __ffma2_rn(p, d[e], missed) : __fadd2_rn(missed, ds);
                wp[c / 2 + e] = pack_bf16(pb.x, pb.y);
                ws[c / 2 + e] = pack_bf16(ds.x, ds.y);
              }
            }
          });
          tmem_st16(tl + M::DP + 32 * half, wp);
          tmem_st16(tl + M::DP + 32 * half + 16, ws);
        }
      }
      if (rem < PARTNER) {
        // Rows of the partner tiles past the last hold whatever follows in memory; a zero weight times NaN or Inf would poison the
        // accumulators, so clear them before those products read the tiles (the first products are over).
        const int which = (tid - 64) >> 6, at = rem + ((tid - 64) & 63);
        if (at < PARTNER) {
          const uint32_t line = base + M::TILES + st * 2 * TILE_BYTES + which * TILE_BYTES + at * 128;
#pragma unroll
          for (int c = 0; c < 8; ++c) st_shared_v4(line + 16 * c, 0, 0, 0, 0);
        }
        fence_async_smem();
      }
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(bars + BAR_W + 8 * (t & 1));
      __syncwarp();
      if (lane == 0) mbar_arrive(bars + BAR_EMPTY + 8 * st);
    }

    grid_dep_launch();   // see scored_tile.cuh
    // ---- results: each thread its own rows of 128 bytes; padded rows +0 ----
    const bool walked = t > 0;
    if (walked) {
      mbar_wait_warp(wc, bars + BAR_ACC, (t - 1) & 1);
      tc_fence_after();
    }
    float scale[2];
    if (KIND == FWD) {
      scale[0] = real && sum != 0.f ? 1.f / sum : 0.f;
      if (a.lse != nullptr && row < o_end)
        a.lse[((int64_t)b * g.heads + h) * a.Lq + a.q_off[s] + row] = real && sum != 0.f ? (ref + log2f(sum)) * LN2 : -INFINITY;
    } else {
      scale[0] = a.scale;
      scale[1] = 1.f;
    }
    float more = 0.f;
    if (KIND == DQ) {
      if (lse2 != INFINITY) more = missed.x + missed.y;
      delta += more;
      if (row < o_end) a.row_stats[stat] = make_float2(lse2, delta);
    }
    const bool store = real && (KIND == FWD ? scale[0] != 0.f : KIND == DQ ? lse2 != INFINITY : true);
    bool broken = MASK && store && KIND == FWD && !finite(sum);
    if (KIND == DQ) broken = broken || (MASK && store && !finite(delta));
#pragma unroll
    for (int k = 0; k < (KIND == DKV ? 2 : 1); ++k) {
      bf16* dst = KIND == FWD  ? static_cast<bf16*>(a.out) + (own_row0 + row) * a.ldo + h * HD
                  : KIND == DQ ? static_cast<bf16*>(a.dq) + (own_row0 + row) * a.lddq + h * HD
                  : k == 0     ? static_cast<bf16*>(a.dk) + (own_row0 + row) * a.lddk + h * HD
                               : static_cast<bf16*>(a.dv) + (own_row0 + row) * a.lddv + h * HD;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t v[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = 0u;
        if (walked) {
          tmem_ld32(tl + M::ACC + 64 * k + 32 * c, v);
          tmem_wait_ld(v);
        }
        if (KIND == DQ && walked) {
          uint32_t along[32];
          tmem_ld32(tl + M::ACC + 64 + 32 * c, along);
          tmem_wait_ld(along);
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) - more * __uint_as_float(along[e]));
        }
        if (row < o_end) {
#pragma unroll
          for (int e = 0; e < 32; e += 8) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float f0 = __uint_as_float(v[e + 2 * i]) * scale[k], f1 = __uint_as_float(v[e + 2 * i + 1]) * scale[k];
              if (MASK && store) broken = broken || !finite(f0) || !finite(f1);
              w[i] = store ? pack_bf16(f0, f1) : 0u;
            }
            *reinterpret_cast<uint4*>(dst + 32 * c + e) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
    }
    if (MASK) {   // zero times NaN or Inf of a closed partner: those rows once more, pair by pair
      uint32_t again = __ballot_sync(0xffffffffu, broken);
      while (again != 0) {
        const int at = o0 + ((warp & 3) << 5) + __ffs(again) - 1;
        again &= again - 1;
        if constexpr (KIND == FWD) attend_row<bf16>(g, a, b, h, s, at);
        else if constexpr (KIND == DQ) dq_row<bf16>(g, a, b, h, s, at);
        else dkv_row<bf16>(g, a, b, h, s, at);
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, M::TMEM);
  }
}

template <int KIND, bool CAP, bool BIAS>
cudaError_t launch_masked(const Maps& maps, const Geometry& g, const ScoredArgs& a, const Tiles& t, dim3 grid, cudaStream_t st) {
  const auto kernel = rule_masks(a) ? scored_tc_kernel<KIND, CAP, BIAS, true> : scored_tc_kernel<KIND, CAP, BIAS, false>;
  const cudaError_t e = sm_count_and_smem_once(reinterpret_cast<const void*>(kernel), Map<KIND>::BYTES, nullptr);
  if (e != cudaSuccess) return e;
  return launch_overlapped(kernel, grid, dim3(THREADS), Map<KIND>::BYTES, st, maps, g, a, t);
}
template <int KIND>
cudaError_t launch(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  alignas(64) Maps maps;
  const int64_t rows = (int64_t)g.batch * g.L, q_rows = (int64_t)g.batch * a.Lq;
  const int kd = a.kv_heads * HD;
  const bool ok = KIND == FWD  ? make_map(&maps.own0, a.q, q_rows, g.d, a.ldq, HD, OWN) && make_map(&maps.own1, a.q, q_rows, g.d, a.ldq, HD, OWN) &&
                                    make_map(&maps.partner0, a.k, rows, kd, a.ldk, HD, PARTNER) && make_map(&maps.partner1, a.v, rows, kd, a.ldv, HD, PARTNER)
                  : KIND == DQ ? make_map(&maps.own0, a.q, rows, g.d, a.ldq, HD, OWN) && make_map(&maps.own1, a.dout, rows, g.d, a.lddo, HD, OWN) &&
                                     make_map(&maps.partner0, a.k, rows, kd, a.ldk, HD, PARTNER) && make_map(&maps.partner1, a.v, rows, kd, a.ldv, HD, PARTNER)
                               : make_map(&maps.own0, a.k, rows, kd, a.ldk, HD, OWN) && make_map(&maps.own1, a.v, rows, kd, a.ldv, HD, OWN) &&
                                     make_map(&maps.partner0, a.q, rows, g.d, a.ldq, HD, PARTNER) && make_map(&maps.partner1, a.dout, rows, g.d, a.lddo, HD, PARTNER);
  if (!ok) return cudaErrorInvalidValue;
  Tiles t = {};
  t.order = segment_order(g, KIND == DKV ? transposed(g.allowed) : g.allowed);
  const int64_t n = make_tiles(&t, KIND == FWD ? a.q_len : g.seg_len, OWN) * (KIND == DKV ? a.kv_heads : g.heads) * g.batch;
  if (n > 0x7fffffffLL) return cudaErrorNotSupported;
  const dim3 grid((unsigned)n);
  const bool cap = a.softcap > 0.f, bias = a.slopes != nullptr;
  return cap ? (bias ? launch_masked<KIND, true, true>(maps, g, a, t, grid, st) : launch_masked<KIND, true, false>(maps, g, a, t, grid, st))
             : (bias ? launch_masked<KIND, false, true>(maps, g, a, t, grid, st) : launch_masked<KIND, false, false>(maps, g, a, t, grid, st));
}

}  // namespace

// Whether these kernels serve a call, or the mma.sync tiles.  A tile of 128 x 64 pairs takes about as long here as 64 x 51 there, a CTA's own time
// 3.5 tiles (tensor memory, barriers, the first and last trips) and 1.5; and here a walk goes in whole tiles.  Fitted to calls without masks, forward /
// gradients, us, here and there, 8 heads:  16 x (50, 500, 500) 40 / 113 and 55 / 187;  4 x (128, 1024, 1024) 27 / 75 and 50 / 187;  64 x (100, 100,
// 100) 39 / 105 and 37 / 129;  64 x (39, 55, 400) 73 / 182 and 51 / 179;  4 heads, 512 x (50, 50, 50) 107 / 254 and 57 / 193;  8 heads, 4 key
// heads, all pairs, 64 x (17, 15, 173) 76 / 201 and 53 / 162, 4 x (27, 13, 898) 43 / 125 and 45 / 169.
bool scored_tc_preferred(const Geometry& g, const int (&rows)[3]) {
  if (g.hd != HD) return false;
  int64_t here = 0, there = 0;   // in quarters of a tile's time, 64 of them to a key
  for (int s = 0; s < 3; ++s) {
    int64_t tiles = 0, keys = 0;
    for (int r = 0; r < 3; ++r)
      if ((g.allowed >> (3 * s + r)) & 1u) {
        tiles += (g.seg_len[r] + PARTNER - 1) / PARTNER;
        keys += g.seg_len[r];
      }
    here += (int64_t)((rows[s] + OWN - 1) / OWN) * 64 * (4 * tiles + 14);
    there += (int64_t)((rows[s] + 63) / 64) * (5 * keys + 64 * 6);
  }
  return here <= there;
}

cudaError_t launch_scored_fwd_tc(const Geometry& g, const ScoredArgs& a, cudaStream_t st) { return launch<FWD>(g, a, st); }

cudaError_t launch_scored_bwd_tc(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  const cudaError_t e = launch<DQ>(g, a, st);
  return e != cudaSuccess ? e : launch<DKV>(g, a, st);
}

}  // namespace gsit

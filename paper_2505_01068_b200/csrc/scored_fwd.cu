// Scored attention, forward, bf16: flash-style tiles on mma.sync (see scored_tile.cuh), scores in registers, running reference and sum.
#include "scored_tile.cuh"

namespace gsit {
namespace {

template <int HD, int MT, int W, bool CAP, bool BIAS, bool MASK>
__global__ void __launch_bounds__(32 * W)
scored_fwd_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const __grid_constant__ Tiles tiles) {
  constexpr int KC = CHUNK_ROWS<HD>, CH = HD / 8, TQ = 16 * MT * W, NT = HD <= 16 ? 8 : 4, STEP = 8 * NT;
  constexpr bool TIMES = BIAS || MASK;
  __shared__ __align__(128) uint8_t s_k[2][KC * HD * 2], s_v[2][KC * HD * 2];
  __shared__ __align__(16) float s_time[2][TIMES ? KC : 4];
  __shared__ int s_doc[2][MASK ? KC : 1];
  const int tid = threadIdx.x, warp = ptx::uniform(tid >> 5), lane = tid & 31;
  const int h = blockIdx.x % g.heads, b = blockIdx.y, hk = h / a.group;
  int s;
  const int tile = find_tile(tiles, blockIdx.x / g.heads, s);
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();

  const int q0 = tile * TQ, q_end = min(q0 + TQ, a.q_len[s]);
  const QueryRows rows = query_rows(g, a, b, s);
  int n_keys[3], chunks = 0, first_chunk[3];
#pragma unroll
  for (int r = 0; r < 3; ++r) {
    n_keys[r] = ((g.allowed >> (3 * s + r)) & 1u) ? valid_rows(g, b, r) : 0;
    first_chunk[r] = chunks;
    chunks += (n_keys[r] + KC - 1) / KC;
  }
  if (max(q0, rows.lo) >= min(q_end, rows.hi)) chunks = 0;

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
      if (TIMES && real[m][i]) {
        own_time[m][i] = time_of(g, a, b, s, row + rows.shift);
        limit[m][i] = latest_seen(a, b, own_time[m][i]);
        own_doc[m][i] = document_of(g, a, b, s, row + rows.shift);
        mine.t_lo = min(mine.t_lo, ordered(limit[m][i]));
        mine.t_hi = max(mine.t_hi, ordered(limit[m][i]));
        mine.d_lo = min(mine.d_lo, own_doc[m][i]);
        mine.d_hi = max(mine.d_hi, own_doc[m][i]);
      } else {
        own_time[m][i] = 0.f;
        limit[m][i] = INFINITY;
        own_doc[m][i] = 0;
      }
    }
    own_rows<HD>(p[0], p[1], lane, qf[m]);
  }
  if (MASK) mine = warp_range(mine.t_lo, mine.t_hi, mine.d_lo, mine.d_hi);
  const bool working = w0 < min(q_end, rows.hi) && w0 + 16 * MT > rows.lo;
  const float slope2 = BIAS ? a.slopes[h] * LOG2E : 0.f;

  // ---- staging ----
  auto segment_of_chunk = [&](int c) { return c >= first_chunk[2] && n_keys[2] > 0 ? 2 : c >= first_chunk[1] && n_keys[1] > 0 ? 1 : 0; };
  auto stage = [&](int c) {
    const int r = segment_of_chunk(c), j0 = (c - first_chunk[r]) * KC, buf = c & 1;
    const int rem = n_keys[r] - j0, need = min(KC, (rem + BLOCK - 1) / BLOCK * BLOCK);   // rows past the last block are not read
    const int64_t row0 = (int64_t)b * g.L + g.off(r) + j0;
    const bf16 *k = static_cast<const bf16*>(a.k) + (int64_t)hk * HD, *v = static_cast<const bf16*>(a.v) + (int64_t)hk * HD;
    const uint32_t dk = smem_u32(s_k[buf]), dv = smem_u32(s_v[buf]);
    for (int i = tid; i < need * CH; i += 32 * W) {
      const int row = i / CH, c16 = i % CH;
      const bool in = row < rem;
      const int64_t at = row0 + (in ? row : 0);
      cp16(dk + piece_at<HD>(row, c16), k + at * a.ldk + 8 * c16, in);
      cp16(dv + piece_at<HD>(row, c16), v + at * a.ldv + 8 * c16, in);
    }
    cp_commit();
    if (TIMES)
      for (int i = tid; i < need; i += 32 * W) {
        s_time[buf][i] = i < rem ? time_of(g, a, b, r, j0 + i) : 0.f;
        if (MASK) s_doc[buf][i] = i < rem ? document_of(g, a, b, r, j0 + i) : 0;
      }
  };

  float o[MT][CH][4], ref[MT][2];
  float2 sum[MT][2];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[m][c][e] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      ref[m][i] = -INFINITY;
      sum[m][i] = make_float2(0.f, 0.f);
    }
  }

  if (chunks > 0) stage(0);
  for (int c = 0; c < chunks; ++c) {
    cp_wait();
    __syncthreads();   // chunk c is there, and nobody reads the other buffer any more
    if (c + 1 < chunks) stage(c + 1);
    if (!working) continue;
    const int r = segment_of_chunk(c), buf = c & 1, rem = min(KC, n_keys[r] - (c - first_chunk[r]) * KC);
    const uint32_t bk = smem_u32(s_k[buf]), bv = smem_u32(s_v[buf]);
    for (int j0 = 0; j0 < rem; j0 += BLOCK) {
      Openness open = ALL;
      if (MASK) {
        Range theirs = NO_ROWS;
#pragma unroll
        for (int i = 0; i < BLOCK; i += 32)
          if (j0 + i + lane < rem) {
            const int t = ordered(s_time[buf][j0 + i + lane]), d = s_doc[buf][j0 + i + lane];
            theirs = {min(theirs.t_lo, t), max(theirs.t_hi, t), min(theirs.d_lo, d), max(theirs.d_hi, d)};
          }
        open = openness(mine, warp_range(theirs.t_lo, theirs.t_hi, theirs.d_lo, theirs.d_hi));
        if (open == SHUT) continue;
      }
#pragma unroll 1
      for (int j = j0; j < min(j0 + BLOCK, rem); j += STEP) {
        float x[MT][NT][4], unused[1][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[m][n][e] = 0.f;
        product_over_features<HD, MT, NT>(x, qf, bk, j, lane);
        uint32_t w[MT][NT][2];
        const bool ragged = j + STEP > rem;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          bend_scores<CAP, false, NT>(x[m], unused, a.inner, a.outer, a.bend_scale);
          if (BIAS) add_bias<NT>(x[m], own_time[m], s_time[buf] + j, lane, slope2);
          if (ragged || (MASK && open == SOME)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int col = j + 8 * n + 2 * (lane & 3) + e;
                const bool in = col < rem;
#pragma unroll
                for (int i = 0; i < 2; ++i)
                  if (!in || (MASK && (s_time[buf][col] > limit[m][i] || s_doc[buf][col] != own_doc[m][i]))) x[m][n][2 * i + e] = -INFINITY;
              }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < NT; ++n) top = ptx::fmax3(top, x[m][n][2 * i], x[m][n][2 * i + 1]);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // the reference follows the maximum only when it has grown by more than 2^8: weights stay below 256
            const bool grow = top > ref[m][i] + 8.f;
            if (__any_sync(0xffffffffu, grow)) {
              const float f = grow ? ptx::ex2(ref[m][i] - top) : 1.f;
              sum[m][i] = __fmul2_rn(sum[m][i], make_float2(f, f));
#pragma unroll
              for (int q = 0; q < CH; ++q) {
                o[m][q][2 * i] *= f;
                o[m][q][2 * i + 1] *= f;
              }
              if (grow) ref[m][i] = top;
            }
            // a row that has seen no open key yet keeps weights of zero
            const float nr = ref[m][i] == -INFINITY ? 0.f : -ref[m][i];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const float2 y = __fadd2_rn(make_float2(x[m][n][2 * i], x[m][n][2 * i + 1]), make_float2(nr, nr));
              const float2 p = make_float2(ptx::ex2(y.x), ptx::ex2(y.y));
              sum[m][i] = __fadd2_rn(sum[m][i], p);
              w[m][n][i] = ptx::pack_bf16(p.x, p.y);
            }
          }
        }
        product_over_partners<HD, MT, NT>(o, w, bv, j, lane);
      }
    }
  }

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

template <int HD, int MT, int W, bool CAP, bool BIAS>
cudaError_t launch_masked(const Geometry& g, const ScoredArgs& a, const Tiles& t, dim3 grid, cudaStream_t st) {
  return rule_masks(a) ? launch_overlapped(scored_fwd_kernel<HD, MT, W, CAP, BIAS, true>, grid, dim3(32 * W), 0, st, g, a, t)
                       : launch_overlapped(scored_fwd_kernel<HD, MT, W, CAP, BIAS, false>, grid, dim3(32 * W), 0, st, g, a, t);
}
template <int HD, int MT, int W>
cudaError_t launch_rule(const Geometry& g, const ScoredArgs& a, const Tiles& t, dim3 grid, cudaStream_t st) {
  const bool cap = a.softcap > 0.f, bias = a.slopes != nullptr;
  return cap ? (bias ? launch_masked<HD, MT, W, true, true>(g, a, t, grid, st) : launch_masked<HD, MT, W, true, false>(g, a, t, grid, st))
             : (bias ? launch_masked<HD, MT, W, false, true>(g, a, t, grid, st) : launch_masked<HD, MT, W, false, false>(g, a, t, grid, st));
}
template <int HD>
cudaError_t launch_width(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  int n_sm = 0;
  const cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  Tiles t = {};
  t.order = segment_order(g, g.allowed);
  // 128 rows a CTA where that still makes several CTAs per SM, 64 below
  const bool tall = make_tiles(&t, a.q_len, 128) * g.heads * g.batch >= 6LL * n_sm;
  const int64_t n = make_tiles(&t, a.q_len, tall ? 128 : 64) * g.heads;
  if (n > 0x7fffffffLL) return cudaErrorNotSupported;
  const dim3 grid((unsigned)n, g.batch);
  constexpr int MT = HD == 64 ? 2 : 1;
  return tall ? launch_rule<HD, MT, 8 / MT>(g, a, t, grid, st) : launch_rule<HD, 1, 4>(g, a, t, grid, st);
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

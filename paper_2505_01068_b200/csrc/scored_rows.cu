// Attention with a rule on its scores, row by row: a warp takes one query row (forward, dq) or one key row (dk, dv).  For float heads
// wider than the tiles of scored_f32.cu, which no configuration of the models has: kept simple.  A pair costs a shuffle tree and a trip
// to L2 that nothing overlaps; 8 samples of (30, 480, 230), 4 heads of 96, inter pattern: 754 us forward, 1.95 ms gradients.
#include "scored.cuh"

namespace gsit {
namespace {

constexpr int WARPS = 4;

enum Pass { FWD, DQ, DKV };

// Rows of the grid: (row of Lq or L) x heads x batch, one warp each.
template <typename T, int PASS>
__global__ void __launch_bounds__(32 * WARPS) scored_rows_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a) {
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int p = blockIdx.x * WARPS + (threadIdx.x >> 5), h = blockIdx.y, b = blockIdx.z;
  if (p >= (PASS == FWD ? a.Lq : g.L)) return;
  const int s = PASS == FWD ? ((p >= a.q_off[2]) ? 2 : (p >= a.q_off[1]) ? 1 : 0) : segment_of(g, p);
  const int i = p - (PASS == FWD ? a.q_off[s] : g.off(s));
  if constexpr (PASS == FWD) attend_row<T>(g, a, b, h, s, i);
  else if constexpr (PASS == DQ) dq_row<T>(g, a, b, h, s, i);
  else dkv_row<T>(g, a, b, h, s, i);
}

template <typename T, int PASS>
cudaError_t launch(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  const dim3 grid(((PASS == FWD ? a.Lq : g.L) + WARPS - 1) / WARPS, PASS == DKV ? a.kv_heads : g.heads, g.batch), block(32 * WARPS);
  return launch_overlapped(scored_rows_kernel<T, PASS>, grid, block, 0, st, g, a);
}

}  // namespace

cudaError_t launch_scored_rows_fwd(const Geometry& g, const ScoredArgs& a, cudaStream_t st) { return launch<float, FWD>(g, a, st); }

cudaError_t launch_scored_rows_bwd(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  const cudaError_t e = launch<float, DQ>(g, a, st);
  return e != cudaSuccess ? e : launch<float, DKV>(g, a, st);
}

}  // namespace gsit

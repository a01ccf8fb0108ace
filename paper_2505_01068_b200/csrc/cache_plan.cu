// Pages and slots for a step of streams (gsit_cache_plan): which blocks open, which pages they get, and where each row goes.
//
// An entry is a (stream, segment).  A warp takes an entry, its lanes 32 blocks of the entry's table at a time, so what an entry needs
// and gives back are ballots; an exclusive scan over all entries, in order, says which pages of the list are whose: no atomics on the
// list, the same pages for the same call every time.  Entries are cut into runs, one to a CTA of a single cluster (one CTA up to
// some hundred entries, eight beyond), which exchange their sums through distributed shared memory.  What an entry reads and writes -- its length, its row of
// the table, its rows' slots -- only its warp touches, so lengths may be updated in place.
// Bound by the chain of dependent loads (count, length, table, list) and the launch.
#include <cooperative_groups.h>

#include "cache.cuh"

namespace gsit {
namespace {

namespace cg = cooperative_groups;

constexpr int THREADS = 1024, WARPS = THREADS / 32;
constexpr int MAX_CTAS = 8;
constexpr int MAX_ENTRIES = 24576;          // of a CTA: 3 * 65535 / 8 and less

struct Sums {
  int need, back;
};

__global__ void __launch_bounds__(THREADS) cache_plan_kernel(const __grid_constant__ Geometry g, const __grid_constant__ Cache c, const int32_t* const held,
                                                             const int32_t* const ended, int32_t* const slots, const int per_cta) {
  extern __shared__ Sums entry[];           // of each entry of this CTA: first its own, then those of all entries before it
  __shared__ Sums s_warp[WARPS], s_total;
  __shared__ int s_used;
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
  const int first = rank * per_cta, here = max(0, min(per_cta, 3 * g.batch - first));
  const uint32_t below = (1u << lane) - 1u;
  ptx::load_params_early(g, c);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();

  struct Entry {
    int old, add, from, to;                 // positions held and added, the blocks [from, to) that the rows lie in
    bool gone, room;
  };
  auto look = [&](int e) {
    Entry x;
    const int b = e / 3, s = e - 3 * b, most = c.blocks * CACHE_BLOCK;
    x.gone = ended != nullptr && ended[b] != 0;
    x.add = valid_rows(g, b, s);
    int n = held != nullptr ? held[e] : c.lengths[e];
    if (n < 0 || n > most) {
      raise_flag(g, GSIT_DEVFLAG_CLAMPED);
      n = n < 0 ? 0 : most;
    }
    x.old = x.gone ? 0 : n;
    x.room = x.add <= most - x.old;
    x.from = x.old / CACHE_BLOCK;
    x.to = x.room && x.add > 0 ? (x.old + x.add + CACHE_BLOCK - 1) / CACHE_BLOCK : x.from;
    return x;
  };

  // what every entry needs and gives back
  for (int i = warp; i < here; i += WARPS) {
    const Entry x = look(first + i);
    const int32_t* table = c.tables + (int64_t)(first + i) * c.blocks;
    Sums n = {x.gone ? x.to - x.from : 0, 0};
    if (x.gone) {
      for (int j = lane; j < c.blocks + lane; j += 32) n.back += __popc(__ballot_sync(0xffffffffu, j < c.blocks && table[j] >= 0));
    } else {
      for (int j = x.from + lane; j < x.to + lane; j += 32) n.need += __popc(__ballot_sync(0xffffffffu, j < x.to && table[j] < 0));
    }
    if (lane == 0) entry[i] = n;
  }
  if (tid == 0) s_used = 0;
  __syncthreads();
  // sums over the entries before each one of this CTA
  const int per = (here + THREADS - 1) / THREADS, lo = min(here, tid * per), hi = min(here, lo + per);
  Sums mine = {0, 0};
  for (int i = lo; i < hi; ++i) {
    mine.need += entry[i].need;
    mine.back += entry[i].back;
  }
  Sums upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int need = __shfl_up_sync(0xffffffffu, upto.need, o), back = __shfl_up_sync(0xffffffffu, upto.back, o);
    if (lane >= o) {
      upto.need += need;
      upto.back += back;
    }
  }
  if (lane == 31) s_warp[warp] = upto;
  __syncthreads();
  if (warp == 0) {
    Sums w = s_warp[lane];
    const Sums own = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int need = __shfl_up_sync(0xffffffffu, w.need, o), back = __shfl_up_sync(0xffffffffu, w.back, o);
      if (lane >= o) {
        w.need += need;
        w.back += back;
      }
    }
    s_warp[lane] = {w.need - own.need, w.back - own.back};
    if (lane == 31) s_total = w;
  }
  const int list = min(max(*c.n_free, 0), c.pages);   // read by every CTA before the first barrier, written behind the last one
  cluster.sync();
  Sums before = {0, 0}, all = {0, 0};
  for (int r = 0; r < ctas; ++r) {
    const Sums t = *cluster.map_shared_rank(&s_total, r);
    if (r < rank) {
      before.need += t.need;
      before.back += t.back;
    }
    all.need += t.need;
    all.back += t.back;
  }
  Sums run = {before.need + s_warp[warp].need + upto.need - mine.need, before.back + s_warp[warp].back + upto.back - mine.back};
  for (int i = lo; i < hi; ++i) {
    const Sums n = entry[i];
    entry[i] = run;
    run.need += n.need;
    run.back += n.back;
  }
  __syncthreads();
  const int avail = min(list + all.back, c.pages);
  // pages of ended streams go back, the first of them on top
  if (all.back > 0) {
    for (int i = warp; i < here; i += WARPS) {
      const int e = first + i;
      if (ended[e / 3] == 0) continue;
      int32_t* table = c.tables + (int64_t)e * c.blocks;
      int rank_of = entry[i].back;
      for (int j = lane; j < c.blocks + lane; j += 32) {
        const int page = j < c.blocks ? table[j] : -1;
        const uint32_t has = __ballot_sync(0xffffffffu, page >= 0);
        const int at = list + all.back - 1 - (rank_of + __popc(has & below));
        if (page >= 0) {
          if (at < c.pages) c.free_list[at] = page;
          table[j] = -1;
        }
        rank_of += __popc(has);
      }
    }
    cluster.sync();
  }
  // pages for blocks that open, slots, lengths
  for (int i = warp; i < here; i += WARPS) {
    const int e = first + i, b = e / 3, s = e - 3 * b;
    const Entry x = look(e);
    int32_t* table = c.tables + (int64_t)e * c.blocks;
    int32_t* out = slots + (int64_t)b * g.L + g.off(s);
    int rank_of = entry[i].need, need = 0;
    for (int j = x.from + lane; j < x.to + lane; j += 32) need += __popc(__ballot_sync(0xffffffffu, j < x.to && table[j] < 0));
    const bool taken = x.room && (need == 0 || rank_of + need <= avail);
    const int add = taken ? x.add : 0;
    for (int j0 = x.from; taken && j0 < x.to; j0 += 32) {
      const int j = j0 + lane;
      int page = j < x.to ? table[j] : 0;
      const uint32_t lacks = __ballot_sync(0xffffffffu, page < 0);
      if (page < 0) {
        page = c.free_list[avail - 1 - (rank_of + __popc(lacks & below))];
        table[j] = page;
      }
      rank_of += __popc(lacks);
      for (int k = 0; k < min(32, x.to - j0); ++k) {
        const int p = __shfl_sync(0xffffffffu, page, k), row = (j0 + k) * CACHE_BLOCK + lane - x.old;
        if (row >= 0 && row < add) out[row] = p * CACHE_BLOCK + lane;
      }
    }
    for (int row = add + lane; row < g.len(s); row += 32) out[row] = -1;
    __syncwarp();   // every lane has read the old length
    if (lane == 0) {
      c.lengths[e] = x.old + add;
      if (need > 0 && taken) atomicMax(&s_used, entry[i].need + need);
      if (!taken && x.add > 0) raise_flag(g, GSIT_DEVFLAG_FULL);
    }
  }
  cluster.sync();
  if (rank == 0 && tid == 0) {
    int used = 0;
    for (int r = 0; r < ctas; ++r) used = max(used, *cluster.map_shared_rank(&s_used, r));
    *c.n_free = avail - used;
  }
  cluster.sync();   // nobody's shared memory goes away while it is read
}

}  // namespace

cudaError_t launch_cache_plan(const Geometry& g, const Cache& c, const int32_t* held, const int32_t* ended, int32_t* slots, cudaStream_t st) {
  const int entries = 3 * g.batch, ctas = entries <= 192 ? 1 : MAX_CTAS, per = (entries + ctas - 1) / ctas;
  if (per > MAX_ENTRIES) return cudaErrorNotSupported;
  const cudaError_t e = sm_count_and_smem_once(reinterpret_cast<const void*>(cache_plan_kernel), MAX_ENTRIES * (int)sizeof(Sums), nullptr);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = per * sizeof(Sums);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, cache_plan_kernel, g, c, held, ended, slots, per);
}

}  // namespace gsit

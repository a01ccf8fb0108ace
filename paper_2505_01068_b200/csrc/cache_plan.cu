// Pages and slots for a step of streams (gsit_cache_plan): which blocks open, which pages they get, and where each row goes.
//
// An entry is a (stream, segment).  A lane takes an entry while all it needs is a few blocks (a step of some hundred rows), so that the entries of a
// warp wait for memory together; a warp takes the longer ones, and the rows of tables of streams that have ended, 32 blocks at a time.  An exclusive
// scan over all entries, in order, says which pages of the list are whose: no atomics on the list, the same pages for the same call every time.  Entries
// are cut into runs, one to a CTA of a single cluster (one CTA up to 192 entries, eight beyond), which exchange their sums through distributed shared
// memory.  What an entry reads and writes -- its length, its row of the table, its rows' slots -- only its warp touches, so lengths may be updated in place.
// Rows' slots are written here as long as there are few entries; beyond, only that of each entry's first row, and a second kernel on all SMs fills in
// the others (1024 streams of up to (16, 100, 100) rows: eight SMs took 21 us for all of it).
// Bound by the chain of dependent loads (count and length, table, list) and the launches: 32 streams' step 5.2 us, 1024 streams' prompts 16.
#include <cooperative_groups.h>

#include "cache.cuh"

namespace gsit {
namespace {

namespace cg = cooperative_groups;

constexpr int THREADS = 1024, WARPS = THREADS / 32;
constexpr int MAX_CTAS = 8;

constexpr int FEW = 8;                      // blocks that a lane looks after

struct Sums {
  int need, back;
};
struct Entry {
  int old, add, from, to;                   // positions held and added, the blocks [from, to) that the rows lie in
  int need, back;                           // pages it takes and gives back
  bool gone, room, few;
};
__device__ __forceinline__ Sums warp_upto(Sums v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int need = __shfl_up_sync(0xffffffffu, v.need, o), back = __shfl_up_sync(0xffffffffu, v.back, o);
    if (lane >= o) {
      v.need += need;
      v.back += back;
    }
  }
  return v;
}

__global__ void __launch_bounds__(THREADS) cache_plan_kernel(const __grid_constant__ Geometry g, const __grid_constant__ Cache c, const int32_t* const held,
                                                             const int32_t* const ended, int32_t* const slots, const int per_cta, const bool first_rows) {
  __shared__ Sums s_warp[WARPS], s_total;
  __shared__ int s_used, s_page[WARPS][32][FEW + 1];
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, warp = ptx::uniform(tid >> 5), lane = tid & 31, rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
  const uint32_t below = (1u << lane) - 1u;
  // this warp's run of entries: [first, last), 32 at a time
  const int cta_last = min((rank + 1) * per_cta, 3 * g.batch), per_warp = (per_cta + WARPS - 1) / WARPS;
  const int first = min(cta_last, rank * per_cta + warp * per_warp), last = min(cta_last, first + per_warp);
  ptx::load_params_early(g, c);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();

  // Entry e of this lane (one that is there), or nothing; lanes of a warp look at theirs together.
  auto look = [&](int e) {
    Entry x = {0, 0, 0, 0, 0, 0, false, true, true};
    const bool mine = e < last;
    const int b = e / 3, s = e - 3 * b, most = c.blocks * CACHE_BLOCK;
    int32_t* const table = c.tables + (int64_t)(mine ? e : 0) * c.blocks;
    if (mine) {
      const int n = held != nullptr ? held[e] : c.lengths[e];
      x.add = valid_rows(g, b, s);
      x.gone = ended != nullptr && ended[b] != 0;
      if (n < 0 || n > most) raise_flag(g, GSIT_DEVFLAG_CLAMPED);
      x.old = x.gone ? 0 : min(max(n, 0), most);
      x.room = x.add <= most - x.old;
      x.from = x.old / CACHE_BLOCK;
      x.to = x.room && x.add > 0 ? (x.old + x.add + CACHE_BLOCK - 1) / CACHE_BLOCK : x.from;
      x.few = x.to - x.from <= FEW;
      if (x.gone) x.need = x.to - x.from;
      else if (x.few)
#pragma unroll
        for (int i = 0; i < FEW; ++i)
          if (x.from + i < x.to) x.need += table[x.from + i] < 0;
    }
    // the whole warp: long ones, and rows of the table that go back
    for (uint32_t todo = __ballot_sync(0xffffffffu, x.gone || !x.few); todo != 0; todo &= todo - 1) {
      const int k = __ffs(todo) - 1;
      const bool gone = __shfl_sync(0xffffffffu, x.gone, k);
      const int from = gone ? 0 : __shfl_sync(0xffffffffu, x.from, k), to = gone ? c.blocks : __shfl_sync(0xffffffffu, x.to, k);
      const int32_t* row = c.tables + (int64_t)__shfl_sync(0xffffffffu, e, k) * c.blocks;
      int n = 0;
      for (int j = from + lane; j < to + lane; j += 32) n += __popc(__ballot_sync(0xffffffffu, j < to && (row[j] < 0) != gone));
      if (lane == k) (gone ? x.back : x.need) = n;
    }
    return x;
  };

  // ---- sums over the entries before this warp's ----
  Sums mine = {0, 0};
  Entry x = look(first + lane);               // (kept where the warp has no more than these)
  for (int e0 = first; e0 < last; e0 += 32) {
    if (e0 > first) x = look(e0 + lane);
    mine.need += __reduce_add_sync(0xffffffffu, x.need);
    mine.back += __reduce_add_sync(0xffffffffu, x.back);
  }
  if (lane == 0) s_warp[warp] = mine;
  if (tid == 0) s_used = 0;
  const int list = min(max(*c.n_free, 0), c.pages);   // read by every CTA before the first barrier, written behind the last one
  __syncthreads();
  if (warp == 0) {
    const Sums own = s_warp[lane], upto = warp_upto(own, lane);
    s_warp[lane] = {upto.need - own.need, upto.back - own.back};
    if (lane == 31) s_total = upto;
  }
  __syncthreads();
  Sums run = s_warp[warp], all = s_total;
  if (ctas > 1) {
    cluster.sync();
    all = {0, 0};
    for (int r = 0; r < ctas; ++r) {
      const Sums t = *cluster.map_shared_rank(&s_total, r);
      if (r < rank) {
        run.need += t.need;
        run.back += t.back;
      }
      all.need += t.need;
      all.back += t.back;
    }
  }
  const int avail = min(list + all.back, c.pages);
  // ---- pages of ended streams go back, the first of them on top ----
  if (all.back > 0) {
    int before = run.back;
    for (int e0 = first; e0 < last; e0 += 32) {
      const int e = e0 + lane;
      for (uint32_t todo = __ballot_sync(0xffffffffu, e < last && ended[min(e, 3 * g.batch - 1) / 3] != 0); todo != 0; todo &= todo - 1) {
        int32_t* table = c.tables + (int64_t)(e0 + __ffs(todo) - 1) * c.blocks;
        for (int j = lane; j < c.blocks + lane; j += 32) {
          const int page = j < c.blocks ? table[j] : -1;
          const uint32_t has = __ballot_sync(0xffffffffu, page >= 0);
          const int at = list + all.back - 1 - (before + __popc(has & below));
          if (page >= 0) {
            if (at < c.pages) c.free_list[at] = page;
            table[j] = -1;
          }
          before += __popc(has);
        }
      }
    }
    if (ctas > 1) cluster.sync();
    else __syncthreads();
  }
  // ---- pages for blocks that open, slots, lengths ----
  for (int e0 = first; e0 < last; e0 += 32) {
    if (last - first > 32) x = look(e0 + lane);   // (lengths of these entries are as they were; rows of ended streams are empty now, and count as they did)
    const int e = e0 + lane;
    const Sums upto = warp_upto({x.need, 0}, lane);
    const int rank_of = run.need + upto.need - x.need;
    run.need += __shfl_sync(0xffffffffu, upto.need, 31);
    const bool taken = x.room && (x.need == 0 || rank_of + x.need <= avail);
    const int add = taken ? x.add : 0;
    if (e < last && x.few && add > 0) {
      int32_t* const table = c.tables + (int64_t)e * c.blocks + x.from;
      int page[FEW], n = 0;
#pragma unroll
      for (int i = 0; i < FEW; ++i) page[i] = x.from + i < x.to ? table[i] : 0;
#pragma unroll
      for (int i = 0; i < FEW; ++i)
        if (page[i] < 0) {
          page[i] = c.free_list[avail - 1 - (rank_of + n++)];
          table[i] = page[i];
        }
#pragma unroll
      for (int i = 0; i < FEW; ++i) s_page[warp][lane][i] = page[i];
    }
    __syncwarp();
    if (first_rows && e < last && g.len(e % 3) > 0 && (x.few || add == 0))
      slots[(int64_t)(e / 3) * g.L + g.off(e % 3)] = add > 0 ? s_page[warp][lane][0] * CACHE_BLOCK + x.old % CACHE_BLOCK : -1;
    // rows, an entry after the other; the lanes are rows
    for (uint32_t todo = __ballot_sync(0xffffffffu, e < last && (!first_rows || (!x.few && add > 0))); todo != 0; todo &= todo - 1) {
      const int k = __ffs(todo) - 1;
      const int from = __shfl_sync(0xffffffffu, x.from, k), to = __shfl_sync(0xffffffffu, x.to, k), old = __shfl_sync(0xffffffffu, x.old, k);
      const int n = __shfl_sync(0xffffffffu, add, k), rank_k = __shfl_sync(0xffffffffu, rank_of, k), b = (e0 + k) / 3, s = e0 + k - 3 * b;
      const bool few = __shfl_sync(0xffffffffu, x.few, k);
      int32_t* const out = slots + (int64_t)b * g.L + g.off(s);
      if (few) {
        for (int row = lane; row < n; row += 32) out[row] = s_page[warp][k][(old + row) / CACHE_BLOCK - from] * CACHE_BLOCK + (old + row) % CACHE_BLOCK;
      } else if (n > 0) {
        int32_t* const table = c.tables + (int64_t)(e0 + k) * c.blocks;
        int taken_of = rank_k;
        for (int j0 = from; j0 < to; j0 += 32) {
          int page = j0 + lane < to ? table[j0 + lane] : 0;
          const uint32_t lacks = __ballot_sync(0xffffffffu, page < 0);
          if (page < 0) {
            page = c.free_list[avail - 1 - (taken_of + __popc(lacks & below))];
            table[j0 + lane] = page;
          }
          taken_of += __popc(lacks);
          for (int i = 0; i < min(32, to - j0); ++i) {
            const int p = __shfl_sync(0xffffffffu, page, i), row = (j0 + i) * CACHE_BLOCK + lane - old;
            if (row >= 0 && row < n) out[row] = p * CACHE_BLOCK + lane;
          }
        }
      }
      for (int row = n + lane; row < g.len(s); row += 32) out[row] = -1;
    }
    if (e < last) {
      c.lengths[e] = x.old + add;
      if (x.need > 0 && taken) atomicMax(&s_used, rank_of + x.need);
      if (!taken && x.add > 0) raise_flag(g, GSIT_DEVFLAG_FULL);
    }
    __syncwarp();
  }
  if (ctas > 1) cluster.sync();
  else __syncthreads();
  if (rank == 0 && tid == 0) {
    int used = 0;
    for (int r = 0; r < ctas; ++r) used = max(used, *cluster.map_shared_rank(&s_used, r));
    *c.n_free = avail - used;
  }
  if (ctas > 1) cluster.sync();   // nobody's shared memory goes away while it is read
}

// Slots of the rows behind each entry's first one, which says whether it was taken.  A thread takes a row.
__global__ void __launch_bounds__(256) cache_slots_kernel(const __grid_constant__ Geometry g, const __grid_constant__ Cache c, int32_t* const slots) {
  ptx::load_params_early(g, c);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (r >= (int64_t)g.batch * g.L) return;
  const int b = (uint32_t)r / (uint32_t)g.L, l = (int)(r - (int64_t)b * g.L), s = segment_of(g, l), i = l - g.off(s);
  if (i == 0) return;
  const int n = valid_rows(g, b, s);
  int slot = -1;
  if (i < n && slots[r - i] >= 0) {
    const int at = c.lengths[3 * b + s] - n + i;
    slot = c.tables[(int64_t)(3 * b + s) * c.blocks + at / CACHE_BLOCK] * CACHE_BLOCK + at % CACHE_BLOCK;
  }
  slots[r] = slot;
}

}  // namespace

cudaError_t launch_cache_plan(const Geometry& g, const Cache& c, const int32_t* held, const int32_t* ended, int32_t* slots, cudaStream_t st) {
  const int entries = 3 * g.batch, ctas = entries <= 192 ? 1 : MAX_CTAS, per = (entries + ctas - 1) / ctas;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(THREADS);
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
  const bool wide = ctas > 1 && g.L > 3;   // (a row for each segment is all there is, else)
  const cudaError_t e = cudaLaunchKernelEx(&cfg, cache_plan_kernel, g, c, held, ended, slots, per, wide);
  if (e != cudaSuccess || !wide) return e;
  return launch_overlapped(cache_slots_kernel, dim3((unsigned)(((int64_t)g.batch * g.L + 255) / 256)), dim3(256), 0, st, g, c, slots);
}

}  // namespace gsit

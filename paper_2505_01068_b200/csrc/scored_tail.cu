// Scored attention for the newest positions of a stream: a handful of query rows against all keys (forward, float and bf16).
//
// The keys and values stream through once, which is all that bounds it, so the work is cut by keys, not by queries: the CTAs that share
// a (sample, key head) form a cluster, and every warp walks its own part of the keys with all query rows that read them -- those of the
// key head's query heads, in every segment.  Each warp keeps its own running reference, sum and weighted values; they are joined over
// the warps in shared memory and over the cluster through distributed shared memory, in a fixed order.
//   bf16   mma.sync on a ring of staged keys and values of each warp's own (scored_tail_tile_kernel): 32 samples of (128, 1024, 1024),
//          8 heads of 64, half of them padding: 107 MB in 28 us, 3.9 TB/s, 0.60 of the measured copy rate; what is left is the launch, the
//          first loads and the join, some 8 us, which small calls take whole
//   float  a lane owns 8 features of a key, so that a load instruction covers whole rows and a score needs log2(head_dim / 8) shuffles;
//          the same call without padding, 285 MB, 61 us, 4.7 TB/s
#include <cooperative_groups.h>

#include "scored_tile.cuh"

namespace gsit {
namespace {

namespace cg = cooperative_groups;

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int STEPS = 4;       // key steps whose loads are in flight together
constexpr int MAX_SPLIT = 8;   // CTAs of a cluster

struct TailRow {
  float time, limit, slope2;
  int doc, opens;              // opens: bit r set where key segment r is open to it
};

// What the parts of a row's softmax are joined through.
template <int HD, int R> struct JoinRoom {
  float acc[WARPS][R][HD], joined[R][HD];
  float2 ml[WARPS][R], joined_ml[R];   // (maximum, sum); a part without a key has a maximum of -inf and takes no part
  float scale[MAX_SPLIT > WARPS ? MAX_SPLIT : WARPS][R];
};
// acc and ml hold the warps' parts: adds them up, and those of the cluster's CTAs, in order; CTA 0 writes the results.  Whole CTAs.
template <typename T, int HD, int R>
__device__ __forceinline__ void join_warps_and_ctas(const Geometry& g, const ScoredArgs& a, JoinRoom<HD, R>& room, int b, int hk, int rank, int split, int n_rows) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid < R) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, room.ml[w][tid].x);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = room.ml[w][tid].x == -INFINITY ? 0.f : ptx::ex2(room.ml[w][tid].x - top);
      room.scale[w][tid] = f;
      sum += f * room.ml[w][tid].y;
    }
    room.joined_ml[tid] = make_float2(top, sum);
  }
  __syncthreads();
  for (int c = tid; c < R * HD; c += THREADS) {
    const int i = c / HD, f = c % HD;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w)
      if (room.scale[w][i] != 0.f) v += room.scale[w][i] * room.acc[w][i][f];
    room.joined[i][f] = v;
  }
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  if (rank == 0) {
    if (tid < R) {
      float top = -INFINITY, sum = 0.f;
      float2 ml[MAX_SPLIT];
      for (int c = 0; c < split; ++c) {
        ml[c] = cluster.map_shared_rank(room.joined_ml, c)[tid];
        top = fmaxf(top, ml[c].x);
      }
      for (int c = 0; c < split; ++c) {
        const float f = ml[c].x == -INFINITY ? 0.f : ptx::ex2(ml[c].x - top);
        room.scale[c][tid] = f;
        sum += f * ml[c].y;
      }
      room.ml[0][tid] = make_float2(top, sum);
    }
    __syncthreads();
    bool broken = false;
    for (int c = tid; c < n_rows * HD; c += THREADS) {
      const int i = c / HD, f = c % HD;
      float v = 0.f;
      for (int k = 0; k < split; ++k)
        if (room.scale[k][i] != 0.f) v += room.scale[k][i] * cluster.map_shared_rank(&room.joined[0][0], k)[c];
      const float sum = room.ml[0][i].y, o = sum != 0.f ? v / sum : 0.f;
      broken = broken || (__float_as_uint(o) & 0x7f800000u) == 0x7f800000u;
      store_as(static_cast<T*>(a.out) + ((int64_t)b * a.Lq + i / a.group) * a.ldo + (int64_t)(hk * a.group + i % a.group) * HD + f, o);
    }
    if (a.lse != nullptr && tid < n_rows) {
      const float2 ml = room.ml[0][tid];
      a.lse[((int64_t)b * g.heads + hk * a.group + tid % a.group) * a.Lq + tid / a.group] = ml.y != 0.f ? (ml.x + log2f(ml.y)) * LN2 : -INFINITY;
    }
    // zero times NaN or Inf of a closed key: the rows once more, pair by pair
    if (__syncthreads_or(broken))
      for (int i = tid >> 5; i < n_rows; i += WARPS) {
        const int p = i / a.group, s = (p >= a.q_off[2]) ? 2 : (p >= a.q_off[1]) ? 1 : 0;
        attend_row<T>(g, a, b, hk * a.group + i % a.group, s, p - a.q_off[s]);
      }
  }
  cluster.sync();   // nobody's shared memory goes away while it is read
}

// The sample's query rows that read key head hk: row i is query row i / group, head hk * group + i % group.
template <int R> __device__ __forceinline__ void find_rows(const Geometry& g, const ScoredArgs& a, int b, int hk, int n_rows, TailRow (&row)[R]) {
  const int i = threadIdx.x;
  if (i < R) {
    TailRow t = {0.f, -INFINITY, 0.f, 0, 0};
    if (i < n_rows) {
      const int p = i / a.group, s = (p >= a.q_off[2]) ? 2 : (p >= a.q_off[1]) ? 1 : 0, at = p - a.q_off[s];
      const QueryRows rows = query_rows(g, a, b, s);
      if (at >= rows.lo && at < rows.hi) {
        t.time = time_of(g, a, b, s, at + rows.shift);
        t.limit = latest_seen(a, b, t.time);
        t.slope2 = a.slopes != nullptr ? a.slopes[hk * a.group + i % a.group] * LOG2E : 0.f;
        t.doc = document_of(g, a, b, s, at + rows.shift);
        t.opens = (int)(g.allowed >> (3 * s)) & 7;
      }
    }
    row[i] = t;
  }
}

// 8 elements of a row as they lie in memory.
template <typename T> struct Raw8 {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) w[i] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    if constexpr (sizeof(T) == 2) {
      unpack_bf16(w[0].x, f[0], f[1]);
      unpack_bf16(w[0].y, f[2], f[3]);
      unpack_bf16(w[0].z, f[4], f[5]);
      unpack_bf16(w[0].w, f[6], f[7]);
    } else {
#pragma unroll
      for (unsigned i = 0; i < sizeof(T) / 2; ++i) {
        f[4 * i] = __uint_as_float(w[i].x);
        f[4 * i + 1] = __uint_as_float(w[i].y);
        f[4 * i + 2] = __uint_as_float(w[i].z);
        f[4 * i + 3] = __uint_as_float(w[i].w);
      }
    }
  }
};

// Sums over the LANES lanes of a key, of P values each; lane `part` ends with values part * P / LANES and following.
template <int LANES, int P> __device__ __forceinline__ void scatter_sums(float (&v)[P], int part) {
  if constexpr (LANES > 1) {
    constexpr int H = P / 2;
    const bool upper = (part & (LANES / 2)) != 0;
    float keep[H];
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const float mine = upper ? v[H + i] : v[i], other = upper ? v[i] : v[H + i];
      keep[i] = mine + __shfl_xor_sync(0xffffffffu, other, LANES / 2);
    }
    scatter_sums<LANES / 2, H>(keep, part);
#pragma unroll
    for (int i = 0; i < P / LANES; ++i) v[i] = keep[i];
  }
}

template <typename T, int HD, int R, bool RULE>
__global__ void __launch_bounds__(THREADS, R == 1 ? 2 : 1)
scored_tail_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const int split) {
  constexpr int LANES = HD / 8, KEYS = 32 / LANES;   // lanes of a key, keys of a step
  __shared__ TailRow s_row[R];
  __shared__ JoinRoom<HD, R> room;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, part = lane % LANES;
  const int rank = blockIdx.x % split, hk = blockIdx.x / split, b = blockIdx.y;
  const int n_rows = a.Lq * a.group;
  ptx::load_params_early(g, a, split);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();

  find_rows<R>(g, a, b, hk, n_rows, s_row);
  __syncthreads();
  int opens = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) opens |= s_row[i].opens;

  float2 q[R][4], acc[R][4];
  float m[R], l[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    float f[8] = {};
    m[i] = -INFINITY;
    l[i] = 0.f;
    if (s_row[i].opens != 0) load_n(static_cast<const T*>(a.q) + ((int64_t)b * a.Lq + i / a.group) * a.ldq + (int64_t)(hk * a.group + i % a.group) * HD + 8 * part, f);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      q[i][e] = make_float2(f[2 * e], f[2 * e + 1]);
      acc[i][e] = make_float2(0.f, 0.f);
    }
  }

  // Of the STEPS * R scores of a step's keys, score c = u R + i, each lane of a key turns SHARE dots into scores: which ones never changes.
  constexpr int C = STEPS * R, SHARE = (C + LANES - 1) / LANES;
  int key_of[SHARE];
  TailRow row_of[SHARE];
#pragma unroll
  for (int c = 0; c < SHARE; ++c) {
    const int at = min(part * SHARE + c, C - 1), u = at / R;
    key_of[c] = u * KEYS + lane / LANES;
    row_of[c] = s_row[at - u * R];
    if (part * SHARE + c >= C) row_of[c].opens = 0;
  }
#pragma unroll 1
  for (int r = 0; r < 3; ++r) {
    const int n = ((opens >> r) & 1) ? valid_rows(g, b, r) : 0;
    const int share = ((n + split - 1) / split + KEYS - 1) / KEYS * KEYS, first = min(n, rank * share), last = min(n, first + share);   // this CTA's keys
    const int64_t row0 = (int64_t)b * g.L + g.off(r);
    const float* const times = RULE && a.times != nullptr ? a.times + row0 : nullptr;
    const int32_t* const docs = RULE && a.documents != nullptr ? a.documents + row0 : nullptr;
    const int t_first = first + warp * KEYS * STEPS;
    const T* kp = static_cast<const T*>(a.k) + (row0 + t_first + lane / LANES) * a.ldk + (int64_t)hk * HD + 8 * part;
    const T* vp = static_cast<const T*>(a.v) + (row0 + t_first + lane / LANES) * a.ldv + (int64_t)hk * HD + 8 * part;
#pragma unroll 1
    for (int t0 = t_first; t0 < last; t0 += WARPS * KEYS * STEPS, kp += WARPS * KEYS * STEPS * a.ldk, vp += WARPS * KEYS * STEPS * a.ldv) {
      Raw8<T> k[STEPS], v[STEPS];
#pragma unroll
      for (int u = 0; u < STEPS; ++u) {
        k[u].clear();
        v[u].clear();
        if (t0 + u * KEYS + lane / LANES < last) {
          k[u].load(kp + u * KEYS * a.ldk);
          v[u].load(vp + u * KEYS * a.ldv);
        }
      }
      float time[SHARE];
      bool open[SHARE];
#pragma unroll
      for (int c = 0; c < SHARE; ++c) {
        const int t = t0 + key_of[c];
        open[c] = t < last && ((row_of[c].opens >> r) & 1);
        time[c] = (float)t;
        if (RULE && open[c]) {
          if (times != nullptr) time[c] = times[t];
          if (docs != nullptr) open[c] = docs[t] == row_of[c].doc;
        }
      }
      float x[SHARE * LANES];
#pragma unroll
      for (int c = C; c < SHARE * LANES; ++c) x[c] = 0.f;
#pragma unroll
      for (int u = 0; u < STEPS; ++u) {
        float f[8];
        k[u].get(f);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          float2 d = __fmul2_rn(q[i][0], make_float2(f[0], f[1]));
#pragma unroll
          for (int e = 1; e < 4; ++e) d = __ffma2_rn(q[i][e], make_float2(f[2 * e], f[2 * e + 1]), d);
          x[u * R + i] = d.x + d.y;
        }
      }
      scatter_sums<LANES, SHARE * LANES>(x, part);
#pragma unroll
      for (int c = 0; c < SHARE; ++c) {
        float d = x[c] * a.inner;
        if (a.softcap > 0.f) d = tanhf(d) * a.outer;
        if (RULE) d -= row_of[c].slope2 * fabsf(row_of[c].time - time[c]);
        x[c] = open[c] && (!RULE || time[c] <= row_of[c].limit) ? d : -INFINITY;
      }
      // every lane of the key gets all its scores back, to weigh its own features
      float y[C];
      bool all = true;
#pragma unroll
      for (int c = 0; c < C; ++c) {
        y[c] = LANES == 1 ? x[c] : __shfl_sync(0xffffffffu, x[c % SHARE], (lane / LANES) * LANES + c / SHARE);
        all = all && y[c] != -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float top = m[i];
#pragma unroll
        for (int u = 0; u < STEPS; ++u) top = fmaxf(top, y[u * R + i]);
        if (__any_sync(0xffffffffu, top > m[i])) {
          const float f = m[i] == -INFINITY ? 0.f : ptx::ex2(m[i] - top);
          l[i] *= f;
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[i][e] = __fmul2_rn(acc[i][e], make_float2(f, f));
          m[i] = top;
        }
        const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
          y[u * R + i] = ptx::ex2(y[u * R + i] - base);
          l[i] += y[u * R + i];
        }
      }
      auto weigh = [&](bool whole) {
#pragma unroll
        for (int u = 0; u < STEPS; ++u) {
          float f[8];
          v[u].get(f);
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float p = y[u * R + i];
            if (whole || p != 0.f)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[i][e] = __ffma2_rn(make_float2(p, p), make_float2(f[2 * e], f[2 * e + 1]), acc[i][e]);
          }
        }
      };
      if (__all_sync(0xffffffffu, all)) weigh(true);
      else weigh(false);   // what stands in a closed key's value must not count, not even times zero
    }
  }

  // ---- join: lanes, warps, CTAs.  A part without a key has a maximum of -inf and takes no part. ----
#pragma unroll
  for (int i = 0; i < R; ++i) {
    float top = m[i];
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float f = m[i] == -INFINITY ? 0.f : ptx::ex2(m[i] - top);
    l[i] *= f;
#pragma unroll
    for (int o = LANES; o < 32; o <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = m[i] == -INFINITY ? 0.f : (e & 1 ? acc[i][e / 2].y : acc[i][e / 2].x) * f;
#pragma unroll
      for (int o = LANES; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (lane < LANES) room.acc[warp][i][8 * part + e] = v;
    }
    if (lane == 0) room.ml[warp][i] = make_float2(top, l[i]);
  }
  join_warps_and_ctas<T, HD, R>(g, a, room, b, hk, rank, split, n_rows);
}

// bf16 on mma.sync: a warp walks its own keys with all the rows (at most 8, the upper half of a fragment's 16) through a ring of its
// own, so that nothing but its own copies is waited for.  110 instructions to 4 KB of keys and values, where lanes that hold features
// took 600: what bounds it is the copies.
template <int HD> struct TailRing {
  static constexpr int KEYS = 1024 / HD;                                      // of a stage: 2 KB of keys, 2 KB of values
  static constexpr int STAGES = 3, STAGE = 4096 + 8 * KEYS, BYTES = STAGES * STAGE;   // behind them the moments and documents
};
constexpr int TILE_ROWS = 8;

template <int HD, bool CAP, bool RULE>
__global__ void __launch_bounds__(THREADS, 2)
scored_tail_tile_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const int split) {
  using Ring = TailRing<HD>;
  constexpr int KS = Ring::KEYS, CH = HD / 8, NT = HD == 8 ? 4 : 2;
  extern __shared__ __align__(128) uint8_t s_ring[];
  __shared__ TailRow s_row[TILE_ROWS];
  const int tid = threadIdx.x, warp = ptx::uniform(tid >> 5), lane = tid & 31;
  const int rank = blockIdx.x % split, hk = blockIdx.x / split, b = blockIdx.y, n_rows = a.Lq * a.group;
  ptx::load_params_early(g, a, split);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  find_rows<TILE_ROWS>(g, a, b, hk, n_rows, s_row);
  __syncthreads();
  int opens = 0;
#pragma unroll
  for (int i = 0; i < TILE_ROWS; ++i) opens |= s_row[i].opens;
  const TailRow own = s_row[lane >> 2];
  uint32_t qf[1][(HD + 15) / 16][4];
  own_rows<HD>(own.opens != 0 ? static_cast<const bf16*>(a.q) + ((int64_t)b * a.Lq + (lane >> 2) / a.group) * a.ldq + (int64_t)(hk * a.group + (lane >> 2) % a.group) * HD
                              : nullptr, nullptr, lane, qf[0]);

  // this warp's stages: every WARPS-th of the CTA's share of every segment
  Walk ahead = {};
  int first[3];
#pragma unroll
  for (int r = 0; r < 3; ++r) {
    const int n = ((opens >> r) & 1) ? valid_rows(g, b, r) : 0, share = ((n + split - 1) / split + KS - 1) / KS * KS;
    first[r] = min(n, rank * share) + warp * KS;
    ahead.n[r] = min(n, min(n, rank * share) + share);
  }
  auto settle = [&](Walk& w) {
    if (w.seg == 0 && w.pos >= w.n[0]) { w.seg = 1; w.pos = first[1]; }
    if (w.seg == 1 && w.pos >= w.n[1]) { w.seg = 2; w.pos = first[2]; }
    if (w.seg == 2 && w.pos >= w.n[2]) w.seg = 3;
  };
  ahead.pos = first[0];
  settle(ahead);
  Walk now = ahead;
  const uint32_t ring = smem_u32(s_ring) + warp * Ring::BYTES;
  // this lane's piece of a sample's row lane / CH
  const bf16* const k0 = static_cast<const bf16*>(a.k) + ((int64_t)b * g.L + lane / CH) * a.ldk + (int64_t)hk * HD + 8 * (lane % CH);
  const bf16* const v0 = static_cast<const bf16*>(a.v) + ((int64_t)b * g.L + lane / CH) * a.ldv + (int64_t)hk * HD + 8 * (lane % CH);
  const int64_t k_step = 32 / CH * a.ldk, v_step = 32 / CH * a.ldv;
  auto request = [&](Walk& w, int stage) {
    if (!w.over()) {
      const int rem = w.left(), row0 = (w.seg == 0 ? g.seg_off[0] : w.seg == 1 ? g.seg_off[1] : g.seg_off[2]) + w.pos;
      const uint32_t at = ring + stage * Ring::STAGE;
      const bf16 *kp = k0 + (int64_t)row0 * a.ldk, *vp = v0 + (int64_t)row0 * a.ldv;
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // 32 lanes take 32 / CH rows at a time
        const int row = lane / CH + i * (32 / CH);
        const bool real = row < rem;    // past the last key: zeros, from an address that is one
        cp16(at + piece_at<HD>(row, lane % CH), real ? kp : static_cast<const bf16*>(a.k), real);
        cp16(at + 2048 + piece_at<HD>(row, lane % CH), real ? vp : static_cast<const bf16*>(a.v), real);
        kp += k_step;
        vp += v_step;
      }
      if (RULE)
        for (int i = lane; i < KS; i += 32)
          if (i < rem) {
            const int64_t from = (int64_t)b * g.L + row0 + i;
            if (a.times != nullptr) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at + 4096 + 4 * i), "l"(a.times + from) : "memory");
            if (a.documents != nullptr) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at + 4096 + 4 * (KS + i)), "l"(a.documents + from) : "memory");
          }
      w.pos += WARPS * KS;
      settle(w);
    }
    cp_commit();
  };
#pragma unroll
  for (int i = 0; i < Ring::STAGES - 1; ++i) request(ahead, i);

  float o[1][CH][4], ref = -INFINITY;
  float2 sum = make_float2(0.f, 0.f);
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[0][c][e] = 0.f;
  const LaneAt<HD> as_n = lane_as_n<HD>(ring, lane), as_k = lane_as_k<HD>(ring + 2048, lane);
#pragma unroll 1
  for (int stage = 0; !now.over(); stage = stage + 1 == Ring::STAGES ? 0 : stage + 1) {
    asm volatile("cp.async.wait_group %0;" ::"n"(Ring::STAGES - 2) : "memory");
    __syncwarp();   // every lane's copies are there, and every lane is done with the stage that is filled next
    request(ahead, stage == 0 ? Ring::STAGES - 1 : stage - 1);
    const int rem = now.left();
    const float* const times = reinterpret_cast<const float*>(s_ring + warp * Ring::BYTES + stage * Ring::STAGE + 4096);
    const int* const docs = reinterpret_cast<const int*>(times + KS);
    const bool mine = (own.opens >> now.seg) & 1;
#pragma unroll 1
    for (int j = 0; j < min(KS, rem); j += 8 * NT) {
      float x[1][NT][4];
      product_over_features<HD, 1, NT>(x, qf, as_n, stage * Ring::STAGE + j * HD * 2, from_zero);
      uint32_t w[1][NT][2];
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float2 y = __fmul2_rn(make_float2(x[0][n][0], x[0][n][1]), make_float2(a.inner, a.inner));
        if constexpr (CAP) y = __fmul2_rn(tanh_any2(y), make_float2(a.outer, a.outer));
        float z[2] = {y.x, y.y};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int col = j + 8 * n + 2 * (lane & 3) + e;
          bool open = mine && col < rem;
          if constexpr (RULE) {
            const float t = a.times != nullptr ? times[col] : (float)(now.pos + col);
            z[e] -= own.slope2 * fabsf(own.time - t);
            open = open && t <= own.limit && (a.documents == nullptr || docs[col] == own.doc);
          }
          x[0][n][e] = open ? z[e] : -INFINITY;
        }
        top = ptx::fmax3(top, x[0][n][0], x[0][n][1]);
      }
      if (__any_sync(0xffffffffu, top > ref + 8.f)) {
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        if (top > ref) {
          const float f = ptx::ex2(ref - top);
          sum = __fmul2_rn(sum, make_float2(f, f));
#pragma unroll
          for (int c = 0; c < CH; ++c) {
            o[0][c][0] *= f;
            o[0][c][1] *= f;
          }
          ref = top;
        }
      }
      const float r = ref == -INFINITY ? 0.f : -ref;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 y = __fadd2_rn(make_float2(x[0][n][0], x[0][n][1]), make_float2(r, r)), p = make_float2(ptx::ex2(y.x), ptx::ex2(y.y));
        sum = __fadd2_rn(sum, p);
        w[0][n][0] = ptx::pack_bf16(p.x, p.y);
        w[0][n][1] = 0u;
      }
      __syncwarp();   // lanes may have taken different ways; matrix instructions need the whole warp
      product_over_partners<HD, 1, NT>(o, w, as_k, stage * Ring::STAGE + j * HD * 2);
    }
    now.pos += WARPS * KS;
    settle(now);
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();   // the rings are free: the parts are joined there
  JoinRoom<HD, TILE_ROWS>& room = *reinterpret_cast<JoinRoom<HD, TILE_ROWS>*>(s_ring);
  float l = sum.x + sum.y;
  l += __shfl_xor_sync(0xffffffffu, l, 1);
  l += __shfl_xor_sync(0xffffffffu, l, 2);
#pragma unroll
  for (int c = 0; c < CH; ++c) *reinterpret_cast<float2*>(&room.acc[warp][lane >> 2][8 * c + 2 * (lane & 3)]) = make_float2(o[0][c][0], o[0][c][1]);
  if ((lane & 3) == 0) room.ml[warp][lane >> 2] = make_float2(ref, l);
  join_warps_and_ctas<bf16, HD, TILE_ROWS>(g, a, room, b, hk, rank, split, n_rows);
}

template <typename K>
cudaError_t launch_cluster(K kernel, size_t bytes, const Geometry& g, const ScoredArgs& a, int split, cudaStream_t st) {
  if (bytes > 0) {
    const cudaError_t e = sm_count_and_smem_once(reinterpret_cast<const void*>(kernel), (int)bytes, nullptr);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.kv_heads * split), g.batch);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = split;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, g, a, split);
}
// CTAs per (sample, key head): until every SM has one, as long as each still gets two turns of its warps, of `turn` keys each.  One
// sample of (128, 1024, 1024), 8 heads of 64, split 1 / 4 / 8 ways: 15.5 / 9.2 / 8.5 us (float 20.9 / 10.7 / 9.4).
int split_keys(const Geometry& g, const ScoredArgs& a, int n_sm, int turn) {
  int split = 1;
  while (split < MAX_SPLIT && (int64_t)g.batch * a.kv_heads * split < n_sm && g.L > 2 * split * WARPS * turn) split *= 2;
  return split;
}
template <int HD>
cudaError_t launch_tile(const Geometry& g, const ScoredArgs& a, int n_sm, cudaStream_t st) {
  const int split = split_keys(g, a, n_sm, TailRing<HD>::KEYS);
  constexpr size_t bytes = WARPS * TailRing<HD>::BYTES;
  static_assert(sizeof(JoinRoom<HD, TILE_ROWS>) <= bytes, "the parts are joined in the rings");
  const bool rule = rule_masks(a) || a.slopes != nullptr;
  if (a.softcap > 0.f) return launch_cluster(rule ? scored_tail_tile_kernel<HD, true, true> : scored_tail_tile_kernel<HD, true, false>, bytes, g, a, split, st);
  return launch_cluster(rule ? scored_tail_tile_kernel<HD, false, true> : scored_tail_tile_kernel<HD, false, false>, bytes, g, a, split, st);
}
template <int HD, int R>
cudaError_t launch_rows(const Geometry& g, const ScoredArgs& a, int n_sm, cudaStream_t st) {
  const bool rule = rule_masks(a) || a.slopes != nullptr;
  return launch_cluster(rule ? scored_tail_kernel<float, HD, R, true> : scored_tail_kernel<float, HD, R, false>, 0, g, a, split_keys(g, a, n_sm, STEPS * 256 / HD), st);
}
template <int HD>
cudaError_t launch_width(const Geometry& g, int dtype, const ScoredArgs& a, cudaStream_t st) {
  int n_sm = 0;
  const cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  if (dtype == GSIT_BF16) return launch_tile<HD>(g, a, n_sm, st);
  const int rows = a.Lq * a.group;
  return rows <= 1 ? launch_rows<HD, 1>(g, a, n_sm, st) : rows <= 3 ? launch_rows<HD, 3>(g, a, n_sm, st) : launch_rows<HD, 6>(g, a, n_sm, st);
}
bool loads_of_16_bytes(const void* p, int64_t ld, int dtype) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % (dtype == GSIT_BF16 ? 8 : 4) == 0;
}

}  // namespace

// bf16: up to eight query rows to a key head, half of a fragment's, and keys enough to pay for the cluster's join.  These kernels /
// the tiles of whole calls, us, three rows to a key head: 1 x 480 keys, 8 heads of 8 8.9 / 6.4; 1 x 1050 9.0 / 11.7; 4 heads of 32 1 x 180
// 7.2 / 5.0, 1 x 480 7.6 / 8.1; 8 heads of 64 1 x 60 7.0 / 5.0, 1 x 300 7.3 / 10.3, 32 x 2176 28 / 113.
// float: up to six rows (one position in each of three segments, two query heads); beyond, the registers of a lane that holds 8 features
// of each row's query and sum are used up.  1 x 30 keys, 4 heads of 8 9.0 / 7.6, 1 x 300, 8 heads of 8 9.8 / 12.2, 32 x 2176, 8 of 64 61 / 1010.
bool scored_tail_supported(const Geometry& g, int dtype, const ScoredArgs& a) {
  const bool rows = dtype == GSIT_BF16 ? a.Lq * a.group <= TILE_ROWS && (int64_t)g.L * g.hd >= 6144 : a.Lq * a.group <= 6;
  return a.tail && rows && (g.hd == 8 || g.hd == 16 || g.hd == 32 || g.hd == 64) &&
         loads_of_16_bytes(a.q, a.ldq, dtype) && loads_of_16_bytes(a.k, a.ldk, dtype) && loads_of_16_bytes(a.v, a.ldv, dtype);
}

cudaError_t launch_scored_tail(const Geometry& g, int dtype, const ScoredArgs& a, cudaStream_t st) {
  switch (g.hd) {
    case 8: return launch_width<8>(g, dtype, a, st);
    case 16: return launch_width<16>(g, dtype, a, st);
    case 32: return launch_width<32>(g, dtype, a, st);
    default: return launch_width<64>(g, dtype, a, st);
  }
}

}  // namespace gsit

// Scored attention for the newest positions of a stream: a handful of query rows against all keys (forward, float and bf16).
//
// The keys and values stream through once, which is all that bounds it (at 32 samples of 2176 positions, 8 heads of 64, bf16: 143 MB,
// 22 us at the measured copy rate), so the work is cut by keys, not by queries.  All query rows that read a key head -- those of its query heads, in
// every segment -- are held together by every warp; a lane owns 8 features of one key per step (a head of 64 takes 8 lanes, a warp 4
// keys), so that a load instruction covers whole rows and a score needs log2(head_dim / 8) shuffles.  Each group of lanes keeps its own
// running maximum, sum and weighted values; they are joined over the lanes by shuffles, over the warps in shared memory, and over the
// CTAs that share a (sample, key head) through the shared memory of a cluster, in a fixed order.
#include <cooperative_groups.h>

#include "scored.cuh"

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
__global__ void __launch_bounds__(THREADS, R <= 3 ? 2 : 1)
scored_tail_kernel(const __grid_constant__ Geometry g, const __grid_constant__ ScoredArgs a, const int split) {
  constexpr int LANES = HD / 8, KEYS = 32 / LANES;   // lanes of a key, keys of a step
  __shared__ TailRow s_row[R];
  __shared__ __align__(16) float s_acc[WARPS][R][HD], s_joined[R][HD];
  __shared__ float2 s_ml[WARPS][R], s_joined_ml[R];
  __shared__ float s_scale[MAX_SPLIT > WARPS ? MAX_SPLIT : WARPS][R];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, part = lane % LANES;
  const int rank = blockIdx.x % split, hk = blockIdx.x / split, b = blockIdx.y;
  const int n_rows = a.Lq * a.group;                 // row i: query row i / group of the sample, head hk * group + i % group
  ptx::load_params_early(g, a, split);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();

  if (tid < R) {
    TailRow t = {0.f, -INFINITY, 0.f, 0, 0};
    if (tid < n_rows) {
      const int p = tid / a.group, s = (p >= a.q_off[2]) ? 2 : (p >= a.q_off[1]) ? 1 : 0, i = p - a.q_off[s];
      const QueryRows rows = query_rows(g, a, b, s);
      if (i >= rows.lo && i < rows.hi) {
        t.time = time_of(g, a, b, s, i + rows.shift);
        t.limit = latest_seen(a, b, t.time);
        t.slope2 = a.slopes != nullptr ? a.slopes[hk * a.group + tid % a.group] * LOG2E : 0.f;
        t.doc = document_of(g, a, b, s, i + rows.shift);
        t.opens = (int)(g.allowed >> (3 * s)) & 7;
      }
    }
    s_row[tid] = t;
  }
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
        if (a.softcap > 0.f) d = tanh_any(d) * a.outer;
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
      if (lane < LANES) s_acc[warp][i][8 * part + e] = v;
    }
    if (lane == 0) s_ml[warp][i] = make_float2(top, l[i]);
  }
  __syncthreads();
  if (tid < R) {
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, s_ml[w][tid].x);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = s_ml[w][tid].x == -INFINITY ? 0.f : ptx::ex2(s_ml[w][tid].x - top);
      s_scale[w][tid] = f;
      sum += f * s_ml[w][tid].y;
    }
    s_joined_ml[tid] = make_float2(top, sum);
  }
  __syncthreads();
  for (int c = tid; c < R * HD; c += THREADS) {
    const int i = c / HD, f = c % HD;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w)
      if (s_scale[w][i] != 0.f) v += s_scale[w][i] * s_acc[w][i][f];
    s_joined[i][f] = v;
  }
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  if (rank == 0) {
    if (tid < R) {
      float top = -INFINITY, sum = 0.f;
      float2 ml[MAX_SPLIT];
      for (int c = 0; c < split; ++c) {
        ml[c] = cluster.map_shared_rank(s_joined_ml, c)[tid];
        top = fmaxf(top, ml[c].x);
      }
      for (int c = 0; c < split; ++c) {
        const float f = ml[c].x == -INFINITY ? 0.f : ptx::ex2(ml[c].x - top);
        s_scale[c][tid] = f;
        sum += f * ml[c].y;
      }
      s_ml[0][tid] = make_float2(top, sum);
    }
    __syncthreads();
    for (int c = tid; c < n_rows * HD; c += THREADS) {
      const int i = c / HD, f = c % HD;
      float v = 0.f;
      for (int k = 0; k < split; ++k)
        if (s_scale[k][i] != 0.f) v += s_scale[k][i] * cluster.map_shared_rank(&s_joined[0][0], k)[c];
      const float sum = s_ml[0][i].y;
      store_as(static_cast<T*>(a.out) + ((int64_t)b * a.Lq + i / a.group) * a.ldo + (int64_t)(hk * a.group + i % a.group) * HD + f, sum != 0.f ? v / sum : 0.f);
    }
    if (a.lse != nullptr && tid < n_rows) {
      const float2 ml = s_ml[0][tid];
      a.lse[((int64_t)b * g.heads + hk * a.group + tid % a.group) * a.Lq + tid / a.group] = ml.y != 0.f ? (ml.x + log2f(ml.y)) * LN2 : -INFINITY;
    }
  }
  cluster.sync();   // nobody's shared memory goes away while it is read
}

template <typename T, int HD, int R>
cudaError_t launch_rows(const Geometry& g, const ScoredArgs& a, int split, cudaStream_t st) {
  const bool rule = rule_masks(a) || a.slopes != nullptr;
  const auto kernel = rule ? scored_tail_kernel<T, HD, R, true> : scored_tail_kernel<T, HD, R, false>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.kv_heads * split), g.batch);
  cfg.blockDim = dim3(THREADS);
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
template <typename T, int HD>
cudaError_t launch_width(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  int n_sm = 0;
  const cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  // CTAs per (sample, key head): until every SM has one, as long as each still gets two turns of its warps
  int split = 1;
  while (split < MAX_SPLIT && (int64_t)g.batch * a.kv_heads * split < n_sm && g.L > 2 * split * WARPS * STEPS * (256 / HD)) split *= 2;
  const int rows = a.Lq * a.group;
  return rows <= 1   ? launch_rows<T, HD, 1>(g, a, split, st)
         : rows <= 3 ? launch_rows<T, HD, 3>(g, a, split, st)
                     : launch_rows<T, HD, 6>(g, a, split, st);
}
template <typename T>
cudaError_t launch(const Geometry& g, const ScoredArgs& a, cudaStream_t st) {
  switch (g.hd) {
    case 8: return launch_width<T, 8>(g, a, st);
    case 16: return launch_width<T, 16>(g, a, st);
    case 32: return launch_width<T, 32>(g, a, st);
    default: return launch_width<T, 64>(g, a, st);
  }
}
bool loads_of_16_bytes(const void* p, int64_t ld, int dtype) {
  return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % (dtype == GSIT_BF16 ? 8 : 4) == 0;
}

}  // namespace

// Up to six query rows to a key head (one position in each of three segments, two query heads): beyond, the registers of a lane that
// holds 8 features of each row's query and sum are used up, and the tiles of 64 rows take over.
bool scored_tail_supported(const Geometry& g, int dtype, const ScoredArgs& a) {
  return a.tail && a.Lq * a.group <= 6 && (g.hd == 8 || g.hd == 16 || g.hd == 32 || g.hd == 64) && loads_of_16_bytes(a.q, a.ldq, dtype) &&
         loads_of_16_bytes(a.k, a.ldk, dtype) && loads_of_16_bytes(a.v, a.ldv, dtype);
}

cudaError_t launch_scored_tail(const Geometry& g, int dtype, const ScoredArgs& a, cudaStream_t st) {
  return dtype == GSIT_BF16 ? launch<__nv_bfloat16>(g, a, st) : launch<float>(g, a, st);
}

}  // namespace gsit

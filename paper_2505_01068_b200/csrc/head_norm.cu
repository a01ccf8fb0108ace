// Norms of the heads of q and k with the rotary positions in the same pass, and their gradients:
//   y = R (x r gamma),  r = 1 / sqrt(mean(x^2) + eps),  R the rotation of the head's pairs by the row's angles.
// Backward, with u = R^-1 dy, g = u gamma and s = sum(g x):  dx = r (g - x r^2 s / hd),  dgamma = sum over rows and heads of u x r.
// x is read again instead of saving anything; r costs one more sum over a head that is in registers anyway.
//
// Bound by the rows read and written, so everything is arranged around loads in flight: a warp works for itself, without barriers.  It
// takes blocks of a few rows of one of the two tensors; a lane holds two 16-byte pieces of a head (the halves that rotate against each other, or
// neighbours where pairs are interleaved), so that sums over a head are log2(lanes of a head) shuffles and a pair never leaves its lane.  Which
// pieces of a block are a lane's never changes: offsets, weights and the sums for dgamma stay in registers.  The angles of a block are
// computed into a table of the warp's own while the block's loads are under way, one (row, pair) a lane: as many as the heads
// of one tensor share.  q and k have warps of their own, in proportion to their heads: shared tables would halve the angles' work, but
// sums for two weights do not fit the registers beside the loads.
// Angles as in rotary.cu: a double product in turns less its nearest integer, so that far positions keep their phase.
// The gradients of the weights: registers, lanes of a warp, warps of a CTA, CTAs, each in order, the last by a second small kernel.
#include <math.h>

#include <algorithm>

#include "ops.cuh"

namespace gsit {
namespace {

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int ANGLES = 64;            // of a block at most: two a lane
constexpr int MAX_CTAS = 1024;        // partial rows of the workspace

struct NormTensor {
  const void *x, *dy;                 // dy: backward only
  void* out;                          // y or dx
  int64_t ldx, lddy, ldo;
  const float* gamma;
  int heads, rows;                    // rows: of a block
  unsigned blocks;
};
struct HeadNormArgs {
  NormTensor t[2];
  const int32_t* positions;
  int64_t axis_stride, batch_stride;
  int axis1, axis2, pairs, q_ctas;    // first pair of axis 1 and 2; CTAs of q (those of k follow)
  float eps, inv_hd;
  float* partial;                     // [CTAs][hd]
  double turns[MAX_ROTARY_PAIRS];     // frequency of a pair in turns a position
};

// E elements of a row, as they lie in memory: 16 bytes, or 8 (bf16 heads of 8)
template <typename T, int E> struct Piece {
  static constexpr int WORDS = E * (int)sizeof(T) / 4;
  uint32_t w[WORDS];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (WORDS == 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x; w[1] = v.y;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) w[i] = 0u;
  }
  __device__ __forceinline__ void get(float2 (&f)[E / 2]) const {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      if constexpr (sizeof(T) == 2) unpack_bf16(w[i], f[i].x, f[i].y);
      else f[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    }
  }
};
template <int E> __device__ __forceinline__ void store_piece(float* p, const float2 (&f)[E / 2]) {
  static_assert(E == 4, "16 bytes");
  *reinterpret_cast<float4*>(p) = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
}
template <int E> __device__ __forceinline__ void store_piece(__nv_bfloat16* p, const float2 (&f)[E / 2]) {
  if constexpr (E == 8)
    *reinterpret_cast<uint4*>(p) = make_uint4(ptx::pack_bf16(f[0].x, f[0].y), ptx::pack_bf16(f[1].x, f[1].y), ptx::pack_bf16(f[2].x, f[2].y), ptx::pack_bf16(f[3].x, f[3].y));
  else
    *reinterpret_cast<uint2*>(p) = make_uint2(ptx::pack_bf16(f[0].x, f[0].y), ptx::pack_bf16(f[1].x, f[1].y));
}

// (lo, hi) of a lane turned by its angles.  Halves: pair e is (lo[e], hi[e]).  Interleaved: pairs are neighbours, first those of lo.
template <int E, bool ADJACENT>
__device__ __forceinline__ void turn(float2 (&lo)[E / 2], float2 (&hi)[E / 2], const float* cs, const float* sn, float sign) {
  if constexpr (!ADJACENT) {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      const float2 c = *reinterpret_cast<const float2*>(cs + 2 * i), s0 = *reinterpret_cast<const float2*>(sn + 2 * i), s = make_float2(sign * s0.x, sign * s0.y);
      const float2 a = __ffma2_rn(make_float2(-hi[i].x, -hi[i].y), s, __fmul2_rn(lo[i], c)), b = __ffma2_rn(lo[i], s, __fmul2_rn(hi[i], c));
      lo[i] = a;
      hi[i] = b;
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      float2& v = i < E / 2 ? lo[i % (E / 2)] : hi[i % (E / 2)];
      const float c = cs[i], s = sign * sn[i];
      v = make_float2(v.x * c - v.y * s, v.x * s + v.y * c);
    }
  }
}

// Sum over the LANES lanes of a head, in all of them.
template <int LANES> __device__ __forceinline__ float2 head_sum(float2 v) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  return v;
}

template <bool BWD> constexpr int UNITS = BWD ? 1 : 2;   // heads' pieces of a lane whose loads are in flight together

template <typename T, int E, int LANES, bool ADJACENT, bool BWD>
__global__ void __launch_bounds__(THREADS, BWD ? 2 : 4)
head_norm_kernel(const __grid_constant__ Geometry g, const __grid_constant__ HeadNormArgs a) {
  constexpr int HALF = E * LANES, HD = 2 * HALF, N = UNITS<BWD>, H2 = E / 2;
  static_assert(HALF <= ANGLES, "the angles of a row fit the table");
  __shared__ __align__(16) float s_cos[WARPS][2][ANGLES], s_sin[WARPS][2][ANGLES];
  __shared__ uint32_t s_real[WARPS][2];      // bit r: row r of the block is a real one
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, unit = lane % LANES;
  ptx::load_params_early(g, a);
  const int which = (int)blockIdx.x >= a.q_ctas;
  const NormTensor& t = a.t[which];
  const unsigned ctas = which ? gridDim.x - a.q_ctas : a.q_ctas, cta = which ? blockIdx.x - a.q_ctas : blockIdx.x;
  const int rows = g.batch * g.L, row_units = t.heads * LANES, block_rows = t.rows;
  // this lane's features: a piece of the first halves and its partner in the second ones; behind the rotated features, and where interleaved, neighbours
  const int rotated = a.pairs / E;
  const bool neighbours = ADJACENT || unit >= rotated;
  const int lo_at = neighbours ? 2 * unit * E : unit * E, hi_at = neighbours ? lo_at + E : a.pairs + unit * E;

  // this lane's angles of a block
  int angle_row[2], angle_axis[2];
  double turns[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int at = lane + 32 * i, pair = at % HALF;
    angle_row[i] = at / HALF;
    turns[i] = pair < a.pairs ? a.turns[pair] : 0.0;
    angle_axis[i] = pair >= a.pairs ? -1 : pair >= a.axis2 ? 2 : pair >= a.axis1 ? 1 : 0;
  }
  auto angles = [&](unsigned block, int buf) {
    uint32_t real = 0;
    if (block < t.blocks) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = (int)(block * block_rows) + angle_row[i];
        if (angle_row[i] < block_rows && row < rows) {
          const int b = (uint32_t)row / (uint32_t)g.L, l = row - b * g.L, s = segment_of(g, l);
          float sn = 0.f, cs = 1.f;
          if (angle_axis[i] >= 0) {
            const double v = (double)a.positions[angle_axis[i] * a.axis_stride + b * a.batch_stride + l] * turns[i];
            sincospif(2.0f * (float)(v - rint(v)), &sn, &cs);
          }
          s_cos[warp][buf][lane + 32 * i] = cs;
          s_sin[warp][buf][lane + 32 * i] = sn;
          if (l - g.off(s) < valid_rows(g, b, s)) real |= 1u << angle_row[i];
        }
      }
    }
    real = __reduce_or_sync(0xffffffffu, real);
    if (lane == 0) s_real[warp][buf] = real;
  };
  // this lane's pieces of a block (a row of more heads than the lanes take is walked in chunks of them)
  int row_of[N], head_of[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int u = lane + 32 * i;
    row_of[i] = block_rows > 1 ? u / row_units : 0;
    head_of[i] = (u - row_of[i] * row_units) / LANES;
    if (row_of[i] >= block_rows) {   // none
      row_of[i] = 0;
      head_of[i] = t.heads;
    }
  }
  float2 ga_lo[H2], ga_hi[H2], dg_lo[H2], dg_hi[H2];

  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
#pragma unroll
  for (int i = 0; i < H2; ++i) {
    ga_lo[i] = ga_hi[i] = make_float2(1.f, 1.f);
    dg_lo[i] = dg_hi[i] = make_float2(0.f, 0.f);
    if (t.gamma != nullptr) {
      ga_lo[i] = make_float2(t.gamma[lo_at + 2 * i], t.gamma[lo_at + 2 * i + 1]);
      ga_hi[i] = make_float2(t.gamma[hi_at + 2 * i], t.gamma[hi_at + 2 * i + 1]);
    }
  }
  const unsigned step = ctas * WARPS;
  unsigned block = cta * WARPS + warp;
  angles(block, 0);
  __syncwarp();
  for (int buf = 0; block < t.blocks; block += step, buf ^= 1) {
    const int64_t row0 = (int64_t)block * block_rows;
    const uint32_t real = s_real[warp][buf];
    for (int chunk = 0; chunk < t.heads; chunk += 32 * N / LANES) {
      Piece<T, E> x_lo[N], x_hi[N], y_lo[N], y_hi[N];
      bool in[N], keep[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int head = head_of[i] + chunk;
        in[i] = row0 + row_of[i] < rows && head < t.heads;
        keep[i] = in[i] && ((real >> row_of[i]) & 1u);
        x_lo[i].clear();
        x_hi[i].clear();
        if constexpr (BWD) {
          y_lo[i].clear();
          y_hi[i].clear();
        }
        if (keep[i]) {
          const T* x = static_cast<const T*>(t.x) + (row0 + row_of[i]) * t.ldx + (int64_t)head * HD;
          x_lo[i].load(x + lo_at);
          x_hi[i].load(x + hi_at);
          if constexpr (BWD) {
            const T* dy = static_cast<const T*>(t.dy) + (row0 + row_of[i]) * t.lddy + (int64_t)head * HD;
            y_lo[i].load(dy + lo_at);
            y_hi[i].load(dy + hi_at);
          }
        }
      }
      if (chunk == 0) angles(block + step, buf ^ 1);   // while these loads are under way
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float *cs = s_cos[warp][buf] + row_of[i] * HALF + unit * E, *sn = s_sin[warp][buf] + row_of[i] * HALF + unit * E;
        float2 lo[H2], hi[H2];
        x_lo[i].get(lo);
        x_hi[i].get(hi);
        float2 sum = make_float2(0.f, 0.f), other = sum;
#pragma unroll
        for (int e = 0; e < H2; ++e) {
          sum = __ffma2_rn(lo[e], lo[e], sum);
          other = __ffma2_rn(hi[e], hi[e], other);
        }
        sum = __fadd2_rn(sum, other);
        float2 both = make_float2(sum.x + sum.y, 0.f);
        float2 u_lo[H2], u_hi[H2];
        if constexpr (BWD) {
          y_lo[i].get(u_lo);
          y_hi[i].get(u_hi);
          turn<E, ADJACENT>(u_lo, u_hi, cs, sn, -1.f);
          float2 gx = make_float2(0.f, 0.f);
#pragma unroll
          for (int e = 0; e < H2; ++e) {
            gx = __ffma2_rn(__fmul2_rn(u_lo[e], ga_lo[e]), lo[e], gx);
            gx = __ffma2_rn(__fmul2_rn(u_hi[e], ga_hi[e]), hi[e], gx);
          }
          both.y = gx.x + gx.y;
        }
        both = head_sum<LANES>(both);
        const float r = rsqrtf(both.x * a.inv_hd + a.eps);
        const float2 r2 = make_float2(r, r);
        if constexpr (!BWD) {
#pragma unroll
          for (int e = 0; e < H2; ++e) {
            lo[e] = __fmul2_rn(__fmul2_rn(lo[e], r2), ga_lo[e]);
            hi[e] = __fmul2_rn(__fmul2_rn(hi[e], r2), ga_hi[e]);
          }
          turn<E, ADJACENT>(lo, hi, cs, sn, 1.f);
        } else {
          const float back = -r * r * (both.y * a.inv_hd);
          const float2 back2 = make_float2(back, back);
#pragma unroll
          for (int e = 0; e < H2; ++e) {
            const float2 h_lo = __fmul2_rn(lo[e], r2), h_hi = __fmul2_rn(hi[e], r2);
            if (keep[i]) {   // (a row that is not real has an h of 0, but r of a tiny eps may be infinite)
              dg_lo[e] = __ffma2_rn(u_lo[e], h_lo, dg_lo[e]);
              dg_hi[e] = __ffma2_rn(u_hi[e], h_hi, dg_hi[e]);
            }
            lo[e] = __ffma2_rn(h_lo, back2, __fmul2_rn(__fmul2_rn(u_lo[e], ga_lo[e]), r2));
            hi[e] = __ffma2_rn(h_hi, back2, __fmul2_rn(__fmul2_rn(u_hi[e], ga_hi[e]), r2));
          }
        }
        if (in[i]) {
          if (!keep[i])
#pragma unroll
            for (int e = 0; e < H2; ++e) lo[e] = hi[e] = make_float2(0.f, 0.f);
          T* out = static_cast<T*>(t.out) + (row0 + row_of[i]) * t.ldo + (int64_t)(head_of[i] + chunk) * HD;
          store_piece<E>(out + lo_at, lo);
          store_piece<E>(out + hi_at, hi);
        }
      }
    }
    __syncwarp();   // the next block's angles are there, and nobody reads this block's any more
  }
  if constexpr (BWD) {
    if (a.partial == nullptr) return;
    __shared__ float acc[WARPS][HD];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float lo = e & 1 ? dg_lo[e / 2].y : dg_lo[e / 2].x, hi = e & 1 ? dg_hi[e / 2].y : dg_hi[e / 2].x;
#pragma unroll
      for (int o = LANES; o < 32; o <<= 1) {
        lo += __shfl_xor_sync(0xffffffffu, lo, o);
        hi += __shfl_xor_sync(0xffffffffu, hi, o);
      }
      if (lane < LANES) {
        acc[warp][lo_at + e] = lo;
        acc[warp][hi_at + e] = hi;
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < HD; c += THREADS) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) s += acc[w][c];
      a.partial[(int64_t)blockIdx.x * HD + c] = s;
    }
  }
}

// Any head up to 256 features, any stride and address: a warp takes a row, its lanes every 32nd feature of a head; partners are met in shared memory.
constexpr int MAX_HEAD = 256, OWN = MAX_HEAD / 32;
template <typename T, bool BWD>
__global__ void __launch_bounds__(THREADS)
head_norm_any_kernel(const __grid_constant__ Geometry g, const __grid_constant__ HeadNormArgs a, const int adjacent) {
  __shared__ float s_cos[WARPS][MAX_ROTARY_PAIRS], s_sin[WARPS][MAX_ROTARY_PAIRS], s_row[WARPS][MAX_HEAD];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hd = g.hd, rows = g.batch * g.L;
  const int which = (int)blockIdx.x >= a.q_ctas;
  const NormTensor& t = a.t[which];
  const int ctas = which ? (int)gridDim.x - a.q_ctas : a.q_ctas, cta = which ? (int)blockIdx.x - a.q_ctas : (int)blockIdx.x;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  float dg[OWN] = {};
  // the head in s_row turned by the angles: feature f
  auto turned = [&](int f, float sign) {
    const float v = s_row[warp][f];
    if (f >= 2 * a.pairs) return v;
    const int p = adjacent ? f >> 1 : f < a.pairs ? f : f - a.pairs;
    const bool first = adjacent ? (f & 1) == 0 : f < a.pairs;
    const float w = s_row[warp][adjacent ? f ^ 1 : first ? f + a.pairs : f - a.pairs], c = s_cos[warp][p], s = sign * s_sin[warp][p];
    return first ? v * c - w * s : w * s + v * c;
  };
  for (int row = cta * WARPS + warp; row < rows; row += ctas * WARPS) {
    const int b = (uint32_t)row / (uint32_t)g.L, l = row - b * g.L, seg = segment_of(g, l);
    const bool real = l - g.off(seg) < valid_rows(g, b, seg);
    if (real)
      for (int p = lane; p < a.pairs; p += 32) {
        const int axis = p >= a.axis2 ? 2 : p >= a.axis1 ? 1 : 0;
        const double v = (double)a.positions[axis * a.axis_stride + b * a.batch_stride + l] * a.turns[p];
        sincospif(2.0f * (float)(v - rint(v)), &s_sin[warp][p], &s_cos[warp][p]);
      }
    __syncwarp();
    for (int head = 0; head < t.heads; ++head) {
      const T* x = static_cast<const T*>(t.x) + (int64_t)row * t.ldx + (int64_t)head * hd;
      T* out = static_cast<T*>(t.out) + (int64_t)row * t.ldo + (int64_t)head * hd;
      if (!real) {
        for (int f = lane; f < hd; f += 32) store_as(out + f, 0.f);
        continue;
      }
      float v[OWN], ga[OWN], u[OWN], sum = 0.f, gx = 0.f;
#pragma unroll
      for (int i = 0; i < OWN; ++i) {
        const int f = lane + 32 * i;
        v[i] = f < hd ? to_float(x[f]) : 0.f;
        ga[i] = f < hd && t.gamma != nullptr ? t.gamma[f] : 1.f;
        sum += v[i] * v[i];
        u[i] = 0.f;
        if (BWD && f < hd) s_row[warp][f] = to_float(static_cast<const T*>(t.dy)[(int64_t)row * t.lddy + (int64_t)head * hd + f]);
      }
      if (BWD) {
        __syncwarp();
#pragma unroll
        for (int i = 0; i < OWN; ++i)
          if (const int f = lane + 32 * i; f < hd) {
            u[i] = turned(f, -1.f);
            gx += u[i] * ga[i] * v[i];
          }
      }
      const float2 s = head_sum<32>(make_float2(sum, gx));
      const float r = rsqrtf(s.x * a.inv_hd + a.eps), back = -r * r * (s.y * a.inv_hd);
      if (BWD) {
#pragma unroll
        for (int i = 0; i < OWN; ++i)
          if (const int f = lane + 32 * i; f < hd) {
            const float h = v[i] * r;
            dg[i] += u[i] * h;
            store_as(out + f, u[i] * ga[i] * r + h * back);
          }
      } else {
#pragma unroll
        for (int i = 0; i < OWN; ++i)
          if (const int f = lane + 32 * i; f < hd) s_row[warp][f] = v[i] * r * ga[i];
        __syncwarp();
        for (int f = lane; f < hd; f += 32) store_as(out + f, turned(f, 1.f));
      }
      __syncwarp();   // s_row is written by the next head
    }
  }
  if (!BWD || a.partial == nullptr) return;
  // warps in order, through the rows they no longer need
#pragma unroll
  for (int i = 0; i < OWN; ++i)
    if (const int f = lane + 32 * i; f < hd) s_row[warp][f] = dg[i];
  __syncthreads();
  for (int c = threadIdx.x; c < hd; c += THREADS) {
    float s = 0.f;
    for (int w = 0; w < WARPS; ++w) s += s_row[w][c];
    a.partial[(int64_t)blockIdx.x * hd + c] = s;
  }
}

// dgamma of q and k = the partial rows of their CTAs added up.  A CTA takes 32 columns of one of them, its 32 warps a share of the rows each.
__global__ void __launch_bounds__(1024)
head_norm_reduce_kernel(const float* __restrict__ partial, int q_ctas, int ctas, int hd, float* dq_gamma, float* dk_gamma) {
  __shared__ float acc[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane, which = blockIdx.y;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  float s = 0.f;
  if (col < hd)
#pragma unroll 8
    for (int i = (which ? q_ctas : 0) + warp; i < (which ? ctas : q_ctas); i += 32) s += partial[(int64_t)i * hd + col];
  acc[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && col < hd) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) s += acc[w][lane];
    (which ? dk_gamma : dq_gamma)[col] = s;
  }
}

using Kernel = void (*)(const Geometry, const HeadNormArgs);
template <typename T, bool ADJACENT, bool BWD> Kernel wide_kernel(int hd) {
  constexpr int E = 16 / (int)sizeof(T);
  if constexpr (sizeof(T) == 2)
    if (hd == 8) return head_norm_kernel<T, 4, 1, ADJACENT, BWD>;
  switch (hd / (2 * E)) {
    case 1: return head_norm_kernel<T, E, 1, ADJACENT, BWD>;
    case 2: return head_norm_kernel<T, E, 2, ADJACENT, BWD>;
    case 4: return head_norm_kernel<T, E, 4, ADJACENT, BWD>;
    case 8: return head_norm_kernel<T, E, 8, ADJACENT, BWD>;
  }
  return head_norm_kernel<T, E, ANGLES / E, ADJACENT, BWD>;   // the widest head, 128 features
}
template <typename T> Kernel wide_kernel(int hd, bool adjacent, bool bwd) {
  if (bwd) return adjacent ? wide_kernel<T, true, true>(hd) : wide_kernel<T, false, true>(hd);
  return adjacent ? wide_kernel<T, true, false>(hd) : wide_kernel<T, false, false>(hd);
}

}  // namespace

size_t head_norm_scratch(const Geometry& g) { return sizeof(float) * (size_t)g.hd * MAX_CTAS; }

cudaError_t launch_head_norm(const Geometry& g, int dtype, const HeadNormCall& c, cudaStream_t st) {
  const int es = dtype == GSIT_BF16 ? 2 : 4;
  int n_sm = 0;
  cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  HeadNormArgs a = {};
  a.pairs = c.sections[0] + c.sections[1] + c.sections[2];
  a.axis1 = c.sections[0];
  a.axis2 = c.sections[0] + c.sections[1];
  a.positions = c.positions;
  a.axis_stride = c.axis_stride;
  a.batch_stride = c.batch_stride;
  a.eps = c.eps;
  a.inv_hd = 1.0f / g.hd;
  a.partial = c.partial;
  rotary_turns(c.base, a.pairs, a.turns);
  // wide: a head of at most 128 features is 1, 2, 4, 8 or 16 lanes of two pieces, 16 bytes each (8 where a bf16 head has 8 features), and whole
  // pieces of it rotate
  const int piece = dtype == GSIT_BF16 ? (g.hd == 8 ? 4 : 8) : 4, lanes = g.hd / (2 * piece);
  bool wide = g.hd % (2 * piece) == 0 && g.hd <= 2 * ANGLES && (lanes & (lanes - 1)) == 0 && (c.interleaved || a.pairs % piece == 0);
  int total = 0;
  for (int i = 0; i < 2; ++i) {
    NormTensor& t = a.t[i];
    t.x = c.x[i]; t.ldx = c.ldx[i];
    t.dy = c.dy[i]; t.lddy = c.lddy[i];
    t.out = c.out[i]; t.ldo = c.ldo[i];
    t.gamma = c.gamma[i];
    t.heads = c.heads[i];
    total += t.heads;
    if (t.heads == 0) continue;
    wide = wide && ((reinterpret_cast<uintptr_t>(t.x) | reinterpret_cast<uintptr_t>(t.dy) | reinterpret_cast<uintptr_t>(t.out)) % (piece * es)) == 0 &&
           t.ldx % piece == 0 && t.lddy % piece == 0 && t.ldo % piece == 0;
  }
  // CTAs: as many as fit the SMs at once, shared out to q and k by their heads; no more than there are blocks of rows
  const int64_t rows = (int64_t)g.batch * g.L;
  const int most = std::min(MAX_CTAS, (c.backward ? 2 : 4) * n_sm), units = c.backward ? UNITS<true> : UNITS<false>;
  int ctas[2] = {0, 0};
  for (int i = 0; i < 2; ++i) {
    NormTensor& t = a.t[i];
    if (t.heads == 0) continue;
    t.rows = wide ? std::max(1, std::min(2 * ANGLES / g.hd, 32 * units / (t.heads * lanes))) : 1;
    t.blocks = (unsigned)((rows + t.rows - 1) / t.rows);
    const int share = std::max(1, i == 0 ? (most * t.heads + total / 2) / total : most - ctas[0]);
    ctas[i] = (int)std::min<int64_t>(std::min(share, c.heads[1] > 0 ? most - 1 : most), (t.blocks + WARPS - 1) / WARPS);
  }
  a.q_ctas = ctas[0];
  const dim3 grid((unsigned)(ctas[0] + ctas[1]));
  if (wide) {
    const Kernel k = dtype == GSIT_BF16 ? wide_kernel<__nv_bfloat16>(g.hd, c.interleaved, c.backward) : wide_kernel<float>(g.hd, c.interleaved, c.backward);
    e = launch_overlapped(k, grid, dim3(THREADS), 0, st, g, a);
  } else if (dtype == GSIT_BF16) {
    e = c.backward ? launch_overlapped(head_norm_any_kernel<__nv_bfloat16, true>, grid, dim3(THREADS), 0, st, g, a, (int)c.interleaved)
                   : launch_overlapped(head_norm_any_kernel<__nv_bfloat16, false>, grid, dim3(THREADS), 0, st, g, a, (int)c.interleaved);
  } else {
    e = c.backward ? launch_overlapped(head_norm_any_kernel<float, true>, grid, dim3(THREADS), 0, st, g, a, (int)c.interleaved)
                   : launch_overlapped(head_norm_any_kernel<float, false>, grid, dim3(THREADS), 0, st, g, a, (int)c.interleaved);
  }
  if (e != cudaSuccess || a.partial == nullptr) return e;
  return launch_overlapped(head_norm_reduce_kernel, dim3((g.hd + 31) / 32, c.heads[1] > 0 ? 2 : 1), dim3(1024), 0, st, a.partial, ctas[0], ctas[0] + ctas[1], g.hd,
                           c.dgamma[0], c.dgamma[1]);
}

}  // namespace gsit

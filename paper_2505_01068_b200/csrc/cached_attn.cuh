// Attention of a step's rows over a stream's cache (gsit_im_cached_attention_fwd); the kernel, for the files that instantiate it.
//
// Everything streams through once: a warp takes blocks of 32 positions of one key head, loads a block's bytes straight into the registers that its
// matrix instructions take them from -- the pages are laid out for that: 16 bytes a lane, whole lines a warp, nothing staged -- and works on one
// block while the next ones' bytes are under way.  8 query rows of the key head (its query heads, in every segment) are the narrow side of
// m16n8k16 products:
//   S^T = K Q^T      keys x rows: 8-bit integers (or e4m3) are exact in f16; q is brought to f16 by a power of two for each row, which loses nothing
//                    of bf16 worth having (what is 2^-28 of a row's largest feature); float q as two f16 terms, 22 bits
//   O^T += vs V^T P  features x rows: P turned round by movmatrix, in f16 (2^-11 of each weight, relative), as two terms for float; the block's scale
//                    is applied to the product in float, so it never meets the range of f16
// The open block's rows are brought to f16 by a power of two for the block (float: two terms) and go the same way, in the warp whose turn it is.
// The softmax runs over a reference that is raised only where a score passes it by 2^8, so that most blocks need no exchange between lanes.
// Warps' parts are joined in shared memory, CTAs' through the cluster's or, where more CTAs than a cluster holds share a (stream, key head), through
// a workspace and a second small kernel; always in order.
// A closed pair's weight is 0 and the bytes it meets are numbers, so nothing of it counts; blocks whose scale is NaN take a way of their own.
#pragma once
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "cache.cuh"
#include "scored.cuh"

namespace gsit {
namespace {

namespace cg = cooperative_groups;

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int MAX_CLUSTER = 8;

struct QueryRow {
  float time, limit, slope2;
  int opens;                    // bit r: key segment r is open to it
};

__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// What rounding a pair to f16 leaves, in f16.
__device__ __forceinline__ uint32_t f16x2_rest(float lo, float hi, uint32_t rounded) {
  const float2 r = __half22float2(*reinterpret_cast<const __half2*>(&rounded));
  return f16x2(lo - r.x, hi - r.y);
}
__device__ __forceinline__ uint32_t turned_round(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_k8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(b0));
}
// Four bytes as two pairs of f16, exactly.
template <int KIND> __device__ __forceinline__ void unpack8(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (KIND == GSIT_CACHE_INT8) {   // the byte plus 128 as the last bits of 1024 + ..., less 1152
    const uint32_t u = w ^ 0x80808080u;
    const __half2 minus = __halves2half2(__ushort_as_half(0xe480), __ushort_as_half(0xe480));
    uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 x = __hadd2(*reinterpret_cast<__half2*>(&a), minus), y = __hadd2(*reinterpret_cast<__half2*>(&b), minus);
    lo = *reinterpret_cast<const uint32_t*>(&x);
    hi = *reinterpret_cast<const uint32_t*>(&y);
  } else {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
  }
}

// A power of two that brings a largest magnitude `top` (> 0, finite) to [2^to, 2^(to + 1)), and its inverse.  Magnitudes of almost nothing
// come to less: the inverse stays a number.
struct Power {
  float up, down;
};
__device__ __forceinline__ Power power_for(float top, int to) {
  const int e = max(-126, min(126, to - (((__float_as_int(top) >> 23) & 255) - 127)));
  return {__int_as_float((127 + e) << 23), __int_as_float((127 - e) << 23)};
}

// What a lane holds of a block of bytes.
template <int HD> struct Bytes {
  static constexpr int WORDS = HD == 8 ? 2 : HD / 4;   // of keys, and of values
  uint32_t k[WORDS], v[WORDS];
  float ks, vs, time[4];
  int rows;                // positions: 32, or those of an open block (whose rows are not loaded here)
  int seg, at, buffer;     // segment, its first position; buffer of an open block, -1: full
  __device__ __forceinline__ void load(const uint8_t* key, const uint8_t* value) {
    if constexpr (HD == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(key), y = *reinterpret_cast<const uint2*>(value);
      k[0] = x.x; k[1] = x.y;
      v[0] = y.x; v[1] = y.y;
    } else {
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        const uint4 x = *reinterpret_cast<const uint4*>(key + 512 * i);
        k[4 * i] = x.x; k[4 * i + 1] = x.y; k[4 * i + 2] = x.z; k[4 * i + 3] = x.w;
      }
#pragma unroll
      for (int i = 0; i < HD / 16; ++i) {
        const uint4 y = *reinterpret_cast<const uint4*>(value + 512 * i);
        v[4 * i] = y.x; v[4 * i + 1] = y.y; v[4 * i + 2] = y.z; v[4 * i + 3] = y.w;
      }
    }
  }
};

// The parts that are joined: of each warp, then of the CTA.
template <int HD, int R> struct PartRoom {
  float acc[WARPS][R][HD], joined[R][HD];
  float2 ml[WARPS][R], joined_ml[R];      // (reference, sum); a part without a key has a reference of -inf and takes no part
  float scale[WARPS][R];
};
// Factors that bring (at most 8) parts to their common reference, and that reference with the sum.  A part without a number among its scores
// has no reference: its sum is 0, or NaN where a score was, and then so is everything.
template <typename Get, typename Put> __device__ __forceinline__ float2 join_sums(int n, Get get, Put put) {
  float2 p[8];
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    p[i] = i < n ? get(i) : make_float2(-INFINITY, 0.f);
    top = fmaxf(top, p[i].x);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float f = p[i].x == -INFINITY ? 1.f : ptx::ex2(p[i].x - top);
    if (i < n) put(i, f);
    sum += f * p[i].y;
  }
  return make_float2(top, sum);
}

// How many blocks' bytes a lane asks for at once: 16 to 32 registers of them.
template <int HD> constexpr int GROUP = HD == 64 ? 1 : HD == 32 ? 2 : 4;

template <typename T, int HD, int KIND, int NT>
__global__ void __launch_bounds__(THREADS, NT == 1 ? 2 : 1)
cached_attention_kernel(const __grid_constant__ Geometry g, const __grid_constant__ CachedArgs a) {
  constexpr int R = 8 * NT, TERMS = sizeof(T) == 4 ? 2 : 1, KS = HD == 8 ? 1 : HD / 16, MD = KS, B = GROUP<HD>;
  using Room = PartRoom<HD, R>;
  extern __shared__ __align__(16) uint8_t smem[];
  Room& room = *reinterpret_cast<Room*>(smem);
  __shared__ QueryRow s_row[R];
  const Cache& c = a.c;
  const int tid = threadIdx.x, warp = ptx::uniform(tid >> 5), lane = tid & 31, gr = lane >> 2, t = lane & 3;
  const int rank = blockIdx.x % a.split, hk = blockIdx.x / a.split, b = blockIdx.y, row0 = blockIdx.z * R;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();

  // ---- the rows: row r of a key head is row r / group of the step, head hk * group + r % group ----
  for (int i = tid; i < R; i += THREADS) {
    QueryRow x = {0.f, -INFINITY, 0.f, 0};
    if (row0 + i < a.rows) {
      const int l = (row0 + i) / a.group, s = segment_of(g, l), at = l - g.off(s), n = valid_rows(g, b, s);
      if (at < n) {
        x.time = a.times.p != nullptr ? a.times.at(b, l) : (float)(held_rows(c, g.status, b, s) - n + at);
        x.limit = a.causal ? x.time : INFINITY;
        x.slope2 = a.slopes != nullptr ? a.slopes[hk * a.group + (row0 + i) % a.group] * LOG2E : 0.f;
        x.opens = (int)(g.allowed >> (3 * s)) & 7;
      }
    }
    s_row[i] = x;
  }
  __syncthreads();
  int opens = 0;
#pragma unroll
  for (int i = 0; i < R; ++i) opens |= s_row[i].opens;

  // ---- queries as B operands, and what brings a dot back to a score ----
  uint32_t qf[NT][TERMS][KS][2];
  float back[NT][2];                     // of the columns 2 t and 2 t + 1 of each tile
  int col_opens[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = row0 + 8 * n + gr;
    const bool real = s_row[8 * n + gr].opens != 0;
    const T* q = static_cast<const T*>(a.q) + ((int64_t)b * g.L + (real ? r / a.group : 0)) * a.ldq + (int64_t)(hk * a.group + (real ? r % a.group : 0)) * HD;
    float2 f[KS][2];
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f[k][h] = make_float2(0.f, 0.f);
        if (real && (HD > 8 || h == 0)) {
          if constexpr (sizeof(T) == 2) unpack_bf16(*reinterpret_cast<const uint32_t*>(q + 16 * k + 8 * h + 2 * t), f[k][h].x, f[k][h].y);
          else f[k][h] = *reinterpret_cast<const float2*>(q + 16 * k + 8 * h + 2 * t);
        }
        top = ptx::fmax3(top, fabsf(f[k][h].x), fabsf(f[k][h].y));
      }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const Power p = top > 0.f && top < INFINITY ? power_for(top, 10) : Power{1.f, 1.f};   // (a row of NaN or Inf stays one)
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float x = f[k][h].x * p.up, y = f[k][h].y * p.up;
        qf[n][0][k][h] = f16x2(x, y);
        if constexpr (TERMS == 2) qf[n][1][k][h] = f16x2_rest(x, y, qf[n][0][k][h]);
      }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      back[n][e] = __shfl_sync(0xffffffffu, p.down, 4 * (2 * t + e)) * a.inner;
      col_opens[n][e] = s_row[8 * n + 2 * t + e].opens;
    }
  }

  // ---- this warp's blocks: every (split * WARPS)-th group of those of the open segments, one after the other ----
  int len[3], upto[3], blocks = 0;       // upto: blocks of the segments before and of this one
#pragma unroll
  for (int r = 0; r < 3; ++r) {
    len[r] = ((opens >> r) & 1) ? held_rows(c, g.status, b, r) : 0;
    blocks += (len[r] + CACHE_BLOCK - 1) / CACHE_BLOCK;
    upto[r] = blocks;
  }
  const int turn = a.split * WARPS * B;
  const bool timed = a.causal != 0 || a.slopes != nullptr;
  // where block i lies: page, or -1 (an open block; none)
  auto page_of = [&](int i) {
    if (i >= blocks) return -1;
    const int r = i >= upto[1] ? 2 : i >= upto[0] ? 1 : 0, j = i - (r == 0 ? 0 : upto[r - 1]);
    const int page = real_page(c, c.tables[((int64_t)b * 3 + r) * c.blocks + j]);
    if (page < 0) raise_flag(g, GSIT_DEVFLAG_CLAMPED);
    return page;
  };
  // lanes know the pages of the warp's next 32 / B turns
  int ahead = (rank * WARPS + warp) * B, known = 0, pages = -1;
  Bytes<HD> next[B];
  auto request = [&]() {
    if (known == 0) {
      pages = page_of(ahead + lane / B * turn + lane % B);
      known = 32 / B;
    }
#pragma unroll
    for (int u = 0; u < B; ++u) {
      Bytes<HD>& x = next[u];
      const int i = ahead + u, page = __shfl_sync(0xffffffffu, pages, (32 / B - known) * B + u);
      x.rows = 0;
      if (i < blocks) {
        const int r = i >= upto[1] ? 2 : i >= upto[0] ? 1 : 0, j = i - (r == 0 ? 0 : r == 1 ? upto[0] : upto[1]);
        x.seg = r;
        x.at = j * CACHE_BLOCK;
        x.rows = min(CACHE_BLOCK, (r == 0 ? len[0] : r == 1 ? len[1] : len[2]) - x.at);
        x.buffer = x.rows < CACHE_BLOCK ? j & 1 : -1;
        if (timed)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x.time[e] = c.times == nullptr ? (float)(x.at + 8 * e + gr) : page >= 0 ? c.times[(int64_t)page * CACHE_BLOCK + 8 * e + gr] : 0.f;
        if (x.buffer < 0) {
          if (page < 0) x.rows = 0;
          else {
            const int64_t head = (int64_t)page * c.kv_heads + hk;
            x.load(c.keys + head * (CACHE_BLOCK * HD) + (HD == 8 ? 8 : 16) * lane, c.values + head * (CACHE_BLOCK * HD) + (HD == 8 ? 8 : 16) * lane);
            x.ks = c.key_scale[head];
            x.vs = c.value_scale[head];
          }
        }
      }
    }
    ahead += turn;
    --known;
  };

  float o[MD][NT][4], ref[NT][2], sum[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      ref[n][e] = -INFINITY;
      sum[n][e] = 0.f;
    }
#pragma unroll
    for (int m = 0; m < MD; ++m)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[m][n][e] = 0.f;
  }

  // One block: keys(m, k, term, fragment) and values(m, k, term, fragment) give A operands, of TERMS_IN terms.
  auto attend = [&](const Bytes<HD>& x, auto terms_in, float ks, float vs, auto keys, auto values) {
    constexpr int IN = decltype(terms_in)::value;
    float s[2][NT][4];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[m][n][e] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int w = 0; w < IN; ++w) {
          uint32_t f[4];
          keys(m, k, w, f);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int y = 0; y < TERMS - w; ++y) {   // the product of the two smaller terms is left out: 2^-22 of the score's terms
              if constexpr (HD == 8) mma_k8(s[m][n], f[0], f[1], qf[n][y][k][0]);
              else mma(s[m][n], f, qf[n][y][k][0], qf[n][y][k][1]);
            }
        }
    }
    // scores in base 2; closed pairs -inf
    bool raise = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bool mine = (col_opens[n][e] >> x.seg) & 1;
        const float f = back[n][e] * ks;
        float time = 0.f, limit = 0.f, slope2 = 0.f;
        if (timed) {
          const QueryRow& row = s_row[8 * n + 2 * t + e];
          time = row.time;
          limit = row.limit;
          slope2 = row.slope2;
        }
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float& v = s[m][n][2 * h + e];
            v *= f;
            if (a.softcap > 0.f) v = (sizeof(T) == 4 ? tanhf(v) : tanh_any2(make_float2(v, v)).x) * a.outer;
            bool open = mine && 16 * m + 8 * h + gr < x.rows;
            if (timed) {
              v -= slope2 * fabsf(time - x.time[2 * m + h]);
              open = open && x.time[2 * m + h] <= limit;
            }
            v = open ? v : -INFINITY;
            raise = raise || !(v <= ref[n][e] + 8.f);   // NaN, too
          }
      }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = fmaxf(fmaxf(s[0][n][e], s[0][n][2 + e]), fmaxf(s[1][n][e], s[1][n][2 + e]));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
          if (top > ref[n][e]) {
            const float f = ptx::ex2(ref[n][e] - top);
            sum[n][e] *= f;
#pragma unroll
            for (int m = 0; m < MD; ++m) {
              o[m][n][e] *= f;
              o[m][n][2 + e] *= f;
            }
            ref[n][e] = top;
          }
        }
      __syncwarp();
    }
    // weights, turned round into B operands: keys 2 t, 2 t + 1 (and + 8) of row gr
    uint32_t pf[NT][TERMS][2][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const float r0 = ref[n][0] == -INFINITY ? 0.f : ref[n][0], r1 = ref[n][1] == -INFINITY ? 0.f : ref[n][1];
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float p0 = ptx::ex2(s[m][n][2 * h] - r0), p1 = ptx::ex2(s[m][n][2 * h + 1] - r1);
          sum[n][0] += p0;
          sum[n][1] += p1;
          const uint32_t p = f16x2(p0, p1);
          pf[n][0][m][h] = turned_round(p);
          if constexpr (TERMS == 2) pf[n][1][m][h] = turned_round(f16x2_rest(p0, p1, p));
        }
    }
    const bool broken = !(fabsf(vs) < INFINITY);
#pragma unroll
    for (int m = 0; m < MD; ++m) {
      float add[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) add[n][e] = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int w = 0; w < IN; ++w) {
          uint32_t f[4];
          values(m, k, w, f);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int y = 0; y < TERMS - w; ++y) mma(add[n], f, pf[n][y][k][0], pf[n][y][k][1]);
        }
      if (!broken) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[m][n][e] = fmaf(vs, add[n][e], o[m][n][e]);
      }
    }
    if (broken)   // NaN for the rows to which any position of the block is open
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          bool any = false;
#pragma unroll
          for (int m = 0; m < 2; ++m) any = any || s[m][n][e] != -INFINITY || s[m][n][2 + e] != -INFINITY;
          uint32_t which = __ballot_sync(0xffffffffu, any);
          which |= which >> 16;
          which |= which >> 8;
          which |= which >> 4;
          if ((which >> t) & 1u)
#pragma unroll
            for (int m = 0; m < MD; ++m) o[m][n][e] = o[m][n][2 + e] = vs;
        }
  };
  // The open block: rows in memory, brought to f16 by a power of two for all of them.
  auto open_block = [&](const Bytes<HD>& x) {
    const int64_t at = ((((int64_t)b * 3 + x.seg) * 2 + x.buffer) * c.kv_heads + hk) * (CACHE_BLOCK * HD);
    const T* const key = static_cast<const T*>(c.open_keys) + at;
    const T* const value = static_cast<const T*>(c.open_values) + at;
    Power up[2];
    bool broken[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      constexpr int E = 16 / (int)sizeof(T) >= 8 ? 8 : 4;
      uint32_t top = 0;
      for (int i = lane * E; i < x.rows * HD; i += 32 * E) {
        float f[E];
        load_n(w ? value + i : key + i, f);
#pragma unroll
        for (int e = 0; e < E; ++e) top = max(top, __float_as_uint(f[e]) & 0x7fffffffu);
      }
      top = __reduce_max_sync(0xffffffffu, top);
      broken[w] = top >= 0x7f800000u;
      up[w] = top > 0 && !broken[w] ? power_for(__uint_as_float(top), 14) : Power{1.f, 1.f};
    }
    auto terms = [&](float2 v, int w) {
      const uint32_t r = f16x2(v.x, v.y);
      return w == 0 ? r : f16x2_rest(v.x, v.y, r);
    };
    attend(x, std::integral_constant<int, TERMS>{}, broken[0] ? __int_as_float(0x7fffffff) : up[0].down, broken[1] ? __int_as_float(0x7fffffff) : up[1].down,
           [&](int m, int k, int w, uint32_t (&f)[4]) {
#pragma unroll
             for (int i = 0; i < 4; ++i) {   // position halves i % 2, feature halves i / 2
               const int row = 16 * m + 8 * (i % 2) + gr;
               float2 v = make_float2(0.f, 0.f);
               if (row < x.rows && !broken[0] && (HD > 8 || i < 2)) {
                 const T* p = key + row * HD + 16 * k + 8 * (i / 2) + 2 * t;
                 if constexpr (sizeof(T) == 2) unpack_bf16(*reinterpret_cast<const uint32_t*>(p), v.x, v.y);
                 else v = *reinterpret_cast<const float2*>(p);
               }
               f[i] = terms(make_float2(v.x * up[0].up, v.y * up[0].up), w);
             }
           },
           [&](int m, int k, int w, uint32_t (&f)[4]) {
#pragma unroll
             for (int i = 0; i < 4; ++i) {   // feature halves i % 2, position halves i / 2; rows of features come in, turned round
               const int row = 16 * k + 8 * (i / 2) + gr;
               float2 v = make_float2(0.f, 0.f);
               if (row < x.rows && !broken[1] && (HD > 8 || i % 2 == 0)) {
                 const T* p = value + row * HD + 16 * m + 8 * (i % 2) + 2 * t;
                 if constexpr (sizeof(T) == 2) unpack_bf16(*reinterpret_cast<const uint32_t*>(p), v.x, v.y);
                 else v = *reinterpret_cast<const float2*>(p);
               }
               f[i] = turned_round(terms(make_float2(v.x * up[1].up, v.y * up[1].up), w));
             }
           });
  };

  int now = ahead;
  request();
#pragma unroll 1
  for (; now < blocks; now += turn) {
    Bytes<HD> x[B];
#pragma unroll
    for (int u = 0; u < B; ++u) x[u] = next[u];
    request();
#pragma unroll
    for (int u = 0; u < B; ++u) {
      if (x[u].rows == 0) continue;
      if (x[u].buffer >= 0) {
        open_block(x[u]);
        continue;
      }
      attend(x[u], std::integral_constant<int, 1>{}, x[u].ks, x[u].vs,
             [&](int m, int k, int, uint32_t (&f)[4]) {
               if constexpr (HD == 8) unpack8<KIND>(x[u].k[m], f[0], f[1]);
               else {
                 unpack8<KIND>(x[u].k[4 * k + 2 * m], f[0], f[1]);
                 unpack8<KIND>(x[u].k[4 * k + 2 * m + 1], f[2], f[3]);
               }
             },
             [&](int m, int k, int, uint32_t (&f)[4]) {
               if constexpr (HD == 8) {
                 unpack8<KIND>(x[u].v[k], f[0], f[2]);
                 f[1] = f[3] = 0u;
               } else {
                 unpack8<KIND>(x[u].v[4 * m + 2 * k], f[0], f[1]);
                 unpack8<KIND>(x[u].v[4 * m + 2 * k + 1], f[2], f[3]);
               }
             });
    }
  }

  // ---- join: lanes, warps, CTAs ----
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float l = sum[n][e];
      l += __shfl_xor_sync(0xffffffffu, l, 4);
      l += __shfl_xor_sync(0xffffffffu, l, 8);
      l += __shfl_xor_sync(0xffffffffu, l, 16);
      const int row = 8 * n + 2 * t + e;
      if (gr == 0) room.ml[warp][row] = make_float2(ref[n][e], l);
#pragma unroll
      for (int m = 0; m < MD; ++m) {
        room.acc[warp][row][16 * m + gr] = o[m][n][e];
        if constexpr (HD > 8) room.acc[warp][row][16 * m + 8 + gr] = o[m][n][2 + e];
      }
    }
  __syncthreads();
  if (tid < R) room.joined_ml[tid] = join_sums(WARPS, [&](int w) { return room.ml[w][tid]; }, [&](int w, float f) { room.scale[w][tid] = f; });
  __syncthreads();
  const int n_rows = min(R, a.rows - row0);
  for (int i = tid; i < n_rows * HD; i += THREADS) {
    const int r = i / HD, f = i % HD;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) v += room.scale[w][r] * room.acc[w][r][f];
    room.joined[r][f] = v;
  }
  auto write = [&](int r, int f, float v, float l) {
    store_as(static_cast<T*>(a.out) + ((int64_t)b * g.L + (row0 + r) / a.group) * g.d + (int64_t)(hk * a.group + (row0 + r) % a.group) * HD + f, l != 0.f ? v / l : 0.f);
  };
  auto write_lse = [&](int r, float2 ml) {
    a.lse[((int64_t)b * g.heads + hk * a.group + (row0 + r) % a.group) * g.L + (row0 + r) / a.group] = ml.y != 0.f ? (ml.x + log2f(ml.y)) * LN2 : -INFINITY;
  };
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  if (a.split == 1) {
    for (int i = tid; i < n_rows * HD; i += THREADS) write(i / HD, i % HD, room.joined[i / HD][i % HD], room.joined_ml[i / HD].y);
    if (a.lse != nullptr && tid < n_rows) write_lse(tid, room.joined_ml[tid]);
  } else {
    // every CTA joins the rows' values of its own share
    if (tid < R) {
      const float2 ml = join_sums(a.split, [&](int k) { return cluster.map_shared_rank(room.joined_ml, k)[tid]; },
                                               [&](int k, float f) { room.scale[k][tid] = f; });
      room.ml[0][tid] = ml;
      if (rank == 0 && a.lse != nullptr && tid < n_rows) write_lse(tid, ml);
    }
    __syncthreads();
    const int share = (n_rows * HD + a.split - 1) / a.split, last = min(n_rows * HD, (rank + 1) * share);
    for (int i = rank * share + tid; i < last; i += THREADS) {
      const int r = i / HD, f = i % HD;
      float v = 0.f;
      for (int k = 0; k < a.split; ++k) v += room.scale[k][r] * cluster.map_shared_rank(&room.joined[0][0], k)[i];
      write(r, f, v, room.ml[0][r].y);
    }
    cluster.sync();   // nobody's shared memory goes away while it is read
  }
}

// CTAs per (stream, key head): until every SM has one, as long as each still gets a turn of its warps where the tables are full.
inline int split_keys(const Geometry& g, const CachedArgs& a, int n_sm, int tiles, int blocks_a_turn) {
  int split = 1;
  while (split < MAX_CLUSTER && (int64_t)g.batch * a.c.kv_heads * tiles * split < n_sm && 3 * a.c.blocks > split * WARPS * blocks_a_turn) split *= 2;
  return split;
}

template <typename T, int HD, int KIND, int NT>
cudaError_t launch_tiles(const Geometry& g, CachedArgs& a, cudaStream_t st) {
  const auto kernel = cached_attention_kernel<T, HD, KIND, NT>;
  constexpr int bytes = (int)sizeof(PartRoom<HD, 8 * NT>);
  static_assert(WARPS == 8 && MAX_CLUSTER == 8, "join_sums takes either");
  int n_sm = 0;
  const cudaError_t e = sm_count_and_smem_once(reinterpret_cast<const void*>(kernel), bytes, &n_sm);
  if (e != cudaSuccess) return e;
  const int tiles = (a.rows + 8 * NT - 1) / (8 * NT);
  if (tiles > 65535) return cudaErrorNotSupported;
  a.split = split_keys(g, a, n_sm, tiles, GROUP<HD>);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.c.kv_heads * a.split), (unsigned)g.batch, (unsigned)tiles);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.split;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, g, a);
}

template <typename T, int HD, int KIND> cudaError_t launch_rows(const Geometry& g, CachedArgs& a, cudaStream_t st) {
  if (a.rows <= 8) return launch_tiles<T, HD, KIND, 1>(g, a, st);
  if (a.rows <= 16 || sizeof(T) == 4) return launch_tiles<T, HD, KIND, 2>(g, a, st);
  if constexpr (sizeof(T) == 2) return launch_tiles<T, HD, KIND, 4>(g, a, st);
}
template <typename T, int KIND> cudaError_t launch_width(const Geometry& g, CachedArgs& a, cudaStream_t st) {
  switch (a.c.hd) {
    case 8: return launch_rows<T, 8, KIND>(g, a, st);
    case 16: return launch_rows<T, 16, KIND>(g, a, st);
    case 32: return launch_rows<T, 32, KIND>(g, a, st);
    default: return launch_rows<T, 64, KIND>(g, a, st);
  }
}
template <typename T> cudaError_t launch_kind(const Geometry& g, CachedArgs& a, cudaStream_t st) {
  return a.c.kind == GSIT_CACHE_INT8 ? launch_width<T, GSIT_CACHE_INT8>(g, a, st) : launch_width<T, GSIT_CACHE_E4M3>(g, a, st);
}

}  // namespace
}  // namespace gsit

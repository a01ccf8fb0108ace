// Attention of a step's rows over a stream's cache (gsit_im_cached_attention_fwd); the kernel, for the files that instantiate it.
//
// Everything streams through once.  A warp takes blocks of 32 positions of one key head, which one lane has copied into a ring of the warp's own (bulk
// copies, three stages, nobody else is waited for); the pages are laid out so that a lane finds what its matrix instructions take in 16 bytes, without
// bank conflicts.  8 query rows of the key head (its query heads, in every segment) are the narrow side of m16n8k16 products:
//   S^T = K Q^T      keys x rows: 8-bit integers (or e4m3) are exact in f16; q is brought to f16 by a power of two for each row, which loses nothing
//                    of bf16 worth having (what is 2^-28 of a row's largest feature); float q as two f16 terms, 22 bits
//   O^T += vs V^T P  features x rows: P turned round by movmatrix, in f16, as two terms for float; the block's scale is applied to the product in float,
//                    so it never meets the range of f16
// The open block's rows are brought to f16 by a power of two for the block (float: two terms) and go the same way, in the warp whose turn it is.
// The softmax runs over a reference that is raised only where a weight would pass 2^15, the last power of two in f16, so that most blocks need no exchange
// between lanes.  It is set so that the largest weight is 2^14 for float, 2^7 for bf16 then: f16 ends at 2^-24, and what stands out (a first position, silence) must not
// take the bits of a long even tail behind it, whose sum is not rounded.  A weight is off by 2^-11 of itself, or 2^-32 of the largest where that is more; by 2^-22, or
// 2^-39 of the largest, where it has two terms.  (With the largest at 1, 512 positions 17.4 nats below it in a warp lost all of their 1.4e-5.)
// Who takes what: where the step is small, the CTAs of a cluster share a (stream, key head, tile of rows) and join their parts through distributed shared
// memory; where there is much to read, two CTAs an SM share out all blocks of all streams and key heads evenly, whatever their lengths are, and
// a second small kernel joins the parts of those that more than one of them had.  Always in order.
// Measured, bf16: 32 streams of up to (128, 1024, 1024), 8 heads of 64, int8, every rule: 54 MB in 20 - 23 us (floor 8.3; 14 of the 19 that the kernel runs
// are the walk, the others launch, first loads and join); 64 streams of up to (512, 10000, 10000), 8 heads on 2 key heads, e4m3: 253 MB in 69 us (floor 38.7; the
// walk moves 6 TB/s; the ramp is 8 us, second pieces and the joining kernel 15).  Instructions a block: 322 for 8 rows and 399 for 16 (e4m3), 416 and 494 (int8).
// A closed pair's weight is 0 and the bytes it meets are numbers, so nothing of it counts; blocks whose scale is NaN take a way of their own.
#pragma once
#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include <algorithm>

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
// d = a b + c, c = (c0, c1) in both halves of the rows: constants, or a column's start, cost no instruction
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ void mma_k8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0, const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%7,%8,%9,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(b0), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ void add_to(float (&d)[4], const float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const float2 s = __fadd2_rn(make_float2(d[i], d[i + 1]), make_float2(v[i], v[i + 1]));
    d[i] = s.x;
    d[i + 1] = s.y;
  }
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Four bytes as two pairs of f16, exactly; integers by way of 1152 + themselves (the byte plus 128 as the last bits of 1024 + ...).  (Products of values with the
// 1152 in them, taken out of what their sum starts from, are no faster -- 16 x (4, 25, 30) rows: 34.1 us, this way 32.9 -- and lose what is 2^-17 of the block's largest.)
template <int KIND> __device__ __forceinline__ void unpack8(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (KIND == GSIT_CACHE_INT8) {
    const uint32_t u = w ^ 0x80808080u, a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    const __half2 minus = __float2half2_rn(-1152.f), x = __hadd2(*reinterpret_cast<const __half2*>(&a), minus), y = __hadd2(*reinterpret_cast<const __half2*>(&b), minus);
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

// A warp's ring: stages of B blocks -- keys, values and moments of each -- and what is known of them.
template <int HD> struct Ring {
  static constexpr int B = HD == 64 ? 1 : HD == 32 ? 2 : 4;            // blocks of a stage: 4 KB, heads of 8 2 KB
  static constexpr int MATRIX = CACHE_BLOCK * HD, MOMENTS = 4 * CACHE_BLOCK, BLOCK = 2 * MATRIX + MOMENTS;
  static constexpr int STAGES = 3, BYTES = STAGES * B * BLOCK;
};
struct BlockInfo {
  float ks, vs;
  int seg, first;          // segment (3: there is no such block), first position
};

// F features of a result, times `by` (out may lie at any element).
template <int F> __device__ __forceinline__ void store_features(float* out, const float (&v)[F], float by) {
#pragma unroll
  for (int e = 0; e < F; ++e) out[e] = v[e] * by;
}
template <int F> __device__ __forceinline__ void store_features(__nv_bfloat16* out, const float (&v)[F], float by) {
  if (F == 2 && (reinterpret_cast<uintptr_t>(out) & 3u) == 0) *reinterpret_cast<uint32_t*>(out) = ptx::pack_bf16(v[0] * by, v[F - 1] * by);
  else
#pragma unroll
    for (int e = 0; e < F; ++e) store_as(out + e, v[e] * by);
}

// The parts that are joined: of each warp, then of the CTA (in the first warp's place).
template <int HD, int R> struct PartRoom {
  float acc[WARPS][R][HD + 4];            // (rows four banks apart: a fragment's columns meet other banks)
  float2 ml[WARPS][R];                    // (reference, sum)
};
// Lanes 0 .. 7 of a warp have (reference, sum) of eight parts of a row, or (-inf, 0): to the factors that bring them to one reference, and that
// reference with the sum, in all lanes.  A part without a number among its scores has no reference: its sum is 0, or NaN where a score was,
// and then so is everything.
__device__ __forceinline__ float2 join_sums(float2 part, float& factor) {
  float top = part.x;
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  factor = part.x == -INFINITY ? 1.f : ptx::ex2(part.x - top);
  float sum = factor * part.y;
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return make_float2(__shfl_sync(0xffffffffu, top, 0), __shfl_sync(0xffffffffu, sum, 0));
}

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, int bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

// A stream's list of blocks for one tile of rows: the full blocks of the segments that a real row is open to, then their open ones.
struct BlockList {
  int len[3], upto[3];     // positions of the segments that are walked; full blocks up to the end of each
  int full, all;
  __device__ __forceinline__ int segment(int i) const { return i >= upto[1] ? 2 : i >= upto[0] ? 1 : 0; }
};
__device__ __forceinline__ BlockList list_blocks(const Geometry& g, const CachedArgs& a, int b, int row0, int n_rows) {
  BlockList l;
  int real[3], opens = 0;
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    l.len[s] = held_rows(a.c, g.status, b, s);
    real[s] = valid_rows(g, b, s);
  }
#pragma unroll
  for (int s = 0; s < 3; ++s)
    if (max(row0, g.off(s) * a.group) < min(row0 + n_rows, (g.off(s) + real[s]) * a.group)) opens |= (int)(g.allowed >> (3 * s)) & 7;
  l.full = 0;
  int open = 0;
#pragma unroll
  for (int s = 0; s < 3; ++s) {
    if (!((opens >> s) & 1)) l.len[s] = 0;
    l.full += l.len[s] / CACHE_BLOCK;
    l.upto[s] = l.full;
    open += l.len[s] % CACHE_BLOCK != 0;
  }
  l.all = l.full + open;
  return l;
}

// Parts in the workspace: of every CTA its first and its last piece.
template <int HD, int R> struct Part {
  float acc[R][HD];
  float2 ml[R];
};

// CTAs of an SM: two where their registers allow it.  (Tiles of 32 rows, one CTA an SM, took 44 us where those of 16 took 34.)
template <typename T, int NT> constexpr int RESIDENT = NT == 1 || sizeof(T) == 2 ? 2 : 1;

// Weights, in base 2: the largest that f16 takes, and where the reference puts a new largest one.  Sums of rows take them in this unit, so that they stay in
// the range of what they add up.
constexpr float MOST_WEIGHT = 15.f, WEIGHT_UNIT = 32768.f;
template <typename T> constexpr float FIRST_WEIGHT = sizeof(T) == 4 ? 14.f : 7.f;

template <typename T, int HD, int KIND, int NT>
__global__ void __launch_bounds__(THREADS, RESIDENT<T, NT>)
cached_attention_kernel(const __grid_constant__ Geometry g, const __grid_constant__ CachedArgs a) {
  constexpr int R = 8 * NT, TERMS = sizeof(T) == 4 ? 2 : 1, KS = HD == 8 ? 1 : HD / 16, MD = KS;
  constexpr float LIFT = FIRST_WEIGHT<T>;
  using RingOf = Ring<HD>;
  constexpr int B = RingOf::B, STAGES = RingOf::STAGES;
  using Room = PartRoom<HD, R>;
  extern __shared__ __align__(128) uint8_t smem[];
  Room& room = *reinterpret_cast<Room*>(smem);             // where the rings were, when they are done with
  __shared__ QueryRow s_row[WARPS][R];
  __shared__ BlockInfo s_info[WARPS][STAGES][B];
  __shared__ __align__(8) uint64_t s_bar[WARPS][STAGES];
  __shared__ uint32_t s_gave_up;
  __shared__ int s_sum[WARPS];
  __shared__ int2 s_first;                   // stream that the share begins in, blocks before it
  const Cache& c = a.c;
  const int tid = threadIdx.x, warp = ptx::uniform(tid >> 5), lane = tid & 31, gr = lane >> 2, t = lane & 3;
  ptx::load_params_early(g, a);
  const uint32_t bars = smem_u32(s_bar[warp]), ring = smem_u32(smem) + warp * RingOf::BYTES;
  if (lane == 0) {
    for (int i = 0; i < STAGES; ++i) ptx::mbar_init(bars + 8 * i, B);
    ptx::mbar_init_fence();
  }
  if (tid == 0) s_gave_up = 0;
  __syncthreads();
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const ptx::WaitCtx wait = {g.status, smem_u32(&s_gave_up)};
  uint32_t stage = 0, phase = 0;             // of the warp's ring: they go on from piece to piece
  const bool timed = a.causal != 0 || a.slopes != nullptr;

  // One piece: blocks [lo, hi) of the list of stream b for key head hk, rows from row0 on, into the room (the warps' parts).
  auto walk = [&](int b, int hk, int row0, int n_rows, const BlockList& list, int lo, int hi) {
    const int first = lo + warp * B, last = min(hi, list.full);
    constexpr int turn = WARPS * B;
    // Everything that is waited for is asked for as early as it can be: the queries, pages, the first blocks, what the rows are.
    uint32_t raw[NT][KS][2][TERMS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = min(8 * n + gr, n_rows - 1) + row0;
      const T* q = static_cast<const T*>(a.q) + ((int64_t)b * g.L + r / a.group) * a.ldq + (int64_t)(hk * a.group + r % a.group) * HD + 2 * t;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int h = 0; h < (HD > 8 ? 2 : 1); ++h) {
          if constexpr (sizeof(T) == 2) raw[n][k][h][0] = *reinterpret_cast<const uint32_t*>(q + 16 * k + 8 * h);
          else {
            const uint2 v = *reinterpret_cast<const uint2*>(q + 16 * k + 8 * h);
            raw[n][k][h][0] = v.x;
            raw[n][k][h][TERMS - 1] = v.y;
          }
        }
    }
    // lanes know where the blocks of the warp's next 32 / B turns lie, and each sees to its own: copies into the stage, and what is known of it
    int ahead = first, known = 0;
    int64_t head = -1;
    const float* moments = nullptr;
    BlockInfo info = {0.f, 0.f, 3, 0};
    uint32_t to = stage;
    auto copy = [&]() {
      if (known == 0) {
        const int i = ahead + lane / B * turn + lane % B, s = list.segment(i), j = i - (s == 0 ? 0 : s == 1 ? list.upto[0] : list.upto[1]);
        head = -1;
        info.seg = 3;
        if (i < last) {
          const int page = real_page(c, c.tables[((int64_t)b * 3 + s) * c.blocks + j]);
          if (page < 0) raise_flag(g, GSIT_DEVFLAG_CLAMPED);
          else {
            head = (int64_t)page * c.kv_heads + hk;
            info = {c.key_scale[head], c.value_scale[head], s, j * CACHE_BLOCK};
            if (timed && c.times != nullptr) moments = c.times + (int64_t)page * CACHE_BLOCK;
          }
        }
        known = 32 / B;
      }
      const int from = (32 / B - known) * B;
      if (lane >= from && lane < from + B && head >= 0) {
        const uint32_t bar = bars + 8 * to, at = ring + (to * B + lane - from) * RingOf::BLOCK;
        bulk_copy(at, c.keys + head * RingOf::MATRIX, RingOf::MATRIX, bar);
        bulk_copy(at + RingOf::MATRIX, c.values + head * RingOf::MATRIX, RingOf::MATRIX, bar);
        if (moments != nullptr) bulk_copy(at + 2 * RingOf::MATRIX, moments, RingOf::MOMENTS, bar);
      }
      ahead += turn;
      --known;
      to = to + 1 == STAGES ? 0 : to + 1;
    };
    // ... behind the copies, which need not wait for the scales: what is known, and the arrival that lets the stage's phase end
    auto tell = [&](uint32_t stage_of, int from) {
      if (lane >= from && lane < from + B) {
        s_info[warp][stage_of][lane - from] = info;
        ptx::mbar_expect_tx(bars + 8 * stage_of, head < 0 ? 0 : 2 * RingOf::MATRIX + (moments != nullptr ? RingOf::MOMENTS : 0));
      }
    };
    static_assert(STAGES == 3 && 32 / B >= 2, "two stages of one batch of pages are asked for ahead");
    const bool one = first < last, two = first + turn < last;
    if (one) copy();
    if (two) copy();

    // ---- the rows: row r of a key head is row r / group of the step, head hk * group + r % group ----
    QueryRow* const rows_of = s_row[warp];
    if (lane < R) {
      QueryRow x = {0.f, -INFINITY, 0.f, 0};
      if (lane < n_rows) {
        const int l = (row0 + lane) / a.group, s = segment_of(g, l), at = l - g.off(s), n = valid_rows(g, b, s);
        if (at < n) {
          if (timed) {
            x.time = a.times.p != nullptr ? a.times.at(b, l) : (float)(held_rows(c, g.status, b, s) - n + at);
            x.slope2 = a.slopes != nullptr ? a.slopes[hk * a.group + (row0 + lane) % a.group] * LOG2E : 0.f;
          }
          x.limit = a.causal ? x.time : INFINITY;
          x.opens = (int)(g.allowed >> (3 * s)) & 7;
        }
      }
      rows_of[lane] = x;
    }
    __syncwarp();
    if (one) tell(stage, 0);
    if (two) tell(stage + 1 == STAGES ? 0 : stage + 1, B);

    // ---- queries as B operands, and what brings a dot back to a score ----
    uint32_t qf[NT][TERMS][KS][2];
    float2 back[NT];                       // of the columns 2 t and 2 t + 1 of each tile
    uint32_t col_opens = 0, every = 7;     // four bits for each column; segments that all of them are open to
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const bool there = rows_of[8 * n + gr].opens != 0;
      float2 f[KS][2];
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          f[k][h] = make_float2(0.f, 0.f);
          if (there && (HD > 8 || h == 0)) {
            if constexpr (sizeof(T) == 2) unpack_bf16(raw[n][k][h][0], f[k][h].x, f[k][h].y);
            else f[k][h] = make_float2(__uint_as_float(raw[n][k][h][0]), __uint_as_float(raw[n][k][h][TERMS - 1]));
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
      back[n] = make_float2(__shfl_sync(0xffffffffu, p.down, 8 * t) * a.inner, __shfl_sync(0xffffffffu, p.down, 8 * t + 4) * a.inner);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int opens = rows_of[8 * n + 2 * t + e].opens;
        col_opens |= (uint32_t)opens << (4 * (2 * n + e));
        if (8 * n + 2 * t + e < n_rows) every &= opens;   // (columns behind the last row write nothing: whatever they see)
      }
    }
    every = __reduce_and_sync(0xffffffffu, every);
    float2 o[MD][NT][2], ref[NT], sum[NT];   // pairs: columns 2 t, 2 t + 1
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      ref[n] = make_float2(-INFINITY, -INFINITY);
      sum[n] = make_float2(0.f, 0.f);
#pragma unroll
      for (int m = 0; m < MD; ++m) o[m][n][0] = o[m][n][1] = make_float2(0.f, 0.f);
    }

    // One block of segment `seg`: keys(m, k, term, fragment) and values(m, k, term, fragment) give A operands, of IN terms; FULL: all 32 positions.
    auto attend = [&](auto terms_in, auto whole, int seg, int rows, float ks, float vs, const float (&times)[4], auto keys, auto values) {
      constexpr int IN = decltype(terms_in)::value;
      constexpr bool FULL = decltype(whole)::value != 0;
      float zero[4] = {0.f, 0.f, 0.f, 0.f};
      float s[2][NT][4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        float small[NT][4];                // float: the products with a smaller term
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
                auto product = [&](float (&to)[4], const float (&from)[4]) {
                  if constexpr (HD == 8) mma_k8(to, f[0], f[1], qf[n][y][k][0], from);
                  else mma(to, f, qf[n][y][k][0], qf[n][y][k][1], from);
                };
                if (TERMS == 1 || (k == 0 && w + y == 0)) product(s[m][n], k > 0 ? s[m][n] : zero);
                else if (w + y > 0) product(small[n], k > 0 || w > 0 ? small[n] : zero);
                else {   // the matrix instructions cut their sums off, always the same way: float adds them itself, rounded (0 - 3 % of a call's time)
                  float add[4];
                  product(add, zero);
                  add_to(s[m][n], add);
                }
              }
          }
        if (TERMS == 2) {
#pragma unroll
          for (int n = 0; n < NT; ++n) add_to(s[m][n], small[n]);
        }
      }
      // scores in base 2, pairs of columns; positions 16 m + 8 h + gr
      float2 x[NT][2][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 f = __fmul2_rn(back[n], make_float2(ks, ks));
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) x[n][m][h] = __fmul2_rn(make_float2(s[m][n][2 * h], s[m][n][2 * h + 1]), f);
      }
      if (a.softcap > 0.f) {
        // bf16: under caps of 64 by an exponential and a reciprocal (see fast_cap), under wider ones to 2^-20 of the score itself
        auto bend = [&](float2 y) {
          if (sizeof(T) == 4) return make_float2(tanhf(y.x) * a.outer, tanhf(y.y) * a.outer);
          if (!a.fast_cap) return __fmul2_rn(tanh_any2(y), make_float2(a.outer, a.outer));
          auto fast = [&](float v) { return fmaf(-2.f * a.outer, reciprocal(ptx::ex2(v) + 1.f), a.outer); };
          return make_float2(fast(y.x), fast(y.y));
        };
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) x[n][m][h] = bend(x[n][m][h]);
      }
      if (!FULL || timed || !((every >> seg) & 1u)) {   // closed pairs -inf
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const bool m0 = (col_opens >> (8 * n + seg)) & 1u, m1 = (col_opens >> (8 * n + 4 + seg)) & 1u;
          float2 time = make_float2(0.f, 0.f), limit = time, slope2 = time;
          if (timed) {
            const QueryRow &r0 = rows_of[8 * n + 2 * t], &r1 = rows_of[8 * n + 2 * t + 1];
            time = make_float2(r0.time, r1.time);
            limit = make_float2(r0.limit, r1.limit);
            slope2 = make_float2(-r0.slope2, -r1.slope2);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float2& v = x[n][i / 2][i % 2];
            const bool there = FULL || 8 * i + gr < rows;
            bool o0 = m0 && there, o1 = m1 && there;
            if (timed) {
              const float2 d = __fadd2_rn(time, make_float2(-times[i], -times[i]));
              v = __ffma2_rn(slope2, make_float2(fabsf(d.x), fabsf(d.y)), v);
              o0 = o0 && times[i] <= limit.x;
              o1 = o1 && times[i] <= limit.y;
            }
            v = make_float2(o0 ? v.x : -INFINITY, o1 ? v.y : -INFINITY);
          }
        }
      }
      bool raise = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {   // (differences, which are exact where it matters: nothing passes 2^15 by a rounding)
        const float2 top = make_float2(fmaxf(ptx::fmax3(x[n][0][0].x, x[n][0][1].x, x[n][1][0].x), x[n][1][1].x),
                                       fmaxf(ptx::fmax3(x[n][0][0].y, x[n][0][1].y, x[n][1][0].y), x[n][1][1].y));
        const float2 over = __fadd2_rn(top, make_float2(-ref[n].x, -ref[n].y));
        raise = raise || over.x > MOST_WEIGHT || over.y > MOST_WEIGHT;
      }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float2 top = make_float2(fmaxf(ptx::fmax3(x[n][0][0].x, x[n][0][1].x, x[n][1][0].x), x[n][1][1].x),
                                   fmaxf(ptx::fmax3(x[n][0][0].y, x[n][0][1].y, x[n][1][0].y), x[n][1][1].y));
#pragma unroll
          for (int l = 4; l < 32; l <<= 1) top = make_float2(fmaxf(top.x, __shfl_xor_sync(0xffffffffu, top.x, l)), fmaxf(top.y, __shfl_xor_sync(0xffffffffu, top.y, l)));
          auto below = [](float x) {   // (scores of 2^24 and more have no place for the distance)
            const float r = x - LIFT;
            return x - r > MOST_WEIGHT ? x : r;
          };
          top = make_float2(fmaxf(below(top.x), ref[n].x), fmaxf(below(top.y), ref[n].y));
          const float2 f = make_float2(top.x > ref[n].x ? ptx::ex2(ref[n].x - top.x) : 1.f, top.y > ref[n].y ? ptx::ex2(ref[n].y - top.y) : 1.f);
          sum[n] = __fmul2_rn(sum[n], f);
#pragma unroll
          for (int m = 0; m < MD; ++m) {
            o[m][n][0] = __fmul2_rn(o[m][n][0], f);
            o[m][n][1] = __fmul2_rn(o[m][n][1], f);
          }
          ref[n] = top;
        }
      }
      const bool broken = !(fabsf(vs) < INFINITY);
      uint32_t seen = 0;                   // where the block's values are broken: columns that any position is open to
      if (broken)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            bool any = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) any = any || (e ? x[n][i / 2][i % 2].y : x[n][i / 2][i % 2].x) != -INFINITY;
            const uint32_t who = __ballot_sync(0xffffffffu, any) & (0x11111111u << t);
            seen |= (who != 0 ? 1u : 0u) << (2 * n + e);
          }
      // weights, turned round into B operands: keys 2 t, 2 t + 1 (and + 8) of row gr
      uint32_t pf[NT][TERMS][2][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float2 r = make_float2(ref[n].x == -INFINITY ? 0.f : -ref[n].x, ref[n].y == -INFINITY ? 0.f : -ref[n].y);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float2 v = __fadd2_rn(x[n][m][h], r), p = make_float2(ptx::ex2(v.x), ptx::ex2(v.y));
            sum[n] = __fadd2_rn(sum[n], p);
            const uint32_t w = f16x2(p.x, p.y);
            pf[n][0][m][h] = turned_round(w);
            if constexpr (TERMS == 2) pf[n][1][m][h] = turned_round(f16x2_rest(p.x, p.y, w));
          }
      }
#pragma unroll
      for (int m = 0; m < MD; ++m) {
        float add[NT][4];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int w = 0; w < IN; ++w) {
            uint32_t f[4];
            values(m, k, w, f);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int y = 0; y < TERMS - w; ++y) mma(add[n], f, pf[n][y][k][0], pf[n][y][k][1], k + w + y > 0 ? add[n] : zero);
          }
        if (!broken) {
          const float by = vs * (1.f / WEIGHT_UNIT);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            o[m][n][0] = __ffma2_rn(make_float2(by, by), make_float2(add[n][0], add[n][1]), o[m][n][0]);
            if constexpr (HD > 8) o[m][n][1] = __ffma2_rn(make_float2(by, by), make_float2(add[n][2], add[n][3]), o[m][n][1]);
          }
        }
      }
      if (broken)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int m = 0; m < MD; ++m) {
            if ((seen >> (2 * n)) & 1u) o[m][n][0].x = o[m][n][1].x = vs;
            if ((seen >> (2 * n + 1)) & 1u) o[m][n][0].y = o[m][n][1].y = vs;
          }
    };

    // The open blocks, each the next warp's in turn, while the first copies are under way: rows in memory, brought to f16 by a power of two for all of a block's.
#pragma unroll 1
    for (int r = 0, at = list.full; r < 3; ++r) {
      const int n = r == 0 ? list.len[0] : r == 1 ? list.len[1] : list.len[2], rows = n % CACHE_BLOCK, j = n / CACHE_BLOCK;
      if (rows == 0) continue;
      const int i = at++;
      if (i < lo || i >= hi || ((max(0, last - lo) + B - 1) / B + i - max(lo, list.full)) % WARPS != warp) continue;
      const int64_t from = open_at(c, b, r, j, hk);
      const T* const key = static_cast<const T*>(c.open_keys) + from;
      const T* const value = static_cast<const T*>(c.open_values) + from;
      float times[4] = {0.f, 0.f, 0.f, 0.f};
      if (timed) {
        const int page = c.times == nullptr ? 0 : real_page(c, c.tables[((int64_t)b * 3 + r) * c.blocks + j]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          times[i] = c.times == nullptr ? (float)(j * CACHE_BLOCK + 8 * i + gr) : page >= 0 ? c.times[(int64_t)page * CACHE_BLOCK + 8 * i + gr] : 0.f;
      }
      // all of it at once into registers, as the fragments want it: pairs of features of positions 8 i + gr
      uint32_t words[2][4][HD / 8][TERMS];
#pragma unroll
      for (int w = 0; w < 2; ++w)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int k = 0; k < HD / 8; ++k) {
            const T* p = (w ? value : key) + (8 * i + gr) * HD + 8 * k + 2 * t;
            uint2 v = make_uint2(0u, 0u);
            if (8 * i + gr < rows) {
              if constexpr (sizeof(T) == 2) v.x = *reinterpret_cast<const uint32_t*>(p);
              else v = *reinterpret_cast<const uint2*>(p);
            }
            words[w][i][k][0] = v.x;
            if constexpr (TERMS == 2) words[w][i][k][1] = v.y;
          }
      auto pair = [&](int w, int i, int k) {
        float2 v;
        if constexpr (sizeof(T) == 2) unpack_bf16(words[w][i][k][0], v.x, v.y);
        else v = make_float2(__uint_as_float(words[w][i][k][0]), __uint_as_float(words[w][i][k][TERMS - 1]));
        return v;
      };
      Power up[2];
      float by[2];
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int k = 0; k < HD / 8; ++k) {
            const float2 v = pair(w, i, k);
            top = max(top, max(__float_as_uint(v.x) & 0x7fffffffu, __float_as_uint(v.y) & 0x7fffffffu));
          }
        top = __reduce_max_sync(0xffffffffu, top);
        const bool broken = top >= 0x7f800000u;
        up[w] = top > 0 && !broken ? power_for(__uint_as_float(top), 14) : Power{1.f, 1.f};
        by[w] = broken ? __int_as_float(0x7fffffff) : up[w].down;
        if (broken)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < HD / 8; ++k)
#pragma unroll
              for (int e = 0; e < TERMS; ++e) words[w][i][k][e] = 0u;
      }
      auto term = [&](float2 v, float f, int w) {
        v = __fmul2_rn(v, make_float2(f, f));
        const uint32_t x = f16x2(v.x, v.y);
        return w == 0 ? x : f16x2_rest(v.x, v.y, x);
      };
      attend(std::integral_constant<int, TERMS>{}, std::integral_constant<int, 0>{}, r, rows, by[0], by[1], times,
             [&](int m, int k, int w, uint32_t (&f)[4]) {
#pragma unroll
               for (int i = 0; i < 4; ++i)   // position halves i % 2, feature halves i / 2
                 f[i] = HD > 8 || i < 2 ? term(pair(0, 2 * m + i % 2, HD > 8 ? 2 * k + i / 2 : 0), up[0].up, w) : 0u;
             },
             [&](int m, int k, int w, uint32_t (&f)[4]) {
#pragma unroll
               for (int i = 0; i < 4; ++i)   // feature halves i % 2, position halves i / 2; rows of features come in, turned round
                 f[i] = HD > 8 || i % 2 == 0 ? turned_round(term(pair(1, 2 * k + i / 2, HD > 8 ? 2 * m + i % 2 : 0), up[1].up, w)) : 0u;
             });
    }

#pragma unroll 1
    for (int now = first; now < last; now += turn) {
      if (ahead < last) {   // into the stage that was read before this one
        const uint32_t into = to;
        copy();
        tell(into, (32 / B - known - 1) * B);
      }
      ptx::mbar_wait_warp(wait, bars + 8 * stage, phase);
#pragma unroll
      for (int u = 0; u < B; ++u) {
        const BlockInfo x = s_info[warp][stage][u];
        if (x.seg == 3) continue;
        const uint32_t at = ring + (stage * B + u) * RingOf::BLOCK, key = at + (HD == 8 ? 8 : 16) * lane, value = key + RingOf::MATRIX;
        float times[4] = {0.f, 0.f, 0.f, 0.f};
        if (timed)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            times[i] = c.times != nullptr ? *reinterpret_cast<const float*>(smem + (at - smem_u32(smem)) + 2 * RingOf::MATRIX + 4 * (8 * i + gr)) : (float)(x.first + 8 * i + gr);
        // fragments of keys come by (feature group, position half), of values by (feature group, position half), both halves in 16 bytes
        uint4 kw[KS], vw[MD];
        auto take = [&](uint4 (&w)[KS], uint32_t from) {
#pragma unroll
          for (int i = 0; i < KS; ++i) {
            if constexpr (HD == 8) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[i].x), "=r"(w[i].y) : "r"(from) : "memory");
            else w[i] = lds16(from + 512 * i);
          }
        };
        take(kw, key);
        attend(std::integral_constant<int, 1>{}, std::integral_constant<int, 1>{}, x.seg, CACHE_BLOCK, x.ks, x.vs, times,
               [&](int m, int k, int, uint32_t (&f)[4]) {
                 if constexpr (HD == 8) unpack8<KIND>(m ? kw[0].y : kw[0].x, f[0], f[1]);
                 else {
                   unpack8<KIND>(m ? kw[k].z : kw[k].x, f[0], f[1]);
                   unpack8<KIND>(m ? kw[k].w : kw[k].y, f[2], f[3]);
                 }
               },
               [&](int m, int k, int, uint32_t (&f)[4]) {
                 if (m + k == 0) take(vw, value);
                 if constexpr (HD == 8) {
                   unpack8<KIND>(k ? vw[0].y : vw[0].x, f[0], f[2]);
                   f[1] = f[3] = 0u;
                 } else {
                   unpack8<KIND>(k ? vw[m].z : vw[m].x, f[0], f[1]);
                   unpack8<KIND>(k ? vw[m].w : vw[m].y, f[2], f[3]);
                 }
               });
      }
      __syncwarp();   // every lane has used what it read of the stage
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      phase ^= stage == 0;
    }
    // ---- the warps' parts ----
    __syncthreads();   // nobody's ring is in use any more
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = 8 * n + 2 * t;
#pragma unroll
      for (int l = 4; l < 32; l <<= 1) sum[n] = make_float2(sum[n].x + __shfl_xor_sync(0xffffffffu, sum[n].x, l), sum[n].y + __shfl_xor_sync(0xffffffffu, sum[n].y, l));
      if (gr == 0) {
        room.ml[warp][row] = make_float2(ref[n].x, sum[n].x);
        room.ml[warp][row + 1] = make_float2(ref[n].y, sum[n].y);
      }
#pragma unroll
      for (int m = 0; m < MD; ++m)
#pragma unroll
        for (int h = 0; h < (HD > 8 ? 2 : 1); ++h) {
          room.acc[warp][row][16 * m + 8 * h + gr] = o[m][n][h].x;
          room.acc[warp][row + 1][16 * m + 8 * h + gr] = o[m][n][h].y;
        }
    }
    __syncthreads();
  };

  // a warp takes every eighth row of a piece, its lanes the features
  constexpr int F = HD < 32 ? 1 : HD / 32;
  const bool mine = lane * F < HD;
  auto finish = [&](int b, int hk, int row, const float (&v)[F], float2 ml) {
    const int l = row / a.group, head = hk * a.group + row % a.group;
    T* const out = static_cast<T*>(a.out) + ((int64_t)b * g.L + l) * g.d + (int64_t)head * HD + lane * F;
    const float inv = ml.y != 0.f ? WEIGHT_UNIT / ml.y : 0.f;
    if (mine) store_features<F>(out, v, inv);
    if (a.lse != nullptr && lane == 0) a.lse[((int64_t)b * g.heads + head) * g.L + l] = ml.y != 0.f ? (ml.x + log2f(ml.y)) * LN2 : -INFINITY;
  };
  // row r of the room, its warps' parts joined
  auto join_warps = [&](int r, float (&v)[F]) {
    float factor;
    const float2 ml = join_sums(lane < WARPS ? room.ml[lane][r] : make_float2(-INFINITY, 0.f), factor);
#pragma unroll
    for (int e = 0; e < F; ++e) v[e] = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float f = __shfl_sync(0xffffffffu, factor, w);
      if (mine)
#pragma unroll
        for (int e = 0; e < F; ++e) v[e] = fmaf(f, room.acc[w][r][lane * F + e], v[e]);
    }
    return ml;
  };

  // ---- this CTA's share: one piece, or an even share of all streams' blocks, in pieces of one stream and key head ----
  const bool even = a.parts != nullptr;
  const int rank = even ? 0 : (int)blockIdx.x % a.split;
  int row0 = 0, n_rows = a.rows;
  if (a.rows > R && a.mixed) {
    row0 = blockIdx.z * R;
    n_rows = min(R, a.rows - row0);
  } else if (a.rows > R) {   // tiles of one segment's rows, so that a tile walks no more than they see
    int tile = blockIdx.z, seg = 0;
    for (; seg < 2 && tile >= (g.len(seg) * a.group + R - 1) / R; ++seg) tile -= (g.len(seg) * a.group + R - 1) / R;
    row0 = g.off(seg) * a.group + tile * R;
    n_rows = min(R, g.len(seg) * a.group - tile * R);
  }
  int b = even ? 0 : (int)blockIdx.y, hk = even ? 0 : (int)blockIdx.x / a.split, pieces = 0;
  int64_t at = 0, end = 1, base = 0;         // in blocks of all streams and key heads: where the share goes on and ends, where stream b begins
  if (even) {
    // Streams' blocks added up, 256 at a time: the total, then the stream that the share begins in.  CTA 0 leaves the sums for the joining kernel.
    int* const before = reinterpret_cast<int*>(a.parts + (size_t)gridDim.x * 2 * (sizeof(Part<HD, R>) / sizeof(float)));
    int total = 0;
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) {
      at = (int64_t)total * c.kv_heads * blockIdx.x / gridDim.x;
      int run = 0;
#pragma unroll 1
      for (int b0 = 0; b0 < g.batch; b0 += THREADS) {
        const int i = b0 + tid, n = i < g.batch ? list_blocks(g, a, i, 0, a.rows).all : 0;
        int upto = n;
#pragma unroll
        for (int l = 1; l < 32; l <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, upto, l);
          if (lane >= l) upto += x;
        }
        __syncthreads();
        if (lane == 31) s_sum[warp] = upto;
        __syncthreads();
        int here = 0, mine_before = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          if (w < warp) mine_before += s_sum[w];
          here += s_sum[w];
        }
        const int from = run + mine_before + upto - n;
        if (pass == 1) {
          if ((int64_t)from * c.kv_heads <= at && at < (int64_t)(from + n) * c.kv_heads) s_first = make_int2(i, from);
          if (blockIdx.x == 0 && i < g.batch) before[i] = from;
        }
        run += here;
        if (g.batch <= THREADS && pass == 0) {   // the one round that there is answers both
          at = (int64_t)run * c.kv_heads * blockIdx.x / gridDim.x;
          if ((int64_t)from * c.kv_heads <= at && at < (int64_t)(from + n) * c.kv_heads) s_first = make_int2(i, from);
          if (blockIdx.x == 0 && i < g.batch) before[i] = from;
        }
      }
      total = run;
      if (g.batch <= THREADS) break;
    }
    if (blockIdx.x == 0 && tid == 0) before[g.batch] = total;
    __syncthreads();
    const int64_t units = (int64_t)total * c.kv_heads;
    at = units * blockIdx.x / gridDim.x;
    end = units * (blockIdx.x + 1) / gridDim.x;
    if (at >= end) return;
    b = s_first.x;
    base = (int64_t)s_first.y * c.kv_heads;
  }
  BlockList list = list_blocks(g, a, b, row0, n_rows);
#pragma unroll 1
  while (true) {
    int lo, hi;
    if (even) {
      while (at >= base + (int64_t)list.all * c.kv_heads) {   // the next stream that has any
        base += (int64_t)list.all * c.kv_heads;
        list = list_blocks(g, a, ++b, row0, n_rows);
      }
      hk = (int)((at - base) / list.all);
      lo = (int)((at - base) - (int64_t)hk * list.all);
      hi = (int)min((int64_t)list.all, lo + (end - at));
      at += hi - lo;
    } else {
      lo = (int)((int64_t)list.all * rank / a.split);
      hi = (int)((int64_t)list.all * (rank + 1) / a.split);
      at = end;
    }
    walk(b, hk, row0, n_rows, list, lo, hi);
    const bool whole = lo == 0 && hi == list.all;
    Part<HD, R>& part = reinterpret_cast<Part<HD, R>*>(a.parts)[2 * blockIdx.x + (pieces > 0)];
    for (int r = warp; r < n_rows; r += WARPS) {
      float v[F];
      const float2 ml = join_warps(r, v);
      if (a.split == 1 && (!even || whole)) finish(b, hk, row0 + r, v, ml);
      else {
        __syncwarp();
        float* const to = even ? part.acc[r] : room.acc[0][r];
        if (mine)
#pragma unroll
          for (int e = 0; e < F; ++e) to[lane * F + e] = v[e];
        if (lane == 0) (even ? part.ml[r] : room.ml[0][r]) = ml;
      }
    }
    if (at >= end) break;
    ++pieces;
    ptx::fence_async_smem();   // what was joined here lies where the next piece's copies go
    __syncthreads();
  }
  if (a.split == 1) return;
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  for (int r = rank * WARPS + warp; r < n_rows; r += a.split * WARPS) {
    float factor, v[F] = {};
    const float2 ml = join_sums(lane < a.split ? cluster.map_shared_rank(&room, lane)->ml[0][r] : make_float2(-INFINITY, 0.f), factor);
#pragma unroll
    for (int k = 0; k < MAX_CLUSTER; ++k)
      if (k < a.split) {
        const float f = __shfl_sync(0xffffffffu, factor, k);
        if (mine)
#pragma unroll
          for (int e = 0; e < F; ++e) v[e] = fmaf(f, cluster.map_shared_rank(&room, k)->acc[0][r][lane * F + e], v[e]);
      }
    finish(b, hk, row0 + r, v, ml);
  }
  cluster.sync();   // nobody's shared memory goes away while it is read
}

// Joins the parts of the (stream, key head)s that more than one CTA had, and writes the rows of those that none had.  A warp takes one row.
template <typename T, int HD, int R>
__global__ void __launch_bounds__(THREADS) cached_join_kernel(const __grid_constant__ Geometry g, const __grid_constant__ CachedArgs a, const int ctas) {
  const Part<HD, R>* const parts = reinterpret_cast<const Part<HD, R>*>(a.parts);
  const int* const before = reinterpret_cast<const int*>(parts + 2 * ctas);
  const int lane = threadIdx.x & 31, item = (int)(blockIdx.x * WARPS + (threadIdx.x >> 5));
  constexpr int F = HD < 32 ? 1 : HD / 32;
  const bool mine = lane * F < HD;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const int r = item % a.rows, pair = item / a.rows, hk = pair % a.c.kv_heads, b = pair / a.c.kv_heads;
  if (b >= g.batch) return;
  const int start = before[b], n = before[b + 1] - start;
  const int64_t units = (int64_t)before[g.batch] * a.c.kv_heads, from = (int64_t)start * a.c.kv_heads + (int64_t)hk * n, to = from + n;
  auto cta_of = [&](int64_t unit) {   // the last one whose share begins at or before it
    int k = (int)(unit * ctas / units);
    while (k + 1 < ctas && units * (k + 1) / ctas <= unit) ++k;
    while (k > 0 && units * k / ctas > unit) --k;
    return k;
  };
  float v[F] = {};
  float2 ml = make_float2(-INFINITY, 0.f);
  if (n > 0) {
    const int k0 = cta_of(from), k1 = cta_of(to - 1);
    if (k0 == k1) return;   // that CTA has written the row
    auto part_of = [&](int k) -> const Part<HD, R>& { return parts[2 * k + (k == k0 && units * k / ctas < from)]; };
    auto empty = [&](int k) { return units * k / ctas == units * (k + 1) / ctas; };   // more CTAs than blocks
    // 32 parts at a time: lanes have their references and sums, then the features, with several parts' loads under way
    float top = -INFINITY, sum = 0.f;
    for (int k = k0 + lane; k <= k1; k += 32)
      if (!empty(k)) top = fmaxf(top, part_of(k).ml[r].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    for (int k = k0; k <= k1; k += 32) {
      const bool has = k + lane <= k1 && !empty(k + lane);
      const float2 p = has ? part_of(k + lane).ml[r] : make_float2(-INFINITY, 0.f);
      const float f = !has ? 0.f : p.x == -INFINITY ? 1.f : ptx::ex2(p.x - top);
      const uint32_t those = __ballot_sync(0xffffffffu, has);
      sum += f * p.y;
#pragma unroll 8
      for (int i = 0; i < min(32, k1 - k + 1); ++i) {
        const float by = __shfl_sync(0xffffffffu, f, i);
        if (mine && ((those >> i) & 1u))
#pragma unroll
          for (int e = 0; e < F; ++e) v[e] = fmaf(by, part_of(k + i).acc[r][lane * F + e], v[e]);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    ml = make_float2(top, sum);
  }
  const int l = r / a.group, head = hk * a.group + r % a.group;
  if (mine) store_features<F>(static_cast<T*>(a.out) + ((int64_t)b * g.L + l) * g.d + (int64_t)head * HD + lane * F, v, ml.y != 0.f ? WEIGHT_UNIT / ml.y : 0.f);
  if (a.lse != nullptr && lane == 0) a.lse[((int64_t)b * g.heads + head) * g.L + l] = ml.y != 0.f ? (ml.x + log2f(ml.y)) * LN2 : -INFINITY;
}

// Small steps: CTAs per (stream, key head, tile) until every SM has one, as long as each still gets a turn of its warps where the tables are full.
inline int split_keys(const Geometry& g, const CachedArgs& a, int n_sm, int tiles, int blocks_a_turn) {
  int split = 1;
  while (split < MAX_CLUSTER && (int64_t)g.batch * a.c.kv_heads * tiles * split < n_sm && 3 * a.c.blocks > split * WARPS * blocks_a_turn) split *= 2;
  return split;
}
// Even shares for all CTAs that fit the SMs, or a cluster for each (stream, key head): by what a warp has to walk where the tables are full, in
// blocks.  Streams are of unlike lengths, so that clusters wait for the longest (a third more, where they lie between half and full); the second piece of
// a share and the joining kernel cost as much as some 12 stages.  Both sides, us, heads of 64, full tables:          even    clusters
//   64 streams, 8 heads on 2 key heads, (512, 10000, 10000) and (2000, 16000, 16000)                                  69, 93    71, 104
//   one stream, 8 key heads, (8000, 64000, 64000), (4000, 32000, 32000), (1000, 8000, 8000)                           36, 32, 27    43, 31, 13
//   8 and 32 streams, 8 key heads, (2000, 16000, 16000) and (500, 4000, 4000)                                         51, 49    42, 43
// and of short streams in tables that are sixteen times as long: 32 of (128, 1024, 1024), 8 key heads, 29 and 16; one of them 26 and 8.  So the 12 is too few where there are
// few rows, and tables say too much of streams that have just begun: the host knows no lengths, and a share of a few blocks costs what a long one does.
template <int HD> bool even_shares(const Geometry& g, const CachedArgs& a, int tiles, int ctas, int split) {
  const int64_t pairs = (int64_t)g.batch * a.c.kv_heads, turns = pairs * 3 * a.c.blocks / (WARPS * Ring<HD>::B);
  return tiles == 1 && turns * 4 / (3 * std::min<int64_t>(pairs * split, ctas)) > turns / ctas + 12;
}

template <typename T, int HD, int KIND, int NT>
cudaError_t launch_tiles(const Geometry& g, CachedArgs& a, cudaStream_t st, size_t* scratch) {
  constexpr int R = 8 * NT;
  const auto kernel = cached_attention_kernel<T, HD, KIND, NT>;
  constexpr int bytes = std::max((int)sizeof(PartRoom<HD, R>), WARPS * Ring<HD>::BYTES);
  static_assert(WARPS == 8 && MAX_CLUSTER == 8, "join_sums takes either");
  int n_sm = 0;
  cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  // Tiles of rows: one where all fit in; of each segment's rows apart, so that a tile walks only what they see (16 streams of (4, 25, 30) rows, two to a key head,
  // forward ring: 33 us, and 41 with mixed ones); across segments where all of them see the same (all blocks open: 76.5 us, and 78 apart).
  uint32_t sees = 0;
  a.mixed = true;
  for (int i = 0; i < 3; ++i)
    if (g.len(i) > 0) {
      const uint32_t s = g.allowed >> (3 * i) & 7u;
      a.mixed = a.mixed && (sees == 0 || sees == s + 8u);
      sees = s + 8u;
    }
  int tiles = (a.rows + R - 1) / R;
  if (a.rows > R && !a.mixed) {
    tiles = 0;
    for (int i = 0; i < 3; ++i) tiles += (g.len(i) * a.group + R - 1) / R;
  }
  const int ctas = RESIDENT<T, NT> * n_sm;
  if (tiles > 65535) return cudaErrorNotSupported;
  a.split = split_keys(g, a, n_sm, tiles, Ring<HD>::B);
  const bool even = even_shares<HD>(g, a, tiles, ctas, a.split);
  const size_t need = even ? 2 * ctas * sizeof(Part<HD, R>) + sizeof(int) * ((size_t)g.batch + 1) : 0;
  if (scratch != nullptr) {
    *scratch = need;
    return cudaSuccess;
  }
  e = sm_count_and_smem_once(reinterpret_cast<const void*>(kernel), bytes, nullptr);
  if (e != cudaSuccess) return e;
  if (even) {
    a.split = 1;
    e = launch_overlapped(kernel, dim3((unsigned)ctas), dim3(THREADS), bytes, st, g, a);
    if (e != cudaSuccess) return e;
    return launch_overlapped(cached_join_kernel<T, HD, R>, dim3((unsigned)(((int64_t)g.batch * a.c.kv_heads * a.rows + WARPS - 1) / WARPS)), dim3(THREADS), 0, st, g, a, ctas);
  }
  a.parts = nullptr;
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

template <typename T, int HD, int KIND> cudaError_t launch_rows(const Geometry& g, CachedArgs& a, cudaStream_t st, size_t* scratch) {
  if (a.rows <= 8) return launch_tiles<T, HD, KIND, 1>(g, a, st, scratch);
  return launch_tiles<T, HD, KIND, 2>(g, a, st, scratch);
}
template <typename T, int KIND> cudaError_t launch_width(const Geometry& g, CachedArgs& a, cudaStream_t st, size_t* scratch) {
  switch (a.c.hd) {
    case 8: return launch_rows<T, 8, KIND>(g, a, st, scratch);
    case 16: return launch_rows<T, 16, KIND>(g, a, st, scratch);
    case 32: return launch_rows<T, 32, KIND>(g, a, st, scratch);
    default: return launch_rows<T, 64, KIND>(g, a, st, scratch);
  }
}
template <typename T> cudaError_t launch_kind(const Geometry& g, CachedArgs& a, cudaStream_t st, size_t* scratch) {
  return a.c.kind == GSIT_CACHE_INT8 ? launch_width<T, GSIT_CACHE_INT8>(g, a, st, scratch) : launch_width<T, GSIT_CACHE_E4M3>(g, a, st, scratch);
}

}  // namespace
}  // namespace gsit

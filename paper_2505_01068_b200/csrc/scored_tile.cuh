// Tiles of the scored attention on mma.sync: staging of partner rows, fragments, the score function on accumulators.
//
// A warp owns 16 * MT rows (queries in the forward pass and for dq, keys for dk and dv) and walks the other side, its partners, in
// chunks that the CTA stages into shared memory (cp.async, two buffers) and in blocks of 64 rows inside a chunk.  A block is skipped
// when none of its pairs can be open -- its documents or moments lie apart from the warp's -- and takes the element-wise mask only
// when some are and some are not.
//
// The next kernel may start only when a CTA has walked: started at once, its CTAs take the places that come free first, and those are all on
// the same few SMs, eight long walks to one of them (16 x (39, 55, 400), 8 heads of 8, forward: 17 us, and 9.1 this way).
#pragma once
#include "scored.cuh"

namespace gsit {
namespace {

using bf16 = __nv_bfloat16;

template <int V> struct IntTag { static constexpr int value = V; };
template <int HD> constexpr int CHUNK_ROWS = HD == 64 ? 64 : 128;

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// d = a b + c; c is an operand of its own, so that a constant start costs no instruction
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ void mma8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t b0, const float (&c)[4]) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%7,%8,%9,%10};"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(b0), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool real) {   // zeros where the row is not real
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }

// Byte offset of 16-byte piece c of row r in a staged tile: pieces are permuted within the 128 bytes that eight rows' worth of
// ldmatrix addresses must spread over.
template <int HD> __device__ __forceinline__ uint32_t piece_at(int r, int c) {
  constexpr int CH = HD / 8;
  return (uint32_t)(r * HD * 2 + ((CH == 1 ? 0 : c ^ ((r / (8 / CH)) % CH)) << 4));
}

// Where a lane's ldmatrix addresses lie from row 0 of a tile on; those of a later group of 16 rows are a multiple of 16 rows further
// (the permutation repeats), those of feature step ks have that bit flipped in.
//   as n: the product runs over features; a load of 16 rows gives {n 0-7 k lo, n 0-7 k hi, n 8-15 k lo, n 8-15 k hi} of a feature step
//   as k: the product runs over the rows; a load gives {features lo: rows 0-7, rows 8-15, features hi: the same} of 16 features
// Rows of 8 features: one load takes 32 of them, 8 to a matrix, either way.
template <int HD> struct LaneAt {
  uint32_t of[(HD + 15) / 16];   // from the tile's first byte, per feature step
};
template <int HD> __device__ __forceinline__ LaneAt<HD> lane_steps(uint32_t base, uint32_t first) {
  LaneAt<HD> at;
#pragma unroll
  for (int ks = 0; ks < (HD + 15) / 16; ++ks) at.of[ks] = base + (first ^ (ks << 5));
  return at;
}
template <int HD> __device__ __forceinline__ LaneAt<HD> lane_as_n(uint32_t base, int lane) {
  return lane_steps<HD>(base, HD == 8 ? lane * 16 : piece_at<HD>(((lane >> 4) << 3) + (lane & 7), (lane >> 3) & 1));
}
template <int HD> __device__ __forceinline__ LaneAt<HD> lane_as_k(uint32_t base, int lane) {
  return lane_steps<HD>(base, HD == 8 ? lane * 16 : piece_at<HD>((((lane >> 3) & 1) << 3) + (lane & 7), lane >> 4));
}

// A operand of a warp's own rows, straight from memory: rows row0 + lane / 4 and + 8, zeros where not real.  Head width 8 uses words 0, 1.
template <int HD> __device__ __forceinline__ void own_rows(const bf16* p0, const bf16* p1, int lane, uint32_t (&f)[(HD + 15) / 16][4]) {
#pragma unroll
  for (int ks = 0; ks < (HD + 15) / 16; ++ks) {
    const int c = 16 * ks + 2 * (lane & 3);
    f[ks][0] = p0 != nullptr ? *reinterpret_cast<const uint32_t*>(p0 + c) : 0u;
    f[ks][1] = p1 != nullptr ? *reinterpret_cast<const uint32_t*>(p1 + c) : 0u;
    f[ks][2] = HD > 8 && p0 != nullptr ? *reinterpret_cast<const uint32_t*>(p0 + c + 8) : 0u;
    f[ks][3] = HD > 8 && p1 != nullptr ? *reinterpret_cast<const uint32_t*>(p1 + c + 8) : 0u;
  }
}

// c[mt][nt] = start(mt, nt) + own rows x partner rows, over features, for NT tiles of 8 partners; the first one's row lies
// `from` bytes behind the tile that `at` (lane_as_n) counts from.
template <int HD, int MT, int NT, typename Start>
__device__ __forceinline__ void product_over_features(float (&c)[MT][NT][4], const uint32_t (&own)[MT][(HD + 15) / 16][4], const LaneAt<HD>& at, uint32_t from, Start start) {
  if constexpr (HD == 8) {
#pragma unroll
    for (int q = 0; q < NT / 4; ++q) {
      uint32_t f[4];
      ldsm4(at.of[0] + from + q * 512, f);
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float z[4];
          start(m, 4 * q + i, z);
          mma8(c[m][4 * q + i], own[m][0][0], own[m][0][1], f[i], z);
        }
    }
  } else {
#pragma unroll
    for (int p = 0; p < NT / 2; ++p)
#pragma unroll
      for (int ks = 0; ks < HD / 16; ++ks) {
        uint32_t f[4];
        ldsm4(at.of[ks] + from + p * 32 * HD, f);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float z[4];
            if (ks == 0) start(m, 2 * p + i, z);
            mma16(c[m][2 * p + i], own[m][ks], f[2 * i], f[2 * i + 1], ks == 0 ? z : c[m][2 * p + i]);
          }
      }
  }
}
// Fragments of partner rows for products over NT tiles of 8 partners, as use(first of their weights' tiles, feature step, fragment); `at`: lane_as_k.
template <int HD, int NT, typename Use>
__device__ __forceinline__ void for_partner_rows(const LaneAt<HD>& at, uint32_t from, Use use) {
#pragma unroll
  for (int p = 0; p < (HD == 8 ? NT / 4 : NT / 2); ++p)
#pragma unroll
    for (int c = 0; c < (HD == 8 ? 1 : HD / 16); ++c) {
      uint32_t f[4];
      ldsm4_t(at.of[c] + from + (HD == 8 ? p * 512 : p * 32 * HD), f);
      use(HD == 8 ? 4 * p : 2 * p, c, f);
    }
}
// o[mt][feature tile] += weights [own rows x partners] x one such fragment; weights as packed accumulators w[mt][nt] = {row g, row g + 8}.
template <int HD, int MT, int NT>
__device__ __forceinline__ void add_product(float (&o)[MT][HD / 8][4], const uint32_t (&w)[MT][NT][2], int first, int c, const uint32_t (&f)[4]) {
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int nt = HD == 8 ? first + 2 * i : first;
      const uint32_t a[4] = {w[m][nt][0], w[m][nt][1], w[m][nt + 1][0], w[m][nt + 1][1]};
      float (&d)[4] = o[m][HD == 8 ? 0 : 2 * c + i];
      mma16(d, a, f[2 * i], f[2 * i + 1], d);
    }
}
template <int HD, int MT, int NT>
__device__ __forceinline__ void product_over_partners(float (&o)[MT][HD / 8][4], const uint32_t (&w)[MT][NT][2], const LaneAt<HD>& at, uint32_t from) {
  for_partner_rows<HD, NT>(at, from, [&](int first, int c, const uint32_t (&f)[4]) { add_product<HD>(o, w, first, c, f); });
}
__device__ __forceinline__ void from_zero(int, int, float (&z)[4]) { z[0] = z[1] = z[2] = z[3] = 0.f; }

// Two dots -> scores in base 2 less m; bend = derivative of the cap, where there is one.  NEAR: tanh's arguments
// are at most 1/4, and both are polynomials of the dot (quadratics of its square: 4 multiply-adds a score with the subtraction, 3 more for
// the derivative; the FMA pipe is what these kernels fill first).
template <bool CAP, bool BEND, bool NEAR> __device__ __forceinline__ float2 score_pair(float2 y, float2 m, float2& bend, const ScoredArgs& a) {
  auto both = [](float v) { return make_float2(v, v); };
  m = make_float2(-m.x, -m.y);
  if constexpr (!CAP) {
    return __ffma2_rn(y, both(a.inner), m);
  } else if constexpr (NEAR) {
    const float2 z = __fmul2_rn(y, y);
    if constexpr (BEND) bend = __ffma2_rn(__ffma2_rn(z, both(a.near_b[2]), both(a.near_b[1])), z, both(a.near_b[0]));
    return __ffma2_rn(__ffma2_rn(__ffma2_rn(z, both(a.near_p[2]), both(a.near_p[1])), z, both(a.near_p[0])), y, m);
  } else {
    const float2 t = tanh_any2(__fmul2_rn(y, both(a.inner)));
    if constexpr (BEND) bend = __ffma2_rn(make_float2(-t.x, -t.y), t, both(1.f));
    return __ffma2_rn(t, both(a.outer), m);
  }
}
// What rounding a pair to bf16 leaves, in bf16: the two terms together hold 16 bits.
__device__ __forceinline__ uint32_t pack_rest(float2 v, uint32_t rounded) {
  float2 r;
  unpack_bf16(rounded, r.x, r.y);
  const float2 rest = __fadd2_rn(v, make_float2(-r.x, -r.y));
  return ptx::pack_bf16(rest.x, rest.y);
}
template <bool CAP> __device__ __forceinline__ float2 times_bend(float2 v, float2 bend) {
  if constexpr (CAP) return __fmul2_rn(v, bend);
  return v;
}
// score -= slope2 * |own time - partner time| for a pair of partners
__device__ __forceinline__ float2 bias_pair(float2 y, float2 times, float own, float slope2) {
  const float2 d = __fadd2_rn(times, make_float2(-own, -own));
  return __ffma2_rn(make_float2(fabsf(d.x), fabsf(d.y)), make_float2(-slope2, -slope2), y);
}
// Runs body(NEAR) for the dots of a step.  One decision for the warp, ahead of everything, so that the multiply-adds of some columns and
// the exponentials of others are one stream of instructions.
template <bool CAP, int MT, int NT, typename Body>
__device__ __forceinline__ void in_form(const float (&x)[MT][NT][4], const ScoredArgs& a, Body body) {
  if constexpr (CAP) {
    float top = 0.f;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; i += 2) top = ptx::fmax3(top, fabsf(x[m][n][i]), fabsf(x[m][n][i + 1]));
    if (__any_sync(0xffffffffu, top > a.near_dot)) {
      body(IntTag<0>{});
      return;
    }
  }
  body(IntTag<1>{});
}

// A chunk of rows of two matrices into shared memory, whole blocks of them, zeros from row `rem` on.
template <int HD, int C, int W>
__device__ __forceinline__ void stage_pair(uint32_t d0, uint32_t d1, const bf16* p0, int64_t ld0, const bf16* p1, int64_t ld1, int rem, int tid) {
  constexpr int CH = HD / 8;
  const int need = min(C, (rem + BLOCK - 1) / BLOCK * BLOCK), c = tid % CH;
  int row = tid / CH;
  p0 += (int64_t)row * ld0 + 8 * c;
  p1 += (int64_t)row * ld1 + 8 * c;
#pragma unroll 1
  for (; row < need; row += 32 * W / CH) {
    const bool in = row < rem;
    cp16(d0 + piece_at<HD>(row, c), in ? p0 : p0 - (int64_t)row * ld0, in);
    cp16(d1 + piece_at<HD>(row, c), in ? p1 : p1 - (int64_t)row * ld1, in);
    p0 += (32 * W / CH) * ld0;
    p1 += (32 * W / CH) * ld1;
  }
  cp_commit();
}

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

}  // namespace
}  // namespace gsit

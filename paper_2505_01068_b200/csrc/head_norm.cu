// Norms of the heads of q and k with the rotary positions in the same pass, and their gradients:
//   y = R (x r gamma),  r = 1 / sqrt(mean(x^2) + eps),  R the rotation of the head's pairs by the row's angles.
// Backward, with u = R^-1 dy, g = u gamma and s = sum(g x):  dx = r (g - x r^2 s / hd),  dgamma = sum over rows and heads of u x r.
// x is read again instead of saving anything; r costs one more sum over a head that is in registers anyway.
//
// Bound by the rows read and written, so everything is arranged around loads in flight and few instructions: a warp works for itself, without barriers.
// It takes blocks of a few rows, forward of q and k, backward of one of them (sums for two weights do not fit the registers beside the rest); a lane holds two
// 16-byte pieces of a head (the halves that rotate against each other, or neighbours where pairs are interleaved), so that sums over a head are
// log2(lanes of a head) shuffles and a pair never leaves its lane.  Which pieces of a block are a lane's never changes, so the sums for dgamma stay in
// registers.  The angles of a block are computed into a table of the warp's own, one (row, pair) a lane, and serve all heads; the rows of the block
// after it are on their way into shared memory meanwhile.
// Angles in turns are products of integers that lose their whole turns by themselves: position * (frequency * 2^64) mod 2^64, of which the upper 32 bits are
// the phase, right for every position an int32 holds.  It is at most half a turn and rounded to float, 2^-26 of a turn or 2^-23.3 of the result next to the
// rounding of float itself (with rsqrtf and sums in float a float result is 1.5e-7 off in all); then sincospi for float, and the special functions' sine and cosine
// for bf16 (2^-21 off, where a result keeps 2^-9).
// Measured, bf16, 8 + 8 heads of 64, 128 samples of (128, 1024, 1024), a quarter of them half padding: forward 1071 MB in 184 us, 5.8 TB/s, 0.89 of the measured
// copy rate; backward 1573 MB in 299 us, 5.3 TB/s, 0.80; one after the other as a training step calls them 485 to 547 from machine to machine; 8 + 4 heads, 64 samples, 403 MB in 77 us.  What bounds it
// then are issue slots (65 %).
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
  int heads;
};
struct HeadNormArgs {
  NormTensor t[2];
  const int32_t* positions;
  int64_t axis_stride, batch_stride;
  int axis1, axis2, pairs;            // first pair of axis 1 and 2
  int block_rows[2];                  // forward: the same for both
  int q_ctas;                         // backward: CTAs of q, those of k follow
  float eps, inv_hd;
  float* partial;                     // rows of hd: one of every CTA of q, then those of k
  uint64_t turns[MAX_ROTARY_PAIRS];   // frequency of a pair in turns a position, as a fraction of 2^64
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
// A piece of 16 bytes into the lane's own place in shared memory, zeros where there is none.
template <typename T> __device__ __forceinline__ void copy_piece(void* dst, const T* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
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

// The table of angles: of pairs 2 i and 2 i + 1 of a lane's piece {cos, cos, sin, sin}; pieces lie 16 bytes further apart than they are long, so that the lanes
// of a head meet different banks.
template <int E> constexpr int PIECE_ANGLES = 2 * E + 4;   // floats

// (lo, hi) of a lane turned by its angles.  Halves: pair e is (lo[e], hi[e]).  Interleaved: pairs are neighbours, first those of lo.
template <int E, bool ADJACENT, bool BACK>
__device__ __forceinline__ void turn(float2 (&lo)[E / 2], float2 (&hi)[E / 2], const float* table) {
#pragma unroll
  for (int i = 0; i < E / 2; ++i) {
    const float4 v = *reinterpret_cast<const float4*>(table + 4 * i);
    const float2 c = make_float2(v.x, v.y), s = BACK ? make_float2(-v.z, -v.w) : make_float2(v.z, v.w);
    if constexpr (!ADJACENT) {
      const float2 a = __ffma2_rn(make_float2(-hi[i].x, -hi[i].y), s, __fmul2_rn(lo[i], c)), b = __ffma2_rn(lo[i], s, __fmul2_rn(hi[i], c));
      lo[i] = a;
      hi[i] = b;
    } else {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int p = 2 * i + e;
        float2& w = p < E / 2 ? lo[p % (E / 2)] : hi[p % (E / 2)];
        const float cs = e ? c.y : c.x, sn = e ? s.y : s.x;
        w = __ffma2_rn(make_float2(-w.y, w.x), make_float2(sn, sn), __fmul2_rn(w, make_float2(cs, cs)));
      }
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

constexpr int UNITS = 2;   // heads' pieces of a lane, of each tensor, that are copied together

// Sine and cosine of position * turns, by the phase in turns, at most 1/2.
template <typename T> __device__ __forceinline__ void sine_cosine(int32_t position, uint64_t turns, float* sn, float* cs) {
  const uint32_t low = (uint32_t)turns, phase = __umulhi((uint32_t)position, low) + (uint32_t)position * (uint32_t)(turns >> 32) - (position < 0 ? low : 0u);
  const float v = (float)(int32_t)phase;   // * 2^-32
  if constexpr (sizeof(T) == 4) sincospif(v * 0x1p-31f, sn, cs);
  else __sincosf(v * (6.283185307f * 0x1p-32f), sn, cs);
}
// First row of segment s, and its length, without an index into the parameters.
__device__ __forceinline__ int first_of(const Geometry& g, int s) { return s == 2 ? g.seg_off[2] : s == 1 ? g.seg_off[1] : 0; }
__device__ __forceinline__ int length_of(const Geometry& g, int s) { return s == 2 ? g.seg_len[2] : s == 1 ? g.seg_len[1] : g.seg_len[0]; }
// Whether pieces come through shared memory, the next block's while this one is worked on, or straight into registers when they are needed, which has them sooner
// and takes fewer instructions for what narrow heads hold.  Measured, us forward and back, 8 + 8 heads, rows in samples of (128, 1024, 1024) a quarter of them padding:
//   float   heads of 8, 64 x (50, 500, 500)    17.6 and 28.2 through shared memory    12.9 and 18.7 straight
//           16, 64 x (128, 512, 512)           27.2     41.2                          25.8     41.8
//           32, 64 samples                     92       111                           118      132
//           64, 64 samples                     181      244                           201      253
//           128, 32 samples                    180      239                           206      248
//   bf16    64, 128 samples                    184      299                           216      394
// (Pieces of 8 bytes, bf16 heads of 8, are narrower than a copy.)
template <typename T> __host__ __device__ constexpr bool staged_pieces(int elements, int lanes) {
  return elements * (int)sizeof(T) == 16 && (sizeof(T) == 2 || lanes >= 4);
}

template <typename T, int E, int LANES, bool ADJACENT, bool BWD>
__global__ void __launch_bounds__(THREADS, 2)
head_norm_kernel(const __grid_constant__ Geometry g, const __grid_constant__ HeadNormArgs a) {
  constexpr int HALF = E * LANES, HD = 2 * HALF, N = UNITS, H2 = E / 2, BYTES = E * (int)sizeof(T), PARTS = BWD ? 4 : 2, TABLE = ANGLES / E * PIECE_ANGLES<E>, W = BWD ? 1 : 2,   // W: tensors of a warp
                STAGE = W * N * PARTS * 32 * BYTES;
  constexpr bool STAGED = staged_pieces<T>(E, LANES);
  static_assert(HALF <= ANGLES, "the angles of a row fit the table");
  __shared__ __align__(16) float s_table[WARPS][2][TABLE], s_gamma[W][HD];
  extern __shared__ __align__(16) uint8_t smem[];   // two stages of every warp's
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, unit = lane % LANES;
  ptx::load_params_early(g, a);
  const int which = W == 1 && (int)blockIdx.x >= a.q_ctas, rows = g.batch * g.L, block_rows = a.block_rows[which];
  const NormTensor own = a.t[which];           // of the warp, where it has one alone: in registers
  const unsigned ctas = W == 2 ? gridDim.x : which ? gridDim.x - a.q_ctas : a.q_ctas, cta = blockIdx.x - (which ? a.q_ctas : 0);
  const unsigned blocks = (unsigned)((rows + block_rows - 1) / block_rows);
  // this lane's features: a piece of the first halves and its partner in the second ones; behind the rotated features, and where interleaved, neighbours
  const int rotated = a.pairs / E;
  const bool neighbours = ADJACENT || unit >= rotated;
  const int lo_at = neighbours ? 2 * unit * E : unit * E, hi_at = neighbours ? lo_at + E : a.pairs + unit * E;

  // this lane's angles of a block: their rows' samples and places go on from block to block without a division.  What they are made from is loaded
  // a block before it is needed.
  const unsigned step = ctas * WARPS;
  unsigned block = cta * WARPS + warp;
  const int step_rows = (int)(step * block_rows), step_b = step_rows / g.L, step_l = step_rows - step_b * g.L;
  int angle_row[2], angle_axis[2], angle_b[2], angle_l[2], position[2], within[2], valid[2];   // within: the segment, and the place in it; valid: its real rows
  uint64_t turns[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int at = lane + 32 * i, pair = at % HALF;
    angle_row[i] = at / HALF;
    turns[i] = pair < a.pairs ? a.turns[pair] : 0;
    angle_axis[i] = pair >= a.pairs ? -1 : pair >= a.axis2 ? 2 : pair >= a.axis1 ? 1 : 0;
    const uint32_t row = (uint32_t)min((int64_t)block * block_rows + angle_row[i], (int64_t)0x3fffffff);
    angle_b[i] = row / (uint32_t)g.L;
    angle_l[i] = row - angle_b[i] * g.L;
  }
  auto fetch = [&]() {   // for the next block in turn
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      position[i] = 0;
      within[i] = valid[i] = 0;
      if (32 * i < block_rows * HALF && angle_row[i] < block_rows && angle_b[i] < g.batch) {
        const int b = angle_b[i], l = angle_l[i], s = segment_of(g, l);
        if (angle_axis[i] >= 0) position[i] = a.positions[angle_axis[i] * a.axis_stride + b * a.batch_stride + l];
        within[i] = (l - first_of(g, s)) | (int)((uint32_t)s << 30);   // (segments are shorter than 2^29)
        valid[i] = g.valid_len != nullptr ? g.valid_len[3 * b + s] : length_of(g, s);
      }
      angle_b[i] += step_b;
      angle_l[i] += step_l;
      if (angle_l[i] >= g.L) {
        angle_l[i] -= g.L;
        ++angle_b[i];
      }
    }
  };
  auto angles = [&](int buf) {   // of the block that was fetched for; which of its rows are real, a bit each
    uint32_t real = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (32 * i < block_rows * HALF) {
        const int at = lane + 32 * i, pair = at % HALF, s = (uint32_t)within[i] >> 30, n = length_of(g, s);
        float sn = 0.f, cs = 1.f;
        if (angle_axis[i] >= 0) sine_cosine<T>(position[i], turns[i], &sn, &cs);
        if (angle_row[i] < block_rows) {
          float* const to = s_table[warp][buf] + (angle_row[i] * LANES + pair / E) * PIECE_ANGLES<E> + pair % E / 2 * 4 + pair % 2;
          to[0] = cs;
          to[2] = sn;
        }
        if (valid[i] < 0 || valid[i] > n) raise_flag(g, GSIT_DEVFLAG_CLAMPED);
        if ((within[i] & 0x3fffffff) < (valid[i] < 0 ? 0 : min(valid[i], n))) real |= 1u << angle_row[i];
      }
    return __reduce_or_sync(0xffffffffu, real);
  };
  // this lane's pieces of a block (a row of more heads than the lanes take is walked in chunks of them)
  int row_of[W][N], head_of[W][N];
#pragma unroll
  for (int w = 0; w < W; ++w)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int u = lane + 32 * i, row_units = (W == 1 ? own : a.t[w]).heads * LANES;
      row_of[w][i] = block_rows > 1 && row_units > 0 ? u / row_units : 0;
      head_of[w][i] = (u - row_of[w][i] * row_units) / LANES;
      if (row_of[w][i] >= block_rows) {   // none
        row_of[w][i] = 0;
        head_of[w][i] = (W == 1 ? own : a.t[w]).heads;
      }
    }
  float2 dg_lo[H2], dg_hi[H2];
#pragma unroll
  for (int i = 0; i < H2; ++i) dg_lo[i] = dg_hi[i] = make_float2(0.f, 0.f);

  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  for (int i = threadIdx.x; i < W * HD; i += THREADS) {
    const float* gamma = W == 1 ? own.gamma : a.t[i / HD].gamma;
    s_gamma[i / HD][i % HD] = gamma != nullptr ? gamma[i % HD] : 1.f;
  }
  uint32_t real = 0;                         // bit r: row r of the block is a real one
  const int most = W == 1 ? own.heads : max(a.t[0].heads, a.t[1].heads);
  constexpr int CHUNK = 32 * N / LANES;
  Piece<T, E> held[W][N][STAGED ? 1 : PARTS];
  auto load_now = [&](int chunk) {
    const int64_t row0 = (int64_t)block * block_rows;
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const NormTensor& t = W == 1 ? own : a.t[w];
        if (chunk >= t.heads || 32 * i >= block_rows * t.heads * LANES) continue;
        const int head = head_of[w][i] + chunk;
#pragma unroll
        for (int k = 0; k < (STAGED ? 1 : PARTS); ++k) held[w][i][k].clear();
        if (head < t.heads && ((real >> row_of[w][i]) & 1u)) {
#pragma unroll
          for (int k = 0; k < (STAGED ? 1 : PARTS); ++k)
            held[w][i][k].load(static_cast<const T*>(k < 2 ? t.x : t.dy) + (row0 + row_of[w][i]) * (k < 2 ? t.ldx : t.lddy) + head * HD + (k % 2 ? hi_at : lo_at));
        }
      }
  };
  // a lane's own places in the ring: [stage][tensor][piece i][x lo, x hi, dy lo, dy hi], 32 lanes of each side by side
  uint8_t* const ring = smem + warp * 2 * STAGE + lane * BYTES;
  auto place = [&](int stage, int w, int i, int part) { return ring + stage * STAGE + (((w * N + i) * PARTS) + part) * 32 * BYTES; };
  auto taken = [&](int stage, int w, int i, int part) {
    Piece<T, E> p;
    if constexpr (STAGED) p.load(reinterpret_cast<const T*>(place(stage, w, i, part)));
    else p = held[w][i][part];
    return p;
  };
  auto copy = [&](unsigned of, int chunk, uint32_t real, int stage) {
    const int64_t row0 = (int64_t)of * block_rows;
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const NormTensor& t = W == 1 ? own : a.t[w];
        if (chunk >= t.heads || 32 * i >= block_rows * t.heads * LANES) continue;   // no lane has any
        const int head = head_of[w][i] + chunk;
        const bool there = head < t.heads && ((real >> row_of[w][i]) & 1u);
        const T* x = static_cast<const T*>(t.x) + (there ? (row0 + row_of[w][i]) * t.ldx + head * HD : 0);
        copy_piece(place(stage, w, i, 0), x + lo_at, there);
        copy_piece(place(stage, w, i, 1), x + hi_at, there);
        if constexpr (BWD) {
          const T* dy = static_cast<const T*>(t.dy) + (there ? (row0 + row_of[w][i]) * t.lddy + head * HD : 0);
          copy_piece(place(stage, w, i, 2), dy + lo_at, there);
          copy_piece(place(stage, w, i, 3), dy + hi_at, there);
        }
      }
  };
  fetch();
  uint32_t next_real = 0;
  real = angles(0);
  fetch();
  if (STAGED && block < blocks) copy(block, 0, real, 0);
  asm volatile("cp.async.commit_group;" ::: "memory");
  __syncthreads();
  for (int buf = 0, chunk = 0, stage = 0; block < blocks; stage ^= 1) {
    // what comes next, on its way while this is worked on
    const bool last = chunk + CHUNK >= most;
    if constexpr (!STAGED) load_now(chunk);
    if (last) {
      next_real = angles(buf ^ 1);
      fetch();
      if (STAGED && block + step < blocks) copy(block + step, 0, next_real, stage ^ 1);
    } else if (STAGED) {
      copy(block, chunk + CHUNK, real, stage ^ 1);
    }
    if constexpr (STAGED) asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 1;" ::: "memory");
    const int64_t row0 = (int64_t)block * block_rows;
    const int left = (int)min((int64_t)block_rows, rows - row0);
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const NormTensor& t = W == 1 ? own : a.t[w];
        if (chunk >= t.heads || 32 * i >= block_rows * t.heads * LANES) continue;
        const int head = head_of[w][i] + chunk;
        const bool in = row_of[w][i] < left && head < t.heads, keep = in && ((real >> row_of[w][i]) & 1u);
        const float* const table = s_table[warp][buf] + (row_of[w][i] * LANES + unit) * PIECE_ANGLES<E>;
        float2 lo[H2], hi[H2], ga_lo[H2], ga_hi[H2];
        taken(stage, w, i, 0).get(lo);
        taken(stage, w, i, 1).get(hi);
#pragma unroll
        for (int e = 0; e < H2; ++e) {
          ga_lo[e] = *reinterpret_cast<const float2*>(&s_gamma[w][lo_at + 2 * e]);
          ga_hi[e] = *reinterpret_cast<const float2*>(&s_gamma[w][hi_at + 2 * e]);
        }
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
          taken(stage, w, i, 2).get(u_lo);
          taken(stage, w, i, 3).get(u_hi);
          turn<E, ADJACENT, true>(u_lo, u_hi, table);
          float2 gx = make_float2(0.f, 0.f), gy = gx;
#pragma unroll
          for (int e = 0; e < H2; ++e) {
            gx = __ffma2_rn(__fmul2_rn(u_lo[e], ga_lo[e]), lo[e], gx);
            gy = __ffma2_rn(__fmul2_rn(u_hi[e], ga_hi[e]), hi[e], gy);
          }
          gx = __fadd2_rn(gx, gy);
          both.y = gx.x + gx.y;
          both = head_sum<LANES>(both);
        } else {
#pragma unroll
          for (int o = LANES / 2; o > 0; o >>= 1) both.x += __shfl_xor_sync(0xffffffffu, both.x, o);
        }
        const float r = rsqrtf(both.x * a.inv_hd + a.eps);
        const float2 r2 = make_float2(r, r);
        if constexpr (!BWD) {
#pragma unroll
          for (int e = 0; e < H2; ++e) {
            lo[e] = __fmul2_rn(__fmul2_rn(lo[e], r2), ga_lo[e]);
            hi[e] = __fmul2_rn(__fmul2_rn(hi[e], r2), ga_hi[e]);
          }
          turn<E, ADJACENT, false>(lo, hi, table);
        } else {
          const float back = -r * r * (both.y * a.inv_hd);
          const float2 back2 = make_float2(back, back);
#pragma unroll
          for (int e = 0; e < H2; ++e) {
            const float2 h_lo = __fmul2_rn(lo[e], r2), h_hi = __fmul2_rn(hi[e], r2);
            if (keep) {   // (a row that is not real has an x of 0, but r of a tiny eps may be infinite)
              dg_lo[e] = __ffma2_rn(u_lo[e], h_lo, dg_lo[e]);
              dg_hi[e] = __ffma2_rn(u_hi[e], h_hi, dg_hi[e]);
            }
            lo[e] = __ffma2_rn(h_lo, back2, __fmul2_rn(__fmul2_rn(u_lo[e], ga_lo[e]), r2));
            hi[e] = __ffma2_rn(h_hi, back2, __fmul2_rn(__fmul2_rn(u_hi[e], ga_hi[e]), r2));
          }
        }
        if (in) {
          if (!keep)
#pragma unroll
            for (int e = 0; e < H2; ++e) lo[e] = hi[e] = make_float2(0.f, 0.f);
          T* out = static_cast<T*>(t.out) + (row0 + row_of[w][i]) * t.ldo + head * HD;
          store_piece<E>(out + lo_at, lo);
          store_piece<E>(out + hi_at, hi);
        }
      }
    if (last) {
      block += step;
      chunk = 0;
      buf ^= 1;
      real = next_real;
    } else {
      chunk += CHUNK;
    }
    __syncwarp();   // the next block's angles are there, and nobody reads this block's any more
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
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
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  float dg[2][OWN] = {};
  // the head in s_row turned by the angles: feature f
  auto turned = [&](int f, float sign) {
    const float v = s_row[warp][f];
    if (f >= 2 * a.pairs) return v;
    const int p = adjacent ? f >> 1 : f < a.pairs ? f : f - a.pairs;
    const bool first = adjacent ? (f & 1) == 0 : f < a.pairs;
    const float w = s_row[warp][adjacent ? f ^ 1 : first ? f + a.pairs : f - a.pairs], c = s_cos[warp][p], s = sign * s_sin[warp][p];
    return first ? v * c - w * s : w * s + v * c;
  };
  for (int row = blockIdx.x * WARPS + warp; row < rows; row += gridDim.x * WARPS) {
    const int b = (uint32_t)row / (uint32_t)g.L, l = row - b * g.L, seg = segment_of(g, l);
    const bool real = l - g.off(seg) < valid_rows(g, b, seg);
    if (real)
      for (int p = lane; p < a.pairs; p += 32) {
        const int axis = p >= a.axis2 ? 2 : p >= a.axis1 ? 1 : 0;
        sine_cosine<float>(a.positions[axis * a.axis_stride + b * a.batch_stride + l], a.turns[p], &s_sin[warp][p], &s_cos[warp][p]);
      }
    __syncwarp();
#pragma unroll
    for (int which = 0; which < 2; ++which)
      for (int head = 0; head < a.t[which].heads; ++head) {
        const NormTensor& t = a.t[which];
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
              dg[which][i] += u[i] * h;
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
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < OWN; ++i)
      if (const int f = lane + 32 * i; f < hd) s_row[warp][f] = dg[which][i];
    __syncthreads();
    for (int c = threadIdx.x; c < hd; c += THREADS) {
      float s = 0.f;
      for (int w = 0; w < WARPS; ++w) s += s_row[w][c];
      a.partial[((int64_t)which * gridDim.x + blockIdx.x) * hd + c] = s;
    }
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

size_t head_norm_scratch(const Geometry& g) { return sizeof(float) * 2 * (size_t)g.hd * MAX_CTAS; }

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
  double turns[MAX_ROTARY_PAIRS];
  rotary_turns(c.base, a.pairs, turns);
  for (int p = 0; p < a.pairs; ++p) a.turns[p] = (uint64_t)ldexp(turns[p] - floor(turns[p]), 64);   // (whole turns do not count)
  // wide: a head of at most 128 features is 1, 2, 4, 8 or 16 lanes of two pieces, 16 bytes each (8 where a bf16 head has 8 features), and whole
  // pieces of it rotate
  const int piece = dtype == GSIT_BF16 ? (g.hd == 8 ? 4 : 8) : 4, lanes = g.hd / (2 * piece);
  bool wide = g.hd % (2 * piece) == 0 && g.hd <= 2 * ANGLES && (lanes & (lanes - 1)) == 0 && (c.interleaved || a.pairs % piece == 0);
  for (int i = 0; i < 2; ++i) {
    NormTensor& t = a.t[i];
    t.x = c.x[i]; t.ldx = c.ldx[i];
    t.dy = c.dy[i]; t.lddy = c.lddy[i];
    t.out = c.out[i]; t.ldo = c.ldo[i];
    t.gamma = c.gamma[i];
    t.heads = c.heads[i];
    if (t.heads > 0)
      wide = wide && ((reinterpret_cast<uintptr_t>(t.x) | reinterpret_cast<uintptr_t>(t.dy) | reinterpret_cast<uintptr_t>(t.out)) % (piece * es)) == 0 &&
             t.ldx % piece == 0 && t.lddy % piece == 0 && t.ldo % piece == 0;
  }
  // rows of a block: what the lanes' pieces in flight take of the (wider) tensor, and two angles a lane; CTAs: as many as fit the SMs at once
  const int64_t rows = (int64_t)g.batch * g.L;
  const int most = std::min(MAX_CTAS, 2 * n_sm);
  auto block_rows = [&](int heads) { return wide && heads > 0 ? std::max(1, std::min(2 * ANGLES / g.hd, 32 * UNITS / (heads * lanes))) : 1; };
  auto ctas_for = [&](int share, int of_rows) { return (int)std::min<int64_t>(share, (rows + of_rows * WARPS - 1) / (of_rows * WARPS)); };
  int ctas;
  if (wide && c.backward) {   // shared out by heads
    const int total = c.heads[0] + c.heads[1], share = c.heads[1] == 0 ? most : std::min(most - 1, std::max(1, (most * c.heads[0] + total / 2) / total));
    for (int i = 0; i < 2; ++i) a.block_rows[i] = block_rows(c.heads[i]);
    a.q_ctas = ctas_for(share, a.block_rows[0]);
    ctas = a.q_ctas + (c.heads[1] == 0 ? 0 : ctas_for(most - share, a.block_rows[1]));
  } else {
    a.block_rows[0] = a.block_rows[1] = block_rows(std::max(c.heads[0], c.heads[1]));
    ctas = a.q_ctas = ctas_for(most, a.block_rows[0]);
  }
  const dim3 grid((unsigned)ctas);
  if (wide) {
    const Kernel k = dtype == GSIT_BF16 ? wide_kernel<__nv_bfloat16>(g.hd, c.interleaved, c.backward) : wide_kernel<float>(g.hd, c.interleaved, c.backward);
    const bool staged = dtype == GSIT_BF16 ? staged_pieces<__nv_bfloat16>(piece, lanes) : staged_pieces<float>(piece, lanes);
    const int bytes = staged ? WARPS * 2 * (c.backward ? 1 : 2) * UNITS * (c.backward ? 4 : 2) * 512 : 0;
    e = sm_count_and_smem_once(reinterpret_cast<const void*>(k), bytes, nullptr);
    if (e != cudaSuccess) return e;
    e = launch_overlapped(k, grid, dim3(THREADS), bytes, st, g, a);
  } else if (dtype == GSIT_BF16) {
    e = c.backward ? launch_overlapped(head_norm_any_kernel<__nv_bfloat16, true>, grid, dim3(THREADS), 0, st, g, a, (int)c.interleaved)
                   : launch_overlapped(head_norm_any_kernel<__nv_bfloat16, false>, grid, dim3(THREADS), 0, st, g, a, (int)c.interleaved);
  } else {
    e = c.backward ? launch_overlapped(head_norm_any_kernel<float, true>, grid, dim3(THREADS), 0, st, g, a, (int)c.interleaved)
                   : launch_overlapped(head_norm_any_kernel<float, false>, grid, dim3(THREADS), 0, st, g, a, (int)c.interleaved);
  }
  if (e != cudaSuccess || a.partial == nullptr) return e;
  return launch_overlapped(head_norm_reduce_kernel, dim3((g.hd + 31) / 32, c.heads[1] > 0 ? 2 : 1), dim3(1024), 0, st, a.partial, a.q_ctas, wide ? ctas : 2 * ctas, g.hd,
                           c.dgamma[0], c.dgamma[1]);
}

}  // namespace gsit

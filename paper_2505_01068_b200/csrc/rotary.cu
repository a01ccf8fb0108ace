// Rotary positions with several axes: every pair of features (u, v) of a head becomes (u c - v s, u s + v c), with c and s of the
// pair's angle; the backward pass is the same rotation by the opposite angle.
//
// One pass over the rows, q and k read once and written once, which is all that bounds it.  A CTA takes blocks of rows in turn; the
// angles of a block's rows -- one (row, pair) a thread -- are computed into shared memory, where all heads of q and k read them (an
// angle costs as much as some 40 rotated pairs), while the loads of the block before are under way.  What a thread does in a block
// (which rows, heads and features) never changes, so its offsets and its pair's frequency stay in registers.
// Angles: position * frequency in turns as one double product, less its nearest integer: right to 2^-20 turns even at positions near
// 2^31, where a float product keeps no bit of the phase; then sincospi of the float remainder.
// Measured: gradients of 128 samples of (128, 1024, 1024), a quarter of the rows padding, q and k with 8 heads of 64, bf16: 1072 MB in 223 - 229 us, 4.8 TB/s, 0.74 of
// the measured copy rate (lines that are asked for ahead are so for padded rows, too: an eighth of what is read there); 64 x (50, 500, 500), 8 heads of 8: 30 MB in 12 us.
#include <algorithm>

#include "ops.cuh"

namespace gsit {
namespace {

constexpr int THREADS = 256;

constexpr int MAX_ROWS = 64;                // of a block
constexpr int BLOCK_UNITS = 4 * THREADS;    // units of work of a block that a thread's registers hold the offsets of

struct RotaryArgs {
  const void* in[2];
  void* out[2];
  int64_t in_stride[2], out_stride[2];   // elements between rows
  const int32_t* positions;
  int64_t axis_stride, batch_stride;
  float sign;
  int pairs, block_rows, q_heads;
  int row_units, head_units;             // units of work (see Form) of a row and of a head
  int axis1, axis2;                      // first pair of axis 1 and of axis 2
  int adjacent;
  double turns[MAX_ROTARY_PAIRS];        // frequency of a pair in turns a position
};

// What one unit of work is.  One thread loads, rotates and stores it, so that calls may work in place.
//   SPLIT     a 16-byte piece of a head's first halves and its partner in the second ones (all of the head rotated, pairs a multiple
//             of the piece)
//   ADJACENT  a 16-byte piece of whole pairs (interleaved, all of the head rotated)
//   HEAD      a whole bf16 head of 8 features, pairs (p, p + 4)
//   SCALAR    one pair, or one feature that is copied: part of a head rotated, odd strides or addresses
// The wide forms wherever they can: 32 x (128, 1024, 1024), 8 heads of 64, bf16 SPLIT 56 us, ADJACENT 80, SCALAR 338; 64 x (50, 500, 500), 8 heads
// of 8 HEAD 12 us, SCALAR 37.
enum Form { SPLIT, ADJACENT, HEAD, SCALAR };

template <typename T> __device__ __forceinline__ void unpack_piece(const uint4& v, float (&f)[16 / sizeof(T)]) {
  if constexpr (sizeof(T) == 2) {
    unpack_bf16(v.x, f[0], f[1]);
    unpack_bf16(v.y, f[2], f[3]);
    unpack_bf16(v.z, f[4], f[5]);
    unpack_bf16(v.w, f[6], f[7]);
  } else {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
}

// Place of pair p in a row of the table: groups of eight lie ten floats apart, so that the four pieces of a head of 64 that a warp reads
// together meet different banks.  A row takes whole groups of four floats, so some numbers of pairs fill more of the table than a float a
// thread and a quarter (12 pairs: 16 floats, of which 21 rows, one angle a thread, would be 336): TABLE bounds the rows of a block, too.
constexpr int TABLE = THREADS + THREADS / 4;   // floats
__host__ __device__ __forceinline__ int slot(int p) { return p + (p >> 3) * 2; }
__host__ __device__ __forceinline__ int table_row(int pairs) { return (slot(pairs - 1) + 4) & ~3; }

template <typename T, int FORM>
__global__ void __launch_bounds__(THREADS, FORM == SPLIT ? 4 : 3)
rotary_kernel(const __grid_constant__ Geometry g, const __grid_constant__ RotaryArgs a) {
  constexpr int E = 16 / sizeof(T);                         // elements of a piece
  constexpr int BATCH = FORM == SCALAR ? 1 : FORM == SPLIT ? 2 : BLOCK_UNITS / THREADS;   // units whose loads are in flight together
  __shared__ __align__(16) float s_cos[2][TABLE], s_sin[2][TABLE];   // of row r, pair p at [r * row_slots + slot(p)]
  __shared__ int s_real[2][MAX_ROWS];
  const int tid = threadIdx.x, row_slots = table_row(a.pairs), rows = g.batch * g.L, blocks = (rows + a.block_rows - 1) / a.block_rows;
  ptx::load_params_early(g, a);

  // this thread's angle of a block
  const int my_row = tid / a.pairs, my_pair = tid - my_row * a.pairs;
  const double turns = a.turns[my_pair];
  const int axis = (my_pair >= a.axis2) ? 2 : (my_pair >= a.axis1) ? 1 : 0;
  auto angles = [&](int block, int buf) {
    const int row = block * a.block_rows + my_row;
    if (my_row < a.block_rows && block < blocks && row < rows) {
      const int b = (uint32_t)row / (uint32_t)g.L, l = row - b * g.L;
      const double t = (double)a.positions[axis * a.axis_stride + b * a.batch_stride + l] * turns;
      float sn, cs;
      sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
      s_cos[buf][my_row * row_slots + slot(my_pair)] = cs;
      s_sin[buf][my_row * row_slots + slot(my_pair)] = a.sign * sn;
      if (my_pair == 0) {
        const int s = segment_of(g, l);
        s_real[buf][my_row] = l - g.off(s) < valid_rows(g, b, s);
      }
    }
  };
  struct Unit {
    int64_t src, dst;   // element offsets from the block's first row
    int row, k, at;     // row in the block, which tensor, place of its first angle
  };
  auto find = [&](int u) {
    Unit p;
    p.row = u / a.row_units;
    const int in_row = u - p.row * a.row_units;
    int head = in_row / a.head_units;
    const int unit = in_row - head * a.head_units;
    p.k = head >= a.q_heads;
    if (p.k) head -= a.q_heads;
    const int64_t in_head = (int64_t)head * g.hd + (FORM == SCALAR ? 0 : unit * E);
    p.src = p.row * (p.k ? a.in_stride[1] : a.in_stride[0]) + in_head;
    p.dst = p.row * (p.k ? a.out_stride[1] : a.out_stride[0]) + in_head;
    p.at = FORM == SCALAR ? unit : p.row * row_slots + slot(FORM == SPLIT ? unit * E : FORM == ADJACENT ? unit * (E / 2) : 0);
    return p;
  };
  const int n_units = a.block_rows * a.row_units;
  Unit mine[BATCH];
#pragma unroll
  for (int i = 0; i < BATCH; ++i) mine[i] = find(min(tid + i * THREADS, n_units - 1));

  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  angles(blockIdx.x, 0);
  __syncthreads();
  for (int block = blockIdx.x, buf = 0; block < blocks; block += gridDim.x, buf ^= 1) {
    const int row0 = block * a.block_rows, here = min(a.block_rows, rows - row0);
    const T *q = static_cast<const T*>(a.in[0]) + row0 * a.in_stride[0], *k = static_cast<const T*>(a.in[1]) + row0 * a.in_stride[1];
    T *qo = static_cast<T*>(a.out[0]) + row0 * a.out_stride[0], *ko = static_cast<T*>(a.out[1]) + row0 * a.out_stride[1];
    for (int u0 = 0; u0 < n_units; u0 += THREADS * BATCH) {
      if (u0 > 0)
#pragma unroll
        for (int i = 0; i < BATCH; ++i) mine[i] = find(min(u0 + tid + i * THREADS, n_units - 1));
      if constexpr (FORM == SCALAR) {
        if (u0 == 0) angles(block + gridDim.x, buf ^ 1);
        const Unit& p = mine[0];
        if (u0 + tid < n_units && p.row < here) {
          const bool keep = s_real[buf][p.row];
          const T* x = (p.k ? k : q) + p.src;
          T* y = (p.k ? ko : qo) + p.dst;
          if (p.at >= a.pairs) {
            const int f = a.pairs + p.at;
            store_as(y + f, keep ? to_float(x[f]) : 0.f);
          } else {
            const int i = a.adjacent ? 2 * p.at : p.at, j = a.adjacent ? i + 1 : a.pairs + i, t = p.row * row_slots + slot(p.at);
            const float lo = keep ? to_float(x[i]) : 0.f, hi = keep ? to_float(x[j]) : 0.f, cs = s_cos[buf][t], sn = s_sin[buf][t];
            store_as(y + i, keep ? lo * cs - hi * sn : 0.f);
            store_as(y + j, keep ? lo * sn + hi * cs : 0.f);
          }
        }
      } else {
        uint4 v[BATCH], w[FORM == SPLIT ? BATCH : 1];   // as they lie in memory
        bool in[BATCH], keep[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          in[i] = u0 + tid + i * THREADS < n_units && mine[i].row < here;
          keep[i] = in[i] && s_real[buf][mine[i].row];
          if (keep[i]) {
            const T* x = (mine[i].k ? k : q) + mine[i].src;
            v[i] = *reinterpret_cast<const uint4*>(x);
            if constexpr (FORM == SPLIT) w[i] = *reinterpret_cast<const uint4*>(x + a.pairs);
          }
        }
        if (u0 == 0) {   // while these loads are under way: the next block's lines and angles
          const int64_t ahead = (int64_t)gridDim.x * a.block_rows;
#pragma unroll
          for (int i = 0; i < BATCH; ++i)
            if (row0 + ahead + mine[i].row < rows) {
              const T* x = (mine[i].k ? k + ahead * a.in_stride[1] : q + ahead * a.in_stride[0]) + mine[i].src;
              if ((reinterpret_cast<uintptr_t>(x) & 112u) == 0) asm volatile("prefetch.global.L2 [%0];" ::"l"(x));
            }
          angles(block + gridDim.x, buf ^ 1);
        }
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
          if (!in[i]) continue;
          float y[E], z[E];
#pragma unroll
          for (int e = 0; e < E; ++e) y[e] = z[e] = 0.f;
          if (keep[i]) {
            const float *pc = s_cos[buf] + mine[i].at, *ps = s_sin[buf] + mine[i].at;
            float x[E];
            unpack_piece<T>(v[i], x);
            if constexpr (FORM == SPLIT) {
              float x_hi[E];
              unpack_piece<T>(w[i], x_hi);
#pragma unroll
              for (int e = 0; e < E; e += 2) {
                const float2 c = *reinterpret_cast<const float2*>(pc + e), s = *reinterpret_cast<const float2*>(ps + e);
                const float2 lo = make_float2(x[e], x[e + 1]), hi = make_float2(x_hi[e], x_hi[e + 1]);
                const float2 a2 = __ffma2_rn(make_float2(-hi.x, -hi.y), s, __fmul2_rn(lo, c)), b2 = __ffma2_rn(lo, s, __fmul2_rn(hi, c));
                y[e] = a2.x; y[e + 1] = a2.y;
                z[e] = b2.x; z[e + 1] = b2.y;
              }
            } else {
#pragma unroll
              for (int e = 0; e < E / 2; ++e) {
                const float c = pc[e], s = ps[e];
                const int lo = FORM == HEAD ? e : 2 * e, hi = FORM == HEAD ? e + E / 2 : 2 * e + 1;
                y[lo] = x[lo] * c - x[hi] * s;
                y[hi] = x[lo] * s + x[hi] * c;
              }
            }
          }
          T* dst = (mine[i].k ? ko : qo) + mine[i].dst;
          store_n(dst, y);
          if constexpr (FORM == SPLIT) store_n(dst + a.pairs, z);
        }
      }
    }
    if (n_units > THREADS * BATCH)   // back to the first units' offsets
#pragma unroll
      for (int i = 0; i < BATCH; ++i) mine[i] = find(min(tid + i * THREADS, n_units - 1));
    __syncthreads();   // the next block's angles are there, and nobody reads this block's any more
  }
}

template <typename T>
cudaError_t launch(const Geometry& g, const RotaryArgs& a, Form form, unsigned grid, cudaStream_t st) {
  switch (form) {
    case SPLIT: return launch_overlapped(rotary_kernel<T, SPLIT>, dim3(grid), dim3(THREADS), 0, st, g, a);
    case ADJACENT: return launch_overlapped(rotary_kernel<T, ADJACENT>, dim3(grid), dim3(THREADS), 0, st, g, a);
    case HEAD: return launch_overlapped(rotary_kernel<T, HEAD>, dim3(grid), dim3(THREADS), 0, st, g, a);
    default: return launch_overlapped(rotary_kernel<T, SCALAR>, dim3(grid), dim3(THREADS), 0, st, g, a);
  }
}

}  // namespace

cudaError_t launch_rotary(const Geometry& g, int dtype, const RotaryCall& c, cudaStream_t st) {
  const int es = dtype == GSIT_BF16 ? 2 : 4, piece = 16 / es;
  RotaryArgs a = {};
  bool wide = true;
  for (int i = 0; i < 2; ++i) {
    a.in[i] = c.in[i];
    a.out[i] = c.out[i];
    a.in_stride[i] = c.in_stride[i];
    a.out_stride[i] = c.out_stride[i];
    if (c.heads[i] > 0)
      wide = wide && ((reinterpret_cast<uintptr_t>(c.in[i]) | reinterpret_cast<uintptr_t>(c.out[i])) & 15u) == 0 &&
             c.in_stride[i] * es % 16 == 0 && c.out_stride[i] * es % 16 == 0;
  }
  a.positions = c.positions;
  a.axis_stride = c.axis_stride;
  a.batch_stride = c.batch_stride;
  a.sign = c.backward ? -1.f : 1.f;
  a.pairs = c.sections[0] + c.sections[1] + c.sections[2];
  a.axis1 = c.sections[0];
  a.axis2 = c.sections[0] + c.sections[1];
  a.adjacent = c.interleaved;
  a.q_heads = c.heads[0];
  rotary_turns(c.base, a.pairs, a.turns);
  wide = wide && 2 * a.pairs == g.hd && g.hd % piece == 0;
  const Form form = !wide ? SCALAR : c.interleaved ? ADJACENT : a.pairs % piece == 0 ? SPLIT : g.hd == piece ? HEAD : SCALAR;
  a.head_units = form == SPLIT ? a.pairs / piece : form == SCALAR ? g.hd - a.pairs : g.hd / piece;
  a.row_units = a.head_units * (c.heads[0] + c.heads[1]);
  // rows of a block: an angle a thread, all of them in the table, and no more units than the registers keep offsets of
  const int batch = form == SCALAR ? 1 : form == SPLIT ? 2 : BLOCK_UNITS / THREADS;
  a.block_rows = std::max(1, std::min({THREADS / a.pairs, TABLE / table_row(a.pairs), MAX_ROWS, batch * THREADS / a.row_units}));
  int n_sm = 0;
  const cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  // (blocks of equal numbers a CTA, so of fewer rows, gain nothing: 64 x (50, 500, 500), half padded, 8 heads of 8 13.2 us for 12.4)
  const int64_t blocks = ((int64_t)g.batch * g.L + a.block_rows - 1) / a.block_rows;
  const unsigned grid = (unsigned)std::min(blocks, (int64_t)4 * n_sm);
  return dtype == GSIT_BF16 ? launch<__nv_bfloat16>(g, a, form, grid, st) : launch<float>(g, a, form, grid, st);
}

}  // namespace gsit

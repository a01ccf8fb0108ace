// Rotary positions with several axes: every pair of features (u, v) of a head becomes (u c - v s, u s + v c), with c and s of the
// pair's angle; the backward pass is the same rotation by the opposite angle.
//
// One pass over the rows, q and k read once and written once, which is all that bounds it.  A CTA takes as many rows as make 256
// (row, pair) angles -- 64 rows at 4 pairs, 8 at 32 -- so that every thread computes one angle into shared memory and all heads of q
// and k of those rows read it there: an angle costs as much as some 40 rotated pairs, and 2 x heads of them share it.
// Angles: position * frequency in turns as one double product, less its nearest integer: right to 2^-20 turns even at positions near
// 2^31, where a float product keeps no bit of the phase; then sincospi of the float remainder.
#include <math.h>

#include "ops.cuh"

namespace gsit {
namespace {

constexpr int THREADS = 256;

struct RotaryArgs {
  const void* in[2];
  void* out[2];
  int64_t in_stride[2], out_stride[2];   // elements between rows
  const int32_t* positions;
  int64_t axis_stride, batch_stride;
  float sign;
  int pairs, rows_per_cta, q_heads;
  int row_units, head_units;             // units of work (see Form) of a row and of a head
  uint32_t row_magic, head_magic;        // ceil(2^32 / units): division by a multiplication, exact while u * units < 2^32
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
enum Form { SPLIT, ADJACENT, HEAD, SCALAR };

__device__ __forceinline__ int div_magic(int u, int d, uint32_t magic) { return d == 1 ? u : (int)__umulhi((uint32_t)u, magic); }

template <typename T, int FORM>
__global__ void __launch_bounds__(THREADS)
rotary_kernel(const __grid_constant__ Geometry g, const __grid_constant__ RotaryArgs a) {
  constexpr int E = 16 / sizeof(T);                         // elements of a piece
  constexpr int BATCH = FORM == SCALAR ? 1 : FORM == SPLIT ? 2 : 4;   // units whose loads are in flight together
  __shared__ float2 table[THREADS];                         // (cos, sin) of row r, pair p at [r * pairs + p]
  const int tid = threadIdx.x;
  const int64_t row0 = (int64_t)blockIdx.x * a.rows_per_cta;
  const int here = (int)min((int64_t)a.rows_per_cta, (int64_t)g.batch * g.L - row0);
  const int b0 = (int)(row0 / g.L), l0 = (int)(row0 - (int64_t)b0 * g.L);
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();

  // sample and position of the CTA's row r
  auto locate = [&](int r, int& b, int& l) {
    b = b0;
    l = l0 + r;
    if (l >= g.L) {
      b += l / g.L;
      l %= g.L;
    }
  };
  auto angles = [&] {
    if (tid < here * a.pairs) {
      const int r = tid / a.pairs, p = tid - r * a.pairs;
      int b, l;
      locate(r, b, l);
      const int axis = (p >= a.axis2) ? 2 : (p >= a.axis1) ? 1 : 0;
      const double t = (double)a.positions[axis * a.axis_stride + b * a.batch_stride + l] * a.turns[p];
      float sn, cs;
      sincospif(2.0f * (float)(t - rint(t)), &sn, &cs);
      table[tid] = make_float2(cs, a.sign * sn);
    }
    __syncthreads();
  };
  struct Place { int64_t src, dst; int row, k, unit; bool real; };   // element offsets of the head's first feature
  auto place = [&](int u) {
    Place p;
    p.row = FORM == SCALAR ? u / a.row_units : div_magic(u, a.row_units, a.row_magic);
    const int in_row = u - p.row * a.row_units;
    int head = FORM == SCALAR ? in_row / a.head_units : div_magic(in_row, a.head_units, a.head_magic);
    p.unit = in_row - head * a.head_units;
    p.k = head >= a.q_heads;
    if (p.k) head -= a.q_heads;
    p.src = (row0 + p.row) * (p.k ? a.in_stride[1] : a.in_stride[0]) + (int64_t)head * g.hd;
    p.dst = (row0 + p.row) * (p.k ? a.out_stride[1] : a.out_stride[0]) + (int64_t)head * g.hd;
    int b, l;
    locate(p.row, b, l);
    const int s = segment_of(g, l);
    p.real = l - g.off(s) < valid_rows(g, b, s);
    return p;
  };
  auto src = [&](const Place& p) { return static_cast<const T*>(p.k ? a.in[1] : a.in[0]) + p.src; };
  auto dst = [&](const Place& p) { return static_cast<T*>(p.k ? a.out[1] : a.out[0]) + p.dst; };
  const int n_units = here * a.row_units;

  if constexpr (FORM == SCALAR) {
    angles();
    for (int u = tid; u < n_units; u += THREADS) {
      const Place p = place(u);
      const T* x = src(p);
      T* y = dst(p);
      if (p.unit >= a.pairs) {
        const int f = a.pairs + p.unit;
        store_as(y + f, p.real ? to_float(x[f]) : 0.f);
      } else {
        const int i = a.adjacent ? 2 * p.unit : p.unit, j = a.adjacent ? i + 1 : a.pairs + i;
        const float2 cs = table[p.row * a.pairs + p.unit];
        const float lo = p.real ? to_float(x[i]) : 0.f, hi = p.real ? to_float(x[j]) : 0.f;
        store_as(y + i, p.real ? lo * cs.x - hi * cs.y : 0.f);
        store_as(y + j, p.real ? lo * cs.y + hi * cs.x : 0.f);
      }
    }
  } else {
    // the first units' loads are under way while the angles are computed
    for (int u0 = tid, turn = 0; turn == 0 || u0 < n_units; u0 += THREADS * BATCH, ++turn) {
      Place p[BATCH];
      float v[BATCH][E], w[FORM == SPLIT ? BATCH : 1][E];
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const int u = u0 + i * THREADS;
        if (u < n_units) {
          p[i] = place(u);
          if (p[i].real) {
            load_n(src(p[i]) + p[i].unit * E, v[i]);
            if constexpr (FORM == SPLIT) load_n(src(p[i]) + a.pairs + p[i].unit * E, w[i]);
          }
        }
      }
      if (turn == 0) angles();
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        if (u0 + i * THREADS >= n_units) break;
        float y[E], z[E];
        const float2* t = table + p[i].row * a.pairs + (FORM == SPLIT ? p[i].unit * E : FORM == ADJACENT ? p[i].unit * (E / 2) : 0);
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = z[e] = 0.f;
        if (p[i].real) {
          if constexpr (FORM == SPLIT) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float2 cs = t[e];
              y[e] = v[i][e] * cs.x - w[i][e] * cs.y;
              z[e] = v[i][e] * cs.y + w[i][e] * cs.x;
            }
          } else {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
              const float2 cs = t[e];
              const int lo = FORM == HEAD ? e : 2 * e, hi = FORM == HEAD ? e + E / 2 : 2 * e + 1;
              y[lo] = v[i][lo] * cs.x - v[i][hi] * cs.y;
              y[hi] = v[i][lo] * cs.y + v[i][hi] * cs.x;
            }
          }
        }
        store_n(dst(p[i]) + p[i].unit * E, y);
        if constexpr (FORM == SPLIT) store_n(dst(p[i]) + a.pairs + p[i].unit * E, z);
      }
    }
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
  for (int p = 0; p < a.pairs; ++p) a.turns[p] = pow(c.base, -(double)p / a.pairs) / (2.0 * M_PI);
  a.rows_per_cta = THREADS / a.pairs;
  wide = wide && 2 * a.pairs == g.hd && g.hd % piece == 0;
  const Form form = !wide ? SCALAR : c.interleaved ? ADJACENT : a.pairs % piece == 0 ? SPLIT : g.hd == piece ? HEAD : SCALAR;
  a.head_units = form == SPLIT ? a.pairs / piece : form == SCALAR ? g.hd - a.pairs : g.hd / piece;
  a.row_units = a.head_units * (c.heads[0] + c.heads[1]);
  const auto magic = [](int d) { return d < 2 ? 0u : (uint32_t)((0x100000000ull + d - 1) / d); };
  a.head_magic = magic(a.head_units);
  a.row_magic = magic(a.row_units);
  const int64_t grid = ((int64_t)g.batch * g.L + a.rows_per_cta - 1) / a.rows_per_cta;
  return dtype == GSIT_BF16 ? launch<__nv_bfloat16>(g, a, form, (unsigned)grid, st) : launch<float>(g, a, form, (unsigned)grid, st);
}

}  // namespace gsit

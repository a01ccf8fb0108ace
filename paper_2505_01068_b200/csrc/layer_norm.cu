// LayerNorm with its backward pass.  Both are bound by the rows they read and write; everything else is arranged around that.
//
// A group of G threads takes a row and keeps it in registers, so that it is read once and the variance is summed around the mean
// (two passes over registers).  8, 16 or 32 threads up to 512 features (a warp holds 4, 2 or 1 rows), a whole CTA of 256 above, where
// sums cross the warps through shared memory.  Rows whose width, stride or address does not allow vectors of four run with VEC = 1.
// Backward: a thread owns the same columns in every row, so the gradients of gamma and beta are sums in its registers over all rows
// of a persistent CTA; the CTA's groups are added up in order, one partial row per CTA goes to the workspace, and a second small
// kernel adds those in order: no atomics, the same bits every time.
// Measured, bf16, forward / backward: 32 x 2176 rows of 512 31 us (4.6 TB/s) / 85 us (2.5 TB/s; float accumulation of dgamma and dbeta beside
// it); 64 x 1050 rows of 64, 8.6 MB a matrix, which fits L2, 8.4 / 13.8 us, of which launches and the reduction are some 10.
#include "ops.cuh"

namespace gsit {
namespace {

constexpr int THREADS = 256;
constexpr int MAX_PARTIALS = 1024;   // CTAs of the backward kernel at most (workspace)
constexpr int FWD_CTAS_PER_SM = 16;   // of the grid; 4: 36.9 us for 31.3 (32 x 2176 rows of 512), 8: 33.4

template <int G>
struct GroupSum {
  // Sum of a pair of values over the G threads of a row, in every one of them.
  static __device__ __forceinline__ float2 run(float2 v, float2* smem) {
    constexpr int W = G < 32 ? G : 32;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) {
      v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
      v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if constexpr (G > 32) {
      __syncthreads();   // the values of the sum before have been read
      if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
      __syncthreads();
      v = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < G / 32; ++w) {
        v.x += smem[w].x;
        v.y += smem[w].y;
      }
    }
    return v;
  }
};

// Rows that a group has in flight together: four or two where a row is one or two loads of each thread.
template <int NV, int VEC> constexpr int ROWS_AT_ONCE = NV * VEC <= 4 ? 4 : NV * VEC <= 8 ? 2 : 1;

// Whether row `row` is a real position (32-bit division: a call's rows are fewer than 2^29).
__device__ __forceinline__ bool real_row(const Geometry& g, int row) {
  const int b = (uint32_t)row / (uint32_t)g.L, l = row - b * g.L, s = segment_of(g, l);
  return l - g.off(s) < valid_rows(g, b, s);
}

template <typename TX, typename TY, int VEC, int G, int NV>
__global__ void __launch_bounds__(THREADS)
layer_norm_fwd_kernel(const __grid_constant__ Geometry g, const __grid_constant__ NormCall c) {
  __shared__ float2 sums[THREADS / 32];
  constexpr int GROUPS = THREADS / G, U = G > 32 ? 1 : ROWS_AT_ONCE<NV, VEC>;
  const int group = threadIdx.x / G, t = threadIdx.x % G, rows = g.batch * g.L;
  ptx::load_params_early(g, c);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const float inv_d = 1.0f / g.d;
  // whole groups of a warp run together: rows past the last are walked, too, without loads or stores
  for (int first = blockIdx.x * GROUPS * U; first < rows; first += gridDim.x * GROUPS * U) {
    float x[U][NV][VEC];
    bool real[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = first + u * GROUPS + group;
      real[u] = row < rows && real_row(g, row);
      const TX* src = static_cast<const TX*>(c.x) + (int64_t)row * c.ldx;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = (v * G + t) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][v][e] = 0.f;
        if (real[u] && col < g.d) load_n(src + col, x[u][v]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = first + u * GROUPS + group;
      float2 s = make_float2(0.f, 0.f);
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < VEC; ++e) s.x += x[u][v][e];
      const float mean = GroupSum<G>::run(s, sums).x * inv_d;
      s = make_float2(0.f, 0.f);
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float z = (v * G + t) * VEC < g.d ? x[u][v][e] - mean : 0.f;
          s.x += z * z;
        }
      const float rstd = rsqrtf(GroupSum<G>::run(s, sums).x * inv_d + c.eps);
      if (row < rows) {
        TY* dst = static_cast<TY*>(c.y) + (int64_t)row * c.ldy;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int col = (v * G + t) * VEC;
          if (col < g.d) {
            float ga[VEC], be[VEC], y[VEC];
            if (c.gamma != nullptr) load_n(c.gamma + col, ga);
            if (c.beta != nullptr) load_n(c.beta + col, be);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
              const float h = (x[u][v][e] - mean) * rstd, scaled = c.gamma != nullptr ? h * ga[e] : h;
              y[e] = real[u] ? (c.beta != nullptr ? scaled + be[e] : scaled) : 0.f;
            }
            store_n(dst + col, y);
          }
        }
        if (t == 0 && c.mean != nullptr) {
          c.mean[row] = real[u] ? mean : 0.f;
          c.rstd[row] = real[u] ? rstd : 0.f;
        }
      }
    }
  }
}

// Asks for the rows of a group's next turn while it works on this one: registers hold one turn only, and a warp that had to wait for
// memory in every turn left it idle in between (32 x 2176 rows of 512: 102 us without, 87 with; the forward kernel, which has five CTAs an
// SM, gains nothing, and rows of one load are taken several at once instead).
template <typename T, int G> __device__ __forceinline__ void ask_for_row(const void* base, int64_t at, int d, int t) {
  for (int c = t * (128 / (int)sizeof(T)); c < d; c += G * (128 / (int)sizeof(T)))
    asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const T*>(base) + at + c));
}

template <typename TX, typename TY, int VEC, int G, int NV>
__global__ void __launch_bounds__(THREADS)
layer_norm_bwd_kernel(const __grid_constant__ Geometry g, const __grid_constant__ NormCall c) {
  __shared__ float2 sums[THREADS / 32];
  constexpr int GROUPS = THREADS / G, U = G > 32 ? 1 : (ROWS_AT_ONCE<NV, VEC> + 1) / 2;
  const int group = threadIdx.x / G, t = threadIdx.x % G, rows = g.batch * g.L;
  ptx::load_params_early(g, c);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  const float inv_d = 1.0f / g.d;
  float dga[NV][VEC] = {}, dbe[NV][VEC] = {};
  for (int first = blockIdx.x * GROUPS * U; first < rows; first += gridDim.x * GROUPS * U) {
    float x[U][NV][VEC], dy[U][NV][VEC], res[U][NV][VEC], mean[U], rstd[U];
    bool real[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = first + u * GROUPS + group;
      real[u] = row < rows && real_row(g, row);
      mean[u] = rstd[u] = 0.f;
      if (real[u]) {
        mean[u] = c.mean[row];
        rstd[u] = c.rstd[row];
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = (v * G + t) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[u][v][e] = dy[u][v][e] = res[u][v][e] = 0.f;
        if (real[u] && col < g.d) {
          load_n(static_cast<const TX*>(c.x) + (int64_t)row * c.ldx + col, x[u][v]);
          load_n(static_cast<const TY*>(c.dy) + (int64_t)row * c.lddy + col, dy[u][v]);
          if (c.residual != nullptr) load_n(static_cast<const TX*>(c.residual) + (int64_t)row * c.ldres + col, res[u][v]);
        }
      }
    }
    if (const int row = first + gridDim.x * GROUPS + group; U == 1 && row < rows) {
      ask_for_row<TX, G>(c.x, (int64_t)row * c.ldx, g.d, t);
      ask_for_row<TY, G>(c.dy, (int64_t)row * c.lddy, g.d, t);
      if (c.residual != nullptr) ask_for_row<TX, G>(c.residual, (int64_t)row * c.ldres, g.d, t);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = first + u * GROUPS + group;
      float2 s = make_float2(0.f, 0.f);   // sums of g and of g h
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int col = (v * G + t) * VEC;
        float ga[VEC];
        const bool scaled = c.gamma != nullptr && col < g.d;
        if (scaled) load_n(c.gamma + col, ga);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float h = (x[u][v][e] - mean[u]) * rstd[u];   // columns past the last meet a dy of zero
          dga[v][e] += dy[u][v][e] * h;
          dbe[v][e] += dy[u][v][e];
          x[u][v][e] = h;
          dy[u][v][e] = scaled ? dy[u][v][e] * ga[e] : dy[u][v][e];
          s.x += dy[u][v][e];
          s.y += dy[u][v][e] * h;
        }
      }
      s = GroupSum<G>::run(s, sums);
      if (row < rows) {
        const float m1 = s.x * inv_d, m2 = s.y * inv_d;
        TX* dst = static_cast<TX*>(c.dx) + (int64_t)row * c.lddx;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const int col = (v * G + t) * VEC;
          if (col < g.d) {
            float dx[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) dx[e] = real[u] ? (dy[u][v][e] - m1 - x[u][v][e] * m2) * rstd[u] + res[u][v][e] : 0.f;
            store_n(dst + col, dx);
          }
        }
      }
    }
  }
  if (c.partial == nullptr) return;
  // the CTA's groups, added in order: each group in turn adds its columns to the partial row (in shared memory: at most 512 columns
  // where there is more than one group)
  float* out = c.partial + (int64_t)blockIdx.x * 2 * g.d;
  if constexpr (GROUPS > 1) {
    constexpr int COLS = G * NV * VEC;
    static_assert(COLS <= 1024, "columns of a warp's row");
    __shared__ float acc[2 * COLS];
    for (int k = 0; k < GROUPS; ++k) {
      if (group == k)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const int col = (v * G + t) * VEC + e;
            acc[col] = k == 0 ? dga[v][e] : acc[col] + dga[v][e];
            acc[COLS + col] = k == 0 ? dbe[v][e] : acc[COLS + col] + dbe[v][e];
          }
      __syncthreads();
    }
    for (int col = threadIdx.x; col < g.d; col += THREADS) {
      out[col] = acc[col];
      out[g.d + col] = acc[COLS + col];
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int col = (v * G + t) * VEC + e;
        if (col < g.d) {
          out[col] = dga[v][e];
          out[g.d + col] = dbe[v][e];
        }
      }
  }
}

// dgamma, dbeta = the partial rows added up.  A CTA takes 32 columns (of the 2 d), its 32 warps a share of the rows each.
__global__ void __launch_bounds__(1024)
layer_norm_reduce_kernel(const float* __restrict__ partial, int n, int d, float* dgamma, float* dbeta) {
  __shared__ float acc[32][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  float s = 0.f;
  if (col < 2 * d)
#pragma unroll 8
    for (int i = warp; i < n; i += 32) s += partial[(int64_t)i * 2 * d + col];
  acc[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && col < 2 * d) {
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 32; ++w) s += acc[w][lane];
    if (col < d) dgamma[col] = s;
    else dbeta[col - d] = s;
  }
}

template <int FWD, typename TX, typename TY, int VEC, int G, int NV>
cudaError_t launch_form(const Geometry& g, const NormCall& c, unsigned grid, cudaStream_t st) {
  if constexpr (FWD) return launch_overlapped(layer_norm_fwd_kernel<TX, TY, VEC, G, NV>, dim3(grid), dim3(THREADS), 0, st, g, c);
  else return launch_overlapped(layer_norm_bwd_kernel<TX, TY, VEC, G, NV>, dim3(grid), dim3(THREADS), 0, st, g, c);
}

// Threads of a row: 8, 16 or 32 with one vector each up to 128 features (more rows of narrow layers in flight than with idle lanes), a warp
// with up to four up to 512, a CTA above.  Forward / backward, us: 64 x 1050 rows of 64 with 16 threads 8.3 / 13.8, with 32 14.1 / 21.3; 32 x 2176
// rows of 512 with a warp 31 / 85, with a CTA 111 / 174.  Without vectors of four: 50 / 217.
int row_threads(int d) { return d <= 32 ? 8 : d <= 64 ? 16 : d <= 512 ? 32 : THREADS; }

template <int FWD, typename TX, typename TY>
cudaError_t launch_typed(const Geometry& g, const NormCall& c, bool wide, unsigned grid, cudaStream_t st) {
  const int d = g.d;
#define GSIT_FORM(VEC, G, NV) return launch_form<FWD, TX, TY, VEC, G, NV>(g, c, grid, st)
  if (wide) {
    if (d <= 32) GSIT_FORM(4, 8, 1);
    if (d <= 64) GSIT_FORM(4, 16, 1);
    if (d <= 128) GSIT_FORM(4, 32, 1);
    if (d <= 256) GSIT_FORM(4, 32, 2);
    if (d <= 512) GSIT_FORM(4, 32, 4);
    if (d <= 1024) GSIT_FORM(4, 256, 1);
    if (d <= 2048) GSIT_FORM(4, 256, 2);
    if (d <= 4096) GSIT_FORM(4, 256, 4);
    GSIT_FORM(4, 256, 8);
  }
  if (d <= 32) GSIT_FORM(1, 8, 4);
  if (d <= 64) GSIT_FORM(1, 16, 4);
  if (d <= 128) GSIT_FORM(1, 32, 4);
  if (d <= 512) GSIT_FORM(1, 32, 16);
  if (d <= 1024) GSIT_FORM(1, 256, 4);
  if (d <= 2048) GSIT_FORM(1, 256, 8);
  GSIT_FORM(1, 256, 32);
#undef GSIT_FORM
}

template <int FWD>
cudaError_t launch_any(const Geometry& g, const NormCall& c, bool wide, unsigned grid, cudaStream_t st) {
  if (c.x_dtype == GSIT_F32)
    return c.y_dtype == GSIT_F32 ? launch_typed<FWD, float, float>(g, c, wide, grid, st) : launch_typed<FWD, float, __nv_bfloat16>(g, c, wide, grid, st);
  return c.y_dtype == GSIT_F32 ? launch_typed<FWD, __nv_bfloat16, float>(g, c, wide, grid, st)
                               : launch_typed<FWD, __nv_bfloat16, __nv_bfloat16>(g, c, wide, grid, st);
}

// Vectors of four elements can be loaded from rows at `p` with this stride.
bool vectors(const void* p, int64_t ld, int dtype) {
  const int es = dtype == GSIT_BF16 ? 2 : 4;
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) % (4 * es)) == 0 && ld % 4 == 0);
}

int64_t row_groups(const Geometry& g) {
  const int per = THREADS / row_threads(g.d);
  return ((int64_t)g.batch * g.L + per - 1) / per;
}

// 4 CTAs an SM: 64 x 1050 rows of 64 13.8 us with 4, 17.5 with 2; 32 x 1000 rows of 1024 102 and 140; 32 x 2176 rows of 512 85 and 80.
int bwd_ctas(const Geometry& g, int n_sm) { return (int)min((int64_t)min(4 * n_sm, MAX_PARTIALS), row_groups(g)); }

}  // namespace

size_t layer_norm_bwd_scratch(const Geometry& g) { return sizeof(float) * 2 * (size_t)g.d * (size_t)min((int64_t)MAX_PARTIALS, row_groups(g)); }

cudaError_t launch_layer_norm_fwd(const Geometry& g, const NormCall& c, cudaStream_t st) {
  const bool wide = g.d % 4 == 0 && vectors(c.x, c.ldx, c.x_dtype) && vectors(c.y, c.ldy, c.y_dtype) && vectors(c.gamma, 0, GSIT_F32) &&
                    vectors(c.beta, 0, GSIT_F32);
  int n_sm = 0;
  const cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  return launch_any<1>(g, c, wide, (unsigned)min(row_groups(g), (int64_t)FWD_CTAS_PER_SM * n_sm), st);
}

cudaError_t launch_layer_norm_bwd(const Geometry& g, const NormCall& c, cudaStream_t st) {
  int n_sm = 0;
  cudaError_t e = sm_count_and_smem_once(nullptr, 0, &n_sm);
  if (e != cudaSuccess) return e;
  const bool wide = g.d % 4 == 0 && vectors(c.x, c.ldx, c.x_dtype) && vectors(c.dy, c.lddy, c.y_dtype) && vectors(c.gamma, 0, GSIT_F32) &&
                    vectors(c.residual, c.ldres, c.x_dtype) && vectors(c.dx, c.lddx, c.x_dtype);
  const int n = bwd_ctas(g, n_sm);
  e = launch_any<0>(g, c, wide, (unsigned)n, st);
  if (e != cudaSuccess || c.partial == nullptr) return e;
  return launch_overlapped(layer_norm_reduce_kernel, dim3((2 * g.d + 31) / 32), dim3(1024), 0, st, c.partial, n, g.d, c.dgamma, c.dbeta);
}

}  // namespace gsit

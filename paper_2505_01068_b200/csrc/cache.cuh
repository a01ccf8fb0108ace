// What the calls of gsit_stream.h share: the cache as kernels see it, and launch entry points.
#pragma once
#include "gsit_stream.h"
#include "ops.cuh"

namespace gsit {

constexpr int CACHE_BLOCK = GSIT_CACHE_BLOCK;
constexpr float LEAST_SCALE = 8.271806125530277e-25f;   // 2^-80: below, a quotient's remainder would leave the range of float

struct Cache {
  int kind, batch, kv_heads, hd, pages, blocks;
  uint8_t *keys, *values;
  float *key_scale, *value_scale, *times;
  void *open_keys, *open_values;
  int32_t *tables, *lengths, *free_list, *n_free;
};

// Positions held of segment s of stream b, within what its table can say.
__device__ __forceinline__ int held_rows(const Cache& c, unsigned int* status, int b, int s) {
  const int n = c.lengths[3 * b + s], most = c.blocks * CACHE_BLOCK;
  if (n >= 0 && n <= most) return n;
  atomicOr(status, GSIT_DEVFLAG_CLAMPED);
  return n < 0 ? 0 : most;
}
// A page that exists, or -1.
__device__ __forceinline__ int real_page(const Cache& c, int page) { return (unsigned)page < (unsigned)c.pages ? page : -1; }
// Element offset of the open rows of (stream, segment, block, head).
__device__ __forceinline__ int64_t open_at(const Cache& c, int b, int s, int block, int head) {
  return ((((int64_t)b * 3 + s) * 2 + (block & 1)) * c.kv_heads + head) * (CACHE_BLOCK * c.hd);
}

// Moments of a step's rows.
struct RowTimes {
  const float* p;
  int64_t batch, row;                  // elements between streams, and between rows
  __device__ __forceinline__ float at(int b, int i) const { return p[b * batch + i * row]; }
};

// cache_plan.cu
cudaError_t launch_cache_plan(const Geometry& g, const Cache& c, const int32_t* held, const int32_t* ended, int32_t* slots, cudaStream_t st);
// cache_rows.cu
cudaError_t launch_cache_append(const Geometry& g, int dtype, const Cache& c, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* slots,
                                const RowTimes& times, cudaStream_t st);
cudaError_t launch_cache_read(const Geometry& g, int dtype, const Cache& c, void* k, int64_t ldk, void* v, int64_t ldv, cudaStream_t st);

// cached_bf16.cu, cached_f32.cu
struct CachedArgs {
  Cache c;
  const void* q; int64_t ldq;
  void* out;
  float* lse;
  const float* slopes;
  RowTimes times;                      // null: the index inside the segment
  int group, rows, causal;             // rows: query rows of a key head, L * group
  bool mixed;                          // tiles of rows run across segments
  float softcap, inner, outer;         // score = outer * tanh(inner * dot) or inner * dot, base 2
  bool fast_cap;                       // inner holds 2 log2 e, too: tanh(y) = 1 - 2 / (e^2y + 1) by an exponential in base 2
  int split;                           // CTAs of the cluster that shares a (stream, key head, tile of rows)
  float* parts;                        // workspace; null: the CTAs of a cluster share the work and need none
};
// scratch not null: nothing is launched, only the workspace's size is said (0: none).
cudaError_t launch_cached_bf16(const Geometry& g, CachedArgs& a, cudaStream_t st, size_t* scratch);
cudaError_t launch_cached_f32(const Geometry& g, CachedArgs& a, cudaStream_t st, size_t* scratch);

}  // namespace gsit

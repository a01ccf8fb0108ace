// Rows into the cache of a stream and back (gsit_cache_append, gsit_cache_read).
//
// A warp takes one block of 32 positions and one key head.  A block that a step fills is quantised as a whole: its rows (those of earlier steps from
// the open block's buffer, the others from the call) are staged in shared memory, read from there in the order of the page -- pairs of features of
// a position for keys, pairs of positions of a feature for values -- and stay in registers while the largest magnitude, the scale and the bytes are found,
// so that everything is read once and a page's head is written as whole lines.  A block that stays open takes copies of the new rows.  Reading goes
// the other way.  Bound by the bytes moved.
//
// x / scale is rounded once: the quotient in float is brought to the odd one of its two neighbours wherever a remainder is left (its sign
// says on which side), so that the rounding to 8 bits that follows meets a tie only where there is one.
#include <cuda_fp8.h>

#include "cache.cuh"

namespace gsit {
namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;

template <typename T, int HD> constexpr int PITCH = HD * (int)sizeof(T) + 16;   // bytes of a staged row: neighbours meet other banks
template <typename T, int HD> constexpr int STAGE = CACHE_BLOCK * PITCH<T, HD>; // of one matrix

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ void copies_done() {
  asm volatile("cp.async.commit_group;\n\tcp.async.wait_group 0;" ::: "memory");
  __syncwarp();
}
__device__ __forceinline__ uint32_t transposed8(uint32_t v) {   // of the 8 x 8 matrix of 16-bit elements that the warp holds
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// Eight values of a lane, bytes 8 u .. 8 u + 7 of its piece(s) of the page: [c][h][e], or heads of 8: all of them.  `at`: the staged matrix.
template <typename T, int HD, bool VALUES> __device__ __forceinline__ void staged(const uint8_t* at, int lane, int u, float (&f)[8]) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {   // pairs: c = i / 2, h = i % 2;  heads of 8: keys m = i / 2, h = i % 2, values half = i / 2, c = i % 2
    int row, col;                 // of the 16-bit pair's operand row (g) and first column (2 t)
    if constexpr (HD == 8) {
      row = VALUES ? g : 16 * (i / 2) + 8 * (i % 2) + g;
      col = VALUES ? 16 * (i / 2) + 8 * (i % 2) + 2 * t : 2 * t;
    } else {
      row = (VALUES ? 16 * (u / 2) : 16 * (u % 2)) + 8 * (i % 2) + g;
      col = (VALUES ? 16 * (u % 2) : 16 * (u / 2)) + 8 * (i / 2) + 2 * t;
    }
    if constexpr (!VALUES) {
      const T* p = reinterpret_cast<const T*>(at + row * PITCH<T, HD>) + col;
      if constexpr (sizeof(T) == 2) unpack_bf16(*reinterpret_cast<const uint32_t*>(p), f[2 * i], f[2 * i + 1]);
      else {
        const float2 v = *reinterpret_cast<const float2*>(p);
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
      }
    } else if constexpr (sizeof(T) == 2) {   // positions 8 (col / 8) + g, features 8 (row / 8) + 2 t, turned round
      const int position = col / 8 * 8 + g, feature = row / 8 * 8 + 2 * t;
      unpack_bf16(transposed8(*reinterpret_cast<const uint32_t*>(reinterpret_cast<const T*>(at + position * PITCH<T, HD>) + feature)), f[2 * i], f[2 * i + 1]);
    } else {
      f[2 * i] = reinterpret_cast<const T*>(at + col * PITCH<T, HD>)[row];
      f[2 * i + 1] = reinterpret_cast<const T*>(at + (col + 1) * PITCH<T, HD>)[row];
    }
  }
}
// The other way: eight values to the staged matrix.
template <typename T, int HD, bool VALUES> __device__ __forceinline__ void stage(uint8_t* at, int lane, int u, const float (&f)[8]) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int row, col;
    if constexpr (HD == 8) {
      row = VALUES ? g : 16 * (i / 2) + 8 * (i % 2) + g;
      col = VALUES ? 16 * (i / 2) + 8 * (i % 2) + 2 * t : 2 * t;
    } else {
      row = (VALUES ? 16 * (u / 2) : 16 * (u % 2)) + 8 * (i % 2) + g;
      col = (VALUES ? 16 * (u % 2) : 16 * (u / 2)) + 8 * (i / 2) + 2 * t;
    }
    if constexpr (!VALUES) {
      T* p = reinterpret_cast<T*>(at + row * PITCH<T, HD>) + col;
      if constexpr (sizeof(T) == 2) *reinterpret_cast<uint32_t*>(p) = ptx::pack_bf16(f[2 * i], f[2 * i + 1]);
      else *reinterpret_cast<float2*>(p) = make_float2(f[2 * i], f[2 * i + 1]);
    } else if constexpr (sizeof(T) == 2) {
      const int position = col / 8 * 8 + g, feature = row / 8 * 8 + 2 * t;
      *reinterpret_cast<uint32_t*>(reinterpret_cast<T*>(at + position * PITCH<T, HD>) + feature) = transposed8(ptx::pack_bf16(f[2 * i], f[2 * i + 1]));
    } else {
      reinterpret_cast<T*>(at + col * PITCH<T, HD>)[row] = f[2 * i];
      reinterpret_cast<T*>(at + (col + 1) * PITCH<T, HD>)[row] = f[2 * i + 1];
    }
  }
}

template <int HD> constexpr int UNITS = HD == 8 ? 1 : HD / 8;   // of eight bytes of a lane
template <int HD> __device__ __forceinline__ int unit_at(int lane, int u) { return HD == 8 ? 8 * lane : 512 * (u / 2) + 16 * lane + 8 * (u % 2); }

// x / s to one of its two neighbours in float, the odd one unless it is exact
__device__ __forceinline__ float odd_quotient(float x, float s, float inv) {
  float t = x * inv;
  t = fmaf(fmaf(-t, s, x), inv, t);
  const float rest = fmaf(-t, s, x);
  int bits = __float_as_int(t);
  if (rest != 0.f && (bits & 1) == 0) bits += ((__float_as_int(rest) ^ bits) < 0 && t != 0.f) ? -1 : 1;
  return __int_as_float(bits);
}
__device__ __forceinline__ uint32_t bytes4(int kind, float a, float b, float c, float d) {
  if (kind == GSIT_CACHE_INT8) {
    const int i = __float2int_rn(fminf(fmaxf(a, -127.f), 127.f)), j = __float2int_rn(fminf(fmaxf(b, -127.f), 127.f));
    const int k = __float2int_rn(fminf(fmaxf(c, -127.f), 127.f)), l = __float2int_rn(fminf(fmaxf(d, -127.f), 127.f));
    return (uint32_t)(i & 255) | (uint32_t)(j & 255) << 8 | (uint32_t)(k & 255) << 16 | (uint32_t)l << 24;
  }
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | (uint32_t)hi << 16;
}
__device__ __forceinline__ void values4(int kind, uint32_t w, float (&f)[4]) {
  if (kind == GSIT_CACHE_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
    return;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(w >> (16 * i))));
    const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
}

// One staged matrix into a page's head.
template <typename T, int HD, bool VALUES>
__device__ __forceinline__ void quantise(int kind, const uint8_t* at, int lane, uint8_t* bytes, float* scale) {
  constexpr int U = UNITS<HD>;
  float f[U][8];
  uint32_t top = 0;   // magnitudes in order as integers, NaN above them all
#pragma unroll
  for (int u = 0; u < U; ++u) {
    staged<T, HD, VALUES>(at, lane, u, f[u]);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[u][i]) & 0x7fffffffu);
  }
  top = __reduce_max_sync(0xffffffffu, top);
  const bool broken = top >= 0x7f800000u;
  const float s = broken ? 1.f : fmaxf(__fdiv_rn(__uint_as_float(top), kind == GSIT_CACHE_INT8 ? 127.f : 448.f), LEAST_SCALE), inv = __frcp_rn(s);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = broken ? 0.f : odd_quotient(f[u][i], s, inv);
    *reinterpret_cast<uint2*>(bytes + unit_at<HD>(lane, u)) = make_uint2(bytes4(kind, t[0], t[1], t[2], t[3]), bytes4(kind, t[4], t[5], t[6], t[7]));
  }
  if (lane == 0) *scale = broken ? __int_as_float(0x7fffffff) : s;
}

// What a warp works on: block `chunk` of those that a step's rows of segment s of stream b lie in, one key head.
struct Piece {
  int b, s, chunk, head;
};
__device__ __forceinline__ bool find_piece(unsigned item, const int (&chunks)[3], int batch, int heads, Piece* p) {
  const unsigned per = (unsigned)(chunks[0] + chunks[1] + chunks[2]), at = item / (unsigned)heads;
  p->head = (int)(item - at * (unsigned)heads);
  p->b = (int)(at / per);
  int c = (int)(at - (unsigned)p->b * per);
  p->s = 0;
  if (c >= chunks[0]) {
    c -= chunks[0];
    p->s = 1;
    if (c >= chunks[1]) {
      c -= chunks[1];
      p->s = 2;
    }
  }
  p->chunk = c;
  return p->b < batch;
}

// How many rows of a segment have a slot: they come first.  A warp looks at every 32nd part, then at the parts of the one that is left.
__device__ __forceinline__ int leading_rows(const int32_t* slots, int len, int lane) {
  int n = 0;
  for (int span = len; span > 0;) {
    const int stride = (span + 31) / 32, at = n + (lane + 1) * stride - 1;
    n += stride * __popc(__ballot_sync(0xffffffffu, at < n + span && slots[at] >= 0));
    span = min(stride - 1, len - n);
  }
  return n;
}

struct RowArgs {
  Cache c;
  const void *k, *v;              // append: read
  void *k_out, *v_out;            // read: written
  int64_t ldk, ldv;
  const int32_t* slots;
  RowTimes times;
  int chunks[3];
};

template <typename T, int HD>
__global__ void __launch_bounds__(THREADS) cache_append_kernel(const __grid_constant__ Geometry g, const __grid_constant__ RowArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int VECS = HD * (int)sizeof(T) / 16;   // of a row
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Cache& c = a.c;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  Piece p;
  if (!find_piece(blockIdx.x * WARPS + warp, a.chunks, g.batch, c.kv_heads, &p)) return;
  const int64_t row0 = (int64_t)p.b * g.L + g.off(p.s);
  const int32_t* const slots = a.slots + row0;
  const int n = leading_rows(slots, g.len(p.s), lane);
  if (n == 0) return;
  // the rows [i0, i1) of the segment lie in this block, from place `o` on
  const int place0 = slots[0] % CACHE_BLOCK, i0 = max(0, p.chunk * CACHE_BLOCK - place0), i1 = min(n, (p.chunk + 1) * CACHE_BLOCK - place0);
  if (i0 >= i1) return;
  const int o = p.chunk == 0 ? place0 : 0, slot = slots[i0], page = slot < 0 ? -1 : real_page(c, slot / CACHE_BLOCK);
  if (page < 0) {
    raise_flag(g, GSIT_DEVFLAG_CLAMPED);
    return;
  }
  const int block = (held_rows(c, g.status, p.b, p.s) - n + i0) / CACHE_BLOCK;
  if (c.times != nullptr && p.head == 0 && i0 + lane < i1) c.times[(int64_t)page * CACHE_BLOCK + o + lane] = a.times.at(p.b, g.off(p.s) + i0 + lane);
  const T* const k = static_cast<const T*>(a.k) + (row0 + i0) * a.ldk + (int64_t)p.head * HD;
  const T* const v = static_cast<const T*>(a.v) + (row0 + i0) * a.ldv + (int64_t)p.head * HD;
  const int64_t open = open_at(c, p.b, p.s, block, p.head);
  T* const open_k = static_cast<T*>(c.open_keys) + open;
  T* const open_v = static_cast<T*>(c.open_values) + open;
  // rows to the places from `to` on of an open block
  auto keep_open = [&](int to, int rows, const T* k_rows, const T* v_rows) {
    for (int i = lane; i < rows * VECS; i += 32) {
      const int row = i / VECS, at = i % VECS * (16 / (int)sizeof(T));
      *reinterpret_cast<uint4*>(open_k + (to + row) * HD + at) = *reinterpret_cast<const uint4*>(k_rows + row * a.ldk + at);
      *reinterpret_cast<uint4*>(open_v + (to + row) * HD + at) = *reinterpret_cast<const uint4*>(v_rows + row * a.ldv + at);
    }
  };
  // The step's last block, where it stays open, may share its buffer with the rows that the first one still has there: then the first one's warp takes both.
  const int last = (place0 + n - 1) / CACHE_BLOCK, tail = (place0 + n) % CACHE_BLOCK;
  const bool shared = place0 > 0 && last >= 2 && last % 2 == 0 && tail > 0;
  if (o + i1 - i0 < CACHE_BLOCK) {   // stays open
    if (!(shared && p.chunk == last)) keep_open(o, i1 - i0, k, v);
    return;
  }
  uint8_t* const stage_k = smem + warp * 2 * STAGE<T, HD>;
  uint8_t* const stage_v = stage_k + STAGE<T, HD>;
#pragma unroll
  for (int i = lane; i < CACHE_BLOCK * VECS; i += 32) {
    const int row = i / VECS, at = i % VECS * (16 / (int)sizeof(T)), to = row * PITCH<T, HD> + i % VECS * 16;
    copy16(smem_u32(stage_k + to), row < o ? open_k + row * HD + at : k + (row - o) * a.ldk + at);
    copy16(smem_u32(stage_v + to), row < o ? open_v + row * HD + at : v + (row - o) * a.ldv + at);
  }
  copies_done();
  if (shared && p.chunk == 0) keep_open(0, tail, k + (n - tail) * a.ldk, v + (n - tail) * a.ldv);   // (i0 is 0 here)
  const int64_t to = (int64_t)page * c.kv_heads + p.head;
  quantise<T, HD, false>(c.kind, stage_k, lane, c.keys + to * (CACHE_BLOCK * HD), c.key_scale + to);
  quantise<T, HD, true>(c.kind, stage_v, lane, c.values + to * (CACHE_BLOCK * HD), c.value_scale + to);
}

template <typename T, int HD>
__global__ void __launch_bounds__(THREADS) cache_read_kernel(const __grid_constant__ Geometry g, const __grid_constant__ RowArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int VECS = HD * (int)sizeof(T) / 16, U = UNITS<HD>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Cache& c = a.c;
  ptx::load_params_early(g, a);
  ptx::grid_dep_wait();
  ptx::grid_dep_launch();
  Piece p;
  if (!find_piece(blockIdx.x * WARPS + warp, a.chunks, g.batch, c.kv_heads, &p)) return;
  const int first = p.chunk * CACHE_BLOCK, held = held_rows(c, g.status, p.b, p.s), rows = min(CACHE_BLOCK, g.len(p.s) - first);
  const int64_t row0 = (int64_t)p.b * g.L + g.off(p.s) + first;
  T* const k = static_cast<T*>(a.k_out) + row0 * a.ldk + (int64_t)p.head * HD;
  T* const v = static_cast<T*>(a.v_out) + row0 * a.ldv + (int64_t)p.head * HD;
  if (first + CACHE_BLOCK > held) {   // the open block, or behind it
    const int64_t open = open_at(c, p.b, p.s, p.chunk, p.head);
    for (int i = lane; i < rows * VECS; i += 32) {
      const int row = i / VECS, at = i % VECS * (16 / (int)sizeof(T));
      uint4 x = make_uint4(0, 0, 0, 0), y = x;
      if (first + row < held) {
        x = *reinterpret_cast<const uint4*>(static_cast<const T*>(c.open_keys) + open + row * HD + at);
        y = *reinterpret_cast<const uint4*>(static_cast<const T*>(c.open_values) + open + row * HD + at);
      }
      *reinterpret_cast<uint4*>(k + row * a.ldk + at) = x;
      *reinterpret_cast<uint4*>(v + row * a.ldv + at) = y;
    }
    return;
  }
  const int page = real_page(c, c.tables[((int64_t)p.b * 3 + p.s) * c.blocks + p.chunk]);
  if (page < 0) raise_flag(g, GSIT_DEVFLAG_CLAMPED);
  const int64_t from = (int64_t)max(page, 0) * c.kv_heads + p.head;
  uint2 x[U], y[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    x[u] = page < 0 ? make_uint2(0, 0) : *reinterpret_cast<const uint2*>(c.keys + from * (CACHE_BLOCK * HD) + unit_at<HD>(lane, u));
    y[u] = page < 0 ? make_uint2(0, 0) : *reinterpret_cast<const uint2*>(c.values + from * (CACHE_BLOCK * HD) + unit_at<HD>(lane, u));
  }
  const float ks = page < 0 ? 0.f : c.key_scale[from], vs = page < 0 ? 0.f : c.value_scale[from];
  uint8_t* const stage_k = smem + warp * 2 * STAGE<T, HD>;
  uint8_t* const stage_v = stage_k + STAGE<T, HD>;
  auto spread = [&](const uint2& w, float s, float (&f)[8]) {
    float lo[4], hi[4];
    values4(c.kind, w.x, lo);
    values4(c.kind, w.y, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = lo[i] * s;
      f[4 + i] = hi[i] * s;
    }
  };
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float f[8];
    spread(x[u], ks, f);
    stage<T, HD, false>(stage_k, lane, u, f);
    spread(y[u], vs, f);
    stage<T, HD, true>(stage_v, lane, u, f);
  }
  __syncwarp();
  for (int i = lane; i < rows * VECS; i += 32) {
    const int row = i / VECS, at = i % VECS * (16 / (int)sizeof(T)), in = row * PITCH<T, HD> + i % VECS * 16;
    *reinterpret_cast<uint4*>(k + row * a.ldk + at) = *reinterpret_cast<const uint4*>(stage_k + in);
    *reinterpret_cast<uint4*>(v + row * a.ldv + at) = *reinterpret_cast<const uint4*>(stage_v + in);
  }
}

template <typename T, int HD, bool APPEND> cudaError_t launch(const Geometry& g, const RowArgs& a, cudaStream_t st) {
  const auto kernel = APPEND ? cache_append_kernel<T, HD> : cache_read_kernel<T, HD>;
  constexpr int bytes = WARPS * 2 * STAGE<T, HD>;
  const cudaError_t e = sm_count_and_smem_once(reinterpret_cast<const void*>(kernel), bytes, nullptr);
  if (e != cudaSuccess) return e;
  const int64_t items = (int64_t)g.batch * (a.chunks[0] + a.chunks[1] + a.chunks[2]) * a.c.kv_heads, grid = (items + WARPS - 1) / WARPS;
  if (grid > 0x7fffffff / WARPS) return cudaErrorNotSupported;
  return launch_overlapped(kernel, dim3((unsigned)grid), dim3(THREADS), bytes, st, g, a);
}
template <bool APPEND> cudaError_t launch_any(const Geometry& g, int dtype, const RowArgs& a, cudaStream_t st) {
  const bool half = dtype == GSIT_BF16;
  switch (a.c.hd) {
    case 8: return half ? launch<__nv_bfloat16, 8, APPEND>(g, a, st) : launch<float, 8, APPEND>(g, a, st);
    case 16: return half ? launch<__nv_bfloat16, 16, APPEND>(g, a, st) : launch<float, 16, APPEND>(g, a, st);
    case 32: return half ? launch<__nv_bfloat16, 32, APPEND>(g, a, st) : launch<float, 32, APPEND>(g, a, st);
    default: return half ? launch<__nv_bfloat16, 64, APPEND>(g, a, st) : launch<float, 64, APPEND>(g, a, st);
  }
}

}  // namespace

cudaError_t launch_cache_append(const Geometry& g, int dtype, const Cache& c, const void* k, int64_t ldk, const void* v, int64_t ldv, const int32_t* slots,
                                const RowTimes& times, cudaStream_t st) {
  RowArgs a = {c, k, v, nullptr, nullptr, ldk, ldv, slots, times, {0, 0, 0}};
  for (int s = 0; s < 3; ++s) a.chunks[s] = g.len(s) == 0 ? 0 : (g.len(s) + 2 * CACHE_BLOCK - 2) / CACHE_BLOCK;   // n rows from any place on: at most this many blocks
  return launch_any<true>(g, dtype, a, st);
}

cudaError_t launch_cache_read(const Geometry& g, int dtype, const Cache& c, void* k, int64_t ldk, void* v, int64_t ldv, cudaStream_t st) {
  RowArgs a = {c, nullptr, nullptr, k, v, ldk, ldv, nullptr, {nullptr, 0, 0}, {0, 0, 0}};
  for (int s = 0; s < 3; ++s) a.chunks[s] = (g.len(s) + CACHE_BLOCK - 1) / CACHE_BLOCK;
  return launch_any<false>(g, dtype, a, st);
}

}  // namespace gsit

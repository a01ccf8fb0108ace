// Rows into the cache of a stream and back (gsit_cache_append, gsit_cache_read).
//
// A warp takes one block of 32 positions and one key head.  A block that a step fills is quantised as a whole: its rows (those of earlier steps from
// the open block's buffer, the others from the call) are staged in shared memory, read from there in the order of the page -- pairs of features of
// a position for keys, pairs of positions of a feature for values -- and stay in registers while the largest magnitude, the scale and the bytes are found,
// so that everything is read once and a page's head is written as whole lines.  A block that stays open takes copies of the new rows.  Reading goes
// the other way, bound by the bytes moved; an append waits for its rows before it computes, and for issue slots then.
//
// x / scale is rounded once: the quotient in float is brought to the odd one of its two neighbours wherever a remainder is left (its sign
// says on which side), so that the rounding to 8 bits that follows meets a tie only where there is one.
// Measured: prompts of 32 x (128, 1024, 1024), a quarter padding, 8 heads of 64, bf16 -> e4m3 and back, 357 MB: 92 us with the plan; append 47 us (58 % of the
// issue slots: a value takes 14 instructions), read 34 us, 5.8 TB/s.
#include <cuda_fp16.h>

#include <type_traits>

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
// Four 8 x 8 matrices of 16-bit elements between registers and shared memory, as they lie or turned round; lane l gives the address of row l % 8 of matrix l / 8.
template <bool TURN> __device__ __forceinline__ void load_matrices(uint32_t at, uint32_t (&r)[4]) {
  if constexpr (TURN)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <bool TURN> __device__ __forceinline__ void store_matrices(uint32_t at, const uint32_t (&r)[4]) {
  if constexpr (TURN)
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
  else
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}

// Unit u of a lane, bytes 8 u .. 8 u + 7 of its pieces of the page, is eight values, four pairs i = 2 c + h (heads of 8: all there is; keys i = 2 m + h, values
// i = 2 half + c): pair i is row g of an 8 x 8 matrix of positions x features (values: features x positions), columns 2 t and 2 t + 1.  Where
// matrix i of the unit begins in the staged rows:
template <int HD, bool VALUES> __device__ __forceinline__ int2 matrix_at(int u, int i) {   // (position, feature)
  if constexpr (HD == 8) return make_int2(8 * i, 0);
  const int c = i / 2, h = i % 2;
  return VALUES ? make_int2(16 * (u % 2) + 8 * c, 16 * (u / 2) + 8 * h) : make_int2(16 * (u % 2) + 8 * h, 16 * (u / 2) + 8 * c);
}
// One unit of a staged matrix as pairs: 16 bits each as they are, or floats.
template <int HD, bool VALUES> __device__ __forceinline__ void staged(const uint8_t* at, int lane, int u, uint32_t (&w)[4]) {
  const int2 m = matrix_at<HD, VALUES>(u, lane / 8);
  load_matrices<VALUES>(smem_u32(at) + (m.x + lane % 8) * PITCH<__nv_bfloat16, HD> + 2 * m.y, w);
}
template <int HD, bool VALUES> __device__ __forceinline__ void staged(const uint8_t* at, int lane, int u, float2 (&f)[4]) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int2 m = matrix_at<HD, VALUES>(u, i);
    if constexpr (VALUES)
      f[i] = make_float2(reinterpret_cast<const float*>(at + (m.x + 2 * t) * PITCH<float, HD>)[m.y + g], reinterpret_cast<const float*>(at + (m.x + 2 * t + 1) * PITCH<float, HD>)[m.y + g]);
    else
      f[i] = *reinterpret_cast<const float2*>(at + (m.x + g) * PITCH<float, HD> + 4 * (m.y + 2 * t));
  }
}
// ... and the other way.
template <typename T, int HD, bool VALUES> __device__ __forceinline__ void stage(uint8_t* at, int lane, int u, const float2 (&f)[4]) {
  if constexpr (sizeof(T) == 2) {
    const int2 m = matrix_at<HD, VALUES>(u, lane / 8);
    const uint32_t w[4] = {ptx::pack_bf16(f[0].x, f[0].y), ptx::pack_bf16(f[1].x, f[1].y), ptx::pack_bf16(f[2].x, f[2].y), ptx::pack_bf16(f[3].x, f[3].y)};
    store_matrices<VALUES>(smem_u32(at) + (m.x + lane % 8) * PITCH<T, HD> + 2 * m.y, w);
  } else {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int2 m = matrix_at<HD, VALUES>(u, i);
      if constexpr (VALUES) {
        reinterpret_cast<T*>(at + (m.x + 2 * t) * PITCH<T, HD>)[m.y + g] = f[i].x;
        reinterpret_cast<T*>(at + (m.x + 2 * t + 1) * PITCH<T, HD>)[m.y + g] = f[i].y;
      } else {
        *reinterpret_cast<float2*>(at + (m.x + g) * PITCH<T, HD> + 4 * (m.y + 2 * t)) = f[i];
      }
    }
  }
}

template <int HD> constexpr int UNITS = HD == 8 ? 1 : HD / 8;   // of eight bytes of a lane
template <int HD> __device__ __forceinline__ int unit_at(int lane, int u) { return HD == 8 ? 8 * lane : 512 * (u / 2) + 16 * lane + 8 * (u % 2); }

// x / s for pairs, to one of its two neighbours in float, the odd one unless it is exact.  The first quotient's remainder brings it to the nearest float (the
// quotient itself, where that is one); the second remainder, which is exact, brings that to the float next to zero, where nothing is left but to set the
// last bit if there was any remainder.
__device__ __forceinline__ float2 odd_quotients(float2 x, float s, float inv) {
  const float2 less = make_float2(-s, -s), by = make_float2(inv, inv);
  float2 t = __fmul2_rn(x, by);
  t = __ffma2_rn(__ffma2_rn(t, less, x), by, t);
  const float2 rest = __ffma2_rn(t, less, x);
  t = __ffma2_rz(rest, by, t);
  return make_float2(__int_as_float(__float_as_int(t.x) | (rest.x != 0.f)), __int_as_float(__float_as_int(t.y) | (rest.y != 0.f)));
}
// Four quotients (at most 127 or 448 and a little) rounded to bytes.  Integers: the last byte of 3 * 2^22 + the quotient.
template <int KIND> __device__ __forceinline__ uint32_t bytes4(float2 a, float2 b) {
  if constexpr (KIND == GSIT_CACHE_INT8) {
    const float2 big = make_float2(12582912.f, 12582912.f), x = __fadd2_rn(a, big), y = __fadd2_rn(b, big);
    return __byte_perm(__byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x0040), __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x0040), 0x5410);
  } else {
    uint32_t w;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}" : "=r"(w) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return w;
  }
}
template <int KIND> __device__ __forceinline__ void values4(uint32_t w, float2 (&f)[2]) {
  if constexpr (KIND == GSIT_CACHE_INT8) {
    f[0] = make_float2((float)(int8_t)w, (float)(int8_t)(w >> 8));
    f[1] = make_float2((float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24));
  } else {
    uint32_t h[2];
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(h[0]), "=r"(h[1]) : "r"(w));
#pragma unroll
    for (int i = 0; i < 2; ++i) f[i] = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
  }
}
// Largest magnitudes of pairs, and as an integer in the order of floats, NaN above them all.
__device__ __forceinline__ void raise(uint32_t& top, uint32_t w) {
  const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<__nv_bfloat162*>(&top), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w)));
  top = *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ void raise(float2& top, float2 v) {
  top = make_float2(__uint_as_float(max(__float_as_uint(top.x), __float_as_uint(v.x) & 0x7fffffffu)), __uint_as_float(max(__float_as_uint(top.y), __float_as_uint(v.y) & 0x7fffffffu)));
}
__device__ __forceinline__ uint32_t ordered(uint32_t w) { return max(w << 16, w & 0xffff0000u); }
__device__ __forceinline__ uint32_t ordered(float2 v) { return max(__float_as_uint(v.x), __float_as_uint(v.y)); }
__device__ __forceinline__ float2 as_floats(uint32_t w) {
  float2 v;
  unpack_bf16(w, v.x, v.y);
  return v;
}
__device__ __forceinline__ float2 as_floats(float2 v) { return v; }

// One staged matrix into a page's head.
template <typename T, int HD, int KIND, bool VALUES>
__device__ __forceinline__ void quantise(const uint8_t* at, int lane, uint8_t* bytes, float* scale) {
  constexpr int U = UNITS<HD>;
  using Pair = std::conditional_t<sizeof(T) == 2, uint32_t, float2>;
  Pair x[U][4], tops = {};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    staged<HD, VALUES>(at, lane, u, x[u]);
#pragma unroll
    for (int i = 0; i < 4; ++i) raise(tops, x[u][i]);
  }
  const uint32_t top = __reduce_max_sync(0xffffffffu, ordered(tops));
  const bool broken = top >= 0x7f800000u;
  const float s = broken ? 1.f : fmaxf(__fdiv_rn(__uint_as_float(top), KIND == GSIT_CACHE_INT8 ? 127.f : 448.f), LEAST_SCALE), inv = __frcp_rn(s);
  if (lane == 0) *scale = broken ? __int_as_float(0x7fffffff) : s;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t w[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) w[e] = bytes4<KIND>(odd_quotients(as_floats(x[u][2 * e]), s, inv), odd_quotients(as_floats(x[u][2 * e + 1]), s, inv));
    *reinterpret_cast<uint2*>(bytes + unit_at<HD>(lane, u)) = broken ? make_uint2(0u, 0u) : make_uint2(w[0], w[1]);
  }
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
  if (slots[len - 1] >= 0) return len;
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

template <typename T, int HD, int KIND>
__global__ void __launch_bounds__(THREADS, sizeof(T) == 2 ? 6 : 3) cache_append_kernel(const __grid_constant__ Geometry g, const __grid_constant__ RowArgs a) {
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
  const int slot0 = slots[0], held = held_rows(c, g.status, p.b, p.s);   // asked for together
  const int n = leading_rows(slots, g.len(p.s), lane);
  if (n == 0) return;
  if (slot0 < 0) {   // rows that have a slot come first: behind one that has none, no place can be told from the first one's
    raise_flag(g, GSIT_DEVFLAG_CLAMPED);
    return;
  }
  // the rows [i0, i1) of the segment lie in this block, from place `o` on
  const int place0 = slot0 % CACHE_BLOCK, i0 = max(0, p.chunk * CACHE_BLOCK - place0), i1 = min(n, (p.chunk + 1) * CACHE_BLOCK - place0);
  if (i0 >= i1) return;
  const int o = p.chunk == 0 ? place0 : 0, slot = slots[i0], page = slot < 0 ? -1 : real_page(c, slot / CACHE_BLOCK);
  if (page < 0) {
    raise_flag(g, GSIT_DEVFLAG_CLAMPED);
    return;
  }
  const int block = (held - n + i0) / CACHE_BLOCK;
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
  quantise<T, HD, KIND, false>(stage_k, lane, c.keys + to * (CACHE_BLOCK * HD), c.key_scale + to);
  quantise<T, HD, KIND, true>(stage_v, lane, c.values + to * (CACHE_BLOCK * HD), c.value_scale + to);
}

template <typename T, int HD, int KIND>
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
  // keys, then values, through one staged matrix: a warp that takes little shared memory has many beside it
  uint8_t* const staging = smem + warp * STAGE<T, HD>;
  auto spread = [&](const uint2& w, float s, float2 (&f)[4]) {
    float2 lo[2], hi[2];
    values4<KIND>(w.x, lo);
    values4<KIND>(w.y, hi);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f[i] = __fmul2_rn(lo[i], make_float2(s, s));
      f[2 + i] = __fmul2_rn(hi[i], make_float2(s, s));
    }
  };
  auto write = [&](T* to, int64_t ld) {
    __syncwarp();
    for (int i = lane; i < rows * VECS; i += 32) {
      const int row = i / VECS, at = i % VECS * (16 / (int)sizeof(T));
      *reinterpret_cast<uint4*>(to + row * ld + at) = *reinterpret_cast<const uint4*>(staging + row * PITCH<T, HD> + i % VECS * 16);
    }
    __syncwarp();
  };
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float2 f[4];
    spread(x[u], ks, f);
    stage<T, HD, false>(staging, lane, u, f);
  }
  write(k, a.ldk);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float2 f[4];
    spread(y[u], vs, f);
    stage<T, HD, true>(staging, lane, u, f);
  }
  write(v, a.ldv);
}

template <typename T, int HD, int KIND, bool APPEND> cudaError_t launch(const Geometry& g, const RowArgs& a, cudaStream_t st) {
  const auto kernel = APPEND ? cache_append_kernel<T, HD, KIND> : cache_read_kernel<T, HD, KIND>;
  constexpr int bytes = WARPS * (APPEND ? 2 : 1) * STAGE<T, HD>;
  const cudaError_t e = sm_count_and_smem_once(reinterpret_cast<const void*>(kernel), bytes, nullptr);
  if (e != cudaSuccess) return e;
  const int64_t items = (int64_t)g.batch * (a.chunks[0] + a.chunks[1] + a.chunks[2]) * a.c.kv_heads, grid = (items + WARPS - 1) / WARPS;
  if (grid > 0x7fffffff / WARPS) return cudaErrorNotSupported;
  return launch_overlapped(kernel, dim3((unsigned)grid), dim3(THREADS), bytes, st, g, a);
}
template <typename T, int KIND, bool APPEND> cudaError_t launch_width(const Geometry& g, const RowArgs& a, cudaStream_t st) {
  switch (a.c.hd) {
    case 8: return launch<T, 8, KIND, APPEND>(g, a, st);
    case 16: return launch<T, 16, KIND, APPEND>(g, a, st);
    case 32: return launch<T, 32, KIND, APPEND>(g, a, st);
    default: return launch<T, 64, KIND, APPEND>(g, a, st);
  }
}
template <bool APPEND> cudaError_t launch_any(const Geometry& g, int dtype, const RowArgs& a, cudaStream_t st) {
  if (a.c.kind == GSIT_CACHE_INT8)
    return dtype == GSIT_BF16 ? launch_width<__nv_bfloat16, GSIT_CACHE_INT8, APPEND>(g, a, st) : launch_width<float, GSIT_CACHE_INT8, APPEND>(g, a, st);
  return dtype == GSIT_BF16 ? launch_width<__nv_bfloat16, GSIT_CACHE_E4M3, APPEND>(g, a, st) : launch_width<float, GSIT_CACHE_E4M3, APPEND>(g, a, st);
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

// What the operators of gsit_ops.h share: row vectors of either type, geometry checks, launch entry points.
#pragma once
#include <math.h>

#include "common.cuh"
#include "ptx.cuh"

namespace gsit {

constexpr int MAX_ROTARY_PAIRS = 64;

// N elements of a row as floats: 16 bytes a load where N * sizeof(T) is 16 or more.
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void store_as(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_as(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }
template <int N> __device__ __forceinline__ void load_n(const float* p, float (&f)[N]) {
  if constexpr (N == 1) f[0] = *p;
  else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + i);
      f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
    }
  }
}
__device__ __forceinline__ void unpack_bf16(uint32_t w, float& lo, float& hi) {
  lo = __uint_as_float(w << 16);
  hi = __uint_as_float(w & 0xffff0000u);
}
template <int N> __device__ __forceinline__ void load_n(const __nv_bfloat16* p, float (&f)[N]) {
  if constexpr (N == 1) f[0] = __bfloat162float(*p);
  else if constexpr (N == 4) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    unpack_bf16(v.x, f[0], f[1]);
    unpack_bf16(v.y, f[2], f[3]);
  } else {
    static_assert(N == 8, "1, 4 or 8 elements");
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    unpack_bf16(v.x, f[0], f[1]);
    unpack_bf16(v.y, f[2], f[3]);
    unpack_bf16(v.z, f[4], f[5]);
    unpack_bf16(v.w, f[6], f[7]);
  }
}
template <int N> __device__ __forceinline__ void store_n(float* p, const float (&f)[N]) {
  if constexpr (N == 1) *p = f[0];
  else {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
  }
}
template <int N> __device__ __forceinline__ void store_n(__nv_bfloat16* p, const float (&f)[N]) {
  if constexpr (N == 1) *p = __float2bfloat16(f[0]);
  else if constexpr (N == 4) *reinterpret_cast<uint2*>(p) = make_uint2(ptx::pack_bf16(f[0], f[1]), ptx::pack_bf16(f[2], f[3]));
  else *reinterpret_cast<uint4*>(p) = make_uint4(ptx::pack_bf16(f[0], f[1]), ptx::pack_bf16(f[2], f[3]), ptx::pack_bf16(f[4], f[5]), ptx::pack_bf16(f[6], f[7]));
}

// Address of the current device's status word; the checks of a shape that all calls share (gsit_api.cu).
cudaError_t device_status_word(unsigned int** p);
gsit_status basic_geometry(const gsit_shape* s, Geometry* g);

// rotary.cu
struct RotaryCall {
  const void* in[2];
  void* out[2];
  int64_t in_stride[2], out_stride[2];   // elements between rows
  int heads[2];                          // of q and of k (0: no k)
  const int32_t* positions;
  int64_t axis_stride, batch_stride;
  int sections[3];
  bool interleaved, backward;
  double base;
};
cudaError_t launch_rotary(const Geometry& g, int dtype, const RotaryCall& c, cudaStream_t st);
// Frequencies of the pairs, base^(-p / pairs), in turns a position.  They are products of those of p's powers of two (six doubles at most):
// 32 calls of pow are a fifth of a small call.
inline void rotary_turns(double base, int pairs, double (&turns)[MAX_ROTARY_PAIRS]) {
  double power[MAX_ROTARY_PAIRS];
  for (int p = 0; p < pairs; ++p) {
    power[p] = (p & (p - 1)) != 0 ? power[p & (p - 1)] * power[p & -p] : pow(base, -(double)p / pairs);
    turns[p] = power[p] / (2.0 * M_PI);
  }
}

// head_norm.cu
constexpr int MAX_NORM_HEAD = 256;
struct HeadNormCall {
  const void *x[2], *dy[2];              // q and k; backward: gradients of the results
  void* out[2];
  int64_t ldx[2], lddy[2], ldo[2];       // elements between rows
  const float* gamma[2];
  int heads[2];                          // (0: no k)
  const int32_t* positions;
  int64_t axis_stride, batch_stride;
  int sections[3];                       // all 0: no rotation
  bool interleaved, backward;
  double base;
  float eps;
  float *dgamma[2], *partial;            // partial null: gradients of the rows alone
};
cudaError_t launch_head_norm(const Geometry& g, int dtype, const HeadNormCall& c, cudaStream_t st);
size_t head_norm_scratch(const Geometry& g);

// layer_norm.cu
constexpr int MAX_NORM_WIDTH = 8192;
struct NormCall {
  const void* x; int64_t ldx; int x_dtype;
  const float *gamma, *beta;
  float eps;
  void* y; int64_t ldy; int y_dtype;              // forward: written
  float *mean, *rstd;                             // forward: written (may be null)
  const void* dy; int64_t lddy;                   // backward (y_dtype)
  const void* residual; int64_t ldres;
  void* dx; int64_t lddx;
  float *dgamma, *dbeta, *partial;
};
cudaError_t launch_layer_norm_fwd(const Geometry& g, const NormCall& c, cudaStream_t st);
cudaError_t launch_layer_norm_bwd(const Geometry& g, const NormCall& c, cudaStream_t st);
size_t layer_norm_bwd_scratch(const Geometry& g);

}  // namespace gsit

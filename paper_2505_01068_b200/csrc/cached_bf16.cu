// Attention over a stream's cache, bf16 rows (see cached_attn.cuh).
#include "cached_attn.cuh"

namespace gsit {
cudaError_t launch_cached_bf16(const Geometry& g, CachedArgs& a, cudaStream_t st, size_t* scratch) { return launch_kind<__nv_bfloat16>(g, a, st, scratch); }
}  // namespace gsit

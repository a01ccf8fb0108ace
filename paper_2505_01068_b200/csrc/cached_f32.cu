// Attention over a stream's cache, float rows (see cached_attn.cuh).
#include "cached_attn.cuh"

namespace gsit {
cudaError_t launch_cached_f32(const Geometry& g, CachedArgs& a, cudaStream_t st, size_t* scratch) { return launch_kind<float>(g, a, st, scratch); }
}  // namespace gsit

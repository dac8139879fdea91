// kernels_cached_f32.hip -- attention over a cache of pages for queries in fp32, the cache in fp32 or in 8 bits.
#include "seq/attn_cached.hpp"

namespace ntk {

hipError_t launch_attn_cached_f32(hipStream_t s, const CachedArgs& a, bool e4m3, int waves, bool vec) {
  return run_cached_type<float>(s, a, e4m3, waves, vec);
}

}  // namespace ntk

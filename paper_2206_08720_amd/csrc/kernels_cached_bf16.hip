// kernels_cached_bf16.hip -- attention over a cache of pages for queries in bf16, the cache in bf16 or in 8 bits.
#include "seq/attn_cached.hpp"

namespace ntk {

hipError_t launch_attn_cached_bf16(hipStream_t s, const CachedArgs& a, bool e4m3, int waves, bool vec) {
  return run_cached_type<__bf16>(s, a, e4m3, waves, vec);
}

}  // namespace ntk

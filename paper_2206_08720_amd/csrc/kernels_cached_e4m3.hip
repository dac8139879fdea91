// kernels_cached_e4m3.hip -- attention over a cache of pages in 8 bits.
#include "seq/attn_cached.hpp"

namespace ntk {

hipError_t launch_attn_cached_e4m3(hipStream_t s, int dtype, const CachedArgs& a, bool tokens, bool vec) {
  return run_cached_type<true>(s, dtype, a, tokens, vec);
}

}  // namespace ntk

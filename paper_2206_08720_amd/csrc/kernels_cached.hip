// kernels_cached.hip -- attention over a cache of pages in the queries' type, and how a call over either cache runs.
#include "seq/attn_cached.hpp"

namespace ntk {

AttnPlan attn_plan_cached(int dtype, bool e4m3, int B, int Hk, int R, int places, int D) {
  (void)e4m3;
  return attn_plan_fwd(dtype, B, Hk, R, places, D);
}

hipError_t launch_attn_cached(hipStream_t s, int dtype, const CachedArgs& a, bool tokens, bool vec) {
  return run_cached_type<false>(s, dtype, a, tokens, vec);
}

}  // namespace ntk

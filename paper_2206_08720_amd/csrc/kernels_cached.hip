// kernels_cached.hip -- attention over a cache of pages in the queries' type, and how a call over either cache runs.
#include "seq/attn_cached.hpp"

namespace ntk {

CachedPlan attn_plan_cached(int dtype, bool e4m3, int B, int Hk, int R, int places, int D) {
  CachedPlan p;
  const int dp = D <= 64 ? 64 : 128, size = dtype == 0 ? 4 : 2, cell = e4m3 ? 1 : size;
  p.tokens = R <= 32;
  p.tiles = p.tokens ? 1 : (R + kFwdRows - 1) / kFwdRows;
  p.blocks = (long long)B * Hk * p.tiles;
  const int rows = p.tokens ? 32 : kFwdRows, keys = p.tokens ? kCachedKeys : size == 2 ? 64 : 32;
  const long long most = ((long long)places + keys - 1) / keys;   // tiles of keys that a row tile can see
  // Workgroups that run at once: two a compute unit, one where registers or LDS leave room for one.
  const bool two = p.tokens ? dp == 64 || (e4m3 && size == 2) : size * dp <= 256;
  const int slots = two ? 512 : 256;
  // Tokens: 64 KB of keys a workgroup at least.  Many rows: 256 keys, 64 in fp32, whose products take several times as long.
  p.least = p.tokens ? std::max(4, 65536 / (keys * dp * cell)) : size == 2 ? 4 : 2;
  p.workers = most < 2 * p.least || p.blocks >= 8 * slots ? 0 : (int)std::min<long long>(slots, (p.blocks * most + p.least - 1) / p.least);
  if (p.workers >= 8) p.workers &= ~7;                            // an eighth for each die
  p.part_floats = (long long)p.workers * 2 * rows * (dp + 2);
  p.ints = 4LL * p.workers + (p.tokens ? 0 : p.workers ? p.workers : p.blocks);
  return p;
}

hipError_t launch_attn_cached(hipStream_t s, int dtype, const CachedArgs& a, bool tokens, bool vec) {
  return run_cached_type<false>(s, dtype, a, tokens, vec);
}

}  // namespace ntk

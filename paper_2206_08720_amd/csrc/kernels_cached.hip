// kernels_cached.hip -- how a call of attention over a cache of pages runs.
#include "seq/attn_cached.hpp"

namespace ntk {

CachedPlan attn_plan_cached(int dtype, bool e4m3, int B, int Hk, int R, int places, int D) {
  CachedPlan p;
  const int dp = D <= 64 ? 64 : 128, size = dtype == 0 ? 4 : 2, cell = e4m3 ? 1 : size;
  // eight waves: parts of 1200 queries over 14 and 2 thousand places in 8 bits 370 us, with four 399
  p.waves = R <= 32 ? 0 : R > kFwdRows && cached_wide(size, e4m3) ? 8 : 4;
  const int rows = std::max(32, 32 * p.waves);
  p.tiles = (R + rows - 1) / rows;
  p.blocks = (long long)B * Hk * p.tiles;
  const int keys = p.waves == 0 ? kCachedKeys : size == 2 ? 64 : 32;
  const long long most = ((long long)places + keys - 1) / keys;   // tiles of keys that a row tile can see
  // Workgroups that run at once: two a compute unit, one where registers or LDS leave room for one.  Tokens: two where a workgroup's
  // tiles (kCachedBytes) take 64 KB, not 128.  (With two counted where one fits, runs go in two rounds: fp32, heads of 64, one sequence of
  // 131 thousand places 91 us, counted right 63; 32 of six thousand 194 and 164; 350 of 1600 662 and 557.)
  const bool two = p.waves == 0 ? size * dp <= (e4m3 ? 256 : 128) : p.waves == 4 && size * dp <= 256;
  const int slots = two ? 512 : 256;
  // Tokens: 64 KB of keys a workgroup at least (four sequences of 1500 places, 8 heads of 128 in bf16: 31 us, with 128 KB 36, with 32 KB
  // 32; in fp32 40, 48 and 40).  Many rows: 256 keys, 64 in fp32, whose products take several times as long (3 by 380 queries at the end of
  // 2100 places, fp16, 12 heads of 80: 50 us, with 512 keys 53, with 128 50; a workgroup a row tile 91.  fp32, up to 40 queries at the end
  // of up to 400, 4 sequences of 8 heads of 64: 24 us, with 128 keys 27; one of 8 heads of 128: 29 and 36; 64 at the end of 4000, 8 heads of
  // 64: 40 and 35, with 32 keys 41, with 256 43).
  p.least = p.waves == 0 ? std::max(4, 65536 / (keys * dp * cell)) : size == 2 ? 4 : 2;
  // A workgroup a row tile where parts would be short, or row tiles are enough to even out.  Parts are counted in 32 bits.
  const bool whole = most < 2 * p.least || p.blocks >= 8 * slots || p.blocks * most >= (1LL << 30);
  p.workers = whole ? 0 : (int)std::min<long long>(slots, (p.blocks * most + p.least - 1) / p.least);
  if (p.workers >= 8) p.workers &= ~7;                            // an eighth for each die
  p.part_floats = (long long)p.workers * 2 * rows * (dp + 2);
  p.ints = 4LL * p.workers + (p.waves == 0 ? 0 : p.workers ? p.workers : p.blocks);
  return p;
}

hipError_t launch_attn_cached(hipStream_t s, int dtype, const CachedArgs& a, bool e4m3, int waves, bool vec) {
  if (dtype == 1) return launch_attn_cached_bf16(s, a, e4m3, waves, vec);
  if (dtype == 2) return launch_attn_cached_f16(s, a, e4m3, waves, vec);
  return launch_attn_cached_f32(s, a, e4m3, waves, vec);
}

}  // namespace ntk

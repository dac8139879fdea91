// launch_cache.hpp -- host-side launchers of the paged cache's kernels and of the token probabilities (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../index_math.hpp"
#include "launch_attn.hpp"
#include "paging.hpp"

namespace ntk {

// Keys and values of new tokens into a cache; types by number: 0 fp32, 1 bf16, 2 fp16.  `vec`: every operand's rows take
// 16-byte accesses, dim is a multiple of 8 and rot of 16.
struct AppendArgs {
  const void* x[3];                        // q, k, v [batch, length, heads, dim]; no q: heads = 0
  long long xb[3], xs[3], xh[3];
  void* qo;                                // like q
  long long qb, qs, qh;
  void* cell[2];                           // k, v [page, slot, head, dim]
  long long cb[2], cs[2], ch[2];
  float* scale[2];                         // [pages, kv_heads], with quantize
  int quantize;                            // the cache is e4m3, else of the arrays' type
  PageTable pages;
  const int *lens, *news, *positions;      // news, positions may be null
  const float* table;                      // [max_pos][rot / 2][2]: cos, sin; rot = 0: nothing turns
  int max_pos, rot, interleaved;
  int batch, length, heads, kv_heads, dim;
};
long long append_blocks(const AppendArgs& a);   // workgroups, of 256 threads
hipError_t launch_append(hipStream_t s, int dtype, const AppendArgs& a, bool vec);

// Attention over a cache (kernels_cached.hip, the kernels in a file for each type).
struct CachedArgs;
// `waves` of 32 rows a workgroup, 0: the few-row kernel; `tiles` row tiles a key/value head; the tiles of keys are dealt out to
// `workers` workgroups, each at least `least` of them (0: a workgroup a row tile, `blocks` in all).  Workspace: part_floats, then 4 ints
// a worker, then a flag a workgroup.
struct CachedPlan {
  int waves, tiles, workers, least;
  long long blocks, part_floats, ints;
};
// whether there is a form of eight waves: what a tile of 8 bits takes to convert is then shared by 256 rows
constexpr bool cached_wide(int type_bytes, bool e4m3) { return e4m3 && type_bytes == 2; }
CachedPlan attn_plan_cached(int dtype, bool e4m3, int B, int Hk, int R, int places, int D);
hipError_t launch_attn_cached(hipStream_t s, int dtype, const CachedArgs& a, bool e4m3, int waves, bool vec);
hipError_t launch_attn_cached_bf16(hipStream_t s, const CachedArgs& a, bool e4m3, int waves, bool vec);   // one file each
hipError_t launch_attn_cached_f16(hipStream_t s, const CachedArgs& a, bool e4m3, int waves, bool vec);
hipError_t launch_attn_cached_f32(hipStream_t s, const CachedArgs& a, bool e4m3, int waves, bool vec);

// Log probabilities of given tokens (kernels_logprob.hip).
struct LogprobArgs {
  const void* logits;
  long long stride;                        // elements between rows
  const int* tokens;
  float *logp, *entropy, *lse, *top_logp;
  int* top_tokens;
  void* work;                              // logprob_work_bytes
  long long rows;
  int vocab, top, splits;
  float scale;
};
struct LogprobBwdArgs {
  const void* logits;
  void* dlogits;
  long long stride, dstride;
  const int* tokens;
  const float *lse, *entropy, *dlogp, *dentropy;   // the last two may be null
  long long rows;
  int vocab, chunks;
  float scale;
};
int logprob_splits(int dtype, long long rows, int vocab);
long long logprob_work_bytes(long long rows, int top, int splits);
int logprob_bwd_chunks(int dtype, int vocab);
hipError_t launch_logprobs(hipStream_t s, int dtype, const LogprobArgs& a);
hipError_t launch_logprobs_bwd(hipStream_t s, int dtype, const LogprobBwdArgs& a);

}  // namespace ntk

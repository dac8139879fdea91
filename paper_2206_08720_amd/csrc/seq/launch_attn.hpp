// launch_attn.hpp -- host-side launchers of the attention kernels (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

namespace ntk {

struct AttnArgs;

// How a forward call runs: `tokens` the few-row kernel; `tiles` row tiles a key/value head; `splits` ranges
// that the keys are cut into, whose results (part_floats) are joined; flag_ints a flag a
// workgroup, behind them in the workspace.
struct AttnPlan {
  bool tokens;
  int tiles, splits;
  long long part_floats, flag_ints;
};
AttnPlan attn_plan_fwd(int dtype, int B, int Hk, int R, int Sk, int D);
// dtype: 0 fp32, 1 bf16, 2 fp16; vec: every operand's rows take 16-byte loads.
hipError_t launch_attn_fwd(hipStream_t s, int dtype, const AttnArgs& a, bool tokens, bool vec);

// The backward pass: tiles of the rows (dq) and of the keys (dk, dv) a key/value head, the ranges that the other axis
// is cut into, and the floats of their partial sums.
struct AttnBwdPlan {
  int dq_tiles, dq_splits, dkv_tiles, dkv_splits;
  long long part_floats, flag_ints;
};
AttnBwdPlan attn_plan_bwd(int dtype, int B, int Hk, int R, int Sk, int D, bool causal);
// delta[b, h, i] = sum_d dout o, then dq, dk and dv.  work: part_floats, then 2 * batch * heads * q_len floats, then flag_ints.
hipError_t launch_attn_bwd(hipStream_t s, int dtype, AttnArgs& a, const AttnBwdPlan& plan, float* work, bool vec);

}  // namespace ntk

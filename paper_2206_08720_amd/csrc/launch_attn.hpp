// launch_attn.hpp -- host-side launchers of the attention kernels (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

namespace ntk {

struct AttnArgs;

// How a forward call runs: `tokens` the few-row kernel; `tiles` row tiles a key/value head; `splits` ranges
// that the keys are cut into, whose results (part_floats) are joined.
struct AttnPlan {
  bool tokens;
  int tiles, splits;
  long long part_floats;
};
AttnPlan attn_plan_fwd(int B, int Hk, int R, int Sk, int D);
// dtype: 0 fp32, 1 bf16, 2 fp16; vec: every operand's rows take 16-byte loads.
hipError_t launch_attn_fwd(hipStream_t s, int dtype, const AttnArgs& a, bool tokens, bool vec);

// delta[b, h, i] = sum_d dout o, then dq, dk and dv.
hipError_t launch_attn_bwd(hipStream_t s, int dtype, AttnArgs& a, float* delta, bool vec);

}  // namespace ntk

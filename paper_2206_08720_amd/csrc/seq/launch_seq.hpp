// launch_seq.hpp -- host-side launchers of the norm and the rotary kernels (internal to the library).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../index_math.hpp"

namespace ntk {

// Types by number: 0 fp32, 1 bf16, 2 fp16.  `vec`: rows and pointers take 16-byte accesses and the width is a
// multiple of 8.
struct NormArgs {
  const void *x, *residual, *weight;   // residual may be null
  long long x_stride, residual_stride; // elements between rows
  void *y, *h;                         // contiguous; h may be null
  float* scale;                        // not null: y is e4m3 under one scale a row
  long long rows;
  int width;
  float eps;
};
struct NormBwdArgs {
  const void *dy, *h, *dh, *weight;    // dh may be null
  long long dy_stride, h_stride, dh_stride;
  void *dx, *dw;
  float* part;                         // [norm_bwd_parts][width]
  long long rows;
  int width;
  float eps;
};
int norm_threads(int width);         // a workgroup's, and the rows it takes
int norm_rows_per_block(int width);
int norm_bwd_parts(long long rows, int width);
hipError_t launch_rms_norm(hipStream_t s, int dtype, int wtype, const NormArgs& a, bool vec);
hipError_t launch_rms_norm_bwd(hipStream_t s, int dtype, int wtype, const NormBwdArgs& a, bool vec);

// Rotation of the first `rot` elements of every head of up to two arrays [batch, length, heads[k], dim].
struct RotaryArgs {
  const void* x[2];
  void* y[2];
  long long xb[2], xs[2], xh[2], yb[2], ys[2], yh[2];
  int heads[2];
  const float* table;                  // [max_pos][rot / 2][2]: cos, sin
  const int* positions;                // [batch, length], or null: first + index
  int first, max_pos;
  int batch, length, dim, rot, interleaved;
  float sign;                          // 1, or -1 for the inverse
};
long long rotary_blocks(const RotaryArgs& a);   // workgroups, of 256 threads
hipError_t launch_rotary(hipStream_t s, int dtype, const RotaryArgs& a, bool vec);

// table[p][j] = mag (cos, sin)(p f_j); see ntk_rotary_table.
struct RotaryTableArgs {
  float* table;
  int max_pos, rot, scaling;
  double base, factor, original, lo, hi;
};
hipError_t launch_rotary_table(hipStream_t s, const RotaryTableArgs& a);

}  // namespace ntk

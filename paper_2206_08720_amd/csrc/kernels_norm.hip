// kernels_norm.hip -- root-mean-square norm with the residual's addition, its 8-bit output and its gradient.
//
//   h = x + residual,  r = (mean h^2 + eps)^(-1/2),  y = h r w;   8 bits: s = max|y| / 448, q = e4m3(y / s)
//   g = dy w,  dx = r (g - h r^2 mean(g h)) + dh,  dw = sum_rows dy h r
//
// A row is held in registers between its two uses, so every array moves once; only the backward kernels of more than 16384
// columns spill (93 to 150 registers).  Sums are fp32; y follows from the unrounded h, and the gradient from the h that
// was stored, which is all that the backward pass is given: in bf16 its dw is then 1.3 to 1.5 times as far off as from the
// unrounded h.  A row takes 64, 256 or 1024 threads, each with CH groups of 8 elements: short rows share a workgroup, long ones
// fill one (rows of 64 columns leave 56 of a wave's lanes idle, of 128 48: 262144 rows of 128 take 78 us, 3.4 TB/s).  Bound by
// memory: 16384 rows of 4096 in bf16 take 100 us forward (5.4 TB/s; a large copy reaches 4.7), 8192 rows of 2048 30 us backward
// with 5 for the columns' sums, 2048 rows of 32768 323 us, whose spills show.
#include <hip/hip_runtime.h>

#include "seq/launch_seq.hpp"

namespace ntk {
namespace {

constexpr int kE = 8;                       // elements a thread takes at once
constexpr int kBlock = 256;
constexpr float kMostE4m3 = 448.f;

template <class T>
struct Pack8 {
  T v[kE];
};

// The 8 elements of group `c` of thread t: neighbours (VEC), or one from each of 8 runs of TPR, so that the threads of
// a row read neighbours.  Those past n are zero.
template <class T, bool VEC, int TPR>
__device__ __forceinline__ void load8(const T* __restrict__ row, int c, int t, int n, float (&f)[kE]) {
  const int at = VEC ? (c * TPR + t) * kE : c * TPR * kE + t;
  if constexpr (VEC) {
    if (at < n) {
      alignas(16) Pack8<T> p;
      uint4* u = reinterpret_cast<uint4*>(&p);
#pragma unroll
      for (int i = 0; i < (int)sizeof(p) / 16; ++i) u[i] = reinterpret_cast<const uint4*>(row + at)[i];
#pragma unroll
      for (int i = 0; i < kE; ++i) f[i] = (float)p.v[i];
      return;
    }
#pragma unroll
    for (int i = 0; i < kE; ++i) f[i] = 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i) f[i] = at + i * TPR < n ? (float)row[at + i * TPR] : 0.f;
  }
}

template <class T, bool VEC, int TPR>
__device__ __forceinline__ void store8(T* __restrict__ row, int c, int t, int n, const float (&f)[kE]) {
  const int at = VEC ? (c * TPR + t) * kE : c * TPR * kE + t;
  if constexpr (VEC) {
    if (at >= n) return;
    alignas(16) Pack8<T> p;
#pragma unroll
    for (int i = 0; i < kE; ++i) p.v[i] = (T)f[i];
    const uint4* u = reinterpret_cast<const uint4*>(&p);
#pragma unroll
    for (int i = 0; i < (int)sizeof(p) / 16; ++i) reinterpret_cast<uint4*>(row + at)[i] = u[i];
  } else {
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if (at + i * TPR < n) row[at + i * TPR] = (T)f[i];
  }
}

// sum (or maximum) over the TPR threads of a row; every thread gets it
template <int TPR, bool MAX>
__device__ __forceinline__ float row_all(float x, float* s) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const float y = __shfl_xor(x, o);
    x = MAX ? fmaxf(x, y) : x + y;
  }
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) s[wave] = x;
    __syncthreads();
    x = s[0];
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w) x = MAX ? fmaxf(x, s[w]) : x + s[w];
    __syncthreads();
  }
  return x;
}

template <int CH>
__device__ __forceinline__ float squares(const float (&h)[CH][kE]) {
  float ss = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < kE; ++i) ss = fmaf(h[c][i], h[c][i], ss);
  return ss;
}

// A row's sum of squares leaves fp32's range where h passes 2^63 or, with an eps that does not cover it, stays below 2^-40.
// Such a row is multiplied by the power of two that this returns (1 for the others), and its sum formed again:
// r of the row as it was is that power times (ss / n + eps power^2)^(-1/2).
__device__ __forceinline__ float row_power(float ss, float eps) {
  if (!(ss <= 0x1p126f)) return 0x1p-80f;
  return ss < 0x1p-80f && eps < 0x1p-100f ? 0x1p100f : 1.f;
}
template <int CH>
__device__ __forceinline__ void scale_row(float (&h)[CH][kE], float f) {
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < kE; ++i) h[c][i] *= f;
}
__device__ __forceinline__ float inverse_norm(float ss, int n, float eps, float power) {
  return 1.f / sqrtf(ss / (float)n + eps * power * power);
}

template <class T, class W, int TPR, int CH, bool VEC>
__global__ void __launch_bounds__(TPR < kBlock ? kBlock : TPR) k_rms_norm(const NormArgs a) {
  constexpr int RPB = TPR < kBlock ? kBlock / TPR : 1;
  __shared__ float s[16];
  const int t = threadIdx.x % TPR;
  const long long row = (long long)blockIdx.x * RPB + threadIdx.x / TPR;
  if (row >= a.rows) return;                // whole waves: with TPR > 64 the grid is exact
  const T* x = (const T*)a.x + row * a.x_stride;
  const T* res = a.residual ? (const T*)a.residual + row * a.residual_stride : nullptr;
  const int n = a.width;
  float h[CH][kE], w[CH][kE];
#pragma unroll
  for (int c = 0; c < CH; ++c) load8<T, VEC, TPR>(x, c, t, n, h[c]);
  if (res) {
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float e[kE];
      load8<T, VEC, TPR>(res, c, t, n, e);
#pragma unroll
      for (int i = 0; i < kE; ++i) h[c][i] += e[i];
    }
  }
#pragma unroll
  for (int c = 0; c < CH; ++c) load8<W, VEC, TPR>((const W*)a.weight, c, t, n, w[c]);
  float ss = row_all<TPR, false>(squares<CH>(h), s);
  if (a.h) {
#pragma unroll
    for (int c = 0; c < CH; ++c) store8<T, VEC, TPR>((T*)a.h + row * n, c, t, n, h[c]);
  }
  const float power = row_power(ss, a.eps);
  if (power != 1.f) {
    scale_row<CH>(h, power);
    ss = row_all<TPR, false>(squares<CH>(h), s);
  }
  const float r = inverse_norm(ss, n, a.eps, power);
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < kE; ++i) h[c][i] = h[c][i] * r * w[c][i];
  if (!a.scale) {
#pragma unroll
    for (int c = 0; c < CH; ++c) store8<T, VEC, TPR>((T*)a.y + row * n, c, t, n, h[c]);
    return;
  }
  float most = 0.f;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int i = 0; i < kE; ++i) most = fmaxf(most, fabsf(h[c][i]));
  most = row_all<TPR, true>(most, s);
  const float scale = most > 0.f ? fmaxf(most / kMostE4m3, 0x1p-126f) : 1.f;   // its inverse stays finite
  if (t == 0) a.scale[row] = scale;
  const float inv = 1.f / scale;
  unsigned char* q = (unsigned char*)a.y + row * n;
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    unsigned u[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      // the product with 1 / scale may round past 448, where the conversion has no finite value
      float e[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float z = h[c][4 * k + i] * inv;
        e[i] = z != z ? z : fminf(fmaxf(z, -kMostE4m3), kMostE4m3);
      }
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(e[0], e[1], 0, false);
      u[k] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(e[2], e[3], p, true);
    }
    const int at = VEC ? (c * TPR + t) * kE : c * TPR * kE + t;
    if constexpr (VEC) {
      if (at < n) *reinterpret_cast<uint2*>(q + at) = make_uint2(u[0], u[1]);
    } else {
#pragma unroll
      for (int i = 0; i < kE; ++i)
        if (at + i * TPR < n) q[at + i * TPR] = (unsigned char)(u[i >> 2] >> (8 * (i & 3)));
    }
  }
}

// Workgroup g takes the rows g, g + G, ... (times RPB): dw is summed over them in registers and written as one
// partial row a workgroup, which k_norm_columns adds in order.
template <class T, class W, int TPR, int CH, bool VEC>
__global__ void __launch_bounds__(TPR < kBlock ? kBlock : TPR) k_rms_norm_bwd(const NormBwdArgs a) {
  constexpr int RPB = TPR < kBlock ? kBlock / TPR : 1;
  __shared__ float s[16];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const int n = a.width;
  float w[CH][kE], dw[CH][kE];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
    load8<W, VEC, TPR>((const W*)a.weight, c, t, n, w[c]);
#pragma unroll
    for (int i = 0; i < kE; ++i) dw[c][i] = 0.f;
  }
  for (long long row = (long long)blockIdx.x * RPB + sub; row < a.rows; row += (long long)gridDim.x * RPB) {
    float h[CH][kE], g[CH][kE];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      load8<T, VEC, TPR>((const T*)a.h + row * a.h_stride, c, t, n, h[c]);
      load8<T, VEC, TPR>((const T*)a.dy + row * a.dy_stride, c, t, n, g[c]);
    }
    auto sums = [&](float& ss, float& sg) {
      ss = sg = 0.f;
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < kE; ++i) {
          ss = fmaf(h[c][i], h[c][i], ss);
          sg = fmaf(g[c][i] * w[c][i], h[c][i], sg);
        }
      ss = row_all<TPR, false>(ss, s);
      sg = row_all<TPR, false>(sg, s);
    };
    float ss, sg;
    sums(ss, sg);
    const float power = row_power(ss, a.eps);
    if (power != 1.f) {
      scale_row<CH>(h, power);
      sums(ss, sg);
    }
    const float r = inverse_norm(ss, n, a.eps, power);
    const float f = r * r * (sg / (float)n), rp = r * power;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      float e[kE];
      if (a.dh) {
        load8<T, VEC, TPR>((const T*)a.dh + row * a.dh_stride, c, t, n, e);
      } else {
#pragma unroll
        for (int i = 0; i < kE; ++i) e[i] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < kE; ++i) {
        dw[c][i] = fmaf(g[c][i], h[c][i] * r, dw[c][i]);
        e[i] += rp * (g[c][i] * w[c][i] - h[c][i] * f);
      }
      store8<T, VEC, TPR>((T*)a.dx + row * n, c, t, n, e);
    }
  }
  float* part = a.part + ((long long)blockIdx.x * RPB + sub) * n;
#pragma unroll
  for (int c = 0; c < CH; ++c) store8<float, VEC, TPR>(part, c, t, n, dw[c]);
}

// dw[c] = sum_p part[p][c], in a fixed order: 16 columns a workgroup, 64 threads a column, eight loads in flight each.
template <class W>
__global__ void __launch_bounds__(1024) k_norm_columns(const float* __restrict__ part, int parts, int n, W* __restrict__ dw) {
  __shared__ float s[64][17];
  const int c = threadIdx.x & 15, q = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float x = 0.f;
  for (int p0 = q; p0 < parts; p0 += 64 * 8) {
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = col < n && p0 + 64 * u < parts ? part[(long long)(p0 + 64 * u) * n + col] : 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) x += v[u];
  }
  s[q][c] = x;
  __syncthreads();
  if (q) return;
#pragma unroll
  for (int k = 1; k < 64; ++k) x += s[k][c];
  if (col < n) dw[col] = (W)x;
}

// Threads a row and groups a thread.  Up to 1024 columns a wave holds the row: no barrier, four rows a workgroup.
struct Shape {
  int tpr, ch;
};
Shape shape_of(int n) {
  if (n <= 512) return {64, 1};
  if (n <= 1024) return {64, 2};
  if (n <= 2048) return {256, 1};
  if (n <= 4096) return {256, 2};
  if (n <= 8192) return {256, 4};
  if (n <= 16384) return {1024, 2};
  return {1024, 4};
}

template <class T, class W, int TPR, int CH>
hipError_t run(hipStream_t s, const NormArgs* f, const NormBwdArgs* b, bool vec) {
  constexpr int threads = TPR < kBlock ? kBlock : TPR, rpb = TPR < kBlock ? kBlock / TPR : 1;
  if (f) {
    const dim3 grid((unsigned)((f->rows + rpb - 1) / rpb));
    if (vec)
      k_rms_norm<T, W, TPR, CH, true><<<grid, threads, 0, s>>>(*f);
    else
      k_rms_norm<T, W, TPR, CH, false><<<grid, threads, 0, s>>>(*f);
    return hipGetLastError();
  }
  const int parts = norm_bwd_parts(b->rows, b->width);
  const dim3 grid((unsigned)(parts / rpb));
  if (parts && vec)
    k_rms_norm_bwd<T, W, TPR, CH, true><<<grid, threads, 0, s>>>(*b);
  else if (parts)   // no rows: dw is zero
    k_rms_norm_bwd<T, W, TPR, CH, false><<<grid, threads, 0, s>>>(*b);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_norm_columns<W><<<dim3((unsigned)((b->width + 15) / 16)), dim3(1024), 0, s>>>(b->part, parts, b->width, (W*)b->dw);
  return hipGetLastError();
}

template <class T, class W>
hipError_t pick(hipStream_t s, const NormArgs* f, const NormBwdArgs* b, bool vec) {
  const Shape h = shape_of(f ? f->width : b->width);
  if (h.tpr == 64) return h.ch == 1 ? run<T, W, 64, 1>(s, f, b, vec) : run<T, W, 64, 2>(s, f, b, vec);
  if (h.tpr == 256)
    return h.ch == 1 ? run<T, W, 256, 1>(s, f, b, vec) : h.ch == 2 ? run<T, W, 256, 2>(s, f, b, vec) : run<T, W, 256, 4>(s, f, b, vec);
  return h.ch == 2 ? run<T, W, 1024, 2>(s, f, b, vec) : run<T, W, 1024, 4>(s, f, b, vec);
}

hipError_t by_type(hipStream_t s, int dtype, int wtype, const NormArgs* f, const NormBwdArgs* b, bool vec) {
  if (dtype == 1) return wtype == 0 ? pick<__bf16, float>(s, f, b, vec) : pick<__bf16, __bf16>(s, f, b, vec);
  if (dtype == 2) return wtype == 0 ? pick<_Float16, float>(s, f, b, vec) : pick<_Float16, _Float16>(s, f, b, vec);
  return pick<float, float>(s, f, b, vec);
}

}  // namespace

int norm_threads(int width) { return std::max(shape_of(width).tpr, kBlock); }
int norm_rows_per_block(int width) { return norm_threads(width) / shape_of(width).tpr; }

int norm_bwd_parts(long long rows, int width) {
  const Shape h = shape_of(width);
  const int rpb = norm_rows_per_block(width);
  const long long groups = (rows + rpb - 1) / rpb;
  const long long most = h.tpr == 1024 ? 256 : 1024;    // workgroups: four (one of 1024 threads) a compute unit
  return (int)(groups < most ? groups : most) * rpb;
}

hipError_t launch_rms_norm(hipStream_t s, int dtype, int wtype, const NormArgs& a, bool vec) {
  return by_type(s, dtype, wtype, &a, nullptr, vec);
}
hipError_t launch_rms_norm_bwd(hipStream_t s, int dtype, int wtype, const NormBwdArgs& a, bool vec) {
  return by_type(s, dtype, wtype, nullptr, &a, vec);
}

}  // namespace ntk

// kernels_rotary.hip -- rotary positions: the pair (u, v) of a head at position p turns to
// (u c - v s, v c + u s) with (c, s) = table[p][pair].  Pairs are (x[j], x[j + rot / 2]) or, interleaved,
// (x[2 j], x[2 j + 1]); elements past `rot` are copied.  The inverse (the gradient) turns by -s.
//
// Bound by moving the heads once.  A thread takes 8 pairs (16 elements) of one head; the workgroup's rows are
// neighbours, so the table's lines are read from memory once and from the L1 by the other heads.  2 x 8192 positions
// of 32 + 8 heads of 128 in bf16: 68 us, 5.0 TB/s.
#include <hip/hip_runtime.h>

#include "seq/launch_seq.hpp"

namespace ntk {
namespace {

constexpr int kPairs = 8;

template <class T, int N>
__device__ __forceinline__ void load_n(const T* p, float (&f)[N]) {
  alignas(16) T e[N];
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T)) / 16; ++i) reinterpret_cast<uint4*>(e)[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = (float)e[i];
}
template <class T, int N>
__device__ __forceinline__ void store_n(T* p, const float (&f)[N]) {
  alignas(16) T e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) e[i] = (T)f[i];
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T)) / 16; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(e)[i];
}

// items a head: groups of 8 pairs, then groups of 16 of the elements that only move
struct RotaryPlan {
  FastDiv per_row, per_head, length;
  int turn, items, rows_per_block;
};

template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_rotary(const RotaryArgs a, const RotaryPlan p) {
  const long long row0 = (long long)blockIdx.x * p.rows_per_block;
  const long long rows = (long long)a.batch * a.length;
  const int n = (int)min((long long)p.rows_per_block, rows - row0) * (int)p.per_row.d;
  for (int id = threadIdx.x; id < n; id += 256) {
    const int lr = (int)p.per_row.div((uint32_t)id), in_row = id - lr * (int)p.per_row.d;
    const int hd = (int)p.per_head.div((uint32_t)in_row), item = in_row - hd * p.items;
    const uint32_t row = (uint32_t)(row0 + lr);
    const int b = (int)p.length.div(row), s = (int)(row - (uint32_t)b * p.length.d);
    const int k = hd >= a.heads[0], head = k ? hd - a.heads[0] : hd;
    const T* x = (const T*)(k ? a.x[1] : a.x[0]) + b * (k ? a.xb[1] : a.xb[0]) + s * (k ? a.xs[1] : a.xs[0]) + head * (k ? a.xh[1] : a.xh[0]);
    T* y = (T*)(k ? a.y[1] : a.y[0]) + b * (k ? a.yb[1] : a.yb[0]) + s * (k ? a.ys[1] : a.ys[0]) + head * (k ? a.yh[1] : a.yh[0]);
    if (item >= p.turn) {                    // the rest of the head
      const int d0 = a.rot + (item - p.turn) * 2 * kPairs;
      if constexpr (VEC) {
#pragma unroll
        for (int w = 0; w < 2; ++w)
          if (d0 + 8 * w < a.dim) {
            float f[8];
            load_n<T, 8>(x + d0 + 8 * w, f);
            store_n<T, 8>(y + d0 + 8 * w, f);
          }
      } else {
        for (int d = d0; d < min(d0 + 2 * kPairs, a.dim); ++d) y[d] = x[d];
      }
      continue;
    }
    const int at = a.positions ? a.positions[row] : a.first + s;
    const bool in = (unsigned)at < (unsigned)a.max_pos;   // a position that the table lacks gives NaN
    const float* tab = a.table + ((long long)(in ? at : 0) * (a.rot / 2) + item * kPairs) * 2;
    const int half = a.rot / 2, j0 = item * kPairs;
    if constexpr (VEC) {
      float t[2 * kPairs], u[kPairs], v[kPairs];
      load_n<float, 2 * kPairs>(tab, t);
      if (!in) {
#pragma unroll
        for (int i = 0; i < 2 * kPairs; ++i) t[i] = __builtin_nanf("");
      }
      if (a.interleaved) {
        float e[2 * kPairs];
        load_n<T, 2 * kPairs>(x + 2 * j0, e);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          const float c = t[2 * i], sn = t[2 * i + 1] * a.sign, eu = e[2 * i], ev = e[2 * i + 1];
          e[2 * i] = eu * c - ev * sn;
          e[2 * i + 1] = ev * c + eu * sn;
        }
        store_n<T, 2 * kPairs>(y + 2 * j0, e);
      } else {
        load_n<T, kPairs>(x + j0, u);
        load_n<T, kPairs>(x + half + j0, v);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          const float c = t[2 * i], sn = t[2 * i + 1] * a.sign, eu = u[i], ev = v[i];
          u[i] = eu * c - ev * sn;
          v[i] = ev * c + eu * sn;
        }
        store_n<T, kPairs>(y + j0, u);
        store_n<T, kPairs>(y + half + j0, v);
      }
    } else {
      for (int i = 0; i < kPairs && j0 + i < half; ++i) {
        const int du = a.interleaved ? 2 * (j0 + i) : j0 + i, dv = a.interleaved ? du + 1 : du + half;
        const float c = in ? tab[2 * i] : __builtin_nanf(""), sn = tab[2 * i + 1] * a.sign;
        const float eu = (float)x[du], ev = (float)x[dv];
        y[du] = (T)(eu * c - ev * sn);
        y[dv] = (T)(ev * c + eu * sn);
      }
    }
  }
}

// Angles in 64 bits: at position 10^6 an fp32 angle is off by 0.06.
__global__ void __launch_bounds__(256) k_rotary_table(const RotaryTableArgs a) {
  const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
  const int half = a.rot / 2;
  if (id >= (long long)a.max_pos * half) return;
  const int p = (int)(id / half), j = (int)(id - (long long)p * half);
  const double two_pi = 6.283185307179586476925286766559;
  double base = a.base;
  if (a.scaling == 2 && a.rot > 2) base *= pow(a.factor, (double)a.rot / (a.rot - 2));
  double f = pow(base, -2.0 * j / a.rot);
  if (a.scaling == 1) f /= a.factor;
  if (a.scaling == 3) {
    // turns of this pair over the original length: below `lo` the frequency is divided, above `hi` kept
    const double turns = f * a.original / two_pi;
    const double keep = fmin(1.0, fmax(0.0, (turns - a.lo) / (a.hi - a.lo)));
    f = f * keep + f / a.factor * (1.0 - keep);
  }
  const double mag = a.scaling == 3 ? 0.1 * log(a.factor) + 1.0 : 1.0;
  double sn, c;
  sincos(p * f, &sn, &c);
  a.table[2 * id] = (float)(c * mag);
  a.table[2 * id + 1] = (float)(sn * mag);
}

RotaryPlan plan_of(const RotaryArgs& a) {
  RotaryPlan p;
  p.turn = (a.rot / 2 + kPairs - 1) / kPairs;
  p.items = p.turn + (a.dim - a.rot + 2 * kPairs - 1) / (2 * kPairs);
  p.per_head = FastDiv((uint32_t)p.items);
  p.per_row = FastDiv((uint32_t)((a.heads[0] + a.heads[1]) * p.items));
  p.length = FastDiv((uint32_t)a.length);
  const long long rows = (long long)a.batch * a.length;
  // four items a thread, fewer where that would leave compute units idle
  long long rpb = std::max(1u, 1024u / p.per_row.d);
  while (rpb > 1 && (rows + rpb - 1) / rpb < 512) rpb = (rpb + 1) / 2;
  p.rows_per_block = (int)rpb;
  return p;
}
long long blocks_of(const RotaryArgs& a, const RotaryPlan& p) {
  return ((long long)a.batch * a.length + p.rows_per_block - 1) / p.rows_per_block;
}

template <class T>
hipError_t run(hipStream_t s, const RotaryArgs& a, bool vec) {
  const RotaryPlan p = plan_of(a);
  const dim3 grid((unsigned)blocks_of(a, p));
  if (vec)
    k_rotary<T, true><<<grid, dim3(256), 0, s>>>(a, p);
  else
    k_rotary<T, false><<<grid, dim3(256), 0, s>>>(a, p);
  return hipGetLastError();
}

}  // namespace

long long rotary_blocks(const RotaryArgs& a) { return blocks_of(a, plan_of(a)); }

hipError_t launch_rotary(hipStream_t s, int dtype, const RotaryArgs& a, bool vec) {
  if (dtype == 1) return run<__bf16>(s, a, vec);
  if (dtype == 2) return run<_Float16>(s, a, vec);
  return run<float>(s, a, vec);
}

hipError_t launch_rotary_table(hipStream_t s, const RotaryTableArgs& a) {
  const long long n = (long long)a.max_pos * (a.rot / 2);
  k_rotary_table<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace ntk

// kernels_logprob.hip -- log probabilities of given tokens, the entropy, the most likely alternatives, and the gradient.
//
//   x = scale logits, m = max x, l = sum e^(x - m), logp = x_t - m - log l,
//   H = log l - (sum e^(x - m) (x - m)) / l,     dx_j = dlogp (1[j = t] - p_j) - dH p_j (log p_j + H),   p_j = e^(x_j - m) / l.
//
// One pass with the running maximum; the sums carry x - m, not x, and m and log l are handed to the gradient apart, so that
// nothing large cancels (a row that a mask fills with the type's lowest value is a uniform one).  Logits of -inf (tokens that
// are ruled out) have p = 0 and add nothing.  Sums are fp32.
//
// Bound by memory: of 4096 rows of 65536 in bf16 the forward pass takes 129 us (4.2 TB/s of reads), the gradient 168 (6.4 TB/s of
// reads and writes, some of them from the last-level cache); with 8 rows of 131072 by the best candidates' order and the launches
// (14 us and 6 for the join, with top = 20), which also makes 512 such rows take 109 us where they take 31 without
// alternatives.  Results are given off in fp32, the gradient in the logits' type.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "seq/launch_cache.hpp"

namespace ntk {
namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kUnroll = 4;                 // 16-byte loads in flight a thread

typedef unsigned long long u64;

// A running sum in units of e^m: raw maximum m, l = sum 2^((x - m) c), s = sum 2^((x - m) c) (x - m) c with c = scale log2(e).
struct Sum {
  float m, l, s;
};
__device__ __forceinline__ Sum empty_sum() { return Sum{-__builtin_inff(), 0.f, 0.f}; }
// the same sum under a maximum of m1 >= m
__device__ __forceinline__ void raise(Sum& a, float m1, float c) {
  if (m1 == a.m) return;
  const float d = a.m == -__builtin_inff() ? 0.f : (a.m - m1) * c;   // nothing summed yet: l = s = 0
  const float f = __builtin_amdgcn_exp2f(d);
  a.s = f > 0.f ? f * fmaf(a.l, d, a.s) : 0.f;
  a.l *= f;
  a.m = m1;
}
__device__ __forceinline__ Sum add(Sum a, Sum b, float c) {
  const float m = fmaxf(a.m, b.m);
  raise(a, m, c);
  raise(b, m, c);
  return Sum{m, a.l + b.l, a.s + b.s};
}

// A logit and its token in one whole number: larger logits first, of equal ones the lower token; NaN before all.
__device__ __forceinline__ u64 rank_of(float x, int token) {
  x = x == 0.f ? 0.f : x;                       // -0 = 0
  const uint32_t u = x == x ? __float_as_uint(x) : 0x7fffffffu;
  const uint32_t key = u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
  return ((u64)key << 32) | (uint32_t)~token;
}
__device__ __forceinline__ float logit_of(u64 r) {
  const uint32_t key = (uint32_t)(r >> 32);
  return __uint_as_float(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int token_of(u64 r) { return (int)~(uint32_t)r; }

__device__ __forceinline__ u64 lane_of(u64 x, int lane) {
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)x, lane), hi = __builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane);
  return ((u64)hi << 32) | lo;
}

// x of the lane below
__device__ __forceinline__ u64 from_below(u64 x) {
  constexpr int WAVE_SHR1 = 0x138;
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, WAVE_SHR1, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), WAVE_SHR1, 0xf, 0xf, true);
  return ((u64)hi << 32) | lo;
}
// how many of the first n lanes hold more than x (different numbers but for zeros)
__device__ __forceinline__ int rank_among(u64 x, int n) {
  int r = 0;
  for (int j = 0; j < n; ++j) r += lane_of(x, j) > x;
  return r;
}

// The best so far of a wave, in order: lane j holds the j-th (0: none yet).
struct Best {
  u64 mine, last;                              // last: the one at `top` - 1, which a candidate has to beat
  __device__ __forceinline__ Best() : mine(0), last(0) {}
  __device__ __forceinline__ void offer(u64 x, int top, int lane) {
    u64 left;
    while ((left = __ballot(x > last)) != 0) {
      const int from = __builtin_ctzll(left);
      const u64 got = lane_of(x, from);
      if (lane == from) x = 0;
      const int at = __popcll(__ballot(mine > got));
      const u64 up = from_below(mine);
      mine = lane < at ? mine : lane == at ? got : up;
      last = lane_of(mine, top - 1);
    }
  }
  // The first candidates, U a lane (0: none).  Offered one by one, a hundred of two thousand would take a place for a while.  So the
  // `top`-th of the lanes' own largest is found first, which is at most the `top`-th of all: mostly fewer than 64 reach it, and those
  // are put in order at once, by how many are larger.
  template <int U>
  __device__ __forceinline__ void begin(const u64 (&x)[U], int top, int lane, u64* lds) {
    u64 most = x[0];
#pragma unroll
    for (int u = 1; u < U; ++u) most = x[u] > most ? x[u] : most;
    const u64 cut = lane_of(most, (int)__builtin_ctzll(__ballot(most == 0 || rank_among(most, 64) == top - 1) | 1ull << 63));
    int n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) n += __popcll(__ballot(x[u] != 0 && x[u] >= cut));
    if (n > 64) {
#pragma unroll
      for (int u = 0; u < U; ++u) offer(x[u], top, lane);
      return;
    }
    int at = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = x[u] != 0 && x[u] >= cut;
      const u64 all = __ballot(in);
      if (in) lds[at + __popcll(all & ((1ull << lane) - 1))] = x[u];
      at += __popcll(all);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const u64 got = lane < n ? lds[lane] : 0;
    const int place = rank_among(got, n);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (lane < n) lds[place] = got;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    mine = lane < n ? lds[lane] : 0;
    last = lane_of(mine, top - 1);
  }
  __device__ __forceinline__ float floor_logit() const { return last ? logit_of(last) : -__builtin_inff(); }
};

// Elements of a row in groups of 16 aligned bytes: group g holds the elements g EC - skip .. + EC - 1, of which those of the
// row exist.
template <class T>
struct Row {
  static constexpr int EC = 16 / (int)sizeof(T);
  const T* p;
  int skip, n, groups;
  __device__ __forceinline__ Row(const void* base, long long row, long long stride, int vocab) {
    p = (const T*)base + row * stride;
    skip = (int)(((uintptr_t)p & 15) / sizeof(T));
    n = vocab;
    groups = (int)(((long long)skip + n + EC - 1) / EC);
  }
  __device__ __forceinline__ int first(int g) const { return g * EC - skip; }
  __device__ __forceinline__ bool whole(int g) const { return first(g) >= 0 && first(g) + EC <= n; }
  // what the row does not have is -inf
  __device__ __forceinline__ void read(int g, float (&f)[EC]) const {
    const int e = first(g);
    if (whole(g)) {
      alignas(16) T v[EC];
      *reinterpret_cast<uint4*>(v) = *reinterpret_cast<const uint4*>(p + e);
#pragma unroll
      for (int i = 0; i < EC; ++i) f[i] = (float)v[i];
    } else {
#pragma unroll
      for (int i = 0; i < EC; ++i) f[i] = (unsigned)(e + i) < (unsigned)n ? (float)p[e + i] : -__builtin_inff();
    }
  }
};

// log l and the entropy from a row's sum
struct Numbers {
  float logl, entropy;
};
__device__ __forceinline__ Numbers numbers(const Sum& a) {
  Numbers r;
  const bool none = a.m == -__builtin_inff() && a.l == 0.f;   // every token is ruled out
  r.logl = none ? 0.f : logf(a.l);
  r.entropy = none ? 0.f : r.logl - a.s / a.l * kLn2;
  return r;
}
// log p of a raw logit; -inf where every token is ruled out
__device__ __forceinline__ float logp_of(float x, const Sum& a, const Numbers& r, float scale) {
  return x == -__builtin_inff() && a.l == a.l ? x : (x - a.m) * scale - r.logl;
}

template <class T>
__device__ __forceinline__ void finish(const LogprobArgs& a, long long row, const Sum& sum, u64 best, int lane) {
  const Numbers r = numbers(sum);
  if (lane == 0) {
    const int t = a.tokens[row];
    a.logp[row] = t < 0 ? 0.f : t < a.vocab ? logp_of((float)((const T*)a.logits)[row * a.stride + t], sum, r, a.scale) : __builtin_nanf("");
    if (a.entropy) a.entropy[row] = r.entropy;
    if (a.lse) {
      a.lse[2 * row] = sum.m;
      a.lse[2 * row + 1] = r.logl;
    }
  }
  if (lane < a.top) {
    a.top_logp[row * a.top + lane] = logp_of(logit_of(best), sum, r, a.scale);
    a.top_tokens[row * a.top + lane] = token_of(best);
  }
}

// One workgroup: range blockIdx % splits of a row.
template <class T, bool TOP>
__global__ void __launch_bounds__(kThreads) k_logprobs(const LogprobArgs a) {
  using R = Row<T>;
  constexpr int EC = R::EC;
  __shared__ Sum sums[kWaves];
  __shared__ u64 bests[kWaves][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long row = blockIdx.x / a.splits;
  const int split = (int)(blockIdx.x - row * a.splits);
  const R r(a.logits, row, a.stride, a.vocab);
  const int per = (r.groups + a.splits - 1) / a.splits, g0 = split * per, g1 = min(r.groups, g0 + per);
  const float c = a.scale * kLog2e;
  Sum sum = empty_sum();
  Best best;
  for (int base = g0; base < g1; base += kThreads * kUnroll) {     // the same trips for every lane
    float f[kUnroll][EC];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int g = base + u * kThreads + (int)threadIdx.x;
      if (g < g1) {
        r.read(g, f[u]);
      } else {
#pragma unroll
        for (int i = 0; i < EC; ++i) f[u][i] = -__builtin_inff();
      }
    }
    float top = f[0][0];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int i = 0; i < EC; ++i) top = fmaxf(top, f[u][i]);
    if (top > sum.m) raise(sum, top, c);
    const float m = sum.m == -__builtin_inff() ? 0.f : sum.m;
    float l = 0.f, s = 0.f;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int i = 0; i < EC; ++i) {
        const float d = (f[u][i] - m) * c, e = __builtin_amdgcn_exp2f(d);
        l += e;
        s = fmaf(e, fmaxf(d, -200.f), s);         // -inf: 0 times a number
      }
    sum.l += l;
    sum.s += s;
    if constexpr (TOP) {
      if (base == g0) {
        u64 x[kUnroll * EC];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int g = base + u * kThreads + (int)threadIdx.x, e0 = r.first(g);
#pragma unroll
          for (int i = 0; i < EC; ++i)
            x[u * EC + i] = g < g1 && (unsigned)(e0 + i) < (unsigned)a.vocab ? rank_of(f[u][i], e0 + i) : 0;
        }
        best.begin(x, a.top, lane, bests[wave]);
      } else if (__any(!(top < best.floor_logit()) || l != l)) {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          const int g = base + u * kThreads + (int)threadIdx.x, e0 = r.first(g);
#pragma unroll
          for (int i = 0; i < EC; ++i)
            best.offer(g < g1 && (unsigned)(e0 + i) < (unsigned)a.vocab ? rank_of(f[u][i], e0 + i) : 0, a.top, lane);
        }
      }
    }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum = add(sum, Sum{__shfl_xor(sum.m, o), __shfl_xor(sum.l, o), __shfl_xor(sum.s, o)}, c);
  if (lane == 0) sums[wave] = sum;
  if constexpr (TOP) bests[wave][lane] = best.mine;
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) sum = add(sum, sums[w], c);
  if constexpr (TOP) {
    u64 x[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int i = w * 64 + lane, from = i / a.top;               // the waves' lists, one behind the other
      x[w] = from < kWaves ? bests[from][i - from * a.top] : 0;
    }
    __shared__ u64 lds[64];
    best = Best();
    best.begin(x, a.top, lane, lds);
  }
  if (a.splits == 1) {
    finish<T>(a, row, sum, best.mine, lane);
    return;
  }
  const long long at = row * a.splits + split;
  u64* lists = (u64*)a.work;                                        // [rows][splits][top], then the sums
  if (TOP && lane < a.top) lists[at * a.top + lane] = best.mine;
  float* out = (float*)(lists + a.rows * a.splits * a.top);
  if (lane == 0) {
    out[at * 3] = sum.m;
    out[at * 3 + 1] = sum.l;
    out[at * 3 + 2] = sum.s;
  }
}

// One wave a row: the sums and lists of its ranges.
template <class T>
__global__ void __launch_bounds__(64) k_logprobs_join(const LogprobArgs a) {
  const int lane = threadIdx.x;
  const long long row = blockIdx.x;
  const u64* lists = (const u64*)a.work + row * a.splits * a.top;
  const float* in = (const float*)((const u64*)a.work + a.rows * a.splits * a.top) + row * a.splits * 3;
  const float c = a.scale * kLog2e;
  Sum sum = empty_sum();
  for (int i = lane; i < a.splits; i += 64) sum = add(sum, Sum{in[3 * i], in[3 * i + 1], in[3 * i + 2]}, c);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum = add(sum, Sum{__shfl_xor(sum.m, o), __shfl_xor(sum.l, o), __shfl_xor(sum.s, o)}, c);
  Best best;
  if (a.top) {
    constexpr int U = 8;
    __shared__ u64 lds[64];
    const int n = a.splits * a.top;
    u64 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = u * 64 + lane < n ? lists[u * 64 + lane] : 0;
    best.begin(x, a.top, lane, lds);
    for (int i = U * 64; i < n; i += 64) best.offer(i + lane < n ? lists[i + lane] : 0, a.top, lane);
  }
  finish<T>(a, row, sum, best.mine, lane);
}

// The gradient: a workgroup takes kUnroll groups a thread of one row.
template <class T>
__global__ void __launch_bounds__(kThreads) k_logprobs_bwd(const LogprobBwdArgs a) {
  using R = Row<T>;
  constexpr int EC = R::EC;
  const long long row = blockIdx.x / a.chunks;
  const int chunk = (int)(blockIdx.x - row * a.chunks);
  const R r(a.logits, row, a.stride, a.vocab);
  const int t = a.tokens[row];
  const float m = a.lse[2 * row], l2 = a.lse[2 * row + 1] * kLog2e, c = a.scale * kLog2e;
  float gl = t >= 0 && a.dlogp ? a.dlogp[row] : 0.f;
  const float ge = a.dentropy ? a.dentropy[row] : 0.f;
  const float h2 = ge != 0.f ? a.entropy[row] * kLog2e : 0.f;
  if (t >= a.vocab) gl = __builtin_nanf("");
  const bool none = m == -__builtin_inff() && l2 == 0.f;      // every token is ruled out
  T* out = (T*)a.dlogits + row * a.dstride;
  const bool same = ((uintptr_t)out & 15) == ((uintptr_t)r.p & 15);
  const float k0 = -gl * a.scale, k1 = -ge * a.scale * kLn2;
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    const int g = (chunk * kUnroll + u) * kThreads + (int)threadIdx.x;
    if (g >= r.groups) continue;
    float f[EC];
    r.read(g, f);
    const int e0 = r.first(g);
    alignas(16) T v[EC];
#pragma unroll
    for (int i = 0; i < EC; ++i) {
      const float d = fmaf(f[i] - m, c, -l2), p = none ? 0.f : __builtin_amdgcn_exp2f(d);
      float dx = p * fmaf(k1, fmaxf(d, -200.f) + h2, k0);
      if (none) dx = gl != gl ? gl : 0.f;
      if (e0 + i == t && !none) dx = fmaf(gl, a.scale, dx);
      v[i] = (T)dx;
    }
    if (same && r.whole(g)) {
      *reinterpret_cast<uint4*>(out + e0) = *reinterpret_cast<const uint4*>(v);
    } else {
#pragma unroll
      for (int i = 0; i < EC; ++i)
        if ((unsigned)(e0 + i) < (unsigned)r.n) out[e0 + i] = v[i];
    }
  }
}

template <class T>
hipError_t run(hipStream_t s, const LogprobArgs& a) {
  const dim3 grid((unsigned)(a.rows * a.splits));
  if (a.top)
    k_logprobs<T, true><<<grid, dim3(kThreads), 0, s>>>(a);
  else
    k_logprobs<T, false><<<grid, dim3(kThreads), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.splits > 1) {
    k_logprobs_join<T><<<dim3((unsigned)a.rows), dim3(64), 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}
template <class T>
hipError_t run_bwd(hipStream_t s, const LogprobBwdArgs& a) {
  k_logprobs_bwd<T><<<dim3((unsigned)(a.rows * a.chunks)), dim3(kThreads), 0, s>>>(a);
  return hipGetLastError();
}
int elem(int dtype) { return dtype == 0 ? 4 : 2; }

}  // namespace

// Ranges of a row: 1024 workgroups, four a compute unit, each with at least 16 KB.  (One row of 131072 in bf16 takes 8.8 us, with
// ranges of 8 KB 12.7, of 32 KB 11.9; eight with top = 20 21.7, 22.6 and 26.8; 300 of 50000 16.4, with 2048 workgroups 19.3.)
int logprob_splits(int dtype, long long rows, int vocab) {
  const long long bytes = (long long)vocab * elem(dtype);
  return rows < 1 ? 1 : (int)std::max(1LL, std::min((1024 + rows - 1) / rows, bytes / 16384));
}
long long logprob_work_bytes(long long rows, int top, int splits) { return splits > 1 ? rows * splits * (8LL * top + 12) : 0; }
int logprob_bwd_chunks(int dtype, int vocab) {
  const int per = kThreads * kUnroll, groups = (int)(((long long)vocab * elem(dtype) + 15) / 16) + 1;
  return (groups + per - 1) / per;
}

hipError_t launch_logprobs(hipStream_t s, int dtype, const LogprobArgs& a) {
  if (dtype == 1) return run<__bf16>(s, a);
  if (dtype == 2) return run<_Float16>(s, a);
  return run<float>(s, a);
}
hipError_t launch_logprobs_bwd(hipStream_t s, int dtype, const LogprobBwdArgs& a) {
  if (dtype == 1) return run_bwd<__bf16>(s, a);
  if (dtype == 2) return run_bwd<_Float16>(s, a);
  return run_bwd<float>(s, a);
}

}  // namespace ntk

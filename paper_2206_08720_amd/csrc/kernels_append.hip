// kernels_append.hip -- new tokens' keys and values into a cache of pages, keys and queries turned to their positions on
// the way: (u, v) -> (u c - v s, v c + u s) with (c, s) = table[position][pair], in fp32, rounded once.
//
// In a cache of 8 bits (e4m3) a page's cells of one head lie under one power of two s, the least that leaves none above 448 s:
// a power of two, because growing it for a later token then leaves the cells that the page holds as they were (they lose bits in
// the subnormals alone), and because the matrix kernels apply it within the conversion.  A page that holds older tokens
// keeps at least the s it has; where s grows, the older cells are multiplied by s_old / s.
//
// Everything moves once: bound by memory where there is much of it (13.8 thousand tokens of 32 query and 8 key/value heads of 128 in
// bf16: 91 us for 339 MB, 3.7 TB/s, where a copy reaches 4.9; the rest goes to the table's rows, which come from the caches, and to the
// look-ups of page after length that each run of 16 waits for), by the launch where there is little (64 tokens: 7 us).  In 8 bits
// a wave owns the part of a page that one head gets, so that no two write a scale; it reads the new tokens twice, the second time
// from the caches: the same tokens 91 us with pages of 64 places, 311 MB.  Large pages leave few waves with much each: 348 us with pages of
// 1024; one prompt of 8192 tokens 40 us with pages of 64, 96 of 256, 303 of 1024.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "seq/launch_cache.hpp"

namespace ntk {
namespace {

constexpr int kRun = 16;                    // elements of a head that a thread takes: 8 pairs, or 16 neighbours

struct AppendPlan {
  FastDiv per_row, per_head, length, slots;
  int turn, items;                          // runs of a head that turn, runs in all
  int rows_per_block, row_blocks;           // the part of the launch that goes row by row
  int page_slots;                           // pages a sequence can touch (8 bits)
};

template <class T, int N>
__device__ __forceinline__ void read_n(const T* p, float (&f)[N]) {
  alignas(16) T e[N];
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T)) / 16; ++i) reinterpret_cast<uint4*>(e)[i] = reinterpret_cast<const uint4*>(p)[i];
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = (float)e[i];
}
template <class T, int N>
__device__ __forceinline__ void write_n(T* p, const float (&f)[N]) {
  alignas(16) T e[N];
#pragma unroll
  for (int i = 0; i < N; ++i) e[i] = (T)f[i];
#pragma unroll
  for (int i = 0; i < (int)(N * sizeof(T)) / 16; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(e)[i];
}
// two values as e4m3 bytes, four as a word
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) { return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false); }
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, (int)e4m3x2(a, b), true);
}

// A run of 16 elements: i < 8 at d0 + i * step, the others at d1 + (i - 8) * step; n0 and n1 of them exist.
struct Run {
  int d0, d1, step, n0, n1;
  bool turns;
  __device__ __forceinline__ Run(const AppendArgs& a, int turn, int rot, int item) {
    turns = item < turn;
    if (turns) {
      const int j0 = item * (kRun / 2);
      step = a.interleaved ? 2 : 1;
      d0 = j0 * step;
      d1 = a.interleaved ? d0 + 1 : rot / 2 + j0;
      n0 = n1 = min(kRun / 2, rot / 2 - j0);
    } else {
      step = 1;
      d0 = rot + (item - turn) * kRun;
      d1 = d0 + 8;
      n0 = min(8, a.dim - d0);
      n1 = min(8, max(0, a.dim - d1));
    }
  }
};

// A run's values, turned to position `pos` if it turns.
template <class T, bool VEC>
__device__ __forceinline__ void read_run(const AppendArgs& a, const T* x, const Run& r, int pos, int item, float (&f)[kRun]) {
  if constexpr (VEC) {
    if (r.turns && a.interleaved) {
      float e[kRun];
      read_n<T, kRun>(x + r.d0, e);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[i] = e[2 * i];
        f[8 + i] = e[2 * i + 1];
      }
    } else {
      float u[8], v[8] = {};
      read_n<T, 8>(x + r.d0, u);
      if (r.n1 > 0) read_n<T, 8>(x + r.d1, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[i] = u[i];
        f[8 + i] = v[i];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f[i] = i < r.n0 ? (float)x[r.d0 + i * r.step] : 0.f;
      f[8 + i] = i < r.n1 ? (float)x[r.d1 + i * r.step] : 0.f;
    }
  }
  if (!r.turns) return;
  const bool in = (unsigned)pos < (unsigned)a.max_pos;   // a position that the table lacks gives NaN
  const float* tab = a.table + ((long long)(in ? pos : 0) * (a.rot / 2) + item * 8) * 2;
  float t[kRun];
  if constexpr (VEC) {
    read_n<float, kRun>(tab, t);
  } else {
#pragma unroll
    for (int i = 0; i < kRun; ++i) t[i] = i < 2 * r.n0 ? tab[i] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = in ? t[2 * i] : __builtin_nanf(""), s = t[2 * i + 1], u = f[i], v = f[8 + i];
    f[i] = fmaf(u, c, -(v * s));                          // rounded where kernels_rotary.hip rounds
    f[8 + i] = fmaf(v, c, u * s);
  }
}

template <class T, bool VEC>
__device__ __forceinline__ void write_run(const AppendArgs& a, T* y, const Run& r, const float (&f)[kRun]) {
  if constexpr (VEC) {
    if (r.turns && a.interleaved) {
      float e[kRun];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[2 * i] = f[i];
        e[2 * i + 1] = f[8 + i];
      }
      write_n<T, kRun>(y + r.d0, e);
    } else {
      float u[8], v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        u[i] = f[i];
        v[i] = f[8 + i];
      }
      write_n<T, 8>(y + r.d0, u);
      if (r.n1 > 0) write_n<T, 8>(y + r.d1, v);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i < r.n0) y[r.d0 + i * r.step] = (T)f[i];
      if (i < r.n1) y[r.d1 + i * r.step] = (T)f[8 + i];
    }
  }
}
template <bool VEC>
__device__ __forceinline__ void write_run_e4m3(const AppendArgs& a, uint8_t* y, const Run& r, const float (&f)[kRun]) {
  if constexpr (VEC) {
    if (r.turns && a.interleaved) {
      *reinterpret_cast<uint4*>(y + r.d0) = make_uint4(e4m3x4(f[0], f[8], f[1], f[9]), e4m3x4(f[2], f[10], f[3], f[11]),
                                                       e4m3x4(f[4], f[12], f[5], f[13]), e4m3x4(f[6], f[14], f[7], f[15]));
    } else {
      *reinterpret_cast<uint2*>(y + r.d0) = make_uint2(e4m3x4(f[0], f[1], f[2], f[3]), e4m3x4(f[4], f[5], f[6], f[7]));
      if (r.n1 > 0)
        *reinterpret_cast<uint2*>(y + r.d1) = make_uint2(e4m3x4(f[8], f[9], f[10], f[11]), e4m3x4(f[12], f[13], f[14], f[15]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u = e4m3x2(f[i], f[8 + i]);
      if (i < r.n0) y[r.d0 + i * r.step] = (uint8_t)u;
      if (i < r.n1) y[r.d1 + i * r.step] = (uint8_t)(u >> 8);
    }
  }
}

// the largest finite magnitude of a run
__device__ __forceinline__ float most_of(const float (&f)[kRun]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < kRun; ++i) {
    const float x = fabsf(f[i]);
    m = x < __builtin_inff() ? fmaxf(m, x) : m;
  }
  return m;
}

// The type has no infinity: what is not finite becomes NaN.  The last values of the arrays' type would round to a power of two that
// it reads as infinity: they stay one step below, 15/16 of it.  (A sum that a turn takes past fp16's range is no such value.)
template <class T>
__device__ __forceinline__ void to_units(float (&f)[kRun], float inv) {
  constexpr bool HALF = std::is_same_v<T, _Float16>;
  constexpr float most = HALF ? 61440.f : 0x1.ep127f, end = HALF ? 65520.f : __builtin_inff();
#pragma unroll
  for (int k = 0; k < kRun; ++k) {
    float v = f[k];
    if (fabsf(v) > most && fabsf(v) < end) v = copysignf(most, v);
    f[k] = fabsf(v) < __builtin_inff() ? v * inv : __builtin_nanf("");
  }
}

// bytes k0 .. of a cell (at most 16) times g
template <bool VEC>
__device__ __forceinline__ void rescale(uint8_t* c, int k0, int dim, float g) {
  const int n = min(kRun, dim - k0);
  alignas(16) uint32_t w[4] = {0, 0, 0, 0};
  if (VEC && n == kRun) {
    *reinterpret_cast<uint4*>(w) = *reinterpret_cast<const uint4*>(c + k0);
  } else {
#pragma unroll
    for (int k = 0; k < kRun; ++k)
      if (k < n) w[k / 4] |= (uint32_t)c[k0 + k] << (8 * (k % 4));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = e4m3x4(__builtin_amdgcn_cvt_f32_fp8((int)w[i], 0) * g, __builtin_amdgcn_cvt_f32_fp8((int)w[i], 1) * g,
                  __builtin_amdgcn_cvt_f32_fp8((int)w[i], 2) * g, __builtin_amdgcn_cvt_f32_fp8((int)w[i], 3) * g);
  if (VEC && n == kRun) {
    *reinterpret_cast<uint4*>(c + k0) = *reinterpret_cast<const uint4*>(w);
  } else {
#pragma unroll
    for (int k = 0; k < kRun; ++k)
      if (k < n) c[k0 + k] = (uint8_t)(w[k / 4] >> (8 * (k % 4)));
  }
}

// One wave: the cells of one head in one page, of the keys (which = 0) or the values.  Twice over the new tokens: once for s.
template <class T, bool VEC>
__device__ __forceinline__ void append_page(const AppendArgs& a, const AppendPlan& p, int b, int e, int head, int which, int lane) {
  const AppendSpan span(a.pages, a.lens[b], a.news ? a.news[b] : a.length, a.length);
  int lo, hi, token;
  if (!span.slots(a.pages, (span.first >> a.pages.shift) + e, lo, hi, token)) return;
  const int page = a.pages.page(b, span.first + token);
  if (page < 0) return;
  const int rot = which ? 0 : a.rot, turn = which ? 0 : p.turn;
  const int per = turn + (a.dim - rot + kRun - 1) / kRun;       // runs a head: at most 9
  const int at_once = 64 / per, mine = lane / per, item = lane - mine * per;
  const bool busy = mine < at_once;
  const Run r(a, turn, rot, item);
  const T* x = (const T*)a.x[1 + which] + b * a.xb[1 + which] + head * a.xh[1 + which];
  uint8_t* cell = (uint8_t*)a.cell[which] + page * a.cb[which] + head * a.ch[which];
  const int n = busy ? hi - lo : 0;
  auto values = [&](int i, float (&f)[kRun]) {
    const int t = token + i;
    const int pos = !r.turns ? 0 : a.positions ? a.positions[(long long)b * a.length + t] : span.first + t;
    read_run<T, VEC>(a, x + t * a.xs[1 + which], r, pos, item, f);
  };
  float most = 0.f;
  for (int i = mine; i < n; i += at_once) {
    float f[kRun];
    values(i, f);
    most = fmaxf(most, most_of(f));
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) most = fmaxf(most, __shfl_xor(most, o));
  float* sp = a.scale[which] + (long long)page * a.kv_heads + head;
  const float old = lo > 0 ? *sp : 0.f;
  const float s = fmaxf(old, __builtin_ldexpf(1.f, e4m3_exponent(most)));
  const float inv = 1.f / s;                                    // of a power of two: exact
  if (lane == 0) *sp = s;
  for (int i = mine; i < n; i += at_once) {
    float f[kRun];
    values(i, f);
    to_units<T>(f, inv);
    write_run_e4m3<VEC>(a, cell + (long long)(lo + i) * a.cs[which], r, f);
  }
  if (lo > 0 && s > old) {
    const int runs = (a.dim + kRun - 1) / kRun;                 // the bytes lie as neighbours, whatever turned
    for (int i = lane; i < lo * runs; i += 64) {
      const int slot = i / runs;
      rescale<VEC>(cell + (long long)slot * a.cs[which], (i - slot * runs) * kRun, a.dim, old * inv);
    }
  }
}

template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_append(const AppendArgs a, const AppendPlan p) {
  if ((int)blockIdx.x >= p.row_blocks) {
    const long long id = (long long)(blockIdx.x - p.row_blocks) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int per = 2 * a.kv_heads;
    const long long at = id / per;
    if (at >= (long long)a.batch * p.page_slots) return;
    const int in = (int)(id - at * per), b = (int)p.slots.div((uint32_t)at), e = (int)at - b * p.page_slots;
    append_page<T, VEC>(a, p, b, e, in >> 1, in & 1, threadIdx.x & 63);
    return;
  }
  const long long row0 = (long long)blockIdx.x * p.rows_per_block, rows = (long long)a.batch * a.length;
  const int n = (int)min((long long)p.rows_per_block, rows - row0) * (int)p.per_row.d;
  for (int id = threadIdx.x; id < n; id += 256) {
    const int lr = (int)p.per_row.div((uint32_t)id), in_row = id - lr * (int)p.per_row.d;
    const int hd = (int)p.per_head.div((uint32_t)in_row), item = in_row - hd * p.items;
    const uint32_t row = (uint32_t)(row0 + lr);
    const int b = (int)p.length.div(row), t = (int)(row - (uint32_t)b * p.length.d);
    const int which = hd < a.heads ? 0 : hd < a.heads + a.kv_heads ? 1 : 2;
    const int head = hd - (which == 0 ? 0 : which == 1 ? a.heads : a.heads + a.kv_heads);
    const int rot = which == 2 ? 0 : a.rot, turn = which == 2 ? 0 : p.turn;
    if (item >= turn + (a.dim - rot + kRun - 1) / kRun) continue;
    const AppendSpan span(a.pages, a.lens[b], a.news ? a.news[b] : a.length, a.length);
    T* y;
    if (which == 0) {
      y = (T*)a.qo + b * a.qb + t * a.qs + head * a.qh;
    } else {
      const int page = t < span.count ? a.pages.page(b, span.first + t) : -1;
      if (page < 0) continue;
      const int c = which - 1;
      y = (T*)a.cell[c] + page * a.cb[c] + a.pages.slot(span.first + t) * a.cs[c] + head * a.ch[c];
    }
    const Run r(a, turn, rot, item);
    float f[kRun] = {};
    if (t < span.count) {
      const int pos = !r.turns ? 0 : a.positions ? a.positions[row] : span.first + t;
      read_run<T, VEC>(a, (const T*)a.x[which] + b * a.xb[which] + t * a.xs[which] + head * a.xh[which], r, pos, item, f);
    }
    write_run<T, VEC>(a, y, r, f);
  }
}

AppendPlan plan_of(const AppendArgs& a) {
  AppendPlan p;
  const bool e4m3 = a.quantize != 0;
  const int row_heads = a.heads + (e4m3 ? 0 : 2 * a.kv_heads);
  p.turn = (a.rot / 2 + kRun / 2 - 1) / (kRun / 2);
  p.items = std::max(p.turn + (a.dim - a.rot + kRun - 1) / kRun, (a.dim + kRun - 1) / kRun);
  p.per_head = FastDiv((uint32_t)p.items);
  p.per_row = FastDiv((uint32_t)std::max(1, row_heads * p.items));
  p.length = FastDiv((uint32_t)std::max(1, a.length));
  const long long rows = (long long)a.batch * a.length;
  // four items a thread, fewer where that would leave compute units idle
  long long rpb = std::max(1u, 1024u / p.per_row.d);
  while (rpb > 1 && (rows + rpb - 1) / rpb < 512) rpb = (rpb + 1) / 2;
  p.rows_per_block = (int)rpb;
  p.row_blocks = row_heads ? (int)((rows + rpb - 1) / rpb) : 0;   // rows < 2^31
  p.page_slots = e4m3 ? append_pages(a.length, a.pages.shift) : 0;
  p.slots = FastDiv((uint32_t)std::max(1, p.page_slots));
  return p;
}
long long blocks_of(const AppendArgs& a, const AppendPlan& p) {
  return p.row_blocks + ((long long)a.batch * p.page_slots * 2 * a.kv_heads + 3) / 4;
}

template <class T>
hipError_t run(hipStream_t s, const AppendArgs& a, bool vec) {
  const AppendPlan p = plan_of(a);
  const dim3 grid((unsigned)blocks_of(a, p));
  if (vec)
    k_append<T, true><<<grid, dim3(256), 0, s>>>(a, p);
  else
    k_append<T, false><<<grid, dim3(256), 0, s>>>(a, p);
  return hipGetLastError();
}

}  // namespace

long long append_blocks(const AppendArgs& a) { return blocks_of(a, plan_of(a)); }

hipError_t launch_append(hipStream_t s, int dtype, const AppendArgs& a, bool vec) {
  if (dtype == 1) return run<__bf16>(s, a, vec);
  if (dtype == 2) return run<_Float16>(s, a, vec);
  return run<float>(s, a, vec);
}

}  // namespace ntk

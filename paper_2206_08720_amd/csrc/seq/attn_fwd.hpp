// attn_fwd.hpp -- what the forward attention kernels share (kernels_attn.hip, kernels_cached.hip): a wave's 32 query rows
// and their running softmax, the rows' results, and the sum of the states that waves have of the same rows.
#pragma once
#include "attn_core.hpp"

namespace ntk {
namespace {

// keys a tile and query rows a workgroup of the kernels for many rows
template <class T>
constexpr int kFwdKeys = sizeof(T) == 2 ? 64 : 32;
constexpr int kFwdRows = 128;

// One wave's 32 query rows: a lane's row, its limits and its state.
// DOCS: the call may have documents.  EARLY: tiles are written into LDS by the waves.
template <class T, int DP, bool DOCS = true, bool EARLY = false>
struct FwdRows {
  using N = Num<T>;
  using Tile = AttnTile<T, DP>;
  using Frag = typename N::Frag;
  static constexpr int KT = DP / 16, DB = DP / 32;
  Frag q[KT];
  f32x16 acc[DB];
  float m, l;
  int klim, pos, doc;
  float slope2;

  __device__ __forceinline__ void reset() {
    m = -__builtin_inff();
    l = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) zero16(acc[d]);
  }

  // Scores of a block of 32 keys from `key0` in log2 units (or, where neither a cap nor a slope applies, raw);
  // hidden ones are -inf.  Careful: `vis` gets bit v for a visible pair.
  template <class Careful>
  __device__ __forceinline__ void scores(const AttnArgs& a, const char* sk, int nb, int key0, const int* ids, bool masked,
                                         int lane, const typename Tile::Lane& tl, f32x16& s, unsigned& vis) const {
    zero16(s);
#pragma unroll
    for (int t = 0; t < KT; ++t) s = N::template product<Careful::value>(Tile::rows(sk, 32 * nb, t, tl), q[t], s);
    finish_scores<Careful>(a, nb, key0, ids, masked, lane, s, vis);
  }
  // All products of a tile before the first of their scores is used, four operands read ahead (left to itself the compiler
  // waits for each operand where it is used: 16 trips to LDS in a row).
  template <int NB>
  __device__ __forceinline__ void products_early(const char* sk, const typename Tile::Lane& tl, f32x16 (&s)[NB]) const {
    constexpr int N_OPS = KT * NB, AHEAD = sizeof(T) == 2 ? 4 : 1;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) zero16(s[nb]);
    Frag f[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) f[i] = Tile::rows(sk, 32 * (i % NB), i / NB, tl);
#pragma unroll
    for (int i = 0; i < N_OPS; ++i) {
      __builtin_amdgcn_sched_barrier(6);       // arithmetic may pass, reads and products not
      s[i % NB] = N::template product<false>(f[i % AHEAD], q[i / NB], s[i % NB]);
      if (i + AHEAD < N_OPS) f[i % AHEAD] = Tile::rows(sk, 32 * ((i + AHEAD) % NB), (i + AHEAD) / NB, tl);
    }
    __builtin_amdgcn_sched_barrier(6);
  }
  template <class Careful>
  __device__ __forceinline__ void finish_scores(const AttnArgs& a, int nb, int key0, const int* ids, bool masked, int lane, f32x16& s,
                                                unsigned& vis) const {
    const int h4 = 4 * (lane >> 5), base = key0 + 32 * nb + h4;
    if (a.cap_in != 0.f) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] = capped<T>(a, s[v]);
    } else if (a.slopes) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] *= a.c;
    }
    if (a.slopes) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] -= slope2 * (float)abs(pos - (base + 8 * (v >> 2) + (v & 3)));
    }
    if (masked) {
      const int left = klim - base;
      if constexpr (Careful::value) {
        vis = 0xffffu;
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (8 * (v >> 2) + (v & 3) >= left || (DOCS && a.docs && ids[32 * nb + h4 + 8 * (v >> 2) + (v & 3)] != doc)) vis &= ~(1u << v);
      }
      if (DOCS && a.docs) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const i32x4 id = *reinterpret_cast<const i32x4*>(ids + 32 * nb + h4 + 8 * q);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[4 * q + i] = 8 * q + i < left && id[i] == doc ? s[4 * q + i] : -__builtin_inff();
        }
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) s[v] = 8 * (v >> 2) + (v & 3) < left ? s[v] : -__builtin_inff();
      }
    } else if (Careful::value) {
      vis = 0xffffu;
    }
  }

  // A tile of 32 NB keys.  `careful`: with the product that keeps hidden operands out (mma_visible).
  template <int NB, class Careful>
  __device__ __forceinline__ void tile(const AttnArgs& a, const char* sk, const char* sv, const int* ids, int key0, bool masked,
                                       Careful, int lane, typename Tile::Lane& tl) {
    tl.fresh();
    f32x16 s[NB];
    unsigned vis[NB];
    if constexpr (EARLY && !Careful::value) {
      products_early<NB>(sk, tl, s);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) finish_scores<Careful>(a, nb, key0, ids, masked, lane, s[nb], vis[nb]);
    } else {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) scores<Careful>(a, sk, nb, key0, ids, masked, lane, tl, s[nb], vis[nb]);
    }
    float top = s[0][0];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, s[nb][v]);
    top = half_max(top);
    const float unit = a.cap_in != 0.f || a.slopes ? 1.f : a.c;
    // The running maximum moves only where it grew: elsewhere 2^(m - m') is 1.
    if (__any(top > m)) {
      const float mn = fmaxf(m, top);
      const float f = mn == m ? 1.f : exp2_hw((m - mn) * unit);   // m = -inf: 0
      m = mn;
      l *= f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[d][v] *= f;
    }
    // nothing seen yet: every weight is 2^-inf = 0
    const float mu = m == -__builtin_inff() ? 0.f : fmaf(-m, unit, kWeightBits<T>);
    float sum = 0.f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        s[nb][v] = exp2_hw(fmaf(s[nb][v], unit, mu));
        sum += s[nb][v];
      }
    l += sum;
    if constexpr (EARLY) __builtin_amdgcn_s_setprio(1);   // the wave that multiplies goes first
    typename Tile::Cols vc;
    vc.set(sv, tl);
    unrolled<2 * NB>([&](auto step) {
      constexpr int X = decltype(step)::value, nb = X / 2, u = X % 2;
      const Frag p = to_frag<T>(s[nb], u);
      if constexpr (!Careful::value) {
        Frag vt[DB];
        if constexpr (EARLY)
          vc.template read_early<16 * X>(vt, tl);
        else
          vc.template read<16 * X>(vt, tl);
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] = N::mma(vt[d], p, acc[d]);
      } else {
        Frag w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = (T)((vis[nb] >> (8 * u + i)) & 1 ? 1.f : 0.f);
        unrolled<DB>([&](auto block) {
          constexpr int d = decltype(block)::value;
          acc[d] = mma_visible<T, true>(vc.template read_one<16 * X, d>(tl), p, w, acc[d]);
        });
      }
    });
    if constexpr (EARLY) __builtin_amdgcn_s_setprio(0);
  }
};

// Row results: o and lse, or a range's partial sums for k_attn_join.
template <class T, int DP, bool VEC, class Rows>
__device__ __forceinline__ void finish_row(const AttnArgs& a, Rows& w, int b, int hk, int r, int split, int lane) {
  if (r >= a.R) return;
  const float unit = a.cap_in != 0.f || a.slopes ? 1.f : a.c;
  const float m2 = w.m == -__builtin_inff() ? w.m : w.m * unit;
  if (a.splits > 1) {
    const long long row = ((long long)split * a.B * a.Hk + (long long)b * a.Hk + hk) * a.R + r;
    store_owned<float, DP, true>(a.part + row * DP, DP, lane, w.acc, 1.f);
    if (lane < 32) {
      float* ml = a.part + (long long)a.splits * a.B * a.Hk * a.R * DP + row * 2;
      ml[0] = m2;
      ml[1] = w.l;
    }
    return;
  }
  const int i = (int)a.gdiv.div((uint32_t)r), g = r - i * a.G, head = hk * a.G + g;
  const float inv = w.l == 0.f ? 0.f : 1.f / w.l;   // a row that sees nothing is zero
  T* o = (T*)a.o.p + b * a.o.sb + i * a.o.ss + head * a.o.sh;
  store_owned<T, DP, VEC>(o, a.D, lane, w.acc, inv);
  if (a.lse && lane < 32)
    a.lse[((long long)b * a.H + head) * a.Sq + i] = w.l == 0.f ? -__builtin_inff() : m2 * kLn2 + logf(w.l * kWeightOne<T>);
}

// The states of W waves that took keys of the same rows, one after the other, into the first one's; true there.
template <class T, int DP, int W, class Rows>
__device__ __forceinline__ bool join_waves(const AttnArgs& a, Rows& w, char* smem, int wave, int lane) {
  __syncthreads();
  float* sacc = reinterpret_cast<float*>(smem);        // [W - 1][DB * 16][64]
  float* sml = sacc + (W - 1) * FwdRows<T, DP>::DB * 16 * 64;   // [W - 1][2][64]
  if (wave) {
    float* d = sacc + (wave - 1) * FwdRows<T, DP>::DB * 16 * 64;
#pragma unroll
    for (int db = 0; db < FwdRows<T, DP>::DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) d[(db * 16 + v) * 64 + lane] = w.acc[db][v];
    sml[(wave - 1) * 128 + lane] = w.m;
    sml[(wave - 1) * 128 + 64 + lane] = w.l;
  }
  __syncthreads();
  if (wave) return false;
  const float unit = a.cap_in != 0.f || a.slopes ? 1.f : a.c;
#pragma unroll 1
  for (int o = 0; o < W - 1; ++o) {
    const float m1 = sml[o * 128 + lane], l1 = sml[o * 128 + 64 + lane];
    const float mn = fmaxf(w.m, m1);
    const float f0 = w.m == mn ? 1.f : exp2_hw((w.m - mn) * unit), f1 = m1 == mn ? 1.f : exp2_hw((m1 - mn) * unit);
    const float* d = sacc + o * FwdRows<T, DP>::DB * 16 * 64;
    w.m = mn;
    w.l = w.l * f0 + l1 * f1;
#pragma unroll
    for (int db = 0; db < FwdRows<T, DP>::DB; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) w.acc[db][v] = w.acc[db][v] * f0 + d[(db * 16 + v) * 64 + lane] * f1;
  }
  return true;
}
template <class T, int DP, int W>
constexpr int kJoinBytes = (W - 1) * (DP / 32 * 16 * 64 + 128) * 4;   // LDS it takes

}  // namespace
}  // namespace ntk

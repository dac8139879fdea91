// kernels_attn_bwd.hip -- attention, backward: dq, dk and dv from dout and the forward pass's o and lse.
//
// With p = exp(s - lse) formed again from q and k, and delta = sum_d dout o:
//   dv = p^T dout,  dp = dout v^T,  ds = p (dp - delta) (1 - (c / cap)^2) scale,  dq = ds k,  dk = ds^T q
// (c the capped score; the factor is 1 without a cap).  Two kernels: one owns rows and sums over the keys
// (dq), one owns keys and sums over the rows of every query head that shares them (dk, dv).  Forming the
// scores twice costs 7 products instead of 5, and buys results that no order of atomics changes.
// p and ds are rounded to the inputs' type for the products; everything else is fp32.
#include "attn_core.hpp"
#include "launch_attn.hpp"

namespace ntk {
namespace {

// p and ds of 16 (row, key) pairs of a lane: `s` the raw products q k, `dp` the products dout v.  In: hidden pairs
// as cleared bits of vis.  dist(v): |position - key| for the slope.
template <class T, class L, class Dl, class Sl, class Dist>
__device__ __forceinline__ void weights(const AttnArgs& a, f32x16& s, f32x16& dp, unsigned vis, L lse2, Dl delta, Sl slope2,
                                        Dist dist) {
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    float x = s[v], fac = 1.f;
    if (a.cap_in != 0.f) {
      const float t = tanh_of<T>(x * a.cap_in);
      fac = 1.f - t * t;
      x = a.cap_out * t;
    } else {
      x *= a.c;
    }
    if (a.slopes) x -= slope2(v) * dist(v);
    const float p = exp2_hw(x - lse2(v));
    const bool on = (vis >> v) & 1;
    s[v] = on ? p : 0.f;
    dp[v] = on ? p * (dp[v] - delta(v)) * fac : 0.f;
  }
}

// delta of a row; rows that see nothing (lse = -inf) get weights 0 through lse2 = inf.
__device__ __forceinline__ float lse_units(float lse) { return lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e; }

template <class T>
__global__ void __launch_bounds__(256) k_attn_delta(const AttnArgs a, float* __restrict__ delta, long long rows) {
  // 16 lanes a row (b, i, head)
  const int lane = threadIdx.x & 15;
  const long long id = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (id >= rows) return;
  const int head = (int)(id % a.H);
  const long long bi = id / a.H;
  const int i = (int)(bi % a.Sq), b = (int)(bi / a.Sq);
  const T* o = (const T*)a.o.p + b * a.o.sb + i * a.o.ss + head * a.o.sh;
  const T* g = (const T*)a.dout.p + b * a.dout.sb + i * a.dout.ss + head * a.dout.sh;
  float s = 0.f;
  for (int d = lane; d < a.D; d += 16) s = fmaf((float)o[d], (float)g[d], s);
#pragma unroll
  for (int w = 8; w; w >>= 1) s += __shfl_xor(s, w);
  if (lane == 0) delta[((long long)b * a.H + head) * a.Sq + i] = s;
}

// ---- dq: four waves of 32 rows over the key tiles -----------------------------------------------------
template <class T>
constexpr int kBwdKeys = sizeof(T) == 2 ? 64 : 32;
constexpr int kBwdRows = 128;

template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) k_attn_dq(const AttnArgs a) {
  constexpr int BN = kBwdKeys<T>, KT = DP / 16, DB = DP / 32;
  using N = Num<T>;
  using Tile = AttnTile<T, DP>;
  using Frag = typename N::Frag;
  using Load = AttnLoad<T, DP, BN, 4, VEC>;
  extern __shared__ __align__(1024) char smem[];
  char* sk = smem;
  char* sv = smem + 2 * Load::BYTES;
  int* sids = reinterpret_cast<int*>(smem + 4 * Load::BYTES);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int id = die_order(blockIdx.x, gridDim.x);
  const int mt = a.tiles - 1 - id % a.tiles;
  id /= a.tiles;
  const int hk = id % a.Hk, b = id / a.Hk;
  const AttnScope sc(a, b);
  const int r0 = mt * kBwdRows, r = r0 + wave * 32 + (lane & 31), rc = min(r, a.R - 1);
  const int i = (int)a.gdiv.div((uint32_t)rc), head = hk * a.G + rc - i * a.G;
  const int* docs = a.docs ? a.docs + (long long)b * a.Sk : nullptr;
  const int pos = sc.off + i;
  const int doc = docs && pos >= 0 ? docs[pos] : 0;
  const int klim = doc < 0 ? 0 : sc.klim(pos);
  const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.f;
  const long long stat = ((long long)b * a.H + head) * a.Sq + i;
  const float lse2 = r < a.R ? lse_units(a.lse[stat]) : __builtin_inff();
  const float delta = a.delta[stat];
  Frag q[KT], g[KT];
  load_owned<T, DP, VEC>((const T*)a.q.p + b * a.q.sb + i * a.q.ss + head * a.q.sh, r < a.R, a.D, lane, q);
  load_owned<T, DP, VEC>((const T*)a.dout.p + b * a.dout.sb + i * a.dout.ss + head * a.dout.sh, r < a.R, a.D, lane, g);

  const int p_lo = sc.off + (int)a.gdiv.div((uint32_t)r0);
  const int p_hi = sc.off + (int)a.gdiv.div((uint32_t)(min(r0 + kBwdRows, a.R) - 1));
  const int all = sc.klim(p_lo), any = sc.klim(p_hi);
  KeyTiles kt;
  kt.t1 = (any + BN - 1) / BN;
  kt.len = sc.len;
  kt.base = -1;
  kt.bn = BN;
  kt.docs = docs;
  if (docs) doc_range(docs, p_lo, p_hi, lane, kt.lo, kt.hi);
  const T* kh = (const T*)a.k.p + b * a.k.sb + hk * a.k.sh;
  const T* vh = (const T*)a.v.p + b * a.v.sb + hk * a.v.sh;

  f32x16 acc[DB];
  auto pass = [&](auto careful) {
#pragma unroll
    for (int d = 0; d < DB; ++d) zero16(acc[d]);
    int t = kt.from(0, lane), st = 0, nid = -1;
    auto issue = [&](int t, int st) {
      if (docs && tid < BN) nid = t * BN + tid < sc.len ? docs[t * BN + tid] : -1;
      Load::positions(kh, a.k.ss, t * BN, sc.len, a.D, sk + st * Load::BYTES, wave, lane);
      Load::positions(vh, a.v.ss, t * BN, sc.len, a.D, sv + st * Load::BYTES, wave, lane);
    };
    if (t < kt.t1) {
      issue(t, 0);
      if (docs && tid < BN) sids[tid] = nid;
    }
    while (t < kt.t1) {
      __builtin_amdgcn_s_waitcnt(0x0070);
      __syncthreads();
      const int tn = kt.from(t + 1, lane);
      if (tn < kt.t1) issue(tn, st ^ 1);
      const bool masked = docs || (t + 1) * BN > all;
      const char *k_ = sk + st * Load::BYTES, *v_ = sv + st * Load::BYTES;
      typename Tile::Cols cols;
      cols.set(k_, lane);
      unrolled<BN / 32>([&](auto block) {
        constexpr int nb = decltype(block)::value;
        f32x16 s, dp;
        zero16(s);
        zero16(dp);
#pragma unroll
        for (int x = 0; x < KT; ++x) {
          s = N::mma(Tile::rows(k_, 32 * nb, x, lane), q[x], s);
          dp = N::mma(Tile::rows(v_, 32 * nb, x, lane), g[x], dp);
        }
        const int h4 = 4 * (lane >> 5), base = t * BN + 32 * nb + h4;
        unsigned vis = 0xffffu;
        if (masked) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (base + 8 * (v >> 2) + (v & 3) >= klim) vis &= ~(1u << v);
          if (docs) {
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (sids[st * BN + 32 * nb + h4 + 8 * (v >> 2) + (v & 3)] != doc) vis &= ~(1u << v);
          }
        }
        weights<T>(a, s, dp, vis, [&](int) { return lse2; }, [&](int) { return delta; }, [&](int) { return slope2; },
                   [&](int v) { return (float)abs(pos - (base + 8 * (v >> 2) + (v & 3))); });
        unrolled<2>([&](auto step) {
          constexpr int u = decltype(step)::value;
          const Frag w = to_frag<T>(dp, u);
          Frag kc[DB];
          cols.template read<32 * nb + 16 * u>(kc, lane);
          if constexpr (decltype(careful)::value) {
            Frag on;
#pragma unroll
            for (int e = 0; e < 8; ++e) on[e] = (T)((vis >> (8 * u + e)) & 1 ? 1.f : 0.f);
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] = mma_visible<T>(kc[d], w, on, acc[d]);
          } else {
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] = N::mma(kc[d], w, acc[d]);
          }
        });
      });
      if (docs && tn < kt.t1 && tid < BN) sids[(st ^ 1) * BN + tid] = nid;
      t = tn;
      st ^= 1;
    }
  };
  pass(std::false_type{});
  if (__syncthreads_or(not_finite(acc))) pass(std::true_type{});
  if (r < a.R)
    store_owned<T, DP, VEC>((T*)a.dq.p + b * a.dq.sb + i * a.dq.ss + head * a.dq.sh, a.D, lane, acc, a.scale);
}

// ---- dk, dv: four waves of 32 keys over the row tiles -----------------------------------------------------
template <class T>
constexpr int kBwdRowTile = sizeof(T) == 2 ? 64 : 32;
constexpr int kBwdKeyTile = 128;

// What a tile of rows brings along, in LDS.
template <int BR>
struct RowStats {
  float lse2[BR], delta[BR], slope2[BR];
  int klim[BR], pos[BR], doc[BR];
};

template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(256, 1) k_attn_dkv(const AttnArgs a) {
  constexpr int BR = kBwdRowTile<T>, KT = DP / 16, DB = DP / 32;
  using N = Num<T>;
  using Tile = AttnTile<T, DP>;
  using Frag = typename N::Frag;
  using Load = AttnLoad<T, DP, BR, 4, VEC>;
  extern __shared__ __align__(1024) char smem[];
  char* sq = smem;
  char* sg = smem + 2 * Load::BYTES;
  RowStats<BR>* stats = reinterpret_cast<RowStats<BR>*>(smem + 4 * Load::BYTES);   // [2]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int id = die_order(blockIdx.x, gridDim.x);
  const int k0 = (id % a.tiles) * kBwdKeyTile;       // the keys that most rows see first
  id /= a.tiles;
  const int hk = id % a.Hk, b = id / a.Hk;
  const AttnScope sc(a, b);
  const int j = k0 + wave * 32 + (lane & 31), jc = min(j, a.Sk - 1);
  const int* docs = a.docs ? a.docs + (long long)b * a.Sk : nullptr;
  const bool live = j < sc.len;
  const int doc = docs ? (live ? docs[jc] : -1) : 0;
  Frag k[KT], vv[KT];
  load_owned<T, DP, VEC>((const T*)a.k.p + b * a.k.sb + jc * a.k.ss + hk * a.k.sh, live, a.D, lane, k);
  load_owned<T, DP, VEC>((const T*)a.v.p + b * a.v.sb + jc * a.v.ss + hk * a.v.sh, live, a.D, lane, vv);

  // the first query that sees one of the keys: positions below 0 do not exist
  int i0 = max(0, -sc.off);
  if (sc.causal && sc.prefix <= k0) i0 = max(i0, k0 - sc.off);
  const int nr = (a.R + BR - 1) / BR;
  const int t_end = k0 < sc.len && i0 < a.Sq ? nr : 0;
  int lo = 0x7fffffff, hi = -1;                       // the keys' documents
  if (docs) doc_range(docs, k0, min(k0 + kBwdKeyTile, sc.len) - 1, lane, lo, hi);
  int base = -1;
  unsigned long long mask = 0;
  auto from = [&](int t) {                            // the next row tile with one of them
    if (!docs) return t;
    while (t < t_end) {
      if (base < 0 || t >= base + 64) {
        base = t;
        mask = doc_tiles(min(64, t_end - t), lo, hi, [&](int x) {
          const int r = (t + x) * BR + lane;
          if (lane >= BR || r >= a.R) return -1;
          const int p = sc.off + (int)a.gdiv.div((uint32_t)r);
          return p >= 0 ? docs[p] : -1;
        });
      }
      const unsigned long long m = mask >> (t - base);
      if (m) return t + (int)__builtin_ctzll(m);
      t = base + 64;
    }
    return t_end;
  };
  const T* qh = (const T*)a.q.p + b * a.q.sb + (long long)hk * a.G * a.q.sh;
  const T* gh = (const T*)a.dout.p + b * a.dout.sb + (long long)hk * a.G * a.dout.sh;

  f32x16 dk[DB], dv[DB];
  auto pass = [&](auto careful) {
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      zero16(dk[d]);
      zero16(dv[d]);
    }
    float n_lse = 0.f, n_delta = 0.f, n_slope = 0.f;
    int n_klim = 0, n_pos = 0, n_doc = 0;
    auto issue = [&](int t, int st) {
      if (tid < BR) {
        const int r = t * BR + tid, rc = min(r, a.R - 1);
        const int i = (int)a.gdiv.div((uint32_t)rc), head = hk * a.G + rc - i * a.G;
        const long long stat = ((long long)b * a.H + head) * a.Sq + i;
        n_pos = sc.off + i;
        n_doc = docs && n_pos >= 0 ? docs[n_pos] : 0;
        n_klim = r < a.R && n_doc >= 0 ? sc.klim(n_pos) : 0;
        n_lse = a.lse[stat];
        n_delta = a.delta[stat];
        if (a.slopes) n_slope = a.slopes[head];
      }
      Load::packed(qh, a.q.ss, a.q.sh, t * BR, a.R, a.gdiv, a.D, sq + st * Load::BYTES, wave, lane);
      Load::packed(gh, a.dout.ss, a.dout.sh, t * BR, a.R, a.gdiv, a.D, sg + st * Load::BYTES, wave, lane);
    };
    auto keep = [&](int st) {
      if (tid < BR) {
        stats[st].lse2[tid] = n_klim > 0 ? lse_units(n_lse) : __builtin_inff();   // rows past the last: weight 0
        stats[st].delta[tid] = n_klim > 0 ? n_delta : 0.f;
        stats[st].slope2[tid] = n_slope * kLog2e;
        stats[st].klim[tid] = n_klim;
        stats[st].pos[tid] = n_pos;
        stats[st].doc[tid] = n_doc;
      }
    };
    int t = from((int)((long long)i0 * a.G / BR)), st = 0;
    if (t < t_end) {
      issue(t, 0);
      keep(0);
    }
    while (t < t_end) {
      __builtin_amdgcn_s_waitcnt(0x0070);
      __syncthreads();
      const int tn = from(t + 1);
      if (tn < t_end) issue(tn, st ^ 1);
      const int p_first = sc.off + (int)a.gdiv.div((uint32_t)(t * BR));
      const bool masked = docs || k0 + kBwdKeyTile > sc.klim(p_first);
      const char *q_ = sq + st * Load::BYTES, *g_ = sg + st * Load::BYTES;
      const RowStats<BR>& rs = stats[st];
      typename Tile::Cols gcols, qcols;
      gcols.set(g_, lane);
      qcols.set(q_, lane);
      unrolled<BR / 32>([&](auto block) {
        constexpr int rb = decltype(block)::value;
        f32x16 s, dp;
        zero16(s);
        zero16(dp);
#pragma unroll
        for (int x = 0; x < KT; ++x) {
          s = N::mma(Tile::rows(q_, 32 * rb, x, lane), k[x], s);
          dp = N::mma(Tile::rows(g_, 32 * rb, x, lane), vv[x], dp);
        }
        const int rr = 32 * rb + 4 * (lane >> 5);
        auto at = [&](int v) { return rr + 8 * (v >> 2) + (v & 3); };
        unsigned vis = 0xffffu;
        if (masked) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (j >= rs.klim[at(v)]) vis &= ~(1u << v);
          if (docs) {
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (rs.doc[at(v)] != doc) vis &= ~(1u << v);
          }
        }
        weights<T>(a, s, dp, vis, [&](int v) { return rs.lse2[at(v)]; }, [&](int v) { return rs.delta[at(v)]; },
                   [&](int v) { return rs.slope2[at(v)]; }, [&](int v) { return (float)abs(rs.pos[at(v)] - j); });
        unrolled<2>([&](auto step) {
          constexpr int u = decltype(step)::value;
          const Frag p = to_frag<T>(s, u), w = to_frag<T>(dp, u);
          Frag gc[DB], qc[DB];
          gcols.template read<32 * rb + 16 * u>(gc, lane);
          if constexpr (decltype(careful)::value) {
            Frag on;
#pragma unroll
            for (int e = 0; e < 8; ++e) on[e] = (T)((vis >> (8 * u + e)) & 1 ? 1.f : 0.f);
#pragma unroll
            for (int d = 0; d < DB; ++d) dv[d] = mma_visible<T>(gc[d], p, on, dv[d]);
            qcols.template read<32 * rb + 16 * u>(qc, lane);
#pragma unroll
            for (int d = 0; d < DB; ++d) dk[d] = mma_visible<T>(qc[d], w, on, dk[d]);
          } else {
#pragma unroll
            for (int d = 0; d < DB; ++d) dv[d] = N::mma(gc[d], p, dv[d]);
            qcols.template read<32 * rb + 16 * u>(qc, lane);
#pragma unroll
            for (int d = 0; d < DB; ++d) dk[d] = N::mma(qc[d], w, dk[d]);
          }
        });
      });
      if (tn < t_end) keep(st ^ 1);
      t = tn;
      st ^= 1;
    }
  };
  pass(std::false_type{});
  if (__syncthreads_or(not_finite(dk) || not_finite(dv))) pass(std::true_type{});
  if (j < a.Sk) {   // keys past the batch entry's length get zeros
    store_owned<T, DP, VEC>((T*)a.dk.p + b * a.dk.sb + j * a.dk.ss + hk * a.dk.sh, a.D, lane, dk, a.scale);
    store_owned<T, DP, VEC>((T*)a.dv.p + b * a.dv.sb + j * a.dv.ss + hk * a.dv.sh, a.D, lane, dv, 1.f);
  }
}

template <class T, int DP, bool VEC>
hipError_t run_bwd(hipStream_t s, AttnArgs& a) {
  {
    constexpr int bytes = 4 * AttnLoad<T, DP, kBwdKeys<T>, 4, VEC>::BYTES + 2 * kBwdKeys<T> * 4;
    a.tiles = (a.R + kBwdRows - 1) / kBwdRows;
    const hipError_t e = hipFuncSetAttribute((const void*)k_attn_dq<T, DP, VEC>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    if (a.tiles) k_attn_dq<T, DP, VEC><<<dim3(a.B * a.Hk * a.tiles), dim3(256), bytes, s>>>(a);
  }
  {
    constexpr int BR = kBwdRowTile<T>;
    constexpr int bytes = 4 * AttnLoad<T, DP, BR, 4, VEC>::BYTES + 2 * (int)sizeof(RowStats<BR>);
    a.tiles = (a.Sk + kBwdKeyTile - 1) / kBwdKeyTile;
    const hipError_t e = hipFuncSetAttribute((const void*)k_attn_dkv<T, DP, VEC>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    if (a.tiles) k_attn_dkv<T, DP, VEC><<<dim3(a.B * a.Hk * a.tiles), dim3(256), bytes, s>>>(a);
  }
  return hipGetLastError();
}

template <class T>
hipError_t run_bwd_dim(hipStream_t s, AttnArgs& a, float* delta, bool vec) {
  const long long rows = (long long)a.B * a.Sq * a.H;
  if (rows) k_attn_delta<T><<<dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, s>>>(a, delta, rows);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.delta = delta;
  if (a.D <= 64) return vec ? run_bwd<T, 64, true>(s, a) : run_bwd<T, 64, false>(s, a);
  return vec ? run_bwd<T, 128, true>(s, a) : run_bwd<T, 128, false>(s, a);
}

}  // namespace

hipError_t launch_attn_bwd(hipStream_t s, int dtype, AttnArgs& a, float* delta, bool vec) {
  if (dtype == 1) return run_bwd_dim<__bf16>(s, a, delta, vec);
  if (dtype == 2) return run_bwd_dim<_Float16>(s, a, delta, vec);
  return run_bwd_dim<float>(s, a, delta, vec);
}

}  // namespace ntk

// kernels_attn.hip -- attention, forward: o = softmax(mask(score(q k^T))) v.
//
// One pass over the keys with the running maximum m and sum l of the softmax: for a tile of keys
//   s = score(k q^T), m' = max(m, max s), p = 2^(s - m'), l' = l 2^(m - m') + sum p,
//   o' = o 2^(m - m') + v^T p,
// and o / l at the end, lse = m + log l.  Scores are held in fp32 in units of log2; p is rounded to the
// inputs' type for the value product (its sum l is not), in fp16 times 2^14 (kWeightBits); o and l are fp32.
#include "seq/attn_core.hpp"
#include "seq/launch_attn.hpp"

namespace ntk {
namespace {

// One wave's 32 query rows: a lane's row, its limits and its state.
template <class T, int DP>
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
          if (8 * (v >> 2) + (v & 3) >= left || (a.docs && ids[32 * nb + h4 + 8 * (v >> 2) + (v & 3)] != doc)) vis &= ~(1u << v);
      }
      if (a.docs) {
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
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) scores<Careful>(a, sk, nb, key0, ids, masked, lane, tl, s[nb], vis[nb]);
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
    typename Tile::Cols vc;
    vc.set(sv, tl);
    unrolled<2 * NB>([&](auto step) {
      constexpr int X = decltype(step)::value, nb = X / 2, u = X % 2;
      const Frag p = to_frag<T>(s[nb], u);
      if constexpr (!Careful::value) {
        Frag vt[DB];
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
  }
};

// Row results: o and lse, or a range's partial sums for k_attn_join.
template <class T, int DP, bool VEC>
__device__ __forceinline__ void finish_row(const AttnArgs& a, FwdRows<T, DP>& w, int b, int hk, int r, int split, int lane) {
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

// ---- many rows: four waves of 32 rows share the key tiles in LDS ---------------------------------------
// Two LDS stages, filled straight from global memory: the next tile is in flight while one is multiplied,
// one barrier a tile.  A wave's 32 MFMAs of a tile of 64 keys (heads of 128) take 1024 cycles of the matrix cores, its
// softmax about as many of the vector unit, of which the exponentials half: two waves a SIMD, on 256 registers
// each, let one multiply while the other exponentiates.  bf16, 16 heads over 4 of 128, 8192 positions: 325 us causal
// (850 TFLOP/s of the visible pairs), 595 us in full (920; a library product of 8192^3 reaches 1200 on this card).
template <class T>
constexpr int kFwdKeys = sizeof(T) == 2 ? 64 : 32;
constexpr int kFwdRows = 128;

template <class T, int DP, bool VEC, bool CAREFUL>
__device__ __forceinline__ bool fwd_body(const AttnArgs& a, char* smem, int block) {
  constexpr int BN = kFwdKeys<T>;
  using Load = AttnLoad<T, DP, BN, 4, VEC>;
  char* sk = smem;                                  // [2][BN][DP]
  char* sv = smem + 2 * Load::BYTES;
  int* sids = reinterpret_cast<int*>(smem + 4 * Load::BYTES);   // [2][BN]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int bh, item;
  place(block, a.B * a.Hk, bh, item);
  const int split = item % a.splits, mt = a.tiles - 1 - item / a.splits;   // the rows that see most keys first
  const int hk = bh % a.Hk, b = bh / a.Hk;
  const AttnScope sc(a, b);
  const int r0 = mt * kFwdRows, r = r0 + wave * 32 + (lane & 31);
  const int i = (int)a.gdiv.div((uint32_t)min(r, a.R - 1)), g = min(r, a.R - 1) - i * a.G;
  const int* docs = a.docs ? a.docs + (long long)b * a.Sk : nullptr;

  FwdRows<T, DP> w;
  typename AttnTile<T, DP>::Lane tl(lane);
  w.pos = sc.off + i;
  w.klim = sc.klim(w.pos);
  w.doc = docs && w.pos >= 0 ? docs[w.pos] : 0;
  const bool one = __all(w.doc >= 0 && w.doc == __builtin_amdgcn_readfirstlane(w.doc));   // this wave's rows: one document
  if (w.doc < 0) w.klim = 0;
  w.slope2 = a.slopes ? a.slopes[hk * a.G + g] * kLog2e : 0.f;
  load_owned<T, DP, VEC>((const T*)a.q.p + b * a.q.sb + i * a.q.ss + (hk * a.G + g) * a.q.sh, r < a.R, a.D, lane, w.q);

  const int p_lo = sc.off + (int)a.gdiv.div((uint32_t)r0);
  const int p_hi = sc.off + (int)a.gdiv.div((uint32_t)(min(r0 + kFwdRows, a.R) - 1));
  const int all = sc.klim(p_lo), any = sc.klim(p_hi);   // keys that every row sees, that some row sees
  const int nt = (any + BN - 1) / BN, per = (nt + a.splits - 1) / a.splits;
  TileList kt;
  kt.t0 = split * per;
  kt.t1 = min(nt, kt.t0 + per);
  kt.words = nullptr;
  if (docs) {
    __shared__ unsigned long long words[kDocWords];
    int lo, hi;
    doc_range(docs, p_lo, p_hi, lane, lo, hi);
    kt.find(words, 4, wave, lane, lo, hi, [&](int t) {
      const int j = t * BN + lane % BN, d = docs[min(j, sc.len - 1)];
      return j < sc.len ? d : -1;
    });
    __syncthreads();
  }
  const T* kh = (const T*)a.k.p + b * a.k.sb + hk * a.k.sh;
  const T* vh = (const T*)a.v.p + b * a.v.sb + hk * a.v.sh;

  auto pass = [&](auto careful) {
    w.reset();
    int t = kt.from(kt.t0), st = 0;
    int nid = -1;
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
      __builtin_amdgcn_s_waitcnt(0x0070);   // this wave's part of the tile has landed, and its LDS reads are done
      __syncthreads();
      const int tn = kt.from(t + 1);
      if (tn < kt.t1) issue(tn, st ^ 1);
      const bool masked = (t + 1) * BN > all || (docs && !(one && __all(sids[st * BN + lane % BN] == w.doc)));
      w.template tile<BN / 32>(a, sk + st * Load::BYTES, sv + st * Load::BYTES, sids + st * BN, t * BN, masked, careful, lane, tl);
      if (docs && tn < kt.t1 && tid < BN) sids[(st ^ 1) * BN + tid] = nid;
      t = tn;
      st ^= 1;
    }
  };
  pass(std::integral_constant<bool, CAREFUL>{});
  // 0 * inf of a hidden pair (or a visible one): once more, with the product that tells them apart
  if (!CAREFUL && __syncthreads_or(not_finite(w.acc))) return true;
  w.l = half_sum(w.l);
  finish_row<T, DP, VEC>(a, w, b, hk, r, split, lane);
  return false;
}
template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(256, (sizeof(T) * DP <= 256 ? 2 : 1)) k_attn_fwd(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  const bool bad = fwd_body<T, DP, VEC, false>(a, smem, blockIdx.x);
  if (threadIdx.x == 0) a.flags[blockIdx.x] = bad;
}
template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(256, 1) k_attn_fwd_again(const AttnArgs a, int blocks) {
  extern __shared__ __align__(1024) char smem[];
  again(a.flags, blocks, [&](int id) { fwd_body<T, DP, VEC, true>(a, smem, id); });
}

// ---- few rows (at most 32 a key/value head: single tokens, short drafts) ---------------------------------
// Bound by reading the cache: each of W waves takes every W-th tile of 32 keys of the workgroup's
// range through two LDS stages of its own (nothing is shared, so no barrier), and the states are
// joined in LDS at the end.  The ranges that the cache is cut into are joined by k_attn_join.  16 sequences of 32
// heads over 4 of 128, caches of 16 to 32 thousand: 163 us with the join, 5.0 TB/s (a large copy: 4.7).
constexpr int kTokKeys = 32;
// four waves, or as many as their stages (of 32 fp32 rows of 128: 64 KB a wave) leave room for
template <class T, int DP>
constexpr int kTokWaves = kTokKeys * DP * (int)sizeof(T) * 16 <= 128 * 1024 ? 4 : 2;

template <class T, int DP, bool VEC, bool CAREFUL>
__device__ __forceinline__ bool tokens_body(const AttnArgs& a, char* smem) {
  constexpr int BN = kTokKeys, W = kTokWaves<T, DP>;
  using Load = AttnLoad<T, DP, BN, 1, VEC>;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  char* mine = smem + wave * 4 * Load::BYTES;          // [2][k, v]
  int* ids = reinterpret_cast<int*>(smem + 4 * W * Load::BYTES) + wave * BN;

  int bh, split;
  place(blockIdx.x, a.B * a.Hk, bh, split);
  const int hk = bh % a.Hk, b = bh / a.Hk;
  const AttnScope sc(a, b);
  const int r = lane & 31;
  const int i = (int)a.gdiv.div((uint32_t)min(r, a.R - 1)), g = min(r, a.R - 1) - i * a.G;
  const int* docs = a.docs ? a.docs + (long long)b * a.Sk : nullptr;

  FwdRows<T, DP> w;
  typename AttnTile<T, DP>::Lane tl(lane);
  w.pos = sc.off + i;
  w.klim = sc.klim(w.pos);
  w.doc = docs && w.pos >= 0 ? docs[w.pos] : 0;
  if (w.doc < 0) w.klim = 0;
  w.slope2 = a.slopes ? a.slopes[hk * a.G + g] * kLog2e : 0.f;
  load_owned<T, DP, VEC>((const T*)a.q.p + b * a.q.sb + i * a.q.ss + (hk * a.G + g) * a.q.sh, r < a.R, a.D, lane, w.q);

  const int all = sc.klim(sc.off), any = sc.klim(sc.off + (a.R - 1) / a.G);
  const int nt = (any + BN - 1) / BN, per = (nt + a.splits - 1) / a.splits;
  TileList kt;
  kt.t0 = split * per;
  kt.t1 = min(nt, kt.t0 + per);
  kt.words = nullptr;
  if (docs) {
    __shared__ unsigned long long words[kDocWords];
    int lo, hi;
    doc_range(docs, sc.off, sc.off + (a.R - 1) / a.G, lane, lo, hi);
    kt.find(words, W, wave, lane, lo, hi, [&](int t) {
      const int j = t * BN + lane % BN, d = docs[min(j, sc.len - 1)];
      return j < sc.len ? d : -1;
    });
    __syncthreads();
  }
  const T* kh = (const T*)a.k.p + b * a.k.sb + hk * a.k.sh;
  const T* vh = (const T*)a.v.p + b * a.v.sb + hk * a.v.sh;

  auto next = [&](int t) {       // the next of this wave's tiles: every W-th, documents skipped over
    t = kt.from(t);
    while (t < kt.t1 && ((t - kt.t0) & (W - 1)) != wave) t = kt.from(t + 1);
    return t;
  };
  auto pass = [&](auto careful) {
    w.reset();
    auto issue = [&](int t, int st) {
      char* s = mine + st * 2 * Load::BYTES;
      Load::positions(kh, a.k.ss, t * BN, sc.len, a.D, s, 0, lane);
      Load::positions(vh, a.v.ss, t * BN, sc.len, a.D, s + Load::BYTES, 0, lane);
    };
    int t = next(kt.t0), st = 0;
    if (t < kt.t1) issue(t, 0);
    while (t < kt.t1) {
      const int tn = next(t + 1);
      const bool masked = docs || (t + 1) * BN > all;
      if (docs && lane < BN) ids[lane] = t * BN + lane < sc.len ? docs[t * BN + lane] : -1;
      if (VEC && tn < kt.t1) {
        issue(tn, st ^ 1);
        wait_loads<2 * Load::NI>();    // the current tile has landed; the next stays in flight
      } else {
        __builtin_amdgcn_s_waitcnt(0x0070);
      }
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_sched_barrier(0);
      const char* s = mine + st * 2 * Load::BYTES;
      w.template tile<1>(a, s, s + Load::BYTES, ids, t * BN, masked, careful, lane, tl);
      __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's LDS reads are done: the stage may be filled again
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_sched_barrier(0);
      if (!VEC && tn < kt.t1) issue(tn, st ^ 1);
      t = tn;
      st ^= 1;
    }
  };
  pass(std::integral_constant<bool, CAREFUL>{});
  if (!CAREFUL && __syncthreads_or(not_finite(w.acc))) return true;
  w.l = half_sum(w.l);

  // the waves' states, one after the other, into the first one's
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
  finish_row<T, DP, VEC>(a, w, b, hk, r, split, lane);
  return false;
}
template <class T, int DP, bool VEC>
__global__ void __launch_bounds__((64 * kTokWaves<T, DP>), 1) k_attn_tokens(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  if (tokens_body<T, DP, VEC, false>(a, smem)) tokens_body<T, DP, VEC, true>(a, smem);
}

// ---- the ranges of a row, joined -----------------------------------------------------------------------
template <class T, int DP>
__global__ void __launch_bounds__(DP) k_attn_join(const AttnArgs a) {
  const int d = threadIdx.x, r = blockIdx.x % a.R, bh = blockIdx.x / a.R, hk = bh % a.Hk, b = bh / a.Hk;
  const long long rows = (long long)a.B * a.Hk * a.R, row = (long long)bh * a.R + r;
  const float* ml = a.part + (long long)a.splits * rows * DP;
  // online, eight ranges' numbers in flight at a time
  float m = -__builtin_inff(), l = 0.f, o = 0.f;
  for (int s0 = 0; s0 < a.splits; s0 += 8) {
    float ms[8], ls[8], os[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const long long at = (long long)min(s0 + u, a.splits - 1) * rows + row;
      ms[u] = s0 + u < a.splits ? ml[at * 2] : -__builtin_inff();
      ls[u] = ml[at * 2 + 1];
      os[u] = a.part[at * DP + d];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (s0 + u >= a.splits) break;
      const float mn = fmaxf(m, ms[u]);
      const float f = m == mn ? 1.f : exp2_hw(m - mn), g = ms[u] == mn ? 1.f : exp2_hw(ms[u] - mn);
      l = l * f + ls[u] * g;
      o = o * f + os[u] * g;
      m = mn;
    }
  }
  const int i = (int)a.gdiv.div((uint32_t)r), head = hk * a.G + r - i * a.G;
  if (d < a.D) ((T*)a.o.p)[b * a.o.sb + i * a.o.ss + head * a.o.sh + d] = (T)(l == 0.f ? 0.f : o / l);
  if (a.lse && d == 0)
    a.lse[((long long)b * a.H + head) * a.Sq + i] = l == 0.f ? -__builtin_inff() : m * kLn2 + logf(l * kWeightOne<T>);
}

template <class T, int DP, bool VEC>
hipError_t run_fwd(hipStream_t s, const AttnArgs& a, bool tokens) {
  if (tokens) {
    constexpr int W = kTokWaves<T, DP>;
    constexpr int bytes = 4 * W * AttnLoad<T, DP, kTokKeys, 1, VEC>::BYTES + W * kTokKeys * 4;
    static_assert(bytes >= (W - 1) * (DP / 32 * 16 * 64 + 128) * 4, "the join fits the stages");
    const hipError_t e = hipFuncSetAttribute((const void*)k_attn_tokens<T, DP, VEC>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    k_attn_tokens<T, DP, VEC><<<dim3(a.B * a.Hk * a.splits), dim3(64 * W), bytes, s>>>(a);
  } else {
    constexpr int bytes = 4 * AttnLoad<T, DP, kFwdKeys<T>, 4, VEC>::BYTES + 2 * kFwdKeys<T> * 4;
    const hipError_t e = hipFuncSetAttribute((const void*)k_attn_fwd<T, DP, VEC>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    const int blocks = a.B * a.Hk * a.tiles * a.splits;
    k_attn_fwd<T, DP, VEC><<<dim3(blocks), dim3(256), bytes, s>>>(a);
    const hipError_t e1 = hipGetLastError();
    if (e1 != hipSuccess) return e1;
    const hipError_t e2 = hipFuncSetAttribute((const void*)k_attn_fwd_again<T, DP, VEC>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e2 != hipSuccess) return e2;
    k_attn_fwd_again<T, DP, VEC><<<dim3(std::min(blocks, kAgainBlocks)), dim3(256), bytes, s>>>(a, blocks);
  }
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && a.splits > 1) {
    k_attn_join<T, DP><<<dim3(a.B * a.Hk * a.R), dim3(DP), 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

template <class T>
hipError_t run_fwd_dim(hipStream_t s, const AttnArgs& a, bool tokens, bool vec) {
  if (a.D <= 64) return vec ? run_fwd<T, 64, true>(s, a, tokens) : run_fwd<T, 64, false>(s, a, tokens);
  return vec ? run_fwd<T, 128, true>(s, a, tokens) : run_fwd<T, 128, false>(s, a, tokens);
}

}  // namespace

AttnPlan attn_plan_fwd(int dtype, int B, int Hk, int R, int Sk, int D) {
  AttnPlan p;
  p.tokens = R <= 32;
  p.tiles = (R + kFwdRows - 1) / kFwdRows;
  const long long blocks = (long long)B * Hk * (p.tokens ? 1 : p.tiles);
  // Ranges of the keys.  Tokens: 512 workgroups or more, two for each of 256 compute units (heads over 64 leave room for one at
  // a time, by their registers and LDS; the second evens out what lengths of their own leave idle), each with at least 64 KB of
  // keys: a call over 777 keys of 8 heads of 64 takes 13.5 us in one range and 20 in four, with the join and its
  // launch; with heads of 128 the ranges pay on the GPU (12 us against 18).  Many rows: as many as run at once, of
  // at least 256 keys (64 in fp32, whose products take several times as long); from 192 tiles on the join's traffic
  // would cost more than idle units do.
  const int row_bytes = (D <= 64 ? 64 : 128) * (dtype == 0 ? 4 : 2);
  if (p.tokens)
    p.splits = (int)std::max(1LL, std::min((512 + blocks - 1) / blocks, (long long)Sk * row_bytes / 65536));
  else
    p.splits = blocks >= 192 ? 1 : (int)std::max(1LL, std::min(512 / blocks, (long long)Sk / (dtype == 0 ? 64 : 256)));
  const int dp = D <= 64 ? 64 : 128;
  p.part_floats = p.splits > 1 ? (long long)p.splits * B * Hk * R * (dp + 2) : 0;
  p.flag_ints = p.tokens ? 0 : blocks * p.splits;
  return p;
}

hipError_t launch_attn_fwd(hipStream_t s, int dtype, const AttnArgs& a, bool tokens, bool vec) {
  if (dtype == 1) return run_fwd_dim<__bf16>(s, a, tokens, vec);
  if (dtype == 2) return run_fwd_dim<_Float16>(s, a, tokens, vec);
  return run_fwd_dim<float>(s, a, tokens, vec);
}

}  // namespace ntk

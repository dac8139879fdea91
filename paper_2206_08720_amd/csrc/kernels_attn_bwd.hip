// kernels_attn_bwd.hip -- attention, backward: dq, dk and dv from dout and the forward pass's o and lse.
//
// With p = exp(s - lse) formed again from q and k, and delta = sum_d dout o:
//   dv = p^T dout,  dp = dout v^T,  ds = p (dp - delta) (1 - (c / cap)^2) scale,  dq = ds k,  dk = ds^T q
// (c the capped score; the factor is 1 without a cap).  Two kernels: one owns rows and sums over the keys
// (dq), one owns keys and sums over the rows of every query head that shares them (dk, dv).  Forming the
// scores twice costs 7 products instead of 5, and buys results that no order of atomics changes.
// p and ds are rounded to the inputs' type for the products, as the matrix cores take them (fp16: in powers of two that keep
// them in its range), and delta is formed with the o that the forward pass stored; everything else is fp32.
#include "seq/attn_core.hpp"
#include "seq/launch_attn.hpp"

namespace ntk {
namespace {

// p and ds of 16 (row, key) pairs of a lane: `s` the raw products q k, `dp` the products dout v.  The functions give the
// numbers of registers 4 q .. 4 q + 3; far(q): |position - key| for the slope.
template <class T, class L, class Dl, class Sl, class Far>
__device__ __forceinline__ void weights(const AttnArgs& a, f32x16& s, f32x16& dp, L lse2, Dl delta, Sl slope2, Far far) {
  // a few numbers at a time (sched_barrier): registers are short
  unrolled<4>([&](auto quad) {
    constexpr int q = decltype(quad)::value;
    const f32x4 d = delta(q);
#pragma unroll
    for (int i = 0; i < 4; ++i) dp[4 * q + i] -= d[i];
  });
  float c = a.c;
  if (a.cap_in != 0.f || a.slopes) {
    // to scores in log2 units, the cap's factor taken along
    c = 1.f;
    if (a.cap_in != 0.f) {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        float slope;
        s[v] = capped<T>(a, s[v], slope);
        dp[v] *= slope;
      }
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[v] *= a.c;
    }
    if (a.slopes)
      unrolled<4>([&](auto quad) {
        constexpr int q = decltype(quad)::value;
        const f32x4 m = slope2(q), f = far(q);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * q + i] -= m[i] * f[i];
        __builtin_amdgcn_sched_barrier(0);
      });
  }
  unrolled<4>([&](auto quad) {
    constexpr int q = decltype(quad)::value;
    const f32x4 l = lse2(q);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[4 * q + i] = exp2_hw(fmaf(s[4 * q + i], c, -l[i]));
      dp[4 * q + i] *= s[4 * q + i];
    }
  });
}
// the hidden ones (cleared bits of vis) are zero, whatever their operands held
__device__ __forceinline__ void hide(f32x16& s, f32x16& dp, unsigned vis) {
#pragma unroll
  for (int v = 0; v < 16; ++v) {
    const bool on = (vis >> v) & 1;
    s[v] = on ? s[v] : 0.f;
    dp[v] = on ? dp[v] : 0.f;
  }
}

// delta, and lse in units of log2; a row that sees nothing (lse = -inf) gets weights 0 through inf.
// fp16: p is formed times 2^14, as in the forward pass (its offset is in lse2).  ds, whose size is that of the gradient,
// is multiplied by a power of two that follows the lane's largest so far, as the running maximum of a softmax does; the sums of
// the lane change with it.
template <class T>
constexpr bool kIsF16 = std::is_same_v<T, _Float16>;
constexpr float kDsTop = 16384.f;         // a quarter of the largest fp16

template <class T, int N>
struct DsScale {
  float mul = kIsF16<T> ? 0x1p100f : 1.f;
  __device__ __forceinline__ void apply(f32x16& ds, f32x16 (&acc)[N]) {
    if constexpr (kIsF16<T>) {
      float top = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) top = fmaxf(top, fabsf(ds[v]));
      top = half_max(top);
      if (__any(top * mul > kDsTop)) {
        // 2^14 over the power of two above top (inf counts as 2^127)
        const int e = min((int)(__float_as_uint(top) >> 23) - 127 + 1, 127);
        const float to = top * mul > kDsTop ? __uint_as_float((uint32_t)(14 - e + 127) << 23) : mul, f = to / mul;
        mul = to;
#pragma unroll
        for (int d = 0; d < N; ++d)
#pragma unroll
          for (int v = 0; v < 16; ++v) acc[d][v] *= f;
      }
#pragma unroll
      for (int v = 0; v < 16; ++v) ds[v] *= mul;
    }
  }
  // what the sums are multiplied by at the end
  __device__ __forceinline__ float undo() const { return kWeightOne<T> / mul; }
};

// With heads of 128 the wave that multiplies into dq, dk or dv goes before the other one of its SIMD (2 x 16 heads over 8,
// 4096 positions: 924 us a backward pass against 990, 600 against 634-666 causal).  Heads of 64 gain nothing, nor does
// the forward kernel.
template <int DP>
__device__ __forceinline__ void multiply_first(int on) {
  if constexpr (DP == 128) {
    if (on)
      __builtin_amdgcn_s_setprio(1);
    else
      __builtin_amdgcn_s_setprio(0);
  }
}

template <class T, bool VEC>
__global__ void __launch_bounds__(256) k_attn_delta(const AttnArgs a, float* __restrict__ lse2, float* __restrict__ delta,
                                                    long long rows) {
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
  if constexpr (VEC) {
    constexpr int EC = 16 / (int)sizeof(T);
    for (int d = lane * EC; d < a.D; d += 16 * EC) {
      const uint4 uo = *reinterpret_cast<const uint4*>(o + d), ug = *reinterpret_cast<const uint4*>(g + d);
      T x[EC], y[EC];
      __builtin_memcpy(x, &uo, 16);
      __builtin_memcpy(y, &ug, 16);
#pragma unroll
      for (int i = 0; i < EC; ++i) s = fmaf((float)x[i], (float)y[i], s);
    }
  } else {
    for (int d = lane; d < a.D; d += 16) s = fmaf((float)o[d], (float)g[d], s);
  }
#pragma unroll
  for (int w = 8; w; w >>= 1) s += __shfl_xor(s, w);
  if (lane) return;
  const long long at = ((long long)b * a.H + head) * a.Sq + i;
  const float l = a.lse[at];
  const bool empty = l == -__builtin_inff();
  lse2[at] = empty ? __builtin_inff() : l * kLog2e - kWeightBits<T>;
  delta[at] = empty ? 0.f : s;
}

// ---- dq: four waves of 32 rows over the key tiles -----------------------------------------------------
// The forward kernel's plan with a third product.  bf16, 2 x 16 heads over 8 of 128, 4096 positions, causal: 210 us,
// 982 TFLOP/s of its three products.
template <class T>
constexpr int kBwdKeys = sizeof(T) == 2 ? 64 : 32;
constexpr int kBwdRows = 128;

template <class T, int DP, bool VEC, bool CAREFUL>
__device__ __forceinline__ bool dq_body(const AttnArgs& a, char* smem, int block) {
  constexpr int BN = kBwdKeys<T>, KT = DP / 16, DB = DP / 32;
  using N = Num<T>;
  using Tile = AttnTile<T, DP>;
  using Frag = typename N::Frag;
  using Load = AttnLoad<T, DP, BN, 4, VEC>;
  char* sk = smem;
  char* sv = smem + 2 * Load::BYTES;
  int* sids = reinterpret_cast<int*>(smem + 4 * Load::BYTES);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int bh, item;
  place(block, a.B * a.Hk, bh, item);
  const int split = item % a.splits, mt = a.tiles - 1 - item / a.splits;   // the rows that see most keys first
  const int hk = bh % a.Hk, b = bh / a.Hk;
  const AttnScope sc(a, b);
  const int r0 = mt * kBwdRows, r = r0 + wave * 32 + (lane & 31), rc = min(r, a.R - 1);
  const int i = (int)a.gdiv.div((uint32_t)rc), head = hk * a.G + rc - i * a.G;
  const int* docs = a.docs ? a.docs + (long long)b * a.Sk : nullptr;
  const int pos = sc.off + i;
  const int doc = docs && pos >= 0 ? docs[pos] : 0;
  const bool one = __all(doc >= 0 && doc == __builtin_amdgcn_readfirstlane(doc));   // this wave's rows: one document
  const int klim = doc < 0 ? 0 : sc.klim(pos);
  const float slope2 = a.slopes ? a.slopes[head] * kLog2e : 0.f;
  const long long stat = ((long long)b * a.H + head) * a.Sq + i;
  const float lse2 = a.lse2[stat];
  const float delta = a.delta[stat];
  Frag q[KT], g[KT];
  load_owned<T, DP, VEC>((const T*)a.q.p + b * a.q.sb + i * a.q.ss + head * a.q.sh, r < a.R, a.D, lane, q);
  load_owned<T, DP, VEC>((const T*)a.dout.p + b * a.dout.sb + i * a.dout.ss + head * a.dout.sh, r < a.R, a.D, lane, g);

  const int p_lo = sc.off + (int)a.gdiv.div((uint32_t)r0);
  const int p_hi = sc.off + (int)a.gdiv.div((uint32_t)(min(r0 + kBwdRows, a.R) - 1));
  const int all = sc.klim(p_lo), any = sc.klim(p_hi);
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

  typename Tile::Lane tl(lane);
  f32x16 acc[DB];
  DsScale<T, DB> dscale;
  auto pass = [&](auto careful) {
#pragma unroll
    for (int d = 0; d < DB; ++d) zero16(acc[d]);
    dscale = {};
    int t = kt.from(kt.t0), st = 0, nid = -1;
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
      const int tn = kt.from(t + 1);
      if (tn < kt.t1) issue(tn, st ^ 1);
      const bool masked = (t + 1) * BN > all || (docs && !(one && __all(sids[st * BN + lane % BN] == doc)));
      tl.fresh();
      const char *k_ = sk + st * Load::BYTES, *v_ = sv + st * Load::BYTES;
      typename Tile::Cols cols;
      cols.set(k_, tl);
      unrolled<BN / 32>([&](auto block) {
        constexpr int nb = decltype(block)::value;
        f32x16 s, dp;
        zero16(s);
        zero16(dp);
#pragma unroll
        for (int x = 0; x < KT; ++x) {
          s = N::template product<CAREFUL>(Tile::rows(k_, 32 * nb, x, tl), q[x], s);
          dp = N::template product<CAREFUL>(Tile::rows(v_, 32 * nb, x, tl), g[x], dp);
          if (x % 2) __builtin_amdgcn_sched_barrier(0);
        }
        const int h4 = 4 * (lane >> 5), base = t * BN + 32 * nb + h4;
        unsigned vis = 0xffffu;
        if (masked) {
#pragma unroll
          for (int v = 0; v < 16; ++v)
            if (base + 8 * (v >> 2) + (v & 3) >= klim) vis &= ~(1u << v);
          if (docs) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const i32x4 id = *reinterpret_cast<const i32x4*>(sids + st * BN + 32 * nb + h4 + 8 * q);
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (id[i] != doc) vis &= ~(1u << (4 * q + i));
            }
          }
        }
        auto same = [](float x) { return f32x4{x, x, x, x}; };
        weights<T>(a, s, dp, [&](int) { return same(lse2); }, [&](int) { return same(delta); }, [&](int) { return same(slope2); },
                   [&](int q) {
                     f32x4 f;
#pragma unroll
                     for (int i = 0; i < 4; ++i) f[i] = (float)abs(pos - (base + 8 * q + i));
                     return f;
                   });
        if (masked) hide(s, dp, vis);
        dscale.apply(dp, acc);
        multiply_first<DP>(1);
        unrolled<2>([&](auto step) {
          constexpr int u = decltype(step)::value;
          const Frag w = to_frag<T>(dp, u);
          if constexpr (decltype(careful)::value) {
            Frag on;
#pragma unroll
            for (int e = 0; e < 8; ++e) on[e] = (T)((vis >> (8 * u + e)) & 1 ? 1.f : 0.f);
            unrolled<DB>([&](auto db) {
              constexpr int d = decltype(db)::value;
              acc[d] = mma_visible<T, false>(cols.template read_one<32 * nb + 16 * u, d>(tl), w, on, acc[d]);
            });
          } else {
            Frag kc[DB];
            cols.template read<32 * nb + 16 * u>(kc, tl);
#pragma unroll
            for (int d = 0; d < DB; ++d) acc[d] = N::mma(kc[d], w, acc[d]);
          }
        });
        multiply_first<DP>(0);
      });
      if (docs && tn < kt.t1 && tid < BN) sids[(st ^ 1) * BN + tid] = nid;
      t = tn;
      st ^= 1;
    }
  };
  pass(std::integral_constant<bool, CAREFUL>{});
  if (!CAREFUL && __syncthreads_or(not_finite(acc))) return true;
  if (r >= a.R) return false;
  if (a.splits > 1)
    store_owned<float, DP, true>(a.part + (((long long)split * a.B * a.Hk + (long long)b * a.Hk + hk) * a.R + r) * DP, DP, lane, acc, dscale.undo());
  else
    store_owned<T, DP, VEC>((T*)a.dq.p + b * a.dq.sb + i * a.dq.ss + head * a.dq.sh, a.D, lane, acc, a.scale * dscale.undo());
  return false;
}
template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) k_attn_dq(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  const bool bad = dq_body<T, DP, VEC, false>(a, smem, blockIdx.x);
  if (threadIdx.x == 0) a.flags[blockIdx.x] = bad;
}

// ---- dk, dv: four waves of 32 keys over the row tiles -----------------------------------------------------
// A wave's keys stay in registers and its values in LDS: with both in registers (and dk, dv in 128 more) only one
// wave a SIMD would fit, and nothing would run beside its MFMAs.  The loop is written to need no more than 256
// registers: a reload from scratch memory would wait for the next tile's loads too.  The same sizes as dq's: 365 us, 750
// TFLOP/s of the four products (in full 650 us, 850), and 32 more for the sums of two ranges.  Counters: the matrix cores are busy
// 39 % of the time (42 % in full), the vector units 41 %, LDS 30 % with no bank conflict, and the compute units throughout; so it is
// two waves a SIMD that mostly take turns that bound it, neither LDS nor the unequal work of the causal order.  dk and dv in
// workgroups of their own, with one product more, took 520 where this took 440.
constexpr int kBwdRowTile = 32;
constexpr int kBwdKeyTile = 128;

// What a tile of rows brings along, in LDS.
struct RowStats {
  float lse2[64], delta[64];         // a wave's worth: loaded straight into LDS, the first kBwdRowTile count
  float slope2[kBwdRowTile];
  int klim[kBwdRowTile], pos[kBwdRowTile], doc[kBwdRowTile];
};

template <class T, int DP, bool VEC, bool CAREFUL>
__device__ __forceinline__ bool dkv_body(const AttnArgs& a, char* smem, int block) {
  constexpr int BR = kBwdRowTile, KT = DP / 16, DB = DP / 32;
  using N = Num<T>;
  using Tile = AttnTile<T, DP>;
  using Frag = typename N::Frag;
  using Load = AttnLoad<T, DP, BR, 4, VEC>;
  using LoadV = AttnLoad<T, DP, kBwdKeyTile, 4, VEC>;
  char* sq = smem;                                   // [2][BR][DP]
  char* sg = smem + 2 * Load::BYTES;
  char* sv = smem + 4 * Load::BYTES;                 // [128][DP]
  RowStats* stats = reinterpret_cast<RowStats*>(sv + LoadV::BYTES);   // [2]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  int bh, item;
  place(block, a.B * a.Hk, bh, item);
  const int split = item % a.splits, k0 = item / a.splits * kBwdKeyTile;   // the keys that most rows see first
  const int hk = bh % a.Hk, b = bh / a.Hk;
  const AttnScope sc(a, b);
  const int j = k0 + wave * 32 + (lane & 31), jc = min(j, a.Sk - 1);
  const int* docs = a.docs ? a.docs + (long long)b * a.Sk : nullptr;
  const bool live = j < sc.len;
  const int doc = docs ? (live ? docs[jc] : -1) : 0;
  Frag k[KT];
  load_owned<T, DP, VEC>((const T*)a.k.p + b * a.k.sb + jc * a.k.ss + hk * a.k.sh, live, a.D, lane, k);
  if (k0 < sc.len)
    LoadV::positions((const T*)a.v.p + b * a.v.sb + hk * a.v.sh, a.v.ss, k0, sc.len, a.D, sv, wave, lane);

  // the first query that sees one of the keys: positions below 0 do not exist
  int i0 = max(0, -sc.off);
  if (sc.causal && sc.prefix <= k0) i0 = max(i0, k0 - sc.off);
  const int all_t = k0 < sc.len && i0 < a.Sq ? (a.R + BR - 1) / BR : 0;
  const int first = min((int)((long long)i0 * a.G / BR), all_t), per = (all_t - first + a.splits - 1) / a.splits;
  TileList rt;
  rt.t0 = __builtin_amdgcn_readfirstlane(first + split * per);
  rt.t1 = __builtin_amdgcn_readfirstlane(min(all_t, first + split * per + per));
  rt.words = nullptr;
  if (docs) {
    __shared__ unsigned long long words[kDocWords];
    int lo, hi;                                       // the keys' documents
    doc_range(docs, k0, min(k0 + kBwdKeyTile, sc.len) - 1, lane, lo, hi);
    rt.find(words, 4, wave, lane, lo, hi, [&](int t) {
      const int r = t * BR + lane, p = sc.off + (int)a.gdiv.div((uint32_t)min(r, a.R - 1)), d = docs[max(p, 0)];
      return lane < BR && r < a.R && p >= 0 ? d : -1;
    });
    __syncthreads();
  }

  const long long stat = ((long long)b * a.H + (long long)hk * a.G) * a.Sq;   // [group][q_len] of this head

  typename Tile::Lane tl(lane);
  f32x16 dk[DB], dv[DB];
  DsScale<T, DB> dscale;
  auto pass = [&](auto careful) {
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      zero16(dk[d]);
      zero16(dv[d]);
    }
    dscale = {};
    auto issue = [&](const AttnArgs& a, int t, int st) {
      int lane = tid & 63;
      asm volatile("" : "+v"(lane));   // the places are formed here, not held over the products
      const T* qh = (const T*)a.q.p + b * a.q.sb + (long long)hk * a.G * a.q.sh;
      const T* gh = (const T*)a.dout.p + b * a.dout.sb + (long long)hk * a.G * a.dout.sh;
      Load::packed(qh, a.q.ss, a.q.sh, t * BR, a.R, a.gdiv, a.D, sq + st * Load::BYTES, wave, lane);
      Load::packed(gh, a.dout.ss, a.dout.sh, t * BR, a.R, a.gdiv, a.D, sg + st * Load::BYTES, wave, lane);
      if (wave == 0) {   // rows past the last read zeros, and see no key
        const int r = t * BR + lane, i = (int)a.gdiv.div((uint32_t)r), g = r - i * a.G;
        const uint32_t off = lane < BR && r < a.R ? (uint32_t)((g * a.Sq + i) * 4) : 0x80000000u;
        buffer_dma4(buffer_rsrc(a.lse2 + stat, (uint32_t)a.R * 4u), off, stats[st].lse2);
        buffer_dma4(buffer_rsrc(a.delta + stat, (uint32_t)a.R * 4u), off, stats[st].delta);
      }
    };
    // what only masks and slopes ask for, formed after the tile before
    auto keep = [&](const AttnArgs& a, int t, int st) {
      if (tid < BR) {
        const int rc = min(t * BR + tid, a.R - 1), i = (int)a.gdiv.div((uint32_t)rc), pos = sc.off + i;
        const int d = docs && pos >= 0 ? docs[pos] : 0;
        stats[st].slope2[tid] = a.slopes ? a.slopes[hk * a.G + rc - i * a.G] * kLog2e : 0.f;
        stats[st].klim[tid] = d >= 0 && t * BR + tid < a.R ? sc.klim(pos) : 0;
        stats[st].pos[tid] = pos;
        stats[st].doc[tid] = d;
      }
    };
    int t = rt.from(rt.t0), st = 0;
    if (t < rt.t1) {
      issue(a, t, 0);
      keep(a, t, 0);
    }
    while (t < rt.t1) {
      __builtin_amdgcn_s_waitcnt(0x0070);
      __syncthreads();
      const AttnArgs& a = args_again();
      const int tn = rt.from(t + 1);
      if (tn < rt.t1) issue(a, tn, st ^ 1);
      const int p_first = sc.off + (int)a.gdiv.div((uint32_t)(t * BR));
      // rows past the last have operands of zeros, but a weight that is not finite would make them NaN
      const bool masked = docs || k0 + kBwdKeyTile > sc.klim(p_first) || (t + 1) * BR > a.R;
      tl.fresh();
      const char *q_ = sq + st * Load::BYTES, *g_ = sg + st * Load::BYTES;
      const RowStats& rs = stats[st];
      f32x16 s, dp;
      zero16(s);
      zero16(dp);
#pragma unroll
      for (int x = 0; x < KT; ++x) {
        s = N::template product<CAREFUL>(Tile::rows(q_, 0, x, tl), k[x], s);
        dp = N::template product<CAREFUL>(Tile::rows(g_, 0, x, tl), Tile::rows(sv, 32 * wave, x, tl), dp);
        if (x % 2) __builtin_amdgcn_sched_barrier(0);   // no more fragments in flight than the accumulators leave room for
      }
      const int rr = 4 * (lane >> 5);
      auto four = [&](const float* x, int q) { return *reinterpret_cast<const f32x4*>(x + rr + 8 * q); };
      auto four_i = [&](const int* x, int q) { return *reinterpret_cast<const i32x4*>(x + rr + 8 * q); };
      weights<T>(a, s, dp, [&](int q) { return four(rs.lse2, q); }, [&](int q) { return four(rs.delta, q); },
                 [&](int q) { return four(rs.slope2, q); },
                 [&](int q) {
                   const i32x4 p = four_i(rs.pos, q);
                   f32x4 f;
#pragma unroll
                   for (int i = 0; i < 4; ++i) f[i] = (float)abs(p[i] - j);
                   return f;
                 });
      unsigned vis = 0xffffu;
      if (masked) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const i32x4 lim = four_i(rs.klim, q), id = four_i(rs.doc, q);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (j >= lim[i] || (docs && id[i] != doc)) vis &= ~(1u << (4 * q + i));
          __builtin_amdgcn_sched_barrier(0);
        }
        hide(s, dp, vis);
      }
      constexpr int GQ = 2 * Load::BYTES;                // from the tile of q to that of dout
      typename Tile::Cols qcols;
      qcols.set(q_, tl);
      dscale.apply(dp, dk);
      const Frag pf[2] = {to_frag<T>(s, 0), to_frag<T>(s, 1)}, wf[2] = {to_frag<T>(dp, 0), to_frag<T>(dp, 1)};
      __builtin_amdgcn_sched_barrier(0);
      multiply_first<DP>(1);
      unrolled<2>([&](auto step) {
        constexpr int u = decltype(step)::value;
        const Frag p = pf[u], w = wf[u];
        if constexpr (decltype(careful)::value) {
          Frag on;
#pragma unroll
          for (int e = 0; e < 8; ++e) on[e] = (T)((vis >> (8 * u + e)) & 1 ? 1.f : 0.f);
          unrolled<DB>([&](auto db) {
            constexpr int d = decltype(db)::value;
            dv[d] = mma_visible<T, true>(qcols.template read_one<16 * u, d, GQ>(tl), p, on, dv[d]);
            dk[d] = mma_visible<T, false>(qcols.template read_one<16 * u, d>(tl), w, on, dk[d]);
          });
        } else {
          Frag gc[DB], qc[DB];
          qcols.template read<16 * u, GQ>(gc, tl);
#pragma unroll
          for (int d = 0; d < DB; ++d) dv[d] = N::mma(gc[d], p, dv[d]);
          __builtin_amdgcn_sched_barrier(0);   // these products run while the next fragments are read
          qcols.template read<16 * u>(qc, tl);
#pragma unroll
          for (int d = 0; d < DB; ++d) dk[d] = N::mma(qc[d], w, dk[d]);
          __builtin_amdgcn_sched_barrier(0);
        }
      });
      multiply_first<DP>(0);
      if (tn < rt.t1) keep(a, tn, st ^ 1);
      t = tn;
      st ^= 1;
    }
  };
  pass(std::integral_constant<bool, CAREFUL>{});
  if (!CAREFUL && __syncthreads_or(not_finite(dk) || not_finite(dv))) return true;
  if (j >= a.Sk) return false;
  if (a.splits > 1) {
    const long long keys = (long long)a.B * a.Hk * a.Sk, row = (long long)bh * a.Sk + j;
    store_owned<float, DP, true>(a.part + ((long long)split * keys + row) * DP, DP, lane, dk, dscale.undo());
    store_owned<float, DP, true>(a.part + ((long long)(a.splits + split) * keys + row) * DP, DP, lane, dv, kWeightOne<T>);
    return false;
  }
  // keys past the batch entry's length get zeros
  store_owned<T, DP, VEC>((T*)a.dk.p + b * a.dk.sb + j * a.dk.ss + hk * a.dk.sh, a.D, lane, dk, a.scale * dscale.undo());
  store_owned<T, DP, VEC>((T*)a.dv.p + b * a.dv.sb + j * a.dv.ss + hk * a.dv.sh, a.D, lane, dv, kWeightOne<T>);
  return false;
}
template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) k_attn_dkv(const AttnArgs a) {
  extern __shared__ __align__(1024) char smem[];
  const bool bad = dkv_body<T, DP, VEC, false>(a, smem, blockIdx.x);
  if (threadIdx.x == 0) a.flags[blockIdx.x] = bad;
}

template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(256, 1) k_attn_dq_again(const AttnArgs a, int blocks) {
  extern __shared__ __align__(1024) char smem[];
  again(a.flags, blocks, [&](int id) { dq_body<T, DP, VEC, true>(a, smem, id); });
}
template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(256, 1) k_attn_dkv_again(const AttnArgs a, int blocks) {
  extern __shared__ __align__(1024) char smem[];
  again(a.flags, blocks, [&](int id) { dkv_body<T, DP, VEC, true>(a, smem, id); });
}

// ---- the ranges' partial sums, added in order -------------------------------------------------------------
// y[row] = f sum_s part[s][row]; a row is a position of a key/value head (gdiv.d = 1), or a packed query row.
template <class T, int DP>
__global__ void __launch_bounds__(256) k_attn_sum(const float* __restrict__ part, AttnView y, FastDiv gdiv, int heads, int per_head,
                                                  long long rows, int D, int splits, float f) {
  constexpr int TPR = DP / 4;
  const long long row = (long long)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  if (row >= rows) return;
  const int d = (threadIdx.x % TPR) * 4;
  f32x4 x = *reinterpret_cast<const f32x4*>(part + row * DP + d);
#pragma unroll 4
  for (int s = 1; s < splits; ++s) {
    const f32x4 z = *reinterpret_cast<const f32x4*>(part + ((long long)s * rows + row) * DP + d);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] += z[i];
  }
  const long long bh = row / per_head;
  const int r = (int)(row - bh * per_head), hk = (int)(bh % heads), b = (int)(bh / heads);
  const int i = (int)gdiv.div((uint32_t)r), head = hk * (int)gdiv.d + r - i * (int)gdiv.d;
  T* o = (T*)y.p + b * y.sb + i * y.ss + head * y.sh;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (d + e < D) o[d + e] = (T)(x[e] * f);
}

template <class T, int DP>
hipError_t run_sum(hipStream_t s, const AttnArgs& a, const float* part, const AttnView& y, const FastDiv& g, int per_head, int splits,
                   float f) {
  const long long rows = (long long)a.B * a.Hk * per_head;
  constexpr int rpb = 256 / (DP / 4);
  k_attn_sum<T, DP><<<dim3((unsigned)((rows + rpb - 1) / rpb)), dim3(256), 0, s>>>(part, y, g, a.Hk, per_head, rows, a.D, splits, f);
  return hipGetLastError();
}

// `k` on `blocks` workgroups, then `k_again` on those it flagged
template <class K, class A>
hipError_t run_twice(hipStream_t s, const AttnArgs& a, K k, A k_again, int bytes, int blocks) {
  hipError_t e = hipFuncSetAttribute((const void*)k, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) e = hipFuncSetAttribute((const void*)k_again, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  k<<<dim3(blocks), dim3(256), bytes, s>>>(a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  k_again<<<dim3(std::min(blocks, kAgainBlocks)), dim3(256), bytes, s>>>(a, blocks);
  return hipGetLastError();
}

template <class T, int DP, bool VEC>
hipError_t run_bwd(hipStream_t s, AttnArgs& a, const AttnBwdPlan& plan) {
  if (plan.dq_tiles) {
    constexpr int bytes = 4 * AttnLoad<T, DP, kBwdKeys<T>, 4, VEC>::BYTES + 2 * kBwdKeys<T> * 4;
    a.tiles = plan.dq_tiles;
    a.splits = plan.dq_splits;
    hipError_t e = run_twice(s, a, k_attn_dq<T, DP, VEC>, k_attn_dq_again<T, DP, VEC>, bytes, a.B * a.Hk * a.tiles * a.splits);
    if (e == hipSuccess && a.splits > 1) e = run_sum<T, DP>(s, a, a.part, a.dq, a.gdiv, a.R, a.splits, a.scale);
    if (e != hipSuccess) return e;
  }
  if (plan.dkv_tiles) {
    constexpr int bytes = 4 * AttnLoad<T, DP, kBwdRowTile, 4, VEC>::BYTES + AttnLoad<T, DP, kBwdKeyTile, 4, VEC>::BYTES + 2 * (int)sizeof(RowStats);
    a.tiles = plan.dkv_tiles;
    a.splits = plan.dkv_splits;
    hipError_t e = run_twice(s, a, k_attn_dkv<T, DP, VEC>, k_attn_dkv_again<T, DP, VEC>, bytes, a.B * a.Hk * a.tiles * a.splits);
    if (e == hipSuccess && a.splits > 1) {
      const FastDiv one(1);
      e = run_sum<T, DP>(s, a, a.part, a.dk, one, a.Sk, a.splits, a.scale);
      if (e == hipSuccess) e = run_sum<T, DP>(s, a, a.part + (long long)a.splits * a.B * a.Hk * a.Sk * DP, a.dv, one, a.Sk, a.splits, 1.f);
    }
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class T>
hipError_t run_bwd_dim(hipStream_t s, AttnArgs& a, const AttnBwdPlan& plan, float* work, bool vec) {
  const long long rows = (long long)a.B * a.Sq * a.H;
  float* lse2 = work + plan.part_floats;
  float* delta = lse2 + rows;
  const dim3 grid((unsigned)((rows + 15) / 16));
  if (rows && vec) k_attn_delta<T, true><<<grid, dim3(256), 0, s>>>(a, lse2, delta, rows);
  if (rows && !vec) k_attn_delta<T, false><<<grid, dim3(256), 0, s>>>(a, lse2, delta, rows);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.lse2 = lse2;
  a.delta = delta;
  a.part = work;
  a.flags = reinterpret_cast<int*>(delta + rows);   // one after the other on the stream
  if (a.D <= 64) return vec ? run_bwd<T, 64, true>(s, a, plan) : run_bwd<T, 64, false>(s, a, plan);
  return vec ? run_bwd<T, 128, true>(s, a, plan) : run_bwd<T, 128, false>(s, a, plan);
}

// Ranges of the summed axis: where the tiles are too few for two workgroups on each of 256 compute units, the axis is cut
// into as many ranges as make 512 of them, of at least 256 keys or rows (64 in fp32, whose products take several
// times as long).  fp32 keeps one workgroup a compute unit busy, but in shorter ranges the causal tiles' unequal work
// evens out: half as many made dk and dv of 2 x 8 heads over 2, 513 positions of 64, a quarter slower.
int ranges(long long blocks, long long axis, int dtype) {
  if (blocks >= 256) return 1;   // the partial sums' traffic would cost more than it gains
  return (int)std::max(1LL, std::min(512 / blocks, axis / (dtype == 0 ? 64 : 256)));
}

}  // namespace

AttnBwdPlan attn_plan_bwd(int dtype, int B, int Hk, int R, int Sk, int D, bool causal) {
  AttnBwdPlan p{};
  const int dp = D <= 64 ? 64 : 128;
  const long long bh = (long long)B * Hk;
  p.dq_splits = p.dkv_splits = 1;
  if (bh == 0) return p;
  p.dq_tiles = (R + kBwdRows - 1) / kBwdRows;
  p.dkv_tiles = (Sk + kBwdKeyTile - 1) / kBwdKeyTile;
  if (p.dq_tiles) p.dq_splits = ranges(bh * p.dq_tiles, Sk, dtype);
  if (p.dkv_tiles) p.dkv_splits = ranges(bh * p.dkv_tiles, R, dtype);
  // A causal tile's work falls with its place: where all workgroups run at once the first ones last twice as long as
  // the mean.  Halved, they leave room that others fill (2 x 16 heads over 8, 4096 positions of 128: 467 us with the sums' addition against
  // 626).  Measured at this size; the traffic of the sums, which short rows feel most, is not weighed against it.
  if (causal && p.dkv_splits == 1 && bh * p.dkv_tiles < 2048 && p.dkv_tiles > 2) p.dkv_splits = 2;
  const long long dq = p.dq_splits > 1 ? p.dq_splits * bh * R * dp : 0, dkv = p.dkv_splits > 1 ? 2 * p.dkv_splits * bh * Sk * dp : 0;
  p.flag_ints = bh * std::max(p.dq_tiles * p.dq_splits, p.dkv_tiles * p.dkv_splits);
  p.part_floats = std::max(dq, dkv);   // one after the other on the stream
  return p;
}

hipError_t launch_attn_bwd(hipStream_t s, int dtype, AttnArgs& a, const AttnBwdPlan& plan, float* work, bool vec) {
  if (dtype == 1) return run_bwd_dim<__bf16>(s, a, plan, work, vec);
  if (dtype == 2) return run_bwd_dim<_Float16>(s, a, plan, work, vec);
  return run_bwd_dim<float>(s, a, plan, work, vec);
}

}  // namespace ntk

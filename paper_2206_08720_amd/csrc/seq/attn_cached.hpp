// attn_cached.hpp -- attention over a cache of pages (kernels_cached.hip, kernels_cached_e4m3.hip).
//
// The forward pass of kernels_attn.hip, o = softmax(mask(score(q k^T))) v with a running maximum, with keys and values read through
// a table of pages.  What differs is how a tile comes into LDS: a row's place follows from its page, read one tile ahead, and is
// a 64-bit address of its own (a cache may be larger than a buffer resource spans).  Rows past the sequence's end read
// zeros, rows on a page that the cache does not have NaN.
//
// A cache in 8 bits is read into registers, converted there (one instruction takes two e4m3 values and their page's power of two to
// two values of the queries' type), and written into the same tiles, so that the products are the same ones.
#pragma once
#include "attn_fwd.hpp"
#include "launch_cache.hpp"

namespace ntk {

struct CachedArgs : AttnArgs {             // k, v: sb from page to page, ss from slot to slot, sh from head to head
  PageTable pages;
  const int* q_lens;                       // [batch] or null
  const float *k_scale, *v_scale;          // [pages, kv_heads]: the cache is e4m3
};

namespace {

__device__ const uint4 kZeros = {0, 0, 0, 0};
__device__ const uint4 kNaNs = {~0u, ~0u, ~0u, ~0u};   // NaN in every type, e4m3 among them

// What a batch entry's queries see, as AttnScope: its first `queries` rows are the last of its `len` positions.
struct CachedScope {
  int len, off, queries, causal;
  __device__ __forceinline__ CachedScope(const CachedArgs& a, int b) {
    len = min(max(a.lens[b], 0), a.Sk);
    queries = a.q_lens ? min(max(a.q_lens[b], 0), a.Sq) : a.Sq;
    off = len - queries;
    causal = a.causal;
  }
  __device__ __forceinline__ int klim(int i) const {     // keys below it are seen by query i
    const int pos = off + i;
    return i >= queries || pos < 0 ? 0 : causal ? pos + 1 : len;
  }
  // keys that every one of the queries i0 .. i1 sees, and that some one does
  __device__ __forceinline__ int all(int i0, int i1) const { return min(klim(i0), klim(i1)); }
  __device__ __forceinline__ int any(int i0, int i1) const { return i0 < queries ? klim(min(i1, queries - 1)) : 0; }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// four e4m3 bytes times a power of two
template <class T>
__device__ __forceinline__ void from_e4m3(uint32_t w, float s, T (&y)[4]) {
  if constexpr (std::is_same_v<T, __bf16>) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true);
    y[0] = a[0], y[1] = a[1], y[2] = b[0], y[3] = b[1];
  } else if constexpr (std::is_same_v<T, _Float16>) {
    const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, true);
    y[0] = a[0], y[1] = a[1], y[2] = b[0], y[3] = b[1];
  } else {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, s, true);
    y[0] = a[0], y[1] = a[1], y[2] = b[0], y[3] = b[1];
  }
}

// ROWS positions of one head into an LDS tile of AttnTile's layout, by WAVES waves.  A lane's `NI` chunks of 16 bytes (of the cache)
// lie in rows of the tile that do not change, so their pages are looked up one tile ahead (look).
template <class T, int DP, int ROWS, int WAVES, bool VEC, bool E4M3>
struct PageLoad {
  using Tile = AttnTile<T, DP>;
  static constexpr int CE = E4M3 ? 1 : (int)sizeof(T);           // bytes an element of the cache
  static constexpr int CH = DP * CE / 16, EC = 16 / CE;         // chunks a row, elements a chunk
  static constexpr int BYTES = ROWS * Tile::RB;
  static constexpr int NI = (ROWS * CH + 64 * WAVES - 1) / (64 * WAVES);
  static constexpr bool EVEN = NI * 64 * WAVES == ROWS * CH;    // else some lanes have none (row >= ROWS)
  static_assert(EVEN || E4M3, "chunks split over the lanes");
  struct Where {
    int page[NI];                          // -1: none, -2: past the end
  };
  struct Held {                            // 8 bits: a tile on its way
    uint4 x[NI];
    float s[NI];
  };
  __device__ static __forceinline__ void place(int i, int wave, int lane, int& row, int& chunk) {
    const int o = (i * WAVES + wave) * 64 + lane;
    row = o / CH;
    chunk = o % CH;
    if constexpr (!E4M3) chunk ^= Tile::swz(row);               // straight into LDS: lane l's 16 bytes go to place l
  }
  __device__ static __forceinline__ void look(const CachedArgs& a, int b, int tile0, int len, int wave, int lane, Where& w) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int row, c;
      place(i, wave, lane, row, c);
      w.page[i] = tile0 + row < len && (EVEN || row < ROWS) ? a.pages.page(b, tile0 + row) : -2;
    }
  }
  __device__ static __forceinline__ const char* at(const AttnView& v, const PageTable& t, int hk, int pos, int page) {
    return (const char*)v.p + ((long long)page * v.sb + (long long)t.slot(pos) * v.ss + (long long)hk * v.sh) * CE;
  }
  // the cache in the queries' type: into LDS
  __device__ static __forceinline__ void rows(const CachedArgs& a, const AttnView& v, int hk, int tile0, const Where& w, char* lds, int wave,
                                              int lane) {
    static_assert(!E4M3, "");
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int row, c;
      place(i, wave, lane, row, c);
      const int page = w.page[i];
      const char* p = at(v, a.pages, hk, tile0 + row, max(page, 0));
      if constexpr (VEC) {
        const char* from = page >= 0 && c * EC < a.D ? p + c * 16 : page == -1 ? (const char*)&kNaNs : (const char*)&kZeros;
        typedef const __attribute__((address_space(1))) void G;
        typedef __attribute__((address_space(3))) void L;
        __builtin_amdgcn_global_load_lds((G*)from, (L*)(lds + __builtin_amdgcn_readfirstlane((i * WAVES + wave) * 1024)), 16, 0, 0);
      } else {
        uint4 u = page == -1 ? kNaNs : kZeros;
        if (page >= 0) u = load_chunk_elems((const T*)p, c * EC, a.D);
        *reinterpret_cast<uint4*>(lds + ((i * WAVES + wave) * 64 + lane) * 16) = u;
      }
    }
  }
  // the cache in 8 bits: into registers, and from there into LDS
  __device__ static __forceinline__ void fetch(const CachedArgs& a, const AttnView& v, const float* scale, int hk, int tile0, const Where& w,
                                               int wave, int lane, Held& h) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int row, c;
      place(i, wave, lane, row, c);
      const int page = w.page[i];
      const char* p = at(v, a.pages, hk, tile0 + row, max(page, 0));
      h.s[i] = page >= 0 ? scale[(long long)page * a.Hk + hk] : 1.f;
      if constexpr (VEC) {
        const char* from = page >= 0 && c * EC < a.D ? p + c * 16 : page == -1 ? (const char*)&kNaNs : (const char*)&kZeros;
        h.x[i] = *reinterpret_cast<const uint4*>(from);
      } else {
        uint32_t u[4] = {0, 0, 0, 0};
        if (page == -1) u[0] = u[1] = u[2] = u[3] = ~0u;
        if (page >= 0)
#pragma unroll
          for (int k = 0; k < 16; ++k)
            if (c * EC + k < a.D) u[k / 4] |= (uint32_t)(uint8_t)p[c * EC + k] << (8 * (k % 4));
        h.x[i] = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
  }
  __device__ static __forceinline__ void put(const Held& h, char* lds, int wave, int lane) {
    constexpr int TC = (int)sizeof(T);     // chunks of the tile that a chunk of the cache becomes
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int row, c;
      place(i, wave, lane, row, c);
      if (!EVEN && row >= ROWS) continue;
      const uint32_t w[4] = {h.x[i].x, h.x[i].y, h.x[i].z, h.x[i].w};
      alignas(16) T e[16];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        T y[4];
        from_e4m3<T>(w[k], h.s[i], y);
#pragma unroll
        for (int n = 0; n < 4; ++n) e[4 * k + n] = y[n];
      }
#pragma unroll
      for (int k = 0; k < TC; ++k)
        *reinterpret_cast<uint4*>(lds + Tile::at(row, TC * c + k)) = reinterpret_cast<const uint4*>(e)[k];
    }
  }
};

// A lane's query row: r = i * group + g of key/value head hk.
template <class T, int DP, bool VEC>
__device__ __forceinline__ void set_row(const CachedArgs& a, const CachedScope& sc, int b, int hk, int r, int lane, FwdRows<T, DP>& w) {
  const int rr = min(r, a.R - 1), i = (int)a.gdiv.div((uint32_t)rr), g = rr - i * a.G;
  w.pos = sc.off + i;
  w.klim = sc.klim(i);
  w.doc = 0;
  w.slope2 = a.slopes ? a.slopes[hk * a.G + g] * kLog2e : 0.f;
  load_owned<T, DP, VEC>((const T*)a.q.p + b * a.q.sb + i * a.q.ss + (hk * a.G + g) * a.q.sh, r < a.R, a.D, lane, w.q);
}

// ---- many rows: four waves of 32 rows share the key tiles in two LDS stages -------------------------------------------------
template <class T, int DP, bool VEC, bool E4M3, bool CAREFUL>
__device__ __forceinline__ bool cached_body(const CachedArgs& a, char* smem, int block) {
  constexpr int BN = kFwdKeys<T>;
  using Load = PageLoad<T, DP, BN, 4, VEC, E4M3>;
  char* sk = smem;                                  // [2][BN][DP]
  char* sv = smem + 2 * Load::BYTES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  int bh, item;
  place(block, a.B * a.Hk, bh, item);
  const int split = item % a.splits, mt = a.tiles - 1 - item / a.splits;   // the rows that see most keys first
  const int hk = bh % a.Hk, b = bh / a.Hk;
  const CachedScope sc(a, b);
  const int r0 = mt * kFwdRows, r = r0 + wave * 32 + (lane & 31);
  FwdRows<T, DP> w;
  typename AttnTile<T, DP>::Lane tl(lane);
  set_row<T, DP, VEC>(a, sc, b, hk, r, lane, w);

  const int i_lo = (int)a.gdiv.div((uint32_t)r0), i_hi = (int)a.gdiv.div((uint32_t)(min(r0 + kFwdRows, a.R) - 1));
  const int all = sc.all(i_lo, i_hi), any = sc.any(i_lo, i_hi);
  const int nt = (any + BN - 1) / BN, per = (nt + a.splits - 1) / a.splits;
  const int t0 = split * per, t1 = min(nt, t0 + per);

  auto pass = [&](auto careful) {
    w.reset();
    typename Load::Where where;
    if constexpr (!E4M3) {
      auto issue = [&](int t, int st) {
        Load::rows(a, a.k, hk, t * BN, where, sk + st * Load::BYTES, wave, lane);
        Load::rows(a, a.v, hk, t * BN, where, sv + st * Load::BYTES, wave, lane);
      };
      if (t0 < t1) {
        Load::look(a, b, t0 * BN, sc.len, wave, lane, where);
        issue(t0, 0);
        Load::look(a, b, (t0 + 1) * BN, sc.len, wave, lane, where);
      }
      for (int t = t0, st = 0; t < t1; ++t, st ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0070);   // this wave's part of the tile has landed, and its LDS reads are done
        __syncthreads();
        if (t + 1 < t1) {
          issue(t + 1, st ^ 1);
          Load::look(a, b, (t + 2) * BN, sc.len, wave, lane, where);
        }
        w.template tile<BN / 32>(a, sk + st * Load::BYTES, sv + st * Load::BYTES, nullptr, t * BN, (t + 1) * BN > all, careful, lane, tl);
      }
    } else {
      typename Load::Held hk_, hv_;
      auto fetch = [&](int t) {
        Load::fetch(a, a.k, a.k_scale, hk, t * BN, where, wave, lane, hk_);
        Load::fetch(a, a.v, a.v_scale, hk, t * BN, where, wave, lane, hv_);
      };
      auto put = [&](int st) {
        Load::put(hk_, sk + st * Load::BYTES, wave, lane);
        Load::put(hv_, sv + st * Load::BYTES, wave, lane);
      };
      if (t0 < t1) {
        Load::look(a, b, t0 * BN, sc.len, wave, lane, where);
        fetch(t0);
        Load::look(a, b, (t0 + 1) * BN, sc.len, wave, lane, where);
        put(0);
      }
      for (int t = t0, st = 0; t < t1; ++t, st ^= 1) {
        __syncthreads();                       // tile t is written, and tile t - 1 read
        if (t + 1 < t1) {
          fetch(t + 1);
          Load::look(a, b, (t + 2) * BN, sc.len, wave, lane, where);
        }
        w.template tile<BN / 32>(a, sk + st * Load::BYTES, sv + st * Load::BYTES, nullptr, t * BN, (t + 1) * BN > all, careful, lane, tl);
        if (t + 1 < t1) put(st ^ 1);
      }
    }
  };
  pass(std::integral_constant<bool, CAREFUL>{});
  // 0 * inf of a hidden pair (or a visible one): once more, with the product that tells them apart
  if (!CAREFUL && __syncthreads_or(not_finite(w.acc))) return true;
  w.l = half_sum(w.l);
  finish_row<T, DP, VEC>(a, w, b, hk, r, split, lane);
  return false;
}
template <class T, int DP, bool VEC, bool E4M3>
__global__ void __launch_bounds__(256, (sizeof(T) * DP <= 256 ? 2 : 1)) k_attn_cached(const CachedArgs a) {
  extern __shared__ __align__(1024) char smem[];
  const bool bad = cached_body<T, DP, VEC, E4M3, false>(a, smem, blockIdx.x);
  if (threadIdx.x == 0) a.flags[blockIdx.x] = bad;
}
template <class T, int DP, bool VEC, bool E4M3>
__global__ void __launch_bounds__(256, 1) k_attn_cached_again(const CachedArgs a, int blocks) {
  extern __shared__ __align__(1024) char smem[];
  again(a.flags, blocks, [&](int id) { cached_body<T, DP, VEC, E4M3, true>(a, smem, id); });
}

// ---- few rows (at most 32 a key/value head): each wave takes every W-th tile of 32 keys through LDS of its own ------------------
constexpr int kCachedKeys = 32;
template <class T, int DP, bool E4M3>
constexpr int kCachedStages = E4M3 ? 1 : 2;     // 8 bits: the next tile is on its way in registers
template <class T, int DP, bool E4M3>
constexpr int kCachedWaves = kCachedKeys * DP * (int)sizeof(T) * 2 * kCachedStages<T, DP, E4M3> * 4 <= 128 * 1024 ? 4 : 2;

template <class T, int DP, bool VEC, bool E4M3, bool CAREFUL>
__device__ __forceinline__ bool cached_tokens_body(const CachedArgs& a, char* smem) {
  constexpr int BN = kCachedKeys, W = kCachedWaves<T, DP, E4M3>, S = kCachedStages<T, DP, E4M3>;
  using Load = PageLoad<T, DP, BN, 1, VEC, E4M3>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char* mine = smem + wave * 2 * S * Load::BYTES;          // [S][k, v]

  int bh, split;
  place(blockIdx.x, a.B * a.Hk, bh, split);
  const int hk = bh % a.Hk, b = bh / a.Hk;
  const CachedScope sc(a, b);
  const int r = lane & 31;
  FwdRows<T, DP> w;
  typename AttnTile<T, DP>::Lane tl(lane);
  set_row<T, DP, VEC>(a, sc, b, hk, r, lane, w);

  const int i_hi = (a.R - 1) / a.G, all = sc.all(0, i_hi), any = sc.any(0, i_hi);
  const int nt = (any + BN - 1) / BN, per = (nt + a.splits - 1) / a.splits;
  const int t0 = split * per, t1 = min(nt, t0 + per);

  auto pass = [&](auto careful) {
    w.reset();
    typename Load::Where where;
    int t = t0 + wave;
    if constexpr (!E4M3) {
      auto issue = [&](int t, int st) {
        char* s = mine + st * 2 * Load::BYTES;
        Load::rows(a, a.k, hk, t * BN, where, s, 0, lane);
        Load::rows(a, a.v, hk, t * BN, where, s + Load::BYTES, 0, lane);
      };
      if (t < t1) {
        Load::look(a, b, t * BN, sc.len, 0, lane, where);
        issue(t, 0);
        Load::look(a, b, (t + W) * BN, sc.len, 0, lane, where);
      }
      for (int st = 0; t < t1; t += W, st ^= 1) {
        const bool more = t + W < t1;
        if (VEC && more) {
          issue(t + W, st ^ 1);
          wait_loads<2 * Load::NI>();    // the current tile has landed; the next stays in flight
        } else {
          __builtin_amdgcn_s_waitcnt(0x0070);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if (VEC && more) Load::look(a, b, (t + 2 * W) * BN, sc.len, 0, lane, where);
        const char* s = mine + st * 2 * Load::BYTES;
        w.template tile<1>(a, s, s + Load::BYTES, nullptr, t * BN, (t + 1) * BN > all, careful, lane, tl);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's LDS reads are done: the stage may be filled again
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if (!VEC && more) {
          issue(t + W, st ^ 1);
          Load::look(a, b, (t + 2 * W) * BN, sc.len, 0, lane, where);
        }
      }
    } else {
      typename Load::Held kh, vh;
      auto fetch = [&](int t) {
        Load::fetch(a, a.k, a.k_scale, hk, t * BN, where, 0, lane, kh);
        Load::fetch(a, a.v, a.v_scale, hk, t * BN, where, 0, lane, vh);
      };
      if (t < t1) {
        Load::look(a, b, t * BN, sc.len, 0, lane, where);
        fetch(t);
        Load::look(a, b, (t + W) * BN, sc.len, 0, lane, where);
      }
      for (; t < t1; t += W) {
        Load::put(kh, mine, 0, lane);
        Load::put(vh, mine + Load::BYTES, 0, lane);
        if (t + W < t1) {
          fetch(t + W);
          Load::look(a, b, (t + 2 * W) * BN, sc.len, 0, lane, where);
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);   // the tile is written
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
        w.template tile<1>(a, mine, mine + Load::BYTES, nullptr, t * BN, (t + 1) * BN > all, careful, lane, tl);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // and read
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  pass(std::integral_constant<bool, CAREFUL>{});
  if (!CAREFUL && __syncthreads_or(not_finite(w.acc))) return true;
  w.l = half_sum(w.l);
  if (join_waves<T, DP, W>(a, w, smem, wave, lane)) finish_row<T, DP, VEC>(a, w, b, hk, r, split, lane);
  return false;
}
template <class T, int DP, bool VEC, bool E4M3>
__global__ void __launch_bounds__((64 * kCachedWaves<T, DP, E4M3>), 1) k_attn_cached_tokens(const CachedArgs a) {
  extern __shared__ __align__(1024) char smem[];
  if (cached_tokens_body<T, DP, VEC, E4M3, false>(a, smem)) cached_tokens_body<T, DP, VEC, E4M3, true>(a, smem);
}

template <class T, int DP, bool VEC, bool E4M3>
hipError_t run_cached(hipStream_t s, const CachedArgs& a, bool tokens) {
  hipError_t e;
  if (tokens) {
    constexpr int W = kCachedWaves<T, DP, E4M3>;
    constexpr int bytes = std::max(2 * W * kCachedStages<T, DP, E4M3> * kCachedKeys * AttnTile<T, DP>::RB, kJoinBytes<T, DP, W>);
    e = hipFuncSetAttribute((const void*)k_attn_cached_tokens<T, DP, VEC, E4M3>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    k_attn_cached_tokens<T, DP, VEC, E4M3><<<dim3(a.B * a.Hk * a.splits), dim3(64 * W), bytes, s>>>(a);
  } else {
    constexpr int bytes = 4 * kFwdKeys<T> * AttnTile<T, DP>::RB;
    e = hipFuncSetAttribute((const void*)k_attn_cached<T, DP, VEC, E4M3>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    const int blocks = a.B * a.Hk * a.tiles * a.splits;
    k_attn_cached<T, DP, VEC, E4M3><<<dim3(blocks), dim3(256), bytes, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    e = hipFuncSetAttribute((const void*)k_attn_cached_again<T, DP, VEC, E4M3>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
    k_attn_cached_again<T, DP, VEC, E4M3><<<dim3(std::min(blocks, kAgainBlocks)), dim3(256), bytes, s>>>(a, blocks);
  }
  e = hipGetLastError();
  if (e == hipSuccess && a.splits > 1) {
    k_attn_join<T, DP><<<dim3(a.B * a.Hk * a.R), dim3(DP), 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

template <class T, bool E4M3>
hipError_t run_cached_dim(hipStream_t s, const CachedArgs& a, bool tokens, bool vec) {
  if (a.D <= 64) return vec ? run_cached<T, 64, true, E4M3>(s, a, tokens) : run_cached<T, 64, false, E4M3>(s, a, tokens);
  return vec ? run_cached<T, 128, true, E4M3>(s, a, tokens) : run_cached<T, 128, false, E4M3>(s, a, tokens);
}
template <bool E4M3>
hipError_t run_cached_type(hipStream_t s, int dtype, const CachedArgs& a, bool tokens, bool vec) {
  if (dtype == 1) return run_cached_dim<__bf16, E4M3>(s, a, tokens, vec);
  if (dtype == 2) return run_cached_dim<_Float16, E4M3>(s, a, tokens, vec);
  return run_cached_dim<float, E4M3>(s, a, tokens, vec);
}

}  // namespace
}  // namespace ntk

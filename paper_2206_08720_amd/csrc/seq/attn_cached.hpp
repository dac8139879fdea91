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
__device__ const float kOne = 1.f;

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

// Loads through addresses that were selected: said to be global memory, since a flat load's wait is one for LDS too.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 load16(const void* p) { return *(const __attribute__((address_space(1))) u32x4*)p; }
__device__ __forceinline__ float load_float(const float* p) { return *(const __attribute__((address_space(1))) float*)p; }

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

// ROWS positions of one head into an LDS tile of AttnTile's layout, by WAVES waves, 64 chunks of 16 bytes an instruction.  Pages
// hold at least 8 places and tiles start on multiples of 32, so 8 rows from a multiple of 8 lie in one page: a page's number
// is the same for a whole wave, and addresses are a scalar base and a lane's offset.  Nothing here waits for a load but for the
// one that look() made a tile before (branches on fresh entries, and flat loads, whose waits are LDS waits too, cost 832 us where this form takes 179: 32 sequences
// of up to 32768 places in 8 bits, 4 heads of 128).
template <class T, int DP, int ROWS, int WAVES, bool VEC, bool E4M3>
struct PageLoad {
  using Tile = AttnTile<T, DP>;
  static constexpr int CE = E4M3 ? 1 : (int)sizeof(T);           // bytes an element of the cache
  static constexpr int CH = DP * CE / 16, EC = 16 / CE;         // chunks a row, elements a chunk
  static constexpr int RPI = 64 / CH;                           // rows an instruction: at most 16
  static constexpr int BYTES = ROWS * Tile::RB;
  static constexpr int NI = (ROWS * CH + 64 * WAVES - 1) / (64 * WAVES);
  static constexpr bool EVEN = NI * 64 * WAVES == ROWS * CH;    // else some waves have none (rows >= ROWS)
  static_assert((EVEN || E4M3) && RPI <= 16, "chunks split over the lanes");

  // lane l: the table's entry for the rows 8 (l % (ROWS / 8)) .. + 7 of a tile
  __device__ static __forceinline__ int look(const CachedArgs& a, int b, int tile0, int lane) {
    const int e = min((tile0 + 8 * (lane & (ROWS / 8 - 1))) >> a.pages.shift, a.pages.most - 1);
    return a.pages.table[(long long)b * a.pages.most + e];
  }
  // instruction i's first row
  __device__ static __forceinline__ int first(int i, int wave) { return (i * WAVES + wave) * RPI; }
  // the entry (or its scale) of a lane's row
  __device__ static __forceinline__ int of_row(int entries, int row0, int lane) {
    const int lo = __builtin_amdgcn_readlane(entries, row0 / 8);
    if constexpr (RPI <= 8) return lo;
    return lane < 32 ? lo : __builtin_amdgcn_readlane(entries, row0 / 8 + 1);
  }
  // where a lane's chunk of instruction i is read; `there`: it is the cache's
  __device__ static __forceinline__ const char* source(const CachedArgs& a, const AttnView& v, int hk, int tile0, int len, int entries, int i,
                                                       int wave, int lane, int& c, bool& there) {
    const int row0 = first(i, wave), lr = lane / CH, row = row0 + lr;
    c = lane % CH;
    if constexpr (!E4M3) c ^= Tile::swz(row);                   // straight into LDS: lane l's 16 bytes go to place l
    const int id = of_row(entries, row0, lane);
    const bool in = (unsigned)id < (unsigned)a.pages.pages;
    const int group = RPI <= 8 ? row0 : row0 + (lr & 8);
    const char* base = (const char*)v.p + ((long long)(in ? id : 0) * v.sb + (long long)a.pages.slot(tile0 + group) * v.ss + (long long)hk * v.sh) * CE;
    const bool live = tile0 + row < len && (EVEN || row < ROWS);
    there = live && in && c * EC < a.D;
    const uint32_t off = (uint32_t)(row - group) * (uint32_t)v.ss * CE + (uint32_t)c * 16;   // rows that are not there: unused
    const char* none = live && !in ? (const char*)&kNaNs : (const char*)&kZeros;
    if constexpr (VEC) return there ? base + off : none;
    return there ? base + (long long)(row - group) * v.ss * CE : none;
  }
  // the same where the whole tile is the cache's (ordinary()): nothing to select
  __device__ static __forceinline__ const char* inside(const CachedArgs& a, const AttnView& v, int hk, int tile0, int entries, int i, int wave,
                                                       int lane) {
    const int row0 = first(i, wave), lr = lane / CH, row = row0 + lr;
    int c = lane % CH;
    if constexpr (!E4M3) c ^= Tile::swz(row);
    const int group = RPI <= 8 ? row0 : row0 + (lr & 8);
    const char* base = (const char*)v.p + ((long long)of_row(entries, row0, lane) * v.sb + (long long)a.pages.slot(tile0 + group) * v.ss + (long long)hk * v.sh) * CE;
    return base + ((uint32_t)(row - group) * (uint32_t)v.ss * CE + (uint32_t)c * 16);
  }
  __device__ static __forceinline__ bool ordinary(const CachedArgs& a, int tile0, int len, int entries) {
    return VEC && EVEN && tile0 + ROWS <= len && a.D == DP && __all((unsigned)entries < (unsigned)a.pages.pages);
  }
  // 16 bytes of a chunk that need not be aligned
  __device__ static __forceinline__ u32x4 gather(const char* from, bool there, int c, int D) {
    if (!there) return load16(from);
    if constexpr (!E4M3) return __builtin_bit_cast(u32x4, load_chunk_elems((const T*)from, c * EC, D));
    u32x4 u = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (c * EC + k < D) u[k / 4] |= (uint32_t)(uint8_t)from[c * EC + k] << (8 * (k % 4));
    return u;
  }
  // the cache in the queries' type: into LDS
  __device__ static __forceinline__ void rows(const CachedArgs& a, const AttnView& v, int hk, int tile0, int len, int entries, char* lds, int wave,
                                              int lane) {
    static_assert(!E4M3, "");
    typedef const __attribute__((address_space(1))) void G;
    typedef __attribute__((address_space(3))) void L;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int c;
      bool there;
      const char* from = source(a, v, hk, tile0, len, entries, i, wave, lane, c, there);
      char* to = lds + __builtin_amdgcn_readfirstlane((i * WAVES + wave) * 1024);
      if constexpr (VEC) {
        __builtin_amdgcn_global_load_lds((G*)from, (L*)to, 16, 0, 0);
      } else {
        *reinterpret_cast<u32x4*>(to + lane * 16) = gather(from, there, c, a.D);
      }
    }
  }
  // the cache in 8 bits: into registers, and from there into LDS
  struct Held {
    u32x4 x[NI];
    float s;                               // lane l: the scale of the rows that look() takes for it
  };
  __device__ static __forceinline__ void fetch(const CachedArgs& a, const AttnView& v, const float* scale, int hk, int tile0, int len, int entries,
                                               int wave, int lane, Held& h) {
    if (ordinary(a, tile0, len, entries)) {
      h.s = load_float(scale + ((long long)entries * a.Hk + hk));
#pragma unroll
      for (int i = 0; i < NI; ++i) h.x[i] = load16(inside(a, v, hk, tile0, entries, i, wave, lane));
      return;
    }
    const bool in = (unsigned)entries < (unsigned)a.pages.pages && tile0 + 8 * (lane & (ROWS / 8 - 1)) < len;
    h.s = load_float(in ? scale + ((long long)entries * a.Hk + hk) : &kOne);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int c;
      bool there;
      const char* from = source(a, v, hk, tile0, len, entries, i, wave, lane, c, there);
      if constexpr (VEC)
        h.x[i] = load16(from);
      else
        h.x[i] = gather(from, there, c, a.D);
    }
  }
  __device__ static __forceinline__ void put(const Held& h, char* lds, int wave, int lane) {
    constexpr int TC = (int)sizeof(T);     // chunks of the tile that a chunk of the cache becomes
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = first(i, wave) + lane / CH, c = lane % CH;
      if (!EVEN && row >= ROWS) continue;
      const float s = __int_as_float(of_row(__float_as_int(h.s), first(i, wave), lane));
      alignas(16) T e[16];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        T y[4];
        from_e4m3<T>(h.x[i][k], s, y);
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
template <class T, int DP, bool VEC, class Rows>
__device__ __forceinline__ void set_row(const CachedArgs& a, const CachedScope& sc, int b, int hk, int r, int lane, Rows& w) {
  const int rr = min(r, a.R - 1), i = (int)a.gdiv.div((uint32_t)rr), g = rr - i * a.G;
  w.pos = sc.off + i;
  w.klim = sc.klim(i);
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
  FwdRows<T, DP, false, E4M3> w;
  typename AttnTile<T, DP>::Lane tl(lane);
  set_row<T, DP, VEC>(a, sc, b, hk, r, lane, w);

  const int i_lo = (int)a.gdiv.div((uint32_t)r0), i_hi = (int)a.gdiv.div((uint32_t)(min(r0 + kFwdRows, a.R) - 1));
  const int all = sc.all(i_lo, i_hi), any = sc.any(i_lo, i_hi);
  const int nt = (any + BN - 1) / BN, per = (nt + a.splits - 1) / a.splits;
  const int t0 = split * per, t1 = min(nt, t0 + per);

  auto pass = [&](auto careful) {
    w.reset();
    int entries = 0;                           // of the tile that is read next
    if constexpr (!E4M3) {
      auto issue = [&](int t, int st) {
        Load::rows(a, a.k, hk, t * BN, sc.len, entries, sk + st * Load::BYTES, wave, lane);
        Load::rows(a, a.v, hk, t * BN, sc.len, entries, sv + st * Load::BYTES, wave, lane);
        entries = Load::look(a, b, (t + 1) * BN, lane);
      };
      if (t0 >= t1) return;
      entries = Load::look(a, b, t0 * BN, lane);
      issue(t0, 0);
      for (int t = t0, st = 0; t < t1; ++t, st ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0070);   // this wave's part of the tile has landed, and its LDS reads are done
        __syncthreads();
        if (t + 1 < t1) issue(t + 1, st ^ 1);
        w.template tile<BN / 32>(a, sk + st * Load::BYTES, sv + st * Load::BYTES, nullptr, t * BN, (t + 1) * BN > all, careful, lane, tl);
      }
    } else {
      typename Load::Held kt, vt;
      auto fetch = [&](int t) {
        Load::fetch(a, a.k, a.k_scale, hk, t * BN, sc.len, entries, wave, lane, kt);
        Load::fetch(a, a.v, a.v_scale, hk, t * BN, sc.len, entries, wave, lane, vt);
        entries = Load::look(a, b, (t + 1) * BN, lane);
      };
      auto put = [&](int st) {
        Load::put(kt, sk + st * Load::BYTES, wave, lane);
        Load::put(vt, sv + st * Load::BYTES, wave, lane);
      };
      if (t0 >= t1) return;
      entries = Load::look(a, b, t0 * BN, lane);
      fetch(t0);
      put(0);
      for (int t = t0, st = 0; t < t1; ++t, st ^= 1) {
        __syncthreads();                       // tile t is written, and tile t - 1 read
        if (t + 1 < t1) fetch(t + 1);
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
  FwdRows<T, DP, false, E4M3> w;
  typename AttnTile<T, DP>::Lane tl(lane);
  set_row<T, DP, VEC>(a, sc, b, hk, r, lane, w);

  const int i_hi = (a.R - 1) / a.G, all = sc.all(0, i_hi), any = sc.any(0, i_hi);
  const int nt = (any + BN - 1) / BN, per = (nt + a.splits - 1) / a.splits;
  const int t0 = split * per, t1 = min(nt, t0 + per);

  auto pass = [&](auto careful) {
    w.reset();
    int entries = 0;                           // of the tile that is read next
    int t = t0 + wave;
    if (t >= t1) return;
    entries = Load::look(a, b, t * BN, lane);
    if constexpr (!E4M3) {
      auto issue = [&](int t, int st) {
        char* s = mine + st * 2 * Load::BYTES;
        Load::rows(a, a.k, hk, t * BN, sc.len, entries, s, 0, lane);
        Load::rows(a, a.v, hk, t * BN, sc.len, entries, s + Load::BYTES, 0, lane);
      };
      issue(t, 0);
      entries = Load::look(a, b, (t + W) * BN, lane);
      for (int st = 0; t < t1; t += W, st ^= 1) {
        const bool more = t + W < t1;
        if (VEC && more) {
          const int then = Load::look(a, b, (t + 2 * W) * BN, lane);   // in front of the loads that it would wait for
          issue(t + W, st ^ 1);
          entries = then;
          wait_loads<2 * Load::NI>();    // the current tile has landed; the next stays in flight
        } else {
          __builtin_amdgcn_s_waitcnt(0x0070);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
        const char* s = mine + st * 2 * Load::BYTES;
        w.template tile<1>(a, s, s + Load::BYTES, nullptr, t * BN, (t + 1) * BN > all, careful, lane, tl);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // this wave's LDS reads are done: the stage may be filled again
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
        if (!VEC && more) {
          issue(t + W, st ^ 1);
          entries = Load::look(a, b, (t + 2 * W) * BN, lane);
        }
      }
    } else {
      typename Load::Held kt, vt;
      Load::fetch(a, a.k, a.k_scale, hk, t * BN, sc.len, entries, 0, lane, kt);
      Load::fetch(a, a.v, a.v_scale, hk, t * BN, sc.len, entries, 0, lane, vt);
      entries = Load::look(a, b, (t + W) * BN, lane);
      for (; t < t1; t += W) {
        const bool more = t + W < t1;
        // keys are on their way while values are written, and the other way round
        Load::put(kt, mine, 0, lane);
        if (more) {
          const int then = Load::look(a, b, (t + 2 * W) * BN, lane);   // in front of the loads that it would wait for
          Load::fetch(a, a.k, a.k_scale, hk, (t + W) * BN, sc.len, entries, 0, lane, kt);
          Load::put(vt, mine + Load::BYTES, 0, lane);
          Load::fetch(a, a.v, a.v_scale, hk, (t + W) * BN, sc.len, entries, 0, lane, vt);
          entries = then;
        } else {
          Load::put(vt, mine + Load::BYTES, 0, lane);
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
__global__ void __launch_bounds__((64 * kCachedWaves<T, DP, E4M3>), (E4M3 && sizeof(T) == 2 ? 2 : 1)) k_attn_cached_tokens(const CachedArgs a) {
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

// attn_cached.hpp -- attention over a cache of pages (kernels_cached_bf16.hip, _f16, _f32).
//
// The forward pass of kernels_attn.hip, o = softmax(mask(score(q k^T))) v with a running maximum, with keys and values read through
// a table of pages.  What differs is how a tile comes into LDS: a row's place follows from its page, read one tile ahead, and is
// a 64-bit address of its own (a cache may be larger than a buffer resource spans).  Rows past the sequence's end read
// zeros, rows on a page that the cache does not have NaN.
//
// A cache in 8 bits is read into registers, converted there (one instruction takes two e4m3 values and their page's power of two to
// two values of the queries' type), and written into the same tiles, so that the products are the same ones.
//
// Fewer bits than fp32, by choice: p is rounded to the queries' type for its product (its sum l is not), as in kernels_attn.hip, which
// leaves bf16 results 0.0022 from 64 bits in norm and fp16 ones 0.00024, where rounding the result alone leaves 0.0017 and 0.00021.  p in
// two parts of 16 bits, whose products are added, reaches the latter, and costs as many products of values again: tokens 1 to 5 %, five
// drafted tokens 7, long parts of prompts 21 to 27 (the case below 604 -> 768 us).
#pragma once
#include "attn_fwd.hpp"
#include "dealing.hpp"
#include "launch_cache.hpp"

namespace ntk {

struct CachedArgs : AttnArgs {             // k, v: sb from page to page, ss from slot to slot, sh from head to head
  PageTable pages;
  const int* q_lens;                       // [batch] or null
  const float *k_scale, *v_scale;          // [pages, kv_heads]: the cache is e4m3
  int workers, least;                      // workgroups, tiles that each takes at least; 0: a workgroup a row tile
  int* heads;                              // [workers][4]: row tiles that a worker begins and others go on with
};

namespace {

__device__ const uint4 kZeros = {0, 0, 0, 0};
__device__ const uint4 kNaNs = {~0u, ~0u, ~0u, ~0u};   // NaN in every type, e4m3 among them
__device__ const float kOne = 1.f;

// What a batch entry's queries see, as AttnScope: its first `queries` rows are the last of its `len` positions.
struct CachedScope {
  int len, off, queries, causal;
  CachedScope() = default;
  __device__ __forceinline__ void set(const CachedArgs& a, int b) {
    len = min(max(a.lens[b], 0), a.Sk);
    queries = a.q_lens ? min(max(a.q_lens[b], 0), a.Sq) : a.Sq;
    off = len - queries;
    causal = a.causal;
  }
  // of a sequence that all lanes work on, which the compiler cannot know of what it loads: scalars, and branches without masks
  __device__ __forceinline__ CachedScope(const CachedArgs& a, int b) {
    set(a, b);
    len = __builtin_amdgcn_readfirstlane(len);
    queries = __builtin_amdgcn_readfirstlane(queries);
    off = len - queries;
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
// one that look() made a tile before (branches on fresh entries, and flat loads, whose waits are LDS waits too, cost 832 us where this
// form took 179: 32 sequences of 24 thousand places on average in 8 bits, 4 heads of 128).
template <class T, int DP, int ROWS, int WAVES, bool VEC, bool E4M3>
struct PageLoad {
  using Tile = AttnTile<T, DP>;
  static constexpr int CE = E4M3 ? 1 : (int)sizeof(T);           // bytes an element of the cache
  static constexpr int CH = DP * CE / 16, EC = 16 / CE;         // chunks a row, elements a chunk
  using At = TilePlaces<CH, WAVES>;
  static constexpr int RPI = At::RPI;
  static constexpr int BYTES = ROWS * Tile::RB;
  static constexpr int NI = (ROWS * CH + 64 * WAVES - 1) / (64 * WAVES);
  static constexpr bool EVEN = NI * 64 * WAVES == ROWS * CH;    // else some waves have none (rows >= ROWS)
  static_assert(EVEN || E4M3, "chunks split over the lanes");

  // lane l: the table's entry for the rows 8 (l % (ROWS / 8)) .. + 7 of a tile
  __device__ static __forceinline__ int look(const CachedArgs& a, int b, int tile0, int lane) {
    const int e = min((tile0 + 8 * (lane & (ROWS / 8 - 1))) >> a.pages.shift, a.pages.most - 1);
    return a.pages.table[(long long)b * a.pages.most + e];
  }
  struct Head : HeadCells<VEC> {
    __device__ __forceinline__ Head(const AttnView& v, int hk) : HeadCells<VEC>(v.p, v.sb, v.ss, v.sh, hk, CE) {}
  };
  // A tile's place, with look()'s entry for it.
  struct Where {
    int entry;
    long long scale;                       // lane l: of the rows 8 (l % (ROWS / 8)) ..; -1: none
    int tile0, len;
    bool whole;                            // every row is the cache's
    __device__ __forceinline__ Where(const CachedArgs& a, int hk, int entry_, int tile0_, int len_, int lane)
        : entry(entry_), tile0(tile0_), len(len_) {
      const bool in = (unsigned)entry < (unsigned)a.pages.pages;
      scale = in && tile0 + 8 * (lane & (ROWS / 8 - 1)) < len ? (long long)entry * a.Hk + hk : -1;
      whole = VEC && EVEN && tile0 + ROWS <= len && a.D == DP && __all(in);
    }
  };
  // what look() has (or its scale) for a lane's row of the instruction whose first row is row0
  __device__ static __forceinline__ int of_row(int x, int row0, int lane) {
    const int lo = __builtin_amdgcn_readlane(x, row0 / 8);
    if constexpr (RPI <= 8) return lo;
    return lane < 32 ? lo : __builtin_amdgcn_readlane(x, row0 / 8 + 1);
  }
  // a lane's chunk of a row
  __device__ static __forceinline__ int chunk(int row, int lane) {
    if constexpr (E4M3) return lane % CH;
    return lane % CH ^ Tile::swz(row);                          // straight into LDS: lane l's 16 bytes go to place l
  }
  // where a lane's chunk of instruction i is read; `there`: it is the cache's
  __device__ static __forceinline__ const char* source(const CachedArgs& a, const Head& h, const Where& w, int i, int wave, int lane, int& c, bool& there) {
    const int row0 = At::first(i, wave), row = At::row(i, wave, lane), id = of_row(w.entry, row0, lane);
    c = chunk(row, lane);
    const bool in = (unsigned)id < (unsigned)a.pages.pages;
    const char* base = h.base + h.offset(in ? id : 0, a.pages.slot(w.tile0 + At::group(row0, lane)));
    const bool live = w.tile0 + row < w.len && (EVEN || row < ROWS);
    there = live && in && c * EC < a.D;
    const char* none = live && !in ? (const char*)&kNaNs : (const char*)&kZeros;
    if constexpr (VEC) {
      uint64_t at = (uint64_t)(uintptr_t)(base + (h.within(row) + (uint32_t)c * 16));
      asm volatile("" : "+v"(at));             // formed in any case: a branch around it would cost more
      return there ? (const char*)(uintptr_t)at : none;
    }
    return there ? base + h.within(row) : none;
  }
  // The same in a whole tile: a scalar base and 32 bits of a lane, nothing to select.
  __device__ static __forceinline__ const char* whole(const CachedArgs& a, const Head& h, const Where& w, int i, int wave, int lane) {
    const int row0 = At::first(i, wave), row = At::row(i, wave, lane);
    return h.base + h.offset(of_row(w.entry, row0, lane), a.pages.slot(w.tile0 + At::group(row0, lane))) + (h.within(row) + (uint32_t)chunk(row, lane) * 16);
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
  __device__ static __forceinline__ void rows(const CachedArgs& a, const Head& h, const Where& w, char* lds, int wave, int lane) {
    static_assert(!E4M3, "");
    typedef const __attribute__((address_space(1))) void G;
    typedef __attribute__((address_space(3))) void L;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int c;
      bool there;
      const char* from = source(a, h, w, i, wave, lane, c, there);
      char* to = lds + __builtin_amdgcn_readfirstlane((i * WAVES + wave) * 1024);
      if constexpr (VEC)
        __builtin_amdgcn_global_load_lds((G*)from, (L*)to, 16, 0, 0);
      else
        *reinterpret_cast<u32x4*>(to + lane * 16) = gather(from, there, c, a.D);
    }
  }
  // the cache in 8 bits: into registers, and from there into LDS
  struct Held {
    u32x4 x[NI];
    float s;                               // lane l: the scale of the rows that look() takes for it
  };
  __device__ static __forceinline__ void fetch(const CachedArgs& a, const Head& h, const float* scale, const Where& w, int wave, int lane, Held& to) {
    to.s = load_float(w.scale >= 0 ? scale + w.scale : &kOne);
    if (w.whole) {
#pragma unroll
      for (int i = 0; i < NI; ++i) to.x[i] = load16(whole(a, h, w, i, wave, lane));
      return;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int c;
      bool there;
      const char* from = source(a, h, w, i, wave, lane, c, there);
      if constexpr (VEC)
        to.x[i] = load16(from);
      else
        to.x[i] = gather(from, there, c, a.D);
    }
  }
  __device__ static __forceinline__ void put(const Held& h, char* lds, int wave, int lane) {
    constexpr int TC = (int)sizeof(T);     // chunks of the tile that a chunk of the cache becomes
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int row = At::row(i, wave, lane), c = lane % CH;
      if (!EVEN && row >= ROWS) continue;
      const float s = __int_as_float(of_row(__float_as_int(h.s), At::first(i, wave), lane));
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

// ---- the work, in equal parts ----------------------------------------------------------------------------------------------
// Sequences have lengths of their own, which the host does not know: with a workgroup a row tile, or ranges of a row's keys cut
// alike for all, the longest sequence would keep a few workgroups busy after the others have gone.  So the workgroups that run at once
// deal out all tiles of keys, head by head and row tile by row tile, in equal runs.  A row tile whose run ends early is gone on with
// by the next workers; what each has of it is joined by k_cached_join.  The parts follow from the lengths alone, so that results do
// not depend on timing.  In us, a workgroup a row tile / alike for all / equal runs (tokens of 32 query over 4 key/value heads in
// 8 bits, the parts' over 8, all of 128): 32 sequences of 24 thousand places 359 / 171 / 182, one of 131 thousand and 31 of one
// thousand 1581 / 543 / 71, parts of 1200 queries at the ends of 14 and 2 thousand places 887 / 782 / 373.  What a worker loses by it is
// the look at all lengths, about 5 us.
//
// A stretch costs 7 to 8 us whatever its length (its state, the first loads, the partial results).  So where few rows have fewer row
// tiles than there are workers, and runs get not much longer by it, a worker takes one part of one row tile, and nothing more: one
// token over 8000 places, 8 key/value heads in bf16, 29 us where runs that go on into the next head take 35; four of 1500 places 25
// and 31.  Tiles of many rows cost more than that saves (3 parts of 380 queries, 12 heads of 80: 60 us, this way 66).
//
// A row tile of no keys counts as one: its rows are written, too.
template <int BN, int ROWS>
struct Parts {
  // tiles of keys that row tile mt of sequence b sees (each lane its own)
  __device__ static __forceinline__ int tiles(const CachedArgs& a, int b, int mt) {
    CachedScope sc;
    sc.set(a, b);
    return tiles(a, sc, mt);
  }
  __device__ static __forceinline__ int tiles(const CachedArgs& a, const CachedScope& sc, int mt) {
    const int i0 = (int)a.gdiv.div((uint32_t)(mt * ROWS)), i1 = (int)a.gdiv.div((uint32_t)(min(mt * ROWS + ROWS, a.R) - 1));
    return (sc.any(i0, i1) + BN - 1) / BN;
  }
  int hk, pair, t, per, left;              // where this worker's run stands: pair = b * row tiles + mt, tile t, tiles left
  __device__ __forceinline__ int b(const CachedArgs& a) const { return a.tiles == 1 ? pair : pair / a.tiles; }
  __device__ __forceinline__ int mt(const CachedArgs& a) const { return a.tiles == 1 ? 0 : pair % a.tiles; }

  template <int THREADS>
  __device__ __forceinline__ void find(const CachedArgs& a, int block) {
    __shared__ int counts[1 + Deal::TRIES], sums[THREADS / 64];
    __shared__ Deal::Part found;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.B * a.tiles;
    if (a.workers == 0) {
      int bh, item;
      place(block, a.B * a.Hk, bh, item);
      hk = bh % a.Hk;
      pair = bh / a.Hk * a.tiles + a.tiles - 1 - item;          // the rows that see most keys first
      t = 0;
      left = per = 0x7fffffff;
      return;
    }
    // The plan sees to it that there are fewer than 2^30 tiles in all.
    const bool inside = a.tiles == 1;
    const int times = inside ? a.Hk : 1, heads = inside ? 1 : a.Hk;
    const int chunk = (n + THREADS - 1) / THREADS, p0 = min(n, (int)threadIdx.x * chunk), p1 = min(n, p0 + chunk);
    auto tiles_of = [&](int p) { return max(1, inside ? tiles(a, p, 0) : tiles(a, p / a.tiles, p % a.tiles)); };
    auto sum = [&](auto f) {                                     // of this thread's row tiles
      int x = 0;
      for (int p = p0; p < p1; ++p) x += times * f(tiles_of(p));
      return x;
    };
    if (threadIdx.x <= Deal::TRIES) counts[threadIdx.x] = 0;
    __syncthreads();
    if (p0 < p1) atomicAdd(&counts[0], sum([](int c) { return c; }));
    __syncthreads();
    Deal d(n, times, heads, a.workers, a.least, counts[0]);
    // the least of a few lengths under which parts that end with their row tile need no more workers than there are
    if (ROWS == 32 && d.may_share()) {
#pragma unroll
      for (int k = 0; k < Deal::TRIES; ++k)
        if (p0 < p1) atomicAdd(&counts[1 + k], sum([&](int c) { return (c + d.length(k) - 1) / d.length(k); }));
      __syncthreads();
      d.choose(counts + 1);
    }
    // neighbours in the order read the same keys: a die (workgroups are dealt out to the eight in turn) takes a run of workers
    const int w = number(a, block), at = d.at(w);
    const int mine = sum([&](int c) { return d.units(c); });
    int upto = mine;                                             // inclusive sum
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < THREADS / 64; ++i)
      if (i < wave) upto += sums[i];
    if (at >= upto - mine && at < upto) {
      int x = upto - mine, p = p0;
      for (;; ++p) {
        const int c = tiles_of(p), u = times * d.units(c);
        if (at < x + u) {
          found = d.within(p, c, x, w);
          break;
        }
        x += u;
      }
    }
    __syncthreads();
    const Deal::Part part = d.taken(found, w);
    pair = part.pair, t = part.t, hk = part.hk, left = part.left, per = part.per;
    pair = __builtin_amdgcn_readfirstlane(pair);                 // (from `part` itself, 25 more vector registers)
    t = __builtin_amdgcn_readfirstlane(t);
    hk = __builtin_amdgcn_readfirstlane(hk);
    left = __builtin_amdgcn_readfirstlane(left);
    per = __builtin_amdgcn_readfirstlane(per);
  }
  // the row tile behind: a sequence's heads in turn, whose parts of a page are neighbours, or, where many rows read the same keys,
  // all of a head's rows
  __device__ __forceinline__ void next(const CachedArgs& a) {
    if (a.tiles == 1) {
      if (++hk < a.Hk) return;
      hk = 0;
      ++pair;
    } else if (++pair == a.B * a.tiles) {
      pair = 0;
      ++hk;
    }
  }
  // this worker's number in the order of the work
  __device__ static __forceinline__ int number(const CachedArgs& a, int block) {
    return a.workers % 8 ? block : (block % 8) * (a.workers / 8) + block / 8;
  }
};

// A stretch [t0, t1) of a row tile's `nt` tiles of keys.
struct Stretch {
  int b, hk, mt, t0, t1, nt, slot;         // slot: where its partial results go, -1: it is all of them
};

// Calls f(stretch) for a worker's stretches and notes the row tile that it begins and does not end.  What it goes on with for another
// comes last: the workers of a head then begin at its first key together, and read the same keys at about the same time.
template <class P, int THREADS, class F>
__device__ __forceinline__ void each_stretch(const CachedArgs& a, int block, F f) {
  P p;
  p.template find<THREADS>(a, block);
  const int w = P::number(a, block);
  if (a.workers && threadIdx.x == 0) a.heads[4 * w + 2] = 0;
  if (p.left <= 0) return;
  P late = p;
  late.left = 0;
  for (;;) {
    const bool end = p.left <= 0;
    if (end) {
      if (late.left <= 0) return;
      p = late;
      late.left = 0;
    }
    Stretch s;
    s.b = p.b(a);
    s.mt = p.mt(a);
    s.hk = p.hk;
    s.nt = P::tiles(a, CachedScope(a, s.b), s.mt);
    const int count = max(1, s.nt), take = min(count - p.t, p.left);
    const bool first = p.t == 0, last = p.t + take == count;
    if (!first && !end && take < p.left) {
      late = p;
      late.left = take;
    } else {
      s.t0 = p.t;
      s.t1 = min(s.nt, p.t + take);
      s.slot = first && last ? -1 : first ? 2 * w + 1 : 2 * w;
      f(s);
      if (a.workers == 0) return;
      if (first && !last && threadIdx.x == 0) {
        a.heads[4 * w] = p.pair;
        a.heads[4 * w + 1] = p.hk;
        a.heads[4 * w + 2] = (count - take + p.per - 1) / p.per;   // workers behind this one
      }
    }
    p.left -= take;
    p.t = 0;
    p.next(a);
  }
}

// The rows' results, or their partial sums: [slot][ROWS] rows of DP, behind them maximum (in units of log2) and sum.
template <class T, int DP, int ROWS, bool VEC, class Rows>
__device__ __forceinline__ void finish_stretch(const CachedArgs& a, Rows& w, const Stretch& s, int row, int lane) {
  if (s.slot < 0) {
    finish_row<T, DP, VEC>(a, w, s.b, s.hk, s.mt * ROWS + row, 0, lane);
    return;
  }
  const long long at = (long long)s.slot * ROWS + row;
  store_owned<float, DP, true>(a.part + at * DP, DP, lane, w.acc, 1.f);
  if (lane < 32) {
    float* ml = a.part + (long long)a.workers * 2 * ROWS * DP + at * 2;
    ml[0] = w.m == -__builtin_inff() ? w.m : w.m * (a.cap_in != 0.f || a.slopes ? 1.f : a.c);
    ml[1] = w.l;
  }
}

// Rows of a row tile that one worker began: its sums and those of the workers behind it.  A thread takes four elements of a row, with
// those of four workers in flight (a row at a time it took 18 us where 16 workers have parts of 40 rows each, and takes 8 this way).
template <int DP, int ROWS>
struct JoinShape {
  static constexpr int LANES = DP / 4, BLOCK_ROWS = 256 / LANES, PARTS = ROWS / BLOCK_ROWS, DEPTH = 4;
};
template <class T, int DP, int ROWS>
__global__ void __launch_bounds__(256) k_cached_join(const CachedArgs a) {
  using S = JoinShape<DP, ROWS>;
  const int w = blockIdx.x / S::PARTS, row = blockIdx.x % S::PARTS * S::BLOCK_ROWS + threadIdx.x / S::LANES;
  const int pair = a.heads[4 * w], hk = a.heads[4 * w + 1], behind = a.heads[4 * w + 2];
  if (behind == 0) return;
  const int b = pair / a.tiles, mt = pair - b * a.tiles, d = threadIdx.x % S::LANES * 4, r = mt * ROWS + row;
  if (r >= a.R) return;
  const float* ml = a.part + (long long)a.workers * 2 * ROWS * DP;
  float m = -__builtin_inff(), l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 <= behind; s0 += S::DEPTH) {
    float ms[S::DEPTH], ls[S::DEPTH];
    f32x4 os[S::DEPTH];
#pragma unroll
    for (int u = 0; u < S::DEPTH; ++u) {
      const int x = min(s0 + u, behind), slot = x == 0 ? 2 * w + 1 : 2 * (w + x);
      const long long at = (long long)slot * ROWS + row;
      ms[u] = s0 + u <= behind ? ml[at * 2] : -__builtin_inff();
      ls[u] = ml[at * 2 + 1];
      os[u] = *reinterpret_cast<const f32x4*>(a.part + at * DP + d);
    }
#pragma unroll
    for (int u = 0; u < S::DEPTH; ++u) {                         // no branch: it would have the loads behind it wait
      const float mn = fmaxf(m, ms[u]), there = s0 + u <= behind ? 1.f : 0.f;
      const float f = m == mn ? 1.f : exp2_hw(m - mn), g = there * (ms[u] == mn ? 1.f : exp2_hw(ms[u] - mn));
      l = l * f + ls[u] * g;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = o[k] * f + (s0 + u <= behind ? os[u][k] : 0.f) * g;   // the last one's may be infinite
      m = mn;
    }
  }
  const int i = (int)a.gdiv.div((uint32_t)r), head = hk * a.G + r - i * a.G;
  T* out = (T*)a.o.p + b * a.o.sb + i * a.o.ss + head * a.o.sh;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (d + k < a.D) out[d + k] = (T)(l == 0.f ? 0.f : o[k] / l);
  if (a.lse && d == 0)
    a.lse[((long long)b * a.H + head) * a.Sq + i] = l == 0.f ? -__builtin_inff() : m * kLn2 + logf(l * kWeightOne<T>);
}

// ---- many rows: NW waves of 32 rows share the key tiles in two LDS stages ----------------------------------------------------
// Bound by two waves a SIMD that take turns at the matrix cores (34 % of the cycles) and at the exponentials (vector 45 %), as in
// kernels_attn.hip; in 8 bits with eight waves a workgroup, so that what a tile takes to bring in and to convert is shared by 256 rows
// (bf16, parts of 1212 and 1839 queries over 14187 and 8463 places, 32 heads over 8 of 128: 578 us in a long run, 860 TFLOP/s; in a short
// one, at the clock that it begins with, 691, and 750 with four waves, of which bringing in takes 110 and converting 70; a cache in bf16,
// with four waves, 691 in a long run; in fp32, parts half as long over half as many places, 16 heads over 8, 587).  Results that are
// not finite are formed again by a kernel of its own: within this one its registers cost long parts 2 to 7 %, which is more than the launch.
template <class T, int DP, int NW, bool VEC, bool E4M3, bool CAREFUL>
__device__ __forceinline__ bool cached_stretch(const CachedArgs& a, char* smem, const Stretch& x) {
  constexpr int BN = kFwdKeys<T>;
  using Load = PageLoad<T, DP, BN, NW, VEC, E4M3>;
  char* sk = smem;                                  // [2][BN][DP]
  char* sv = smem + 2 * Load::BYTES;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = x.b, hk = x.hk, t0 = x.t0, t1 = x.t1;
  const CachedScope sc(a, b);
  const int row = wave * 32 + (lane & 31), r0 = x.mt * (32 * NW) + wave * 32;
  FwdRows<T, DP, false, E4M3> w;
  typename AttnTile<T, DP>::Lane tl(lane);
  set_row<T, DP, VEC>(a, sc, b, hk, x.mt * (32 * NW) + row, lane, w);

  // keys that all of this wave's rows see, that some row sees
  const int i_lo = (int)a.gdiv.div((uint32_t)min(r0, a.R - 1)), i_hi = (int)a.gdiv.div((uint32_t)(min(r0 + 32, a.R) - 1));
  const int all = sc.all(i_lo, i_hi), any = r0 < a.R ? sc.any(i_lo, i_hi) : 0;

  const typename Load::Head keys(a.k, hk), values(a.v, hk);

  auto pass = [&](auto careful) {
    w.reset();
    auto multiply = [&](int t, int st) {
      if (t * BN < any)
        w.template tile<BN / 32>(a, sk + st * Load::BYTES, sv + st * Load::BYTES, nullptr, t * BN, (t + 1) * BN > all, careful, lane, tl);
    };
    if (t0 >= t1) return;
    int entry = Load::look(a, b, t0 * BN, lane);                 // of the tile that is read next
    if constexpr (!E4M3) {
      auto issue = [&](int t, int st) {
        const typename Load::Where at(a, hk, entry, t * BN, sc.len, lane);
        entry = Load::look(a, b, (t + 1) * BN, lane);
        Load::rows(a, keys, at, sk + st * Load::BYTES, wave, lane);
        Load::rows(a, values, at, sv + st * Load::BYTES, wave, lane);
      };
      issue(t0, 0);
      for (int t = t0, st = 0; t < t1; ++t, st ^= 1) {
        __builtin_amdgcn_s_waitcnt(0x0070);   // this wave's part of the tile has landed, and its LDS reads are done
        __syncthreads();
        if (t + 1 < t1) issue(t + 1, st ^ 1);
        multiply(t, st);
      }
    } else {
      typename Load::Held kt, vt;
      auto fetch = [&](int t) {
        const typename Load::Where at(a, hk, entry, t * BN, sc.len, lane);
        entry = Load::look(a, b, (t + 1) * BN, lane);
        Load::fetch(a, keys, a.k_scale, at, wave, lane, kt);
        Load::fetch(a, values, a.v_scale, at, wave, lane, vt);
      };
      auto put = [&](int st) {
        Load::put(kt, sk + st * Load::BYTES, wave, lane);
        Load::put(vt, sv + st * Load::BYTES, wave, lane);
      };
      fetch(t0);
      put(0);
      for (int t = t0, st = 0; t < t1; ++t, st ^= 1) {
        __syncthreads();                       // tile t is written, and tile t - 1 read
        if (t + 1 < t1) fetch(t + 1);
        multiply(t, st);
        if (t + 1 < t1) put(st ^ 1);
      }
    }
  };
  pass(std::integral_constant<bool, CAREFUL>{});
  // 0 * inf of a hidden pair (or a visible one): once more, with the product that tells them apart
  const bool bad = !CAREFUL && not_finite(w.acc);
  w.l = half_sum(w.l);
  finish_stretch<T, DP, 32 * NW, VEC>(a, w, x, row, lane);
  return __syncthreads_or(bad);                // and the next stretch fills the same LDS
}
template <class T, int DP, int NW, bool VEC, bool E4M3>
__global__ void __launch_bounds__(64 * NW, (sizeof(T) * DP <= 256 ? 2 : 1)) k_attn_cached(const CachedArgs a) {
  extern __shared__ __align__(1024) char smem[];
  bool bad = false;
  each_stretch<Parts<kFwdKeys<T>, 32 * NW>, 64 * NW>(
      a, blockIdx.x, [&](const Stretch& x) { bad |= cached_stretch<T, DP, NW, VEC, E4M3, false>(a, smem, x); });
  if (threadIdx.x == 0) a.flags[blockIdx.x] = bad;
}
template <class T, int DP, int NW, bool VEC, bool E4M3>
__global__ void __launch_bounds__(64 * NW, 1) k_attn_cached_again(const CachedArgs a, int blocks) {
  extern __shared__ __align__(1024) char smem[];
  again(a.flags, blocks, [&](int id) {
    each_stretch<Parts<kFwdKeys<T>, 32 * NW>, 64 * NW>(a, id, [&](const Stretch& x) { cached_stretch<T, DP, NW, VEC, E4M3, true>(a, smem, x); });
  });
}

// ---- few rows (at most 32 a key/value head): each wave takes every W-th tile of 32 keys through LDS of its own ------------------
// Bound by memory where there is enough to read: 96 sequences of 3 thousand places on average, 8 heads of 128 in bf16, 234 us, 5.2 TB/s (a
// large copy reaches 4.9); in 8 bits 32 sequences of 24 thousand, 4 heads, 163 us, 4.8 TB/s, where a wave's conversions and products
// take turns with its loads (vector 32 %, LDS 32 %, matrix 12 % of the cycles).  fp32 queries, 32 sequences of 6 thousand, 8 heads: of 64
// 159 us, 5.0 TB/s; of 128, whose 439 registers leave one wave a SIMD, 474, 3.3 TB/s, over 8 bits 285.  Rows of 8 bits that are no multiple
// of 16 bytes are read byte by byte: 4 heads of 72 over 24 thousand places 929 us, of 80 152.  The careful pass comes after the loop over the
// stretches: inside it, its registers would be spilled with theirs.
constexpr int kCachedKeys = 32;
template <class T, int DP, bool E4M3>
constexpr int kCachedStages = E4M3 ? 1 : 2;     // 8 bits: the next tile is on its way in registers
template <class T, int DP, bool E4M3>
constexpr int kCachedWaves = kCachedKeys * DP * (int)sizeof(T) * 2 * kCachedStages<T, DP, E4M3> * 4 <= 128 * 1024 ? 4 : 2;
template <class T, int DP, bool E4M3>
constexpr int kCachedBytes = std::max(2 * kCachedWaves<T, DP, E4M3> * kCachedStages<T, DP, E4M3> * kCachedKeys * AttnTile<T, DP>::RB,
                                      kJoinBytes<T, DP, kCachedWaves<T, DP, E4M3>>);

template <class T, int DP, bool VEC, bool E4M3, bool CAREFUL>
__device__ __forceinline__ bool tokens_stretch(const CachedArgs& a, char* smem, const Stretch& x) {
  constexpr int BN = kCachedKeys, W = kCachedWaves<T, DP, E4M3>, S = kCachedStages<T, DP, E4M3>;
  using Load = PageLoad<T, DP, BN, 1, VEC, E4M3>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  char* mine = smem + wave * 2 * S * Load::BYTES;          // [S][k, v]
  const int b = x.b, hk = x.hk, t1 = x.t1;
  const CachedScope sc(a, b);
  const int r = lane & 31;
  FwdRows<T, DP, false, E4M3> w;
  typename AttnTile<T, DP>::Lane tl(lane);
  set_row<T, DP, VEC>(a, sc, b, hk, r, lane, w);
  const int all = sc.all(0, (a.R - 1) / a.G);

  const typename Load::Head keys(a.k, hk), values(a.v, hk);

  auto pass = [&](auto careful) {
    w.reset();
    int t = x.t0 + wave;
    if (t >= t1) return;
    // Every step brings in the wave's next tile, past its last one zeros from one address: the loads in flight are the same
    // ones every time, and no wait is for more than it needs.  Entries are looked up a step ahead, in front of the loads that are
    // still on their way when they are used.
    typedef typename Load::Where Where;
    int entry = Load::look(a, b, t * BN, lane);
    const Where at0(a, hk, entry, t * BN, sc.len, lane);
    entry = Load::look(a, b, (t + W) * BN, lane);
    if constexpr (!E4M3) {
      auto issue = [&](const Where& at, int st) {
        char* s = mine + st * 2 * Load::BYTES;
        Load::rows(a, keys, at, s, 0, lane);
        Load::rows(a, values, at, s + Load::BYTES, 0, lane);
      };
      issue(at0, 0);
      for (int st = 0; t < t1; t += W, st ^= 1) {
        const Where at(a, hk, entry, (t + W) * BN, t + W < t1 ? sc.len : 0, lane);
        entry = Load::look(a, b, (t + 2 * W) * BN, lane);
        if constexpr (VEC) {
          issue(at, st ^ 1);
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
        if constexpr (!VEC) issue(at, st ^ 1);
      }
    } else {
      typename Load::Held kt, vt;
      Load::fetch(a, keys, a.k_scale, at0, 0, lane, kt);
      Load::fetch(a, values, a.v_scale, at0, 0, lane, vt);
      for (; t < t1; t += W) {
        const Where at(a, hk, entry, (t + W) * BN, t + W < t1 ? sc.len : 0, lane);
        // keys are on their way while values are written, and the other way round
        Load::put(kt, mine, 0, lane);
        entry = Load::look(a, b, (t + 2 * W) * BN, lane);
        Load::fetch(a, keys, a.k_scale, at, 0, lane, kt);
        Load::put(vt, mine + Load::BYTES, 0, lane);
        Load::fetch(a, values, a.v_scale, at, 0, lane, vt);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // the tile is written
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
        w.template tile<1>(a, mine, mine + Load::BYTES, nullptr, t * BN, (t + 1) * BN > all, careful, lane, tl);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // and read
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // what was brought in past the end goes where the waves' states are joined: it has to have landed before
    __builtin_amdgcn_s_waitcnt(0x0070);
  };
  pass(std::integral_constant<bool, CAREFUL>{});
  if (!CAREFUL && __syncthreads_or(not_finite(w.acc))) return true;
  w.l = half_sum(w.l);
  if (join_waves<T, DP, W>(a, w, smem, wave, lane)) finish_stretch<T, DP, 32, VEC>(a, w, x, r, lane);
  __syncthreads();                             // the next stretch fills the same LDS
  return false;
}
template <class T, int DP, bool VEC, bool E4M3>
__global__ void __launch_bounds__((64 * kCachedWaves<T, DP, E4M3>), (E4M3 && sizeof(T) == 2 ? 2 : 1)) k_attn_cached_tokens(const CachedArgs a) {
  extern __shared__ __align__(1024) char smem[];
  typedef Parts<kCachedKeys, 32> P;
  constexpr int THREADS = 64 * kCachedWaves<T, DP, E4M3>;
  bool bad = false;
  each_stretch<P, THREADS>(a, blockIdx.x, [&](const Stretch& x) { bad |= tokens_stretch<T, DP, VEC, E4M3, false>(a, smem, x); });
  if (bad) each_stretch<P, THREADS>(a, blockIdx.x, [&](const Stretch& x) { tokens_stretch<T, DP, VEC, E4M3, true>(a, smem, x); });
}

template <class T, int DP, int NW, bool VEC, bool E4M3>
hipError_t run_cached_tiles(hipStream_t s, const CachedArgs& a, int blocks) {
  constexpr int bytes = 4 * kFwdKeys<T> * AttnTile<T, DP>::RB;
  const void* kernels[2] = {(const void*)k_attn_cached<T, DP, NW, VEC, E4M3>, (const void*)k_attn_cached_again<T, DP, NW, VEC, E4M3>};
  for (const void* k : kernels) {
    const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return e;
  }
  k_attn_cached<T, DP, NW, VEC, E4M3><<<dim3(blocks), dim3(64 * NW), bytes, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  k_attn_cached_again<T, DP, NW, VEC, E4M3><<<dim3(std::min(blocks, kAgainBlocks)), dim3(64 * NW), bytes, s>>>(a, blocks);
  e = hipGetLastError();
  if (e == hipSuccess && a.workers) {
    k_cached_join<T, DP, 32 * NW><<<dim3(a.workers * JoinShape<DP, 32 * NW>::PARTS), dim3(256), 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

template <class T, int DP, bool VEC, bool E4M3>
hipError_t run_cached(hipStream_t s, const CachedArgs& a, int waves) {
  const int blocks = a.workers ? a.workers : a.B * a.Hk * a.tiles;
  if constexpr (cached_wide(sizeof(T), E4M3))
    if (waves == 8) return run_cached_tiles<T, DP, 8, VEC, E4M3>(s, a, blocks);
  if (waves) return run_cached_tiles<T, DP, 4, VEC, E4M3>(s, a, blocks);
  constexpr int bytes = kCachedBytes<T, DP, E4M3>;
  hipError_t e = hipFuncSetAttribute((const void*)k_attn_cached_tokens<T, DP, VEC, E4M3>, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != hipSuccess) return e;
  k_attn_cached_tokens<T, DP, VEC, E4M3><<<dim3(blocks), dim3(64 * kCachedWaves<T, DP, E4M3>), bytes, s>>>(a);
  e = hipGetLastError();
  if (e == hipSuccess && a.workers) {
    k_cached_join<T, DP, 32><<<dim3(a.workers * JoinShape<DP, 32>::PARTS), dim3(256), 0, s>>>(a);
    e = hipGetLastError();
  }
  return e;
}

template <class T, bool E4M3>
hipError_t run_cached_dim(hipStream_t s, const CachedArgs& a, int waves, bool vec) {
  if (a.D <= 64) return vec ? run_cached<T, 64, true, E4M3>(s, a, waves) : run_cached<T, 64, false, E4M3>(s, a, waves);
  return vec ? run_cached<T, 128, true, E4M3>(s, a, waves) : run_cached<T, 128, false, E4M3>(s, a, waves);
}
template <class T>
hipError_t run_cached_type(hipStream_t s, const CachedArgs& a, bool e4m3, int waves, bool vec) {
  return e4m3 ? run_cached_dim<T, true>(s, a, waves, vec) : run_cached_dim<T, false>(s, a, waves, vec);
}

}  // namespace
}  // namespace ntk

// paging.hpp -- where a position of a sequence lies in a cache of pages (integer arithmetic, for the kernels and for the host).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace ntk {

// A sequence's place `pos` is slot pos % 2^shift of the page that entry pos / 2^shift of its row of the table names.
struct PageTable {
  const int* table = nullptr;    // [batch, most]
  int most = 0, pages = 0, shift = 0;
  __host__ __device__ __forceinline__ int slot(int pos) const { return pos & ((1 << shift) - 1); }
  // the page, or -1 where the row ends before it or names none of the cache's
  __host__ __device__ __forceinline__ int page(int b, int pos) const {
    const int e = pos >> shift;
    if (pos < 0 || e >= most) return -1;
    const int id = table[(long long)b * most + e];
    return (unsigned)id < (unsigned)pages ? id : -1;
  }
};

// How WAVES waves bring a tile of rows of CH 16-byte chunks in, 64 chunks an instruction: instruction i of a wave takes the rows from
// first() on.  Pages hold at least 8 places and tiles start on multiples of 32, so that the eight rows from a multiple of 8 lie side by
// side in one page: a row is `row % 8` slots behind the one that group() names.
template <int CH, int WAVES>
struct TilePlaces {
  static constexpr int RPI = 64 / CH;                           // rows an instruction: at most 16
  static_assert(RPI >= 1 && RPI <= 16, "an instruction takes rows of two groups at most");
  __host__ __device__ static __forceinline__ int first(int i, int wave) { return (i * WAVES + wave) * RPI; }
  __host__ __device__ static __forceinline__ int row(int i, int wave, int lane) { return first(i, wave) + lane / CH; }
  __host__ __device__ static __forceinline__ int group(int row0, int lane) { return (row0 & ~7) + (RPI == 16 ? lane / CH & 8 : 0); }
};

// Whether offsets within a page of a cache fit 32 bits, its slots `stride` elements of `bytes` apart.
inline bool narrow_slots(long long stride, int bytes, int page_size) { return stride < (1LL << 31) / bytes / page_size; }

// One head's part of a cache's array, in bytes.  NARROW: narrow_slots() holds.  Where it does not, slots may lie any distance apart
// (the slots outermost, in a cache of tens of GB), and their offsets have 64 bits.
template <bool NARROW>
struct HeadCells {
  using Offset = std::conditional_t<NARROW, uint32_t, long long>;
  const char* base;
  long long page;                          // from page to page
  Offset slot;                             // from slot to slot
  __host__ __device__ __forceinline__ HeadCells(const void* p, long long pages, long long slots, long long heads, int head, int bytes)
      : base((const char*)p + (long long)head * heads * bytes), page(pages * bytes), slot((Offset)(slots * bytes)) {}
  // where page `id` has its slot `s`
  __host__ __device__ __forceinline__ long long offset(int id, int s) const { return (long long)id * page + (Offset)s * slot; }
  // a row's place behind the first one of its eight
  __host__ __device__ __forceinline__ Offset within(int row) const { return (Offset)(row & 7) * slot; }
};

// The tokens that an append adds to one sequence: positions first .. first + count - 1.
struct AppendSpan {
  int first, count;
  __host__ __device__ __forceinline__ AppendSpan(const PageTable& t, int held, int new_tokens, int length) {
    const int places = t.most << t.shift;    // places + length < 2^31, checked on the host
    first = held < 0 ? 0 : held > places ? places : held;
    count = new_tokens < 0 ? 0 : new_tokens > length ? length : new_tokens;
  }
  // the slots [lo, hi) of the sequence's page number `e` that get new tokens, and the index of the first one's token
  __host__ __device__ __forceinline__ bool slots(const PageTable& t, int e, int& lo, int& hi, int& token) const {
    const int size = 1 << t.shift;
    if (e >= t.most) return false;
    const int at = e << t.shift, end = first + count;
    lo = first > at ? first - at : 0;
    hi = end - at < size ? end - at : size;
    token = at + lo - first;
    return lo < hi;
  }
};
// pages that `length` new tokens of a sequence can touch
__host__ __device__ inline int append_pages(int length, int shift) {
  return length < 1 ? 0 : (int)(((long long)length + (1 << shift) - 2) >> shift) + 1;
}

// The exponent of the least power of two that `most` (finite, >= 0) is at most 448 times of, but at least -126.
__host__ __device__ inline int e4m3_exponent(float most) {
  uint32_t u;
  __builtin_memcpy(&u, &most, 4);
  const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);   // 448 = 1.75 2^8
  return e < -126 ? -126 : e;
}

}  // namespace ntk

// Host check of csrc/seq/paging.hpp: where the cells of a cache lie, slots far apart among them, and the rows that the waves of the
// widest workgroups bring in.
#include <stdio.h>

#include <random>
#include <vector>

#include "seq/paging.hpp"

using namespace ntk;

static int fail(const char* what, long long x) {
  printf("%s %lld\n", what, x);
  return 1;
}

template <bool NARROW>
static int check_cells(long long page, long long slot, long long head, int bytes, int page_size, int id, int hk) {
  const char* p = (const char*)(uintptr_t)4096;
  const HeadCells<NARROW> h(p, page, slot, head, hk, bytes);
  for (int s : {0, 1, 5, 7, 8, page_size / 2 + 3, page_size - 8, page_size - 1}) {
    if (s >= page_size) continue;
    // eight rows from a multiple of 8 on share the address of the first
    const __int128 want = 4096 + ((__int128)id * page + (__int128)s * slot + (__int128)hk * head) * bytes;
    const char* got = h.base + h.offset(id, s & ~7) + h.within(s);
    if ((__int128)(uintptr_t)got != want) return fail(NARROW ? "a cell" : "a cell, slots far apart", s);
  }
  return 0;
}

// Every row of a tile once, from its group's page.
template <int CH, int WAVES>
static int check_tile(int rows) {
  using At = TilePlaces<CH, WAVES>;
  const int ni = (rows * CH + 64 * WAVES - 1) / (64 * WAVES);
  std::vector<int> seen((size_t)ni * 64 * WAVES / CH, 0);
  for (int i = 0; i < ni; ++i)
    for (int wave = 0; wave < WAVES; ++wave)
      for (int lane = 0; lane < 64; ++lane) {
        const int row = At::row(i, wave, lane), g = At::group(At::first(i, wave), lane);
        if (g % 8 || row < g || row >= g + 8) return fail("group", row);
        const int by = At::RPI <= 8 || lane < 32 ? At::first(i, wave) / 8 : At::first(i, wave) / 8 + 1;
        if (by * 8 != g) return fail("entry of a row", row);
        ++seen[row];
      }
  for (int n : seen)
    if (n != CH) return fail("chunks of a row", n);
  return 0;
}

int main() {
  // eight waves share a tile of 64 rows of 8 bits, heads of 64 and 128
  if (check_tile<4, 8>(64) || check_tile<8, 8>(64)) return 1;
  std::mt19937_64 rng(3);
  int narrow = 0, wide = 0;
  for (int trial = 0; trial < 20000; ++trial) {
    const int bytes = 1 << rng() % 3, page_size = 8 << rng() % 8;
    const long long slot = (long long)(rng() >> (29 + rng() % 34)), page = (long long)(rng() >> (29 + rng() % 34)), head = (long long)(rng() >> (29 + rng() % 34));
    const int id = (int)(rng() % 1000000), hk = (int)(rng() % 64);
    if (check_cells<false>(page, slot, head, bytes, page_size, id, hk)) return 1;
    if (narrow_slots(slot, bytes, page_size)) {
      ++narrow;
      if (check_cells<true>(page, slot, head, bytes, page_size, id, hk)) return 1;
    } else {
      ++wide;
    }
  }
  if (narrow < 1000 || wide < 1000) return fail("trials", narrow);
  // the last distance whose offsets fit 32 bits, the first that does not, and those about 2^32 bytes
  for (int bytes : {1, 2, 4})
    for (int page_size : {8, 16, 1024}) {
      const long long edge = (1LL << 31) / bytes / page_size;
      if (!narrow_slots(edge - 1, bytes, page_size) || narrow_slots(edge, bytes, page_size)) return fail("the rule", bytes);
      if (check_cells<true>(edge * page_size, edge - 1, 64, bytes, page_size, 3, 1)) return 1;
      for (long long slot : {edge, (1LL << 32) / bytes - 1, (1LL << 32) / bytes, (1LL << 32) / bytes + 64, (1LL << 33) / bytes})
        if (check_cells<false>(128, slot, 64, bytes, page_size, 5, 1)) return 1;
    }
  printf("ok\n");
  return 0;
}

// Host check of csrc/seq/paging.hpp: pages of places, bad tables, the slots that an append writes, and the scales' exponents.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <random>
#include <set>
#include <vector>

#include "seq/paging.hpp"

using namespace ntk;

static int fail(const char* what, long long x) {
  printf("%s %lld\n", what, x);
  return 1;
}

// Every row of a tile once, at its own slot and in its group's page.
template <int CH, int WAVES>
static int check_tile(int rows) {
  using At = TilePlaces<CH, WAVES>;
  const int ni = (rows * CH + 64 * WAVES - 1) / (64 * WAVES);
  for (int shift = 3; shift <= 10; ++shift) {
    PageTable t;
    t.shift = shift;
    for (int tile0 = 0; tile0 < 4096; tile0 += 32) {
      std::vector<int> seen((size_t)ni * 64 * WAVES / CH, 0);
      for (int i = 0; i < ni; ++i)
        for (int wave = 0; wave < WAVES; ++wave)
          for (int lane = 0; lane < 64; ++lane) {
            const int row = At::row(i, wave, lane), g = At::group(At::first(i, wave), lane);
            if (g % 8 || row < g || row >= g + 8) return fail("group", row);
            if ((tile0 + g) >> shift != (tile0 + row) >> shift) return fail("two pages", row);
            if (t.slot(tile0 + g) + row % 8 != t.slot(tile0 + row)) return fail("slot of a row", row);
            // the lane whose look() has the group, and what an instruction reads it by
            const int by = At::RPI <= 8 || lane < 32 ? At::first(i, wave) / 8 : At::first(i, wave) / 8 + 1;
            if (by * 8 != g) return fail("entry of a row", row);
            ++seen[row];
          }
      for (int n : seen)
        if (n != CH) return fail("chunks of a row", n);
    }
  }
  return 0;
}

int main() {
  if (check_tile<4, 1>(32) || check_tile<4, 4>(64) || check_tile<4, 4>(32) || check_tile<8, 1>(32) || check_tile<8, 4>(64) || check_tile<8, 4>(32) ||
      check_tile<16, 1>(32) || check_tile<16, 4>(64) || check_tile<16, 4>(32) || check_tile<32, 1>(32) || check_tile<32, 4>(32))
    return 1;
  std::mt19937 rng(7);
  for (int trial = 0; trial < 4000; ++trial) {
    PageTable t;
    t.shift = rng() % 7;
    t.most = rng() % 9;
    t.pages = 1 + rng() % 40;
    const int batch = 1 + rng() % 3, size = 1 << t.shift;
    // one entry to spare on either side, which names no page
    std::vector<int> table((size_t)batch * t.most + 2, 12345);
    for (int i = 0; i < batch * t.most; ++i) {
      const int kind = rng() % 8;
      table[i + 1] = kind == 0 ? -1 - (int)(rng() % 5) : kind == 1 ? t.pages + (int)(rng() % 5) : kind == 2 ? 0x7fffffff : (int)(rng() % t.pages);
    }
    t.table = table.data() + 1;
    for (int b = 0; b < batch; ++b)
      for (int pos = -3; pos < t.most * size + 40; ++pos) {
        const int got = t.page(b, pos);
        int want = -1;
        if (pos >= 0 && pos / size < t.most) {
          const int id = t.table[b * t.most + pos / size];
          want = id >= 0 && id < t.pages ? id : -1;
        }
        if (got != want) return fail("page", pos);
        if (pos >= 0 && (t.slot(pos) != pos % size)) return fail("slot", pos);
      }
    // every new token once, at its place, and none past the table
    const int length = rng() % 70;
    const int held = (int)(rng() % (t.most * size + 30)) - 10, fresh = (int)(rng() % (length + 10)) - 5;
    const AppendSpan s(t, held, fresh, length);
    const int first = held < 0 ? 0 : held > t.most * size ? t.most * size : held;
    const int count = fresh < 0 ? 0 : fresh > length ? length : fresh;
    if (s.first != first || s.count != count) return fail("span", trial);
    std::set<int> written;
    for (int e = 0; e < append_pages(length, t.shift); ++e) {
      int lo, hi, token;
      const int at = (s.first >> t.shift) + e;
      if (!s.slots(t, at, lo, hi, token)) continue;
      if (lo < 0 || hi > size || lo >= hi) return fail("slots", trial);
      for (int k = lo; k < hi; ++k) {
        const int i = token + k - lo;
        if (i < 0 || i >= count || at * size + k != first + i || !written.insert(i).second) return fail("token", trial);
      }
      if (lo > 0 && at * size + lo != first) return fail("older", trial);
    }
    int want = 0;
    for (int i = 0; i < count; ++i) want += first + i < t.most * size;
    if ((int)written.size() != want) return fail("written", trial);
  }
  // large caches: no product leaves 32 bits
  {
    PageTable t;
    t.shift = 10;
    t.most = (1 << 21) - 2;
    t.pages = 5;
    const int places = t.most << t.shift;
    const AppendSpan s(t, places - 3, 2000, 2000);
    int lo, hi, token, n = 0;
    for (int e = 0; e < append_pages(2000, t.shift); ++e)
      if (s.slots(t, (s.first >> t.shift) + e, lo, hi, token)) n += hi - lo;
    if (n != 3) return fail("the end of a large cache", n);
  }
  // the least power of two that x is at most 448 times of
  for (int trial = 0; trial < 200000; ++trial) {
    uint32_t u = rng() & 0x7fffffffu;
    if (trial < 600) u = (uint32_t)((trial % 200 + 20) << 23) | (trial < 200 ? 0x600000u : trial < 400 ? 0x600001u : 0x5fffffu);
    float x;
    memcpy(&x, &u, 4);
    if (!isfinite(x)) continue;
    const int e = e4m3_exponent(x);
    if (e < -126 || e > 120) return fail("range of the exponent", trial);
    if (!((double)x <= 448.0 * ldexp(1.0, e))) return fail("too small", trial);
    if (e > -126 && !((double)x > 448.0 * ldexp(1.0, e - 1))) return fail("too large", trial);
  }
  if (e4m3_exponent(0.f) != -126) return fail("zero", 0);
  printf("ok\n");
  return 0;
}

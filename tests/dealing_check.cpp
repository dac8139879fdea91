// Host check of csrc/seq/dealing.hpp: every tile of keys is taken once, and what every worker is told lies within the work, also
// where there is none for it.
#include <stdio.h>

#include <random>
#include <vector>

#include "seq/dealing.hpp"

using namespace ntk;

static int fail(const char* what, long long x) {
  printf("%s %lld\n", what, x);
  return 1;
}

// pairs with `nt` tiles of keys each; `inside`: a sequence's heads in a row
static int check(const std::vector<int>& nt, int Hk, bool inside, bool few_rows, int workers, int least, int& idle, int& shared) {
  const int n = (int)nt.size(), times = inside ? Hk : 1, heads = inside ? 1 : Hk;
  long long all = 0;
  for (int c : nt) all += c;
  Deal d(n, times, heads, workers, least, (int)(all * times));
  if (few_rows && d.may_share()) {
    int parts[Deal::TRIES] = {};
    for (int k = 0; k < Deal::TRIES; ++k) {
      if (d.length(k) < 1) return fail("length", k);
      for (int c : nt) parts[k] += times * ((c + d.length(k) - 1) / d.length(k));
    }
    d.choose(parts);
  }
  shared += d.share > 0;
  std::vector<std::vector<int>> seen((size_t)n * Hk);            // which worker took it
  for (int p = 0; p < n; ++p)
    for (int h = 0; h < Hk; ++h) seen[(size_t)p * Hk + h].assign(nt[p], -1);
  for (int w = 0; w < workers; ++w) {
    // the pair whose units hold the worker's first one; with none, what the array held before
    Deal::Part found = {0x5a5a5a5a, 0x5a5a5a5a, 0x5a5a5a5a, 0x5a5a5a5a, 0x5a5a5a5a};
    int x = 0;
    for (int p = 0; p < n; ++p) {
      const int u = times * d.units(nt[p]);
      if (d.at(w) >= x && d.at(w) < x + u) found = d.within(p, nt[p], x, w);
      x += u;
    }
    Deal::Part t = d.taken(found, w);
    if (t.pair < 0 || t.pair >= n) return fail("pair", t.pair);
    if (t.hk < 0 || t.hk >= Hk) return fail("head", t.hk);
    if (t.t < 0 || t.t >= nt[t.pair]) return fail("tile", t.t);
    if (t.left < 0 || t.left > std::max(d.per, d.share)) return fail("left", t.left);
    if (t.per < 1 || t.per > std::max(d.per, d.share)) return fail("per", t.per);
    idle += t.left == 0;
    for (; t.left > 0; --t.left) {
      int& s = seen[(size_t)t.pair * Hk + t.hk][t.t];
      if (s >= 0) return fail("taken twice", t.t);
      s = w;
      if (++t.t < nt[t.pair]) continue;
      t.t = 0;
      if (d.share && t.left > 1) return fail("a part past its row tile", w);
      if (inside ? ++t.hk == Hk : ++t.pair == n) inside ? (t.hk = 0, ++t.pair) : (t.pair = 0, ++t.hk);
      if (t.left > 1 && (t.pair >= n || t.hk >= Hk)) return fail("past the end", w);
    }
  }
  // whole, and a row tile's parts with workers side by side, each `per` of them but for the last
  for (auto& row : seen)
    for (size_t i = 0; i < row.size(); ++i) {
      if (row[i] < 0) return fail("left out", (long long)i);
      if (i && row[i] != row[i - 1] && row[i] != row[i - 1] + 1) return fail("order of workers", (long long)i);
    }
  return 0;
}

int main() {
  int idle = 0, shared = 0;
  // one token of two heads over 1030, 1 and 0 places, in runs of 16 tiles by 8 workers: five have work
  if (check({33, 1, 1}, 2, true, false, 8, 16, idle, shared)) return 1;
  if (idle != 3) return fail("workers without work", idle);
  if (check({33, 1, 1}, 2, true, true, 8, 16, idle, shared)) return 1;
  std::mt19937 rng(11);
  for (int trial = 0; trial < 60000; ++trial) {
    const bool few = rng() % 2, inside = few || rng() % 2;
    const int n = 1 + rng() % (1 << rng() % 7), Hk = 1 + rng() % 8, workers = rng() % 3 ? 8 * (1 + rng() % 64) : 1 + rng() % 7;
    const int least = 1 + rng() % 32, longest = 1 << rng() % 9;
    std::vector<int> nt(n);
    for (int& c : nt) c = rng() % 4 ? 1 + rng() % longest : 1;
    if (check(nt, Hk, inside, few, workers, least, idle, shared)) return fail("trial", trial);
  }
  if (idle < 1000 || shared < 1000) return fail("trials", idle);
  // as much as there can be
  if (check(std::vector<int>(512, (1 << 16) - 1), 2, false, false, 512, 4, idle, shared)) return 1;
  Deal d(4096, 1, 8, 512, 4, (1 << 27) - 1);
  if (d.start(511) < 0 || (long long)d.per * 512 < ((1LL << 27) - 1) * 8) return fail("2^30 tiles", d.per);
  printf("ok\n");
  return 0;
}

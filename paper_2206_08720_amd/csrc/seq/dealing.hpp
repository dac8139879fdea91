// dealing.hpp -- which tiles of keys each worker of the attention over pages takes (integer arithmetic, for the kernels and for the host).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

namespace ntk {

// `pairs` row tiles, each `times` times in a row (a sequence's heads), and all of it `heads` times over: one of times and heads is 1.  A row
// tile counts as its tiles of keys, at least one.  The workers take equal runs of `per` tiles, or, with `share`, parts of at most
// `share` tiles that end with their row tile.  Fewer than 2^30 tiles in all.
struct Deal {
  static constexpr int TRIES = 6;
  int pairs, times, heads, workers;
  int per, top;                            // tiles a run; the longest parts that are tried instead
  int share, total;                        // total: units (tiles, or parts) of the pairs, `times` included

  // `tiles`: of all pairs, `times` included
  __host__ __device__ __forceinline__ Deal(int pairs_, int times_, int heads_, int workers_, int least, int tiles)
      : pairs(pairs_), times(times_), heads(heads_), workers(workers_), share(0), total(tiles) {
    const int all = tiles * heads;
    per = top = std::max(least, (all + workers - 1) / workers);
    const int spare = workers - pairs * times * heads;
    if (spare > 0) top = std::min(std::max(least, (all + spare - 1) / spare), per + per / 4 + 8);
  }
  // whether parts can be as many as there are workers, and the lengths that are tried, the least first
  __host__ __device__ __forceinline__ bool may_share() const { return pairs * times * heads < workers; }
  __host__ __device__ __forceinline__ int length(int k) const { return per + (top - per) * ((1 << k) >> 1) / 16; }
  // parts: those of the pairs under each length, `times` included
  __host__ __device__ __forceinline__ void choose(const int* parts) {
#pragma unroll
    for (int k = TRIES - 1; k >= 0; --k)
      if (parts[k] * heads <= workers) {
        share = length(k);
        total = parts[k];
      }
  }
  __host__ __device__ __forceinline__ int units(int tiles) const { return share ? (tiles + share - 1) / share : tiles; }
  // the first unit of worker `number`
  __host__ __device__ __forceinline__ int start(int number) const { return number * (share ? 1 : per); }
  // its head, where a head's pairs come together, and its first unit among the pairs
  __host__ __device__ __forceinline__ int head(int number) const { return times > 1 || heads == 1 ? 0 : start(number) / total; }
  __host__ __device__ __forceinline__ int at(int number) const { return start(number) - head(number) * total; }

  // What a worker takes: from tile t of a pair and head on, `left` tiles, in parts of `per`.
  struct Part {
    int pair, t, hk, left, per;
  };
  // from pair p, which has `tiles` tiles, and whose units begin at x <= at(number) and end behind it
  __host__ __device__ __forceinline__ Part within(int p, int tiles, int x, int number) const {
    const int u = units(tiles), i = (at(number) - x) % u, hk = times > 1 ? (at(number) - x) / u : head(number);
    if (!share) return Part{p, i, hk, std::min(per, total * heads - start(number)), per};
    const int equal = (tiles + u - 1) / u, t = i * equal;        // a row tile's parts are equal ones, of which the last may be none
    return t < tiles ? Part{p, t, hk, std::min(equal, tiles - t), equal} : Part{p, 0, hk, 0, equal};
  }
  // `found`: what the thread that has the worker's first unit noted.  Behind the last unit no thread has one, and the worker's part is
  // none of the first pair: `found` then holds anything.
  __host__ __device__ __forceinline__ Part taken(const Part& found, int number) const {
    if (start(number) >= total * heads) return Part{0, 0, 0, 0, per};
    return found;
  }
};

}  // namespace ntk

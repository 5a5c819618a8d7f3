// How the attention of new tokens is cut into units of work: plain arithmetic, also for a host compiler.
//
// A request's n new tokens, the last of its `len`, are taken 2^q_shift to a tile; the cache is read 2^t_shift tokens at a step.  Tile r sees no
// more than the tokens up to its last row's, so it has min(cap, ceil((first + (r + 1) Q) / T)) steps, first = len - n, cap = ceil(len / T); a unit is one
// step of one tile of one KV head.  Q and T are powers of two, so the units before a tile have a closed form, and a unit's tile is found by halving.
#pragma once

#include <cstdint>

namespace pillar {

#ifdef __HIPCC__
#define PILLAR_RULE __host__ __device__ inline
#else
#define PILLAR_RULE inline
#endif

struct PromptSteps {
  int q_shift, t_shift;
  int from;                    // tokens before, rounded up to steps, and a tile: the numerator of the first tile's steps
  int cap;
  int tiles;                   // 0: nothing to do (no new token, or none in the cache)

  PILLAR_RULE PromptSteps(int len, int n, int q_shift_, int t_shift_) : q_shift(q_shift_), t_shift(t_shift_) {
    const int first = len > n ? len - n : 0;             // (rows whose number would be negative see nothing; their tiles have a few steps all the same)
    from = first + (1 << t_shift) - 1 + (1 << q_shift);
    cap = (len + (1 << t_shift) - 1) >> t_shift;
    tiles = len > 0 && n > 0 ? (n + (1 << q_shift) - 1) >> q_shift : 0;
  }
  PILLAR_RULE int steps(int r) const {
    const int64_t s = (from + (static_cast<int64_t>(r) << q_shift)) >> t_shift;
    return s < cap ? static_cast<int>(s) : cap;
  }
  // sum over i < n of i >> d
  static PILLAR_RULE int64_t sum_of_shifted(int64_t n, int d) {
    const int64_t k = n >> d;
    return ((k * (k - 1) / 2) << d) + (n - (k << d)) * k;
  }
  // units of the tiles before r, r <= tiles
  PILLAR_RULE int64_t before(int r) const {
    const int d = q_shift - t_shift;
    if (d >= 0) {                                        // steps(r) = a + (r << d) as long as that is below cap
      const int64_t a = from >> t_shift, room = cap > a ? (cap - a + (1 << d) - 1) >> d : 0, k = room < r ? room : r;
      return k * a + ((k * (k - 1) / 2) << d) + (r - k) * cap;
    }
    const int64_t a = from >> q_shift, room = (static_cast<int64_t>(cap) << -d) - a, k = room < 0 ? 0 : room < r ? room : r;
    return sum_of_shifted(a + k, -d) - sum_of_shifted(a, -d) + (r - k) * cap;
  }
  PILLAR_RULE int units() const { return tiles > 0 ? static_cast<int>(before(tiles)) : 0; }
  // the tile that has unit u, 0 <= u < units()
  PILLAR_RULE int tile_of(int u) const {
    int lo = 0, hi = tiles;                              // before(lo) <= u < before(hi)
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before(mid) <= u) lo = mid;
      else hi = mid;
    }
    return lo;
  }
};

// Tokens of a tile: the largest power of two whose rows, `group` to a token, fit into `rows`.
PILLAR_RULE int tile_tokens_shift(int rows, int group) {
  int s = 0;
  while ((2 << s) * group <= rows) ++s;
  return s;
}

}  // namespace pillar

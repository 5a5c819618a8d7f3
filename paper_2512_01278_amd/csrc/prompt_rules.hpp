// How the attention of new tokens is cut into units of work: plain arithmetic, also for a host compiler.
//
// A request's n new tokens, the last of its `len`, are taken 2^q_shift to a tile; the cache is read 2^t_shift tokens at a step.  Tile r sees no
// more than the tokens up to its last row's, so it has min(cap, ceil((first + (r + 1) Q) / T)) steps, first = len - n, cap = ceil(len / T); a unit is one
// step of one tile of one KV head.  Q and T are powers of two, so the units before a tile have a closed form, and a unit's tile is near a root.
#pragma once

#include <cstdint>

namespace pillar {

#ifdef __HIPCC__
#define PILLAR_RULE __host__ __device__ inline
#else
#define PILLAR_RULE inline
#endif

// Everything below is 32-bit arithmetic without sign: counts of units are below 2^31, and where a term is larger on the way, only differences of such terms are
// taken, which come out right modulo 2^32.  (In 64 bits the search below took the kernels 2 us, and the one that joins partials, where every
// wavefront searches, 17 of its 25.)
struct PromptSteps {
  int q_shift, t_shift;
  uint32_t from;               // tokens before, rounded up to steps, and a tile: the numerator of the first tile's steps
  int cap;
  int tiles;                   // 0: nothing to do (no new token, or none in the cache)
  int setup;                   // units that a tile has beside its steps, ahead of them: what it costs to begin and end one

  PILLAR_RULE PromptSteps(int len, int n, int q_shift_, int t_shift_, int setup_) : q_shift(q_shift_), t_shift(t_shift_), setup(setup_) {
    const uint32_t first = len > n ? len - n : 0;        // (rows whose number would be negative see nothing; their tiles have a few steps all the same)
    from = first + (1u << t_shift) - 1 + (1u << q_shift);
    cap = static_cast<int>((static_cast<uint32_t>(len) + (1u << t_shift) - 1) >> t_shift);
    tiles = len > 0 && n > 0 ? static_cast<int>((static_cast<uint32_t>(n) + (1u << q_shift) - 1) >> q_shift) : 0;
  }
  PILLAR_RULE int steps(int r) const {
    const int s = static_cast<int>((from + (static_cast<uint32_t>(r) << q_shift)) >> t_shift);
    return s < cap ? s : cap;
  }
  // 0 + 1 + ... + k - 1, modulo 2^32
  static PILLAR_RULE uint32_t up_to(uint32_t k) { return (k & 1) ? k * ((k - 1) >> 1) : (k >> 1) * (k - 1); }
  // sum over i < n of i >> d, modulo 2^32
  static PILLAR_RULE uint32_t sum_of_shifted(uint32_t n, int d) {
    const uint32_t k = n >> d;
    return (up_to(k) << d) + (n - (k << d)) * k;
  }
  // the tiles ahead of the first that reads all of the cache: up to there, steps grow (there may be fewer tiles than that)
  PILLAR_RULE int growing() const {
    const int d = q_shift - t_shift;
    if (d >= 0) {
      const int a = static_cast<int>(from >> t_shift);
      return cap > a ? (cap - a + (1 << d) - 1) >> d : 0;
    }
    const int room = static_cast<int>((static_cast<uint32_t>(cap) << -d) - (from >> q_shift));
    return room < 0 ? 0 : room;
  }
  // units of the tiles before r, r <= tiles
  PILLAR_RULE int before(int r) const {
    const int d = q_shift - t_shift, room = growing(), k = room < r ? room : r;
    const uint32_t rest = static_cast<uint32_t>(r - k) * cap + static_cast<uint32_t>(r) * setup;
    if (d >= 0) return static_cast<int>(static_cast<uint32_t>(k) * (from >> t_shift) + (up_to(k) << d) + rest);        // steps(r) = a + (r << d) as long as that is below cap
    const uint32_t a = from >> q_shift;
    return static_cast<int>(sum_of_shifted(a + k, -d) - sum_of_shifted(a, -d) + rest);
  }
  PILLAR_RULE int units() const { return tiles > 0 ? before(tiles) : 0; }
  // The tile that has unit u, 0 <= u < units(), or one near it.  Of growing tiles, where steps grow by g = Q / T from tile to tile, those before r have
  // s r + g r^2 / 2 units, s = steps(0) - g / 2 + setup, and this is its root.  With T > Q steps are stairs of T / Q tiles, (from + r Q) / T - 1/2 (1 - g) on the average, and the
  // sum is off by T / 8 Q units at the most.  The other tiles are alike (with far more new rows than tokens in the cache, nearly all are).
  PILLAR_RULE int tile_near(int u) const {
    const int room = growing(), k = room < tiles ? room : tiles, grown = before(k);
    if (u >= grown) return k + (u - grown) / (cap + setup);
    const float g = static_cast<float>(1 << q_shift) / static_cast<float>(1 << t_shift);
    const float s = setup + (q_shift >= t_shift ? static_cast<float>(from >> t_shift) - 0.5f * g : static_cast<float>(from >> q_shift) * g - 0.5f);
    const int r = static_cast<int>(2.f * static_cast<float>(u) / (s + sqrt_of(s * s + 2.f * g * static_cast<float>(u))));
    return r < 0 ? 0 : r >= k ? k - 1 : r;
  }
  PILLAR_RULE int tile_of(int u) const {
    int r = tile_near(u);
    while (r > 0 && before(r) > u) --r;
    while (r + 1 < tiles && before(r + 1) <= u) ++r;
    return r;
  }
  static PILLAR_RULE float sqrt_of(float x) {
#ifdef __HIP_DEVICE_COMPILE__
    return __builtin_amdgcn_sqrtf(x);
#else
    return __builtin_sqrtf(x);
#endif
  }
};

// Tokens of a tile: the largest power of two whose rows, `group` to a token, fit into `rows`.
PILLAR_RULE int tile_tokens_shift(int rows, int group) {
  int s = 0;
  while ((2 << s) * group <= rows) ++s;
  return s;
}

}  // namespace pillar

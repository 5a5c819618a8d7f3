// What the passes over a paged cache in 32 x 32 products share (verify_tree.hip, prompt_attn.hip): the shape of a workgroup, equal ranges of units of work that every
// wavefront finds by itself, and the rows of a tile on their way from the pages into LDS.
#pragma once

#include <type_traits>

#include "launch.hpp"
#include "tree_tile.hpp"

namespace pillar {

// What a smaller v_scale (that of a page of zeros) counts as: far enough below any other for its rows to add nothing to O, and a token's share of l, which passes
// through an exponential with v_scale in its exponent, is flushed (at 2^-126) only from 2^-46 of the largest scale on.  (2^-100: from 2^-26, 2000 tokens of
// 2^-20 beside a page of scale 2^12 were missing from l.)  2^8 / kLeastScale times all tokens there may be stays below 2^128.
constexpr float kLeastScale = 0x1p-80f;

// As many ranges as the chip holds workgroups, or `few` (one to a compute unit) where those would have fewer than eight units each: a range costs a
// partial result of RT rows that is written and read back, and a second workgroup on the compute unit gains less than that.  Two / one to a
// compute unit: one request of 8000 tokens with 26 nodes 42 / 33 us, 4 of 2100 38 / 32, with 60 nodes 48 / 40, 8 of 2100 46 / 39; 16 of 4000
// (16 units each) 78 / 79, 32 of 4096 with 32 nodes 118 / 130.
constexpr int kFewUnits = 8;
// And never so many that a tile's partials take longer to join than its units: with U units to a tile, a range has sqrt(U / 8) of them at the least.  One
// unit / the rule: one request of 2100 tokens (33 units) with 26 nodes 25.7 / 22.2 us, with 60 34.0 / 28.5, of 20000 with one kv head 48 / 29.5;
// of 8000 with 8 kv heads and 500 the same; with one node 15.2 / 17.  sqrt(U / 4) and sqrt(U / 16) are slower by up to 3.  An fp32 unit takes
// far longer than the joining of a partial: 2 of 2100 tokens with 26 nodes 35 / 48, so there the rule is off.
constexpr int kMostUnits = 16;                           // (where the root is more, the number of workgroups decides)

// Range w of n has units range_begin(w) .. range_begin(w + 1) - 1.
struct Ranges {
  int n, each, longer;         // the first `longer` ranges have each + 1 units, the others `each`
  __device__ __forceinline__ Ranges(int total, int workgroups, int few, int tiles8) {
    const int eighth = (total - 1) / tiles8;
    int least = 1;                                       // sqrt(total / tiles8), rounded up; in integers, so that all kernels agree
    while (least < kMostUnits && least * least <= eighth) ++least;
    n = max(1, min(total / least, total < kFewUnits * workgroups ? few : workgroups));
    each = total / n;
    longer = total - each * n;
  }
  __device__ __forceinline__ int begin(int w) const { return w * each + min(w, longer); }
  __device__ __forceinline__ int of(int u) const {          // the range that has unit u
    const int split = longer * (each + 1);
    return u < split ? u / (each + 1) : longer + (u - split) / each;
  }
};

// What a workgroup finds out about its share of the work, every wavefront for itself: 64 requests at a time, a request per lane.
struct Share {
  int w, u0, u1;               // its range, first unit and past the last
  int b, ub;                   // the request that has unit u0, and that request's first unit
  int total;                   // units of the launch
  // units: of a request; each(c): called for every 64 requests; prefix: the first workgroup leaves the units before every request, and all of them, there
  template <typename F, typename Each>
  __device__ __forceinline__ Share(int batch, int workgroups, int few, int tiles8, int32_t* prefix, F units, Each each) {
    const int lane = threadIdx.x & 63;
    int mine = 0, upto = 0;
    total = 0;
    for (int c = 0; c < batch; c += 64) {
      mine = c + lane < batch ? units(c + lane) : 0;
      upto = total + wave_inclusive(mine);
      total = __builtin_amdgcn_readlane(upto, 63);
      each(c);
    }
    const Ranges ranges(total, workgroups, few, tiles8);
    // neighbouring ranges, whose row tiles may share K and V, on one XCD (workgroups go round the XCDs in turn)
    w = blockIdx.x;
    u0 = u1 = b = ub = 0;
    if (w >= ranges.n) return;
    if (ranges.n % 8 == 0) w = (w & 7) * (ranges.n >> 3) + (w >> 3);
    u0 = ranges.begin(w);
    u1 = ranges.begin(w + 1);
    const bool leaves = prefix && w == 0 && threadIdx.x < 64;
    bool found = false;
    int before = 0;
    for (int c = 0; c < batch; c += 64) {
      if (batch > 64) {                                  // (else both are still there)
        mine = c + lane < batch ? units(c + lane) : 0;
        upto = before + wave_inclusive(mine);
        before = __builtin_amdgcn_readlane(upto, 63);
      }
      if (leaves && c + lane < batch) prefix[c + lane] = upto - mine;
      const uint64_t after = __ballot(upto > u0);
      if (!found && after) {
        const int at = __builtin_ctzll(after);
        b = c + at;
        ub = __builtin_amdgcn_readlane(upto - mine, at);
        found = true;
      }
      if (found && !leaves) break;
    }
    if (leaves && lane == 0) prefix[batch] = total;
    // (the same in all lanes: kept in scalar registers)
    w = __builtin_amdgcn_readfirstlane(w);
    u0 = __builtin_amdgcn_readfirstlane(u0);
    u1 = __builtin_amdgcn_readfirstlane(u1);
    b = __builtin_amdgcn_readfirstlane(b);
    ub = __builtin_amdgcn_readfirstlane(ub);
  }
};

template <int D_, int KV_, bool F32, int WR_, int WT_, int NS_, bool BYPASS>
struct Cfg {
  static constexpr bool kBypass = BYPASS;                                  // rows of the cache bypass the Infinity Cache
  static constexpr int D = D_, KV = KV_, WR = WR_, WT = WT_, NS = NS_;     // WR x WT wavefronts: groups of 32 rows x groups of tokens
  using E = std::conditional_t<F32, EngineF32<D>, EngineBf16<D>>;
  static constexpr int kWaves = WR * WT, kThreads = 64 * kWaves;
  static constexpr int kGroupTokens = 32 * NS, TS = kGroupTokens * WT, RT = 32 * WR;
  static constexpr int kPieces = D * kv_bytes<KV>() / 16;                  // 16-byte pieces of a row
  static constexpr int kLoads = (TS * kPieces + kThreads - 1) / kThreads;  // of K, and as many of V, per thread and tile
  static constexpr bool kAllLoad = TS * kPieces >= kThreads;
  static constexpr bool kScales = KV == PILLAR_FP8_E4M3 && !F32;           // page scales are applied to logits and P
  static constexpr int kTileBytes = TS * (E::kKPitch + E::kVPitch);
  static constexpr int kJoinRow = D + 4;                                   // floats
  static constexpr int kJoinBytes = WT > 1 ? kWaves * 32 * kJoinRow * 4 : 0;
  static constexpr int kLds = kTileBytes > kJoinBytes ? kTileBytes : kJoinBytes;
};

// The pieces of a tile that a thread carries, one place in every kRows-th row, between global memory and LDS.  V: of V too.
template <typename C, bool V>
struct Carrier {
  using E = typename C::E;
  static constexpr int kRows = C::kThreads / C::kPieces;
  const uint8_t* k_rows;       // this head's rows in page 0
  const uint8_t* v_rows;
  const int32_t* table;
  int last;                    // the last token: rows past it are read there
  int row0, piece;
  int pid[C::kLoads];
  u32x4 k[C::kLoads], v[V ? C::kLoads : 1];
  int scale_pid;
  float ks, vs;                // page scales of a token: of the thread's own (bf16 engine) ...
  static constexpr bool kRowScales = E::kF32 && C::KV == PILLAR_FP8_E4M3;
  float row_ks[kRowScales ? C::kLoads : 1], row_vs[kRowScales ? C::kLoads : 1];                  // ... of each row that is carried (fp32)

  __device__ __forceinline__ Carrier(const KvView& kv, int b, int g, int len) {
    const int64_t head = static_cast<int64_t>(g) * kv.stride_head * kv_bytes<C::KV>();
    k_rows = static_cast<const uint8_t*>(kv.k_pool) + head;
    v_rows = static_cast<const uint8_t*>(kv.v_pool) + head;
    table = kv.block_table + static_cast<int64_t>(b) * kv.block_table_stride;
    last = len - 1;
    row0 = threadIdx.x / C::kPieces;
    piece = threadIdx.x % C::kPieces;
  }
  __device__ __forceinline__ int row(int u) const { return row0 + u * kRows; }
  __device__ __forceinline__ bool carries() const { return C::kAllLoad || threadIdx.x < C::TS * C::kPieces; }
  __device__ __forceinline__ int token(int step, int r) const { return min(step * C::TS + r, last); }
  __device__ __forceinline__ void pages(const KvView& kv, int step) {
#pragma unroll
    for (int u = 0; u < C::kLoads; ++u) pid[u] = carries() ? table[token(step, row(u)) >> kv.page_shift] : 0;
    if (C::kScales) scale_pid = table[token(step, min<int>(threadIdx.x, C::TS - 1)) >> kv.page_shift];
  }
  __device__ __forceinline__ float k_scale(int u) const { return kRowScales ? row_ks[u] : 1.f; }
  __device__ __forceinline__ float v_scale(int u) const { return kRowScales ? row_vs[u] : 1.f; }
  static __device__ __forceinline__ u32x4 load(const uint8_t* p) {
    if constexpr (C::kBypass) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    else return *reinterpret_cast<const u32x4*>(p);
  }
  __device__ __forceinline__ void fetch(const KvView& kv, int g, int step, bool aligned) {
    if constexpr (E::kF32) {
      if (!carries()) return;
#pragma unroll
      for (int u = 0; u < C::kLoads; ++u) {
        const int64_t at = static_cast<int64_t>(g) * kv.stride_head + static_cast<int64_t>(pid[u]) * kv.stride_page +
                           static_cast<int64_t>(token(step, row(u)) & (kv.page_size - 1)) * kv.stride_slot + piece * (16 / kv_bytes<C::KV>());
        k[u] = load_piece<C::KV>(kv.k_pool, at, aligned);
        if constexpr (V) v[u] = load_piece<C::KV>(kv.v_pool, at, aligned);
        if constexpr (kRowScales) {
          const int64_t s = static_cast<int64_t>(pid[u]) * kv.num_kv_heads + g;
          row_ks[u] = kv.k_scale[s];
          if constexpr (V) row_vs[u] = kv.v_scale[s];
        }
      }
      return;
    }
    // (strides below 2^32 bytes: a row's offset is two products of 32 bits)
    const uint32_t page_bytes = static_cast<uint32_t>(kv.stride_page * kv_bytes<C::KV>()), slot_bytes = static_cast<uint32_t>(kv.stride_slot * kv_bytes<C::KV>());
    if (carries()) {
#pragma unroll
      for (int u = 0; u < C::kLoads; ++u) {
        const uint64_t at = static_cast<uint64_t>(static_cast<uint32_t>(pid[u])) * page_bytes +
                            static_cast<uint64_t>(static_cast<uint32_t>(token(step, row(u)) & (kv.page_size - 1))) * slot_bytes + 16 * piece;
        k[u] = load(k_rows + at);
        if constexpr (V) v[u] = load(v_rows + at);
      }
    }
    if (C::kScales) {
      const int64_t at = static_cast<int64_t>(scale_pid) * kv.num_kv_heads + g;
      ks = kv.k_scale[at];
      if (V) vs = kv.v_scale[at];
    }
  }
};

// the matrix-core kernels work out a row's offset from strides of 32 bits
inline bool strides_fit(const KvView& kv, int kv_dtype) {
  const int64_t most = (int64_t{1} << 32) / (kv_dtype == PILLAR_BF16 ? 2 : 1) - 1;
  return kv.stride_page <= most && kv.stride_slot <= most;
}

}  // namespace pillar

// Verification of a tree of drafted tokens over the paged cache.
//
// Paper Section 4.1 verifies a chain: query i sees everything up to its own position.  Here the n drafted tokens, the last n of
// the context, form a tree (or any graph): node i sees the tokens before the tree and those nodes whose bit its word has.
//
//   out  = softmax(sm_scale q K^T over what the node sees) V
//   lse  = log sum exp of the same logits
//   scores[t] = 1 / (n G) sum over the rows of exp(sm_scale q k_t - lse)          (the statistic; optional)
//
// Launches:
//   tree_pass    one pass over K and V with the running maximum and sum of every row's softmax.  A unit of work is TS tokens of one (request, KV
//                head, tile of RT rows); all units in a row are cut into equal ranges, one per resident workgroup, so lengths on the
//                device need no plan on the host.  A stretch of one tile that a range does not hold whole leaves a partial (m, l, O).
//   tree_merge   joins the partials.
//   tree_scores  (with scores) K once more against the final log-sum-exp, summed over the rows.  With n G rows a stash of P would be 2 n G
//                bytes a token written and read where K's second read is 2 D: at 64 and more rows the read is less.  With fewer it is not: chains have
//                the calls of verify_range.hip, which stash (in 11 bits).  64 requests of 8192 tokens with the statistic, 4 heads to a KV head, this /
//                those: one node 522 / 391 us, 4 540 / 441, 8 536 / 515, 12 562 / 582, 16 554 / 641; fp8 318 / 218, 327 / 265, 323 / 322, 425 /
//                361, 422 / 453.  A tree of few rows takes the second read all the same, and has fp32 scores.
#include <algorithm>

#include "host_rules.hpp"
#include "launch.hpp"
#include "paged_pass.hpp"

namespace pillar {
namespace {

constexpr int kTreeNodes = 64;
struct TreeParams {
  KvView kv;
  const void* q;
  const int32_t* tree_sizes;   // null: max_nodes each
  const uint64_t* visible;
  void* out;
  float* lse;                  // may be null
  int32_t max_nodes, group, q_dtype;
  bool aligned;                // cache rows can be read 16 bytes at a time,
  bool dense;                  // rows of q and out too
  // workspace
  int32_t* prefix;             // [B+1] units before a request, and all of them
  float* part_ml;              // [slots][RT][2]
  float* part_o;               // [slots][RT][D]
  float* lse2;                 // [B][max_nodes][Hq], in log2 units; only with scores
  int32_t ranges, few;         // workgroups of the pass; of those, with little to do
  int32_t tiles8;              // eight times the tiles there may be, or the largest number where a tile may go into ranges of one unit
};

// Units are counted the same way by the pass and the merge.
struct Shape {
  int len, nodes, rows, steps, tiles;
};
template <int TS, int RT>
__device__ __forceinline__ Shape shape_of(const TreeParams& a, int b) {
  Shape s;
  s.len = min(max(a.kv.seq_lens[b], 0), a.kv.max_seq_len);
  s.nodes = a.tree_sizes ? min(max(a.tree_sizes[b], 0), a.max_nodes) : a.max_nodes;
  s.rows = s.nodes * a.group;
  s.steps = (s.len + TS - 1) / TS;
  s.tiles = (s.rows + RT - 1) / RT;
  return s;
}
template <int TS, int RT>
__device__ __forceinline__ int units_of(const TreeParams& a, int b) {
  const Shape s = shape_of<TS, RT>(a, b);
  return s.steps * s.tiles * a.kv.num_kv_heads;
}

// Which of 32 tokens a row sees that has `word`, the tree beginning `before` tokens on from the first of them (or -before ahead of it).
__device__ __forceinline__ uint32_t sees_of(uint64_t word, int before) {
  if (before >= 32) return ~0u;
  if (before <= -64) return 0;
  return before >= 0 ? static_cast<uint32_t>(word << before) | ((1u << before) - 1) : static_cast<uint32_t>(word >> -before);
}

// four dims of an output row
template <int D>
__device__ __forceinline__ void store_dims(const TreeParams& a, int64_t row, int dim, f32x4 x) {
  const int64_t at = row * D + dim;
  if (a.q_dtype == PILLAR_F32) {
    if (a.dense) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = x;
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) Storage<PILLAR_F32>::store(a.out, at + j, x[j]);
  } else {
    if (a.dense) {
      u32x2 y;
      y.x = f32_to_bf16(x[0]) | static_cast<uint32_t>(f32_to_bf16(x[1])) << 16;
      y.y = f32_to_bf16(x[2]) | static_cast<uint32_t>(f32_to_bf16(x[3])) << 16;
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + at) = y;
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) Storage<PILLAR_BF16>::store(a.out, at + j, x[j]);
  }
}

// Results of the rows of a request that has nothing to see, by a whole workgroup.
template <int D>
__device__ __forceinline__ void see_nothing(const TreeParams& a, int b, int nodes) {
  const int64_t first = static_cast<int64_t>(b) * a.max_nodes * a.kv.num_q_heads;
  const int rows = nodes * a.kv.num_q_heads;
  for (int64_t e = threadIdx.x; e < static_cast<int64_t>(rows) * D; e += blockDim.x) {
    if (a.q_dtype == PILLAR_F32) Storage<PILLAR_F32>::store(a.out, first * D + e, 0.f);
    else Storage<PILLAR_BF16>::store(a.out, first * D + e, 0.f);
  }
  if (a.lse)
    for (int r = threadIdx.x; r < rows; r += blockDim.x) a.lse[first + r] = -INFINITY;
}

template <typename C>
__global__ __launch_bounds__(C::kThreads, C::E::kF32 ? 1 : 2) void tree_pass(TreeParams a) {
  using E = typename C::E;
  constexpr int D = C::D, TS = C::TS, RT = C::RT;
  __shared__ __attribute__((aligned(16))) uint8_t smem[C::kLds];
  // page scales of the tile's tokens: k_scale in the logits' unit, log2 of v_scale, and one over it
  __shared__ __attribute__((aligned(16))) float s_ks[C::kScales ? TS : 4], s_log_vs[C::kScales ? TS : 4], s_inv_vs[C::kScales ? TS : 4];
  __shared__ float s_m[C::kWaves][32], s_l[C::kWaves][32];
  __shared__ uint32_t s_bad[2][2];                       // nodes whose V row is not finite throughout
  const KvView& kv = a.kv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % C::WR, wt = wave / C::WR;
  const int n = lane & 31, g2 = lane >> 5;
  uint8_t* const ktile = smem;
  uint8_t* const vtile = smem + TS * E::kKPitch;
  const float scale2 = kv.sm_scale * kLog2e;
  const float unit = C::kScales ? 1.f : scale2;          // of the logits, in log2: page scales come with it

  const Share share(kv.batch, a.ranges, a.few, a.tiles8, a.prefix, [&](int r) { return units_of<TS, RT>(a, r); }, [&](int c) {
    // contexts without a token have no unit: their rows are shared out among the workgroups
    for (uint64_t none = __ballot(c + lane < kv.batch && kv.seq_lens[min(c + lane, kv.batch - 1)] <= 0); none; none &= none - 1) {
      const int r = c + __builtin_ctzll(none);
      if (r % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x)) see_nothing<D>(a, r, shape_of<TS, RT>(a, r).nodes);
    }
  });
  int b = share.b, ub = share.ub;                        // the request at work and its first unit
  const int w = share.w, u0 = share.u0, u1 = share.u1;
  if (u0 == u1) return;
  if (tid < 2) s_bad[0][tid] = 0;
  int parity = 0;              // of the stretch: the other half of s_bad is cleared meanwhile
  __syncthreads();

  for (int u = u0; u < u1;) {
    b = __builtin_amdgcn_readfirstlane(b);
    const Shape sh = shape_of<TS, RT>(a, b);
    const int units = sh.steps * sh.tiles * kv.num_kv_heads;
    if (u >= ub + units) {     // (a request without units among them)
      ub += units;
      ++b;
      continue;
    }
    const int rel = u - ub, pair = rel / sh.steps, s0 = rel - pair * sh.steps;
    const int g = pair / sh.tiles, tile = pair - g * sh.tiles;
    const int s1 = min(sh.steps, s0 + (u1 - u));
    const bool whole = s0 == 0 && s1 == sh.steps;
    const int slot = 2 * w + (u == u0 ? 0 : 1);
    u += s1 - s0;

    // ---- rows ----
    const int row = tile * RT + wr * 32 + n;             // of the (request, head)'s nodes x group
    const bool there = row < sh.rows, any_row = tile * RT + wr * 32 < sh.rows;
    const int node = there ? row / a.group : 0, head = g * a.group + (there ? row - node * a.group : 0);
    const int64_t out_row = (static_cast<int64_t>(b) * a.max_nodes + node) * kv.num_q_heads + head;
    typename E::Query qf;
    E::load_query(qf, a.q, out_row, there, a.q_dtype, a.dense, g2);
    const uint64_t word = there ? a.visible[static_cast<int64_t>(b) * a.max_nodes + node] & (~0ull >> (64 - sh.nodes)) : 0;
    const int first_node = sh.len - sh.nodes;            // token of node 0 (below 0: it is not in the cache)
    f32x16 o[D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = f32x16{};
    float m_run = -INFINITY, l_run = 0.f;

    Carrier<C, true> c(kv, b, g, sh.len);
    c.pages(kv, s0);
    c.fetch(kv, g, s0, a.aligned);
    if (s0 + 1 < s1) c.pages(kv, s0 + 1);

    // What is not finite in a node's V counts for the rows that see the node only: it is left out of the tile, and added at the end.
    auto park_v = [&](const u32x4& x, float scale, int s, int r, int piece, bool tail) {
      uint8_t* to = vtile + r * E::kVPitch;
      const int t = s * TS + r;
      if (!tail || t < first_node) {
        park_piece<E, C::KV, false>(x, scale, to, piece);
      } else if (park_piece<E, C::KV, true>(x, scale, to, piece) && t < sh.len) {
        atomicOr(&s_bad[parity][(t - first_node) >> 5], 1u << ((t - first_node) & 31));
      }
    };

    for (int s = s0; s < s1; ++s) {
      const bool tail = (s + 1) * TS > first_node;       // some token of the tile is a node, or past the end
      // ---- the tile into LDS, the next one on its way ----
      if (c.carries()) {
#pragma unroll
        for (int i = 0; i < C::kLoads; ++i) {
          park_piece<E, C::KV, false>(c.k[i], c.k_scale(i), ktile + c.row(i) * E::kKPitch, c.piece);
          park_v(c.v[i], c.v_scale(i), s, c.row(i), c.piece, tail);
        }
      }
      // With v_scale in the exponent p v_scale is 1, which bf16 has exactly, for the token that set a row's running maximum; as a factor on P it left the
      // weight of a row that one token dominates off by 2^-8 (64 fp8 requests, out against 64 bits: 0.0024 of its norm, now 0.0018 of which
      // 0.0017 is out's own rounding; 611 / 637 us).  A later token that exceeds the maximum by up to 8 does not move it, and is rounded like any other.
      if (C::kScales && tid < TS) {
        const float log_vs = __builtin_amdgcn_logf(c.vs < kLeastScale ? kLeastScale : c.vs);
        s_ks[tid] = c.ks * scale2;
        s_log_vs[tid] = log_vs;
        s_inv_vs[tid] = fast_exp2(-log_vs);              // (of the rounded logarithm: l is exact to fp32)
      }
      __syncthreads();
      if (s + 1 < s1) {
        c.fetch(kv, g, s + 1, a.aligned);
        if (s + 2 < s1) c.pages(kv, s + 2);
      }
      if (s == s0 && tid < 2) s_bad[parity ^ 1][tid] = 0;

      // ---- 32 tokens at a time ----
      if (any_row) {
        // Two workgroups of four wavefronts side by side on the rows: those at work on a tile go before those that fetch one (64 requests of 8192
        // tokens with 32 nodes 441 / 430 and 446 / 419 us without / with, fp8 394 / 379; other shapes gain nothing).
        if (C::WR == 4) __builtin_amdgcn_s_setprio(1);
        const int at = wt * C::kGroupTokens, t0 = s * TS + at;
        const bool masked = t0 + C::kGroupTokens > first_node;
        f32x16 x[C::NS];
#pragma unroll
        for (int sub = 0; sub < C::NS; ++sub) {
          x[sub] = E::qk(ktile + (at + 32 * sub) * E::kKPitch, qf, lane);
          if constexpr (C::kScales) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const f32x4 f = *reinterpret_cast<const f32x4*>(s_ks + at + 32 * sub + elem_of(i, g2));
              const f32x4 d = *reinterpret_cast<const f32x4*>(s_log_vs + at + 32 * sub + elem_of(i, g2));
#pragma unroll
              for (int j = 0; j < 4; ++j) x[sub][i + j] = __builtin_fmaf(x[sub][i + j], f[j], d[j]);
            }
          }
        }
        // The first half's K operands, then a product and an operand of the second half in turn: left to itself the compiler fetches two at a
        // time and waits (32 fp8 requests of 8192 tokens with 64 nodes 345 / 334 us; bf16 the same either way).
        if constexpr (C::WR == 8) {
          __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
          __builtin_amdgcn_sched_group_barrier(0x8, 8, 0);
        }
        uint32_t sees[C::NS];                            // bit elem_of(i, 0): this row sees the token of element i
        if (masked) {
#pragma unroll
          for (int sub = 0; sub < C::NS; ++sub) {
            sees[sub] = sees_of(word, first_node - (t0 + 32 * sub)) >> (4 * g2);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[sub][i] = (sees[sub] >> elem_of(i, 0) & 1u) ? x[sub][i] : -INFINITY;
          }
        }
        float top = x[0][0];
#pragma unroll
        for (int sub = 0; sub < C::NS; ++sub)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, x[sub][i]);
        top = other_half_max(top) * unit;
        // The maximum that exponentials are relative to moves only when a logit exceeds it by more than 8 (in log2 units): P stays below
        // 2^8, which costs no precision in floating point, and the accumulators are rescaled a few times per stretch.  Each row goes by its own
        // logits: what other rows see moves no bit of it.
        const bool moves = top > m_run + 8.f;
        if (__any(moves)) {
          const float f = !moves ? 1.f : m_run == -INFINITY ? 0.f : fast_exp2(m_run - top);
          m_run = moves ? top : m_run;
          l_run *= f;
#pragma unroll
          for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] *= f;
        }
        const float m_use = m_run == -INFINITY ? 0.f : m_run;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int sub = 0; sub < C::NS; ++sub) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            x[sub][i] = fast_exp2(C::kScales ? x[sub][i] - m_use : __builtin_fmaf(x[sub][i], scale2, -m_use));
            if (!C::kScales) sum[i & 1] += x[sub][i];
          }
          if constexpr (C::kScales) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const f32x4 f = *reinterpret_cast<const f32x4*>(s_inv_vs + at + 32 * sub + elem_of(i, g2));
              if (masked) {                              // (the scale of a page that no row sees may be anything)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j & 1] += (sees[sub] >> elem_of(i + j, 0) & 1u) ? x[sub][i + j] * f[j] : 0.f;
              } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[j & 1] = __builtin_fmaf(x[sub][i + j], f[j], sum[j & 1]);
              }
            }
          }
          E::pv(vtile + (at + 32 * sub) * E::kVPitch, x[sub], o, lane);
        }
        l_run += sum[0] + sum[1];
        if (C::WR == 4) __builtin_amdgcn_s_setprio(0);
      }
      __syncthreads();
    }

    const uint64_t bad = nodes_of(__builtin_amdgcn_readfirstlane(s_bad[parity][0]), __builtin_amdgcn_readfirstlane(s_bad[parity][1]));
    for (uint64_t left = bad; left; left &= left - 1) {
      const int j = __builtin_ctzll(left), t = first_node + j;
      if (t >= sh.len) break;                            // (there is no such row)
      if ((t % TS) / C::kGroupTokens != wt) continue;    // (the wavefronts whose maximum has seen the token)
      int page;
      const int64_t at = row_offset(kv, b, g, t, &page);
      float vs = 1.f;
      if constexpr (C::KV == PILLAR_FP8_E4M3) vs = kv.v_scale[static_cast<int64_t>(page) * kv.num_kv_heads + g];
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float val = Storage<C::KV>::load(kv.v_pool, at + 32 * db + elem_of(i, g2)) * vs;
          const float was = val;
          if (drop_nonfinite(val) && (word >> j & 1)) o[db][i] += was;
          __builtin_amdgcn_sched_barrier(0);
        }
    }
    parity ^= 1;

    // ---- what the stretch leaves ----
    l_run = other_half_sum(l_run);
    const int tile_row = wr * 32 + n;
    auto leave_row = [&](int64_t to_row, int in_tile, float m, float l) {        // one lane per row
      if (whole) {
        const float y = l == 0.f ? -INFINITY : m + log2f(l);
        if (a.lse) a.lse[to_row] = y * kLn2;
        if (a.lse2) a.lse2[to_row] = y;
      } else {
        float* ml = a.part_ml + (static_cast<int64_t>(slot) * RT + in_tile) * 2;
        ml[0] = m;
        ml[1] = l;
      }
    };
    auto leave_dims = [&](int64_t to_row, int in_tile, int dim, f32x4 x, float inv) {
      if (!whole) {
        *reinterpret_cast<f32x4*>(a.part_o + (static_cast<int64_t>(slot) * RT + in_tile) * D + dim) = x;
      } else {
        store_dims<D>(a, to_row, dim, x * inv);
      }
    };
    if constexpr (C::WT == 1) {
      if (there) {
        if (g2 == 0) leave_row(out_row, tile_row, m_run, l_run);
        const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            leave_dims(out_row, tile_row, 32 * db + elem_of(i, g2), f32x4{o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]}, inv);
      }
    } else {
      // the wavefronts that shared the rows join in LDS, where the tile was
      float* join = reinterpret_cast<float*>(smem);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<f32x4*>(join + (wave * 32 + n) * C::kJoinRow + 32 * db + elem_of(i, g2)) = f32x4{o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]};
      if (g2 == 0) { s_m[wave][n] = m_run; s_l[wave][n] = l_run; }
      __syncthreads();
      constexpr int kQuads = D / 4;
      for (int e = tid; e < RT * kQuads; e += C::kThreads) {
        const int r = e / kQuads, dim = 4 * (e % kQuads), rr = tile * RT + r;
        if (rr >= sh.rows) continue;
        float m = -INFINITY;
#pragma unroll
        for (int k = 0; k < C::WT; ++k) m = fmaxf(m, s_m[k * C::WR + (r >> 5)][r & 31]);
        const float m_use = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        f32x4 x = {};
#pragma unroll
        for (int k = 0; k < C::WT; ++k) {
          const int from = k * C::WR + (r >> 5);
          const float f = fast_exp2(s_m[from][r & 31] - m_use);
          l += s_l[from][r & 31] * f;
          x += *reinterpret_cast<const f32x4*>(join + (from * 32 + (r & 31)) * C::kJoinRow + dim) * f;
        }
        const int nd = rr / a.group;
        const int64_t to = (static_cast<int64_t>(b) * a.max_nodes + nd) * kv.num_q_heads + g * a.group + (rr - nd * a.group);
        if (dim == 0) leave_row(to, r, m, l);
        leave_dims(to, r, dim, x, l == 0.f ? 0.f : 1.f / l);
      }
      __syncthreads();
    }
  }
}

// ---- joins what several ranges left of a tile.  A tile is cut where a range begins inside it, so there is a row of workgroups for each range, which
// do nothing unless theirs is the first to begin inside its tile.  A row has D/4 lanes: they fetch (m, l) of as many partials side by
// side, and the partials of O kAhead at a time. ----
template <int D, int TS, int RT, int kAhead>
__global__ __launch_bounds__(128) void tree_merge(TreeParams a) {
  constexpr int kLanes = D / 4, kRows = 128 / kLanes;
  const KvView& kv = a.kv;
  const int lane = threadIdx.x & 63, part = threadIdx.x % kLanes;
  const Ranges ranges(a.prefix[kv.batch], a.ranges, a.few, a.tiles8);
  const int w = blockIdx.x + 1;
  if (w >= ranges.n) return;
  const int u = ranges.begin(w);
  int b = 0;
  for (int c = 0; c < kv.batch; c += 64) {
    const uint64_t after = __ballot(c + lane < kv.batch && a.prefix[min(c + lane, kv.batch - 1) + 1] > u);
    if (after) {
      b = c + __builtin_ctzll(after);
      break;
    }
  }
  b = __builtin_amdgcn_readfirstlane(b);
  const Shape sh = shape_of<TS, RT>(a, b);
  const int before = a.prefix[b], index = (u - before) / sh.steps, first = before + index * sh.steps;
  if (first == u) return;                                // the range begins with the tile
  const int w0 = ranges.of(first), w1 = ranges.of(first + sh.steps - 1);
  if (w0 != w - 1) return;
  const int first_slot = 2 * w0 + (ranges.begin(w0) < first ? 1 : 0);      // the others begin their range
  const int g = index / sh.tiles, tile = index - g * sh.tiles;
  const int count = w1 - w0 + 1, r_end = min(RT, sh.rows - tile * RT);
  for (int r = blockIdx.y * kRows + threadIdx.x / kLanes; r < r_end; r += gridDim.y * kRows) {
    const int row = tile * RT + r;
    auto at = [&](int i) { return static_cast<int64_t>(i == 0 ? first_slot : 2 * (w0 + i)) * RT + r; };
    f32x4 o[kAhead];
    auto fetch = [&](int i) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j) o[j] = *reinterpret_cast<const f32x4*>(a.part_o + at(min(i + j, count - 1)) * D + 4 * part);
    };
    fetch(0);                                            // (beside the (m, l) that it is weighed by)
    float m = -INFINITY;
    for (int c = part; c < count; c += kLanes) m = fmaxf(m, a.part_ml[2 * at(c)]);
#pragma unroll
    for (int k = kLanes / 2; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k, kLanes));
    const float m_use = m == -INFINITY ? 0.f : m;
    float l = 0.f, f = 0.f;
    f32x4 x = {};
    for (int i = 0; i < count; i += kAhead) {
      if (i % kLanes == 0) {                             // the weights of the next partials, one to a lane
        f = 0.f;
        if (i + part < count) {
          const float* ml = a.part_ml + 2 * at(i + part);
          f = fast_exp2(ml[0] - m_use);
          l += ml[1] * f;
        }
      }
      if (i > 0) fetch(i);
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < count) x += o[j] * __shfl(f, i % kLanes + j, kLanes);
    }
#pragma unroll
    for (int k = kLanes / 2; k > 0; k >>= 1) l += __shfl_xor(l, k, kLanes);
    const int node = row / a.group;
    const int64_t to = (static_cast<int64_t>(b) * a.max_nodes + node) * kv.num_q_heads + g * a.group + (row - node * a.group);
    if (part == 0) {
      const float y = l == 0.f ? -INFINITY : m + log2f(l);
      if (a.lse) a.lse[to] = y * kLn2;
      if (a.lse2) a.lse2[to] = y;
    }
    store_dims<D>(a, to, 4 * part, x * (l == 0.f ? 0.f : 1.f / l));
  }
}

// ---- the statistic: exp(logit - lse) summed over the rows.  Tiles of K pass as in tree_pass, but with the roles of the product exchanged (A = Q, B = K^T): a
// lane has one token and 16 of the 32 rows, and sums over rows without asking another lane but its other half.  Wavefronts that have
// other rows of the same tokens join in LDS.  More rows than a workgroup has (256): again for the next rows, adding to what
// the same threads wrote before. ----
// wavefronts per SIMD that the statistic's kernel is compiled for: what the registers allow without spilling
template <typename C>
constexpr int score_waves() { return C::E::kF32 && C::WR == 1 && C::D == 128 ? 1 : C::E::kF32 || C::WR == 1 ? 2 : C::WR == 8 ? 4 : 3; }

template <typename C>
__global__ __launch_bounds__(C::kThreads, score_waves<C>()) void tree_scores(TreeParams a, float* scores, int64_t score_stride) {
  using E = typename C::E;
  constexpr int TS = C::TS, RT = C::RT;
  __shared__ __attribute__((aligned(16))) uint8_t ktile[TS * E::kKPitch];
  __shared__ float s_ks[C::kScales ? TS : 1];
  __shared__ float s_part[C::WR][TS];
  __shared__ __attribute__((aligned(16))) float s_y[RT];
  __shared__ uint64_t s_word[RT];
  const KvView& kv = a.kv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % C::WR, wt = wave / C::WR, n = lane & 31, g2 = lane >> 5;
  const float scale2 = kv.sm_scale * kLog2e;
  const Share share(kv.batch, gridDim.x, gridDim.x, INT32_MAX, nullptr, [&](int r) {
    const Shape sh = shape_of<TS, RT>(a, r);
    return sh.rows > 0 ? sh.steps * kv.num_kv_heads : 0;
  }, [](int) {});
  int b = share.b, ub = share.ub;
  for (int u = share.u0; u < share.u1;) {
    b = __builtin_amdgcn_readfirstlane(b);
    const Shape sh = shape_of<TS, RT>(a, b);
    const int units = sh.rows > 0 ? sh.steps * kv.num_kv_heads : 0;
    if (u >= ub + units) {
      ub += units;
      ++b;
      continue;
    }
    const int g = (u - ub) / sh.steps, s0 = u - ub - g * sh.steps, s1 = min(sh.steps, s0 + share.u1 - u);
    u += s1 - s0;
    const int first_node = sh.len - sh.nodes;
    float* out = scores + (static_cast<int64_t>(b) * kv.num_kv_heads + g) * score_stride;
    Carrier<C, false> c(kv, b, g, sh.len);

    for (int r0 = 0; r0 < sh.rows; r0 += RT) {
      const int row = r0 + wr * 32 + n;
      const bool there = row < sh.rows, any_row = r0 + wr * 32 < sh.rows;
      const int node = there ? row / a.group : 0;
      const int64_t q_row = (static_cast<int64_t>(b) * a.max_nodes + node) * kv.num_q_heads + g * a.group + (there ? row - node * a.group : 0);
      typename E::Query qf;
      E::load_query(qf, a.q, q_row, there, a.q_dtype, a.dense, g2);
      float mine = there ? a.lse2[q_row] : INFINITY;
      if (mine == -INFINITY) mine = INFINITY;            // a row that sees nothing has no share
      const bool ragged = __any(mine == INFINITY);
      if (wt == 0 && g2 == 0) {
        s_y[wr * 32 + n] = mine;
        s_word[wr * 32 + n] = there ? a.visible[static_cast<int64_t>(b) * a.max_nodes + node] : 0;
      }
      c.pages(kv, s0);
      c.fetch(kv, g, s0, a.aligned);
      if (s0 + 1 < s1) c.pages(kv, s0 + 1);
      __syncthreads();
      float y[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = s_y[wr * 32 + elem_of(i, g2)];

      for (int s = s0; s < s1; ++s) {
        if (c.carries()) {
#pragma unroll
          for (int i = 0; i < C::kLoads; ++i) park_piece<E, C::KV, false>(c.k[i], c.k_scale(i), ktile + c.row(i) * E::kKPitch, c.piece);
        }
        if (C::kScales && tid < TS) s_ks[tid] = c.ks;
        __syncthreads();
        if (s + 1 < s1) {
          c.fetch(kv, g, s + 1, a.aligned);
          if (s + 2 < s1) c.pages(kv, s + 2);
        }
#pragma unroll
        for (int sub = 0; sub < C::NS; ++sub) {
          const int at = wt * C::kGroupTokens + 32 * sub, t = s * TS + at + n;
          float sum = 0.f;
          if (any_row && t - n < sh.len) {
            const f32x16 x = E::qk_token(ktile + at * E::kKPitch, qf, lane);
            const float f = C::kScales ? s_ks[at + n] * scale2 : scale2;
            if (ragged || t - n + 32 > first_node) {
              const int j = t - first_node;
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const bool vis = j < 0 || (j < sh.nodes && (s_word[wr * 32 + elem_of(i, g2)] >> (j & 63) & 1));
                const float p = fast_exp2(__builtin_fmaf(x[i], f, -y[i]));
                sum += vis && y[i] != INFINITY ? p : 0.f;
              }
            } else {
#pragma unroll
              for (int i = 0; i < 16; ++i) sum += fast_exp2(__builtin_fmaf(x[i], f, -y[i]));
            }
            sum = other_half_sum(sum);
          }
          if (g2 == 0) s_part[wr][at + n] = sum;
        }
        __syncthreads();
        if (tid < TS && s * TS + tid < sh.len) {
          float sum = s_part[0][tid];
#pragma unroll
          for (int i = 1; i < C::WR; ++i) sum += s_part[i][tid];
          float* to = out + s * TS + tid;
          if (r0 > 0) sum += *to;
          *to = r0 + RT >= sh.rows ? sum / static_cast<float>(sh.rows) : sum;
        }
      }
      __syncthreads();                                   // s_y and s_word are about to change
    }
  }
}

// ------------------------------------------------------------------ host --
struct TreePlan {
  int rt, ts, ranges, steps_max;
  int64_t tiles, slots;        // (request, head, tile of rows) there may be; partial results
};

// Wavefronts side by side on the rows: as many groups of 32 as there are rows, up to 8; the others of a workgroup of four take other tokens.
TreePlan plan_of(const KvView& kv, int max_nodes, bool f32) {
  TreePlan p;
  const int rows = max_nodes * (kv.num_q_heads / kv.num_kv_heads);
  const int groups = (rows + 31) / 32;
  int per_cu;
  if (f32) {
    p.rt = groups <= 1 ? 32 : groups <= 2 ? 64 : 128;
    p.ts = groups <= 1 ? 128 : 64;
    per_cu = kv.head_dim == 64 ? 2 : 1;
  } else {
    // 256 rows to a workgroup read K and V once for them, 128 make twice as many units: one request of 2100 tokens with 60 nodes 36 / 30 us, 4 49 / 40,
    // 128 of 1-8 K tokens 788 / 992
    const bool many = static_cast<int64_t>(kv.batch) * kv.num_kv_heads * ((rows + 255) / 256) * ((kv.max_seq_len + 63) / 64) >= 8 * static_cast<int64_t>(num_cus());
    p.rt = groups <= 1 ? 32 : groups <= 2 ? 64 : groups <= 4 || !many ? 128 : 256;
    p.ts = groups <= 1 ? 128 : 64;
    per_cu = p.rt <= 128 ? 2 : 1;
  }
  p.steps_max = (kv.max_seq_len + p.ts - 1) / p.ts;
  p.tiles = static_cast<int64_t>(kv.batch) * kv.num_kv_heads * ((rows + p.rt - 1) / p.rt);
  p.ranges = static_cast<int>(std::min<int64_t>(p.tiles * p.steps_max, static_cast<int64_t>(per_cu) * num_cus()));
  p.slots = 2 * static_cast<int64_t>(p.ranges);
  return p;
}

struct TreeWs {
  size_t ml, o, lse2, bytes;
};
TreeWs carve(const KvView& kv, int max_nodes, const TreePlan& p) {
  TreeWs w;
  size_t at = align_up((static_cast<size_t>(kv.batch) + 1) * 4, 256);
  w.ml = at;
  at = align_up(at + static_cast<size_t>(p.slots) * p.rt * 8, 256);
  w.o = at;
  at = align_up(at + static_cast<size_t>(p.slots) * p.rt * kv.head_dim * 4, 256);
  w.lse2 = at;
  at = align_up(at + static_cast<size_t>(kv.batch) * max_nodes * kv.num_q_heads * 4, 256);
  w.bytes = at;
  return w;
}

template <typename C>
hipError_t launch_tree(const TreeParams& p, const TreePlan& plan, const TreeArgs& t, hipStream_t s) {
  static_assert(C::kLds + 12 * C::TS + 64 * C::kWaves * 4 + 64 <= 160 * 1024, "");
  {
    KernelTimer timer("tree_pass", s);
    hipLaunchKernelGGL((tree_pass<C>), dim3(p.ranges), dim3(C::kThreads), 0, s, p);
  }
  if (plan.steps_max > 1 && p.ranges > 1) {
    KernelTimer timer("tree_merge", s);
    constexpr int kThreads = 128, kRows = kThreads / (C::D / 4);
    const int rows = std::min(C::RT, p.max_nodes * p.group);
    // of the workgroups that find work (one of the ranges of a tile) no more than the chip holds at once: 32 requests of 4096 tokens 17 / 15 us,
    // 128 of 1-8 K 24 / 18
    const int64_t busy = std::min<int64_t>(p.ranges - 1, plan.tiles);
    const int room = static_cast<int>(std::max<int64_t>(1, 16 * num_cus() / busy));
    const dim3 grid(p.ranges - 1, std::min(room, (rows + kRows - 1) / kRows));
    // many ranges to a tile: many partials at once, which take registers that two or three to a tile would miss (16 for all: 15 / 20 and 18 / 30 us)
    if (p.ranges > 4 * plan.tiles) hipLaunchKernelGGL((tree_merge<C::D, C::TS, C::RT, 16>), grid, dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((tree_merge<C::D, C::TS, C::RT, 4>), grid, dim3(kThreads), 0, s, p);
  }
  if (t.scores) {
    KernelTimer timer("tree_scores", s);
    const int64_t most = static_cast<int64_t>(p.kv.batch) * p.kv.num_kv_heads * plan.steps_max;
    const int workgroups = static_cast<int>(std::min<int64_t>(most, score_waves<C>() * 4 / C::kWaves * num_cus()));
    hipLaunchKernelGGL((tree_scores<C>), dim3(workgroups), dim3(C::kThreads), 0, s, p, t.scores, t.score_stride);
  }
  return hipGetLastError();
}

template <int D, int KV, bool BYPASS>
hipError_t launch_bf16(const TreeParams& p, const TreePlan& plan, const TreeArgs& t, hipStream_t s) {
  switch (plan.rt) {
    case 32: return launch_tree<Cfg<D, KV, false, 1, 4, 1, BYPASS>>(p, plan, t, s);
    case 64: return launch_tree<Cfg<D, KV, false, 2, 2, 1, BYPASS>>(p, plan, t, s);
    case 128: return launch_tree<Cfg<D, KV, false, 4, 1, 2, BYPASS>>(p, plan, t, s);
    default: return launch_tree<Cfg<D, KV, false, 8, 1, 2, BYPASS>>(p, plan, t, s);
  }
}
template <int D, int KV>
hipError_t launch_bf16(const TreeParams& p, const TreePlan& plan, const TreeArgs& t, hipStream_t s) {
  const KvView& kv = p.kv;
  const bool bypass = tree_bypasses(static_cast<int64_t>(kv.batch) * kv.num_kv_heads * kv.max_seq_len * 2 * D * kv_bytes<KV>());
  return bypass ? launch_bf16<D, KV, true>(p, plan, t, s) : launch_bf16<D, KV, false>(p, plan, t, s);
}
template <int D, int KV>
hipError_t launch_f32(const TreeParams& p, const TreePlan& plan, const TreeArgs& t, hipStream_t s) {
  if (plan.rt == 32) return launch_tree<Cfg<D, KV, true, 1, 4, 1, false>>(p, plan, t, s);
  if (plan.rt == 64) return launch_tree<Cfg<D, KV, true, 2, 2, 1, false>>(p, plan, t, s);
  return launch_tree<Cfg<D, KV, true, 4, 1, 2, false>>(p, plan, t, s);
}

}  // namespace

int tree_nodes_max() { return kTreeNodes; }

// The workspace has room for either engine: which one runs depends on the alignment of the tensors of a call.
size_t verify_tree_workspace(const KvView& kv, int max_nodes) {
  return std::max(carve(kv, max_nodes, plan_of(kv, max_nodes, false)).bytes, carve(kv, max_nodes, plan_of(kv, max_nodes, true)).bytes);
}

// units are counted in 32 bits
bool verify_tree_counts(const KvView& kv, int max_nodes) {
  const int64_t tiles = (static_cast<int64_t>(max_nodes) * (kv.num_q_heads / kv.num_kv_heads) + 31) / 32;
  return static_cast<int64_t>(kv.batch) * kv.num_kv_heads * tiles * ((static_cast<int64_t>(kv.max_seq_len) + 63) / 64) < (int64_t{1} << 30) && kv.batch <= 65535;
}

hipError_t launch_verify_tree(const TreeArgs& t, hipStream_t s) {
  const KvView& kv = t.kv;
  const bool dense = ((reinterpret_cast<uintptr_t>(t.q) | reinterpret_cast<uintptr_t>(t.out)) & 15u) == 0;
  const bool f32 = t.generic || t.q_dtype != PILLAR_BF16 || t.kv_dtype == PILLAR_F32 || !rows_aligned(kv, t.kv_dtype) || !strides_fit(kv, t.kv_dtype) || !dense;
  const TreePlan plan = plan_of(kv, t.max_nodes, f32);
  const TreeWs w = carve(kv, t.max_nodes, plan);
  char* ws = static_cast<char*>(t.workspace);
  TreeParams p;
  p.kv = kv;
  p.q = t.q;
  p.tree_sizes = t.tree_sizes;
  p.visible = t.visible;
  p.out = t.out;
  p.lse = t.lse;
  p.max_nodes = t.max_nodes;
  p.group = kv.num_q_heads / kv.num_kv_heads;
  p.q_dtype = t.q_dtype;
  p.aligned = rows_aligned(kv, t.kv_dtype);
  p.dense = dense;
  p.prefix = reinterpret_cast<int32_t*>(ws);
  p.part_ml = reinterpret_cast<float*>(ws + w.ml);
  p.part_o = reinterpret_cast<float*>(ws + w.o);
  p.lse2 = t.scores ? reinterpret_cast<float*>(ws + w.lse2) : nullptr;
  p.ranges = plan.ranges;
  p.few = std::min(plan.ranges, num_cus());
  p.tiles8 = f32 ? INT32_MAX : static_cast<int32_t>(std::min<int64_t>(8 * plan.tiles, INT32_MAX));
  const bool wide = kv.head_dim == 128;
  if (!f32) {
    if (t.kv_dtype == PILLAR_BF16) return wide ? launch_bf16<128, PILLAR_BF16>(p, plan, t, s) : launch_bf16<64, PILLAR_BF16>(p, plan, t, s);
    return wide ? launch_bf16<128, PILLAR_FP8_E4M3>(p, plan, t, s) : launch_bf16<64, PILLAR_FP8_E4M3>(p, plan, t, s);
  }
  switch (t.kv_dtype) {
    case PILLAR_F32: return wide ? launch_f32<128, PILLAR_F32>(p, plan, t, s) : launch_f32<64, PILLAR_F32>(p, plan, t, s);
    case PILLAR_BF16: return wide ? launch_f32<128, PILLAR_BF16>(p, plan, t, s) : launch_f32<64, PILLAR_BF16>(p, plan, t, s);
    default: return wide ? launch_f32<128, PILLAR_FP8_E4M3>(p, plan, t, s) : launch_f32<64, PILLAR_FP8_E4M3>(p, plan, t, s);
  }
}

}  // namespace pillar

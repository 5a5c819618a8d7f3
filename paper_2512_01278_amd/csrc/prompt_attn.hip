// Causal attention of new tokens over the paged cache: prompts, chunks of prompts, single tokens beside them.
//
//   out = softmax(sm_scale q K^T over tokens 0 .. own) V,   lse = log sum exp of the same logits
//
// The rows of a (request, KV head) are its new tokens times the query heads of the group; a tile is 2^s tokens' rows, at most RT, against K and V up to
// the tile's last token.  With 256 rows a tile reads 2 D e bytes per token and does 4 D 256 operations on them, so for prompts the matrix cores
// and the exponentials are the bound, not the cache.
//
//   prompt_pass   one pass over K and V with the running maximum and sum of every row's softmax (the tile arithmetic of tree_tile.hpp).  All units
//                 (a step of one tile of one KV head) in a row are cut into equal ranges, one per resident workgroup; where a range ends
//                 inside a tile it leaves a partial (m, l, O)
//   prompt_merge  joins the partials
//
// Four prompts of 8 K tokens, 32 heads on 8: 2400 us, 916 TFLOP/s; two chunks of 2 K after 30 K 2190 us, 970 TFLOP/s, where a product of 8192^3 by the library runs at
// 1320 (on another card 2500 us, 877 TFLOP/s, and 1180).
// Between the two lies what it takes to begin and end a tile.  (Two groups of wavefronts half a step apart, one at the products while the other takes
// exponentials, gain nothing: 800 against 830 TFLOP/s at the time.)
#include <algorithm>

#include "host_rules.hpp"
#include "paged_pass.hpp"
#include "prompt_rules.hpp"

namespace pillar {
namespace {

// What a range says about the tile that it begins in, for the joining of its partials.
struct Cut {
  int first, steps;            // the tile's first unit, its units
  int row;                     // the packed row of its first token
  int rows, head;              // rows of the tile (tokens times group), first query head
  int pad[3];
};
static_assert(sizeof(Cut) == 32, "");

struct PromptParams {
  KvView kv;
  const void* q;
  const int32_t* starts;       // null: max_new rows each
  void* out;
  float* lse;                  // may be null
  int32_t total_rows, max_new, group, q_dtype, q_shift;
  int32_t part_rows;           // rows that a partial result has room for
  int32_t setup;               // units that a tile counts for beside its steps
  bool aligned;                // cache rows can be read 16 bytes at a time,
  bool dense;                  // rows of q and out too
  // workspace
  int32_t* total;              // units of the launch
  Cut* cuts;                   // [ranges]
  float* part_ml;              // [slots][RT][2]
  float* part_o;               // [slots][RT][D]
  int32_t ranges, few;         // workgroups of the pass; of those, with little to do
  int32_t tiles8;              // eight times the tiles there may be, or the largest number where a tile may go into ranges of one unit
};

constexpr int shift_of(int x) { return x <= 1 ? 0 : 1 + shift_of(x / 2); }

struct Request {
  int row0, n, len;            // first packed row, new tokens, tokens in the cache
  __device__ __forceinline__ Request(const PromptParams& a, int b) {
    row0 = a.starts ? min(max(a.starts[b], 0), a.total_rows) : b * a.max_new;
    n = a.starts ? min(max(a.starts[b + 1], row0), a.total_rows) - row0 : a.max_new;
    len = min(max(a.kv.seq_lens[b], 0), a.kv.max_seq_len);
  }
};
// A request with few rows (single tokens, a chain) among prompts is read in larger steps, by a workgroup whose wavefronts share the rows: in 64 tokens at a time its
// one wavefront with rows would keep the others waiting.  A step then takes about as long as one of 256 rows, so ranges stay even.  31 single tokens after
// 1-8 K beside a chunk of 1000: 268 / 214 us (with steps of 256 tokens, twice as long as the others, 265).
constexpr int kNarrowRows = 64;
__device__ __forceinline__ bool is_narrow(const PromptParams& a, const Request& r) { return r.n * a.group <= kNarrowRows; }
template <typename C, typename N>
__device__ __forceinline__ PromptSteps steps_of(const PromptParams& a, const Request& r) {
  return PromptSteps(r.len, r.n, a.q_shift, is_narrow(a, r) ? shift_of(N::TS) : shift_of(C::TS), a.setup);
}

// four dims of an output row
__device__ __forceinline__ void store_four(const PromptParams& a, int64_t at, f32x4 x) {
  if (a.q_dtype == PILLAR_F32) {
    if (a.dense) {
      *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = x;
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) Storage<PILLAR_F32>::store(a.out, at + j, x[j]);
  } else {
    if (a.dense) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      *reinterpret_cast<bf16x4*>(static_cast<uint16_t*>(a.out) + at) = __builtin_convertvector(x, bf16x4);
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) Storage<PILLAR_BF16>::store(a.out, at + j, x[j]);
  }
}

// Results of the rows of a request without a token, by a whole workgroup.
__device__ __forceinline__ void see_nothing(const PromptParams& a, const Request& r) {
  const int64_t first = static_cast<int64_t>(r.row0) * a.kv.num_q_heads, rows = static_cast<int64_t>(r.n) * a.kv.num_q_heads;
  for (int64_t e = threadIdx.x; e < rows * a.kv.head_dim; e += blockDim.x) {
    if (a.q_dtype == PILLAR_F32) Storage<PILLAR_F32>::store(a.out, first * a.kv.head_dim + e, 0.f);
    else Storage<PILLAR_BF16>::store(a.out, first * a.kv.head_dim + e, 0.f);
  }
  if (a.lse)
    for (int64_t i = threadIdx.x; i < rows; i += blockDim.x) a.lse[first + i] = -INFINITY;
}

// Of 32 tokens, those that a row sees which sees `upto` of them (any number).
__device__ __forceinline__ uint32_t first_tokens(int upto) { return upto >= 32 ? ~0u : upto <= 0 ? 0u : (1u << upto) - 1; }

// A stretch: steps s0 .. s1 - 1 of a tile.
struct Stretch {
  int b, g, s0, s1;
  int i0, rows;                // the tile's first new token, its rows
  int slot;                    // of the partial result
  bool whole;                  // it is all of the tile
};

template <typename C>
struct PassLds {
  uint8_t* smem;
  float *ks, *log_vs, *inv_vs;                           // page scales of a step's tokens: k_scale in the logits' unit, log2 of v_scale, and one over it
  float (*m)[32], (*l)[32];
  uint32_t (*bad)[8];                                    // the tile's own tokens whose V row is not finite throughout; two sets, cleared in turn
};

template <typename C>
__device__ __forceinline__ void do_stretch(const PromptParams& a, const Stretch& st, const Request& rq, const PassLds<C>& lds, int parity) {
  using E = typename C::E;
  constexpr int D = C::D, TS = C::TS, RT = C::RT;
  constexpr int kBadWords = RT / 32;                     // a tile has at most RT tokens
  const KvView& kv = a.kv;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % C::WR, wt = wave / C::WR;
  const int n = lane & 31, g2 = lane >> 5;
  uint8_t* const ktile = lds.smem;
  uint8_t* const vtile = lds.smem + TS * E::kKPitch;
  const float scale2 = kv.sm_scale * kLog2e;
  const float unit = C::kScales ? 1.f : scale2;          // of the logits, in log2: page scales come with it
  const int b = st.b, g = st.g, s0 = st.s0, s1 = st.s1, i0 = st.i0, rows = st.rows;

  Carrier<C, true> c(kv, b, g, rq.len);                // (first of all: the rows of the cache are at the end of a chain of three loads)
  c.pages(kv, s0);

  // ---- rows ----
  const int first = rq.len - rq.n;                     // number of the first new token (below 0: it is not in the cache)
  const int row = wr * 32 + n;
  const bool there = row < rows, any_row = wr * 32 < rows;
  const int token = i0 + (there ? row / a.group : 0), head = g * a.group + (there ? row % a.group : 0);
  const int64_t out_row = static_cast<int64_t>(rq.row0 + token) * kv.num_q_heads + head;
  typename E::Query qf;
  E::load_query(qf, a.q, out_row, there, a.q_dtype, a.dense, g2);
  const int sees = there ? first + token + 1 : 0;      // tokens that this row sees
  const int wave_sees0 = first + i0 + wr * 32 / a.group + 1;                                // ... the wavefront's first row, its last
  const int wave_sees1 = first + i0 + (min(wr * 32 + 32, rows) - 1) / a.group + 1;
  const int own = max(first + i0, 0);                  // first of the tile's own tokens, which not all rows see
  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) o[db] = f32x16{};
  float m_run = -INFINITY, l_run = 0.f;

  c.fetch(kv, g, s0, a.aligned);
  if (s0 + 1 < s1) c.pages(kv, s0 + 1);

  // What is not finite in V of one of the tile's own tokens counts for the rows that see it only: it is left out of the tile, and added at the end.
  auto park_v = [&](const u32x4& x, float scale, int s, int r, int piece, bool tail) {
    uint8_t* to = vtile + r * E::kVPitch;
    const int t = s * TS + r;
    if (!tail || t < own) {
      park_piece<E, C::KV, false>(x, scale, to, piece);
    } else if (park_piece<E, C::KV, true>(x, scale, to, piece) && t - own < RT) {
      atomicOr(&lds.bad[parity][(t - own) >> 5], 1u << ((t - own) & 31));
    }
  };

  for (int s = s0; s < s1; ++s) {
    const bool tail = (s + 1) * TS > own;              // some token of the step is the tile's own, or later
    // ---- the step's rows into LDS, the next ones on their way ----
    if (c.carries()) {
#pragma unroll
      for (int i = 0; i < C::kLoads; ++i) {
        park_piece<E, C::KV, false>(c.k[i], c.k_scale(i), ktile + c.row(i) * E::kKPitch, c.piece);
        park_v(c.v[i], c.v_scale(i), s, c.row(i), c.piece, tail);
      }
    }
    if (C::kScales && tid < TS) {                      // (v_scale in the exponent: the weightiest token of a row is not rounded)
      const float log_vs = __builtin_amdgcn_logf(c.vs < kLeastScale ? kLeastScale : c.vs);
      lds.ks[tid] = c.ks * scale2;
      lds.log_vs[tid] = log_vs;
      lds.inv_vs[tid] = fast_exp2(-log_vs);              // (of the rounded logarithm: l is exact to fp32)
    }
    __syncthreads();
    if (s + 1 < s1) {
      c.fetch(kv, g, s + 1, a.aligned);
      if (s + 2 < s1) c.pages(kv, s + 2);
    }
    if (s == s0 && tid < 8) lds.bad[parity ^ 1][tid] = 0;

    const int at = wt * C::kGroupTokens, t0 = s * TS + at;
    if (any_row && t0 < wave_sees1) {
      if (C::WR == 4) __builtin_amdgcn_s_setprio(1);
      const bool masked = t0 + C::kGroupTokens > wave_sees0;
      f32x16 x[C::NS];
#pragma unroll
      for (int sub = 0; sub < C::NS; ++sub) {
        x[sub] = E::qk(ktile + (at + 32 * sub) * E::kKPitch, qf, lane);
        if constexpr (C::kScales) {
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const f32x4 f = *reinterpret_cast<const f32x4*>(lds.ks + at + 32 * sub + elem_of(i, g2));
            const f32x4 d = *reinterpret_cast<const f32x4*>(lds.log_vs + at + 32 * sub + elem_of(i, g2));
#pragma unroll
            for (int j = 0; j < 4; ++j) x[sub][i + j] = __builtin_fmaf(x[sub][i + j], f[j], d[j]);
          }
        }
      }
      uint32_t seen[C::NS];                            // bit elem_of(i, 0): this row sees the token of element i
      if (masked) {
#pragma unroll
        for (int sub = 0; sub < C::NS; ++sub) {
          seen[sub] = first_tokens(sees - t0 - 32 * sub) >> (4 * g2);
#pragma unroll
          for (int i = 0; i < 16; ++i) x[sub][i] = (seen[sub] >> elem_of(i, 0) & 1u) ? x[sub][i] : -INFINITY;
        }
      }
      float top = x[0][0];
#pragma unroll
      for (int sub = 0; sub < C::NS; ++sub)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, x[sub][i]);
      top = other_half_max(top) * unit;
      // the maximum moves only when a logit exceeds it by more than 8 (log2): P stays below 2^8, and the accumulators are rescaled a few times per stretch
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
            const f32x4 f = *reinterpret_cast<const f32x4*>(lds.inv_vs + at + 32 * sub + elem_of(i, g2));
            if (masked) {                              // (the scale of a page that no row sees may be anything)
#pragma unroll
              for (int j = 0; j < 4; ++j) sum[j & 1] += (seen[sub] >> elem_of(i + j, 0) & 1u) ? x[sub][i + j] * f[j] : 0.f;
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

  const uint32_t bad = lane < kBadWords ? lds.bad[parity][lane] : 0;
  for (uint64_t some = __ballot(bad != 0); some; some &= some - 1) {
    const int word = __builtin_ctzll(some);
    for (uint32_t left = __builtin_amdgcn_readlane(bad, word); left; left &= left - 1) {
      const int t = own + 32 * word + __builtin_ctz(left);
      if (t >= rq.len) break;                          // (there is no such row)
      if ((t % TS) / C::kGroupTokens != wt) continue;  // (the wavefronts whose maximum has seen the token)
      int page;
      const int64_t from = row_offset(kv, b, g, t, &page);
      float vs = 1.f;
      if constexpr (C::KV == PILLAR_FP8_E4M3) vs = kv.v_scale[static_cast<int64_t>(page) * kv.num_kv_heads + g];
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float val = Storage<C::KV>::load(kv.v_pool, from + 32 * db + elem_of(i, g2)) * vs;
          const float was = val;
          if (drop_nonfinite(val) && t < sees) o[db][i] += was;
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  }

  // ---- what the stretch leaves ----
  l_run = other_half_sum(l_run);
  auto leave_row = [&](int64_t to_row, int in_tile, float m, float l) {        // one lane per row
    if (st.whole) {
      if (a.lse) a.lse[to_row] = (l == 0.f ? -INFINITY : m + log2f(l)) * kLn2;
    } else {
      float* ml = a.part_ml + (static_cast<int64_t>(st.slot) * a.part_rows + in_tile) * 2;
      ml[0] = m;
      ml[1] = l;
    }
  };
  auto leave_dims = [&](int64_t to_row, int in_tile, int dim, f32x4 x, float inv) {
    if (!st.whole) *reinterpret_cast<f32x4*>(a.part_o + (static_cast<int64_t>(st.slot) * a.part_rows + in_tile) * D + dim) = x;
    else store_four(a, to_row * D + dim, x * inv);
  };
  if constexpr (C::WT == 1) {
    if (there) {
      if (g2 == 0) leave_row(out_row, row, m_run, l_run);
      const float inv = l_run == 0.f ? 0.f : 1.f / l_run;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          leave_dims(out_row, row, 32 * db + elem_of(i, g2), f32x4{o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]}, inv);
    }
  } else {
    // the wavefronts that shared the rows join in LDS, where the step's rows were
    float* join = reinterpret_cast<float*>(lds.smem);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<f32x4*>(join + (wave * 32 + n) * C::kJoinRow + 32 * db + elem_of(i, g2)) = f32x4{o[db][i], o[db][i + 1], o[db][i + 2], o[db][i + 3]};
    if (g2 == 0) { lds.m[wave][n] = m_run; lds.l[wave][n] = l_run; }
    __syncthreads();
    constexpr int kQuads = D / 4;
    for (int e = tid; e < RT * kQuads; e += C::kThreads) {
      const int r = e / kQuads, dim = 4 * (e % kQuads);
      if (r >= rows) continue;
      float m = -INFINITY;
#pragma unroll
      for (int k = 0; k < C::WT; ++k) m = fmaxf(m, lds.m[k * C::WR + (r >> 5)][r & 31]);
      const float m_use = m == -INFINITY ? 0.f : m;
      float l = 0.f;
      f32x4 x = {};
#pragma unroll
      for (int k = 0; k < C::WT; ++k) {
        const int from = k * C::WR + (r >> 5);
        const float f = fast_exp2(lds.m[from][r & 31] - m_use);
        l += lds.l[from][r & 31] * f;
        x += *reinterpret_cast<const f32x4*>(join + (from * 32 + (r & 31)) * C::kJoinRow + dim) * f;
      }
      const int64_t to = static_cast<int64_t>(rq.row0 + i0 + r / a.group) * kv.num_q_heads + g * a.group + r % a.group;
      if (dim == 0) leave_row(to, r, m, l);
      leave_dims(to, r, dim, x, l == 0.f ? 0.f : 1.f / l);
    }
    __syncthreads();
  }
}

template <typename C, typename N>
__global__ __launch_bounds__(C::kThreads, C::E::kF32 ? 1 : 2) void prompt_pass(PromptParams a) {
  static_assert(C::kThreads == N::kThreads && (std::is_same_v<C, N> || N::RT >= kNarrowRows), "");
  constexpr int kTokens = C::TS > N::TS ? C::TS : N::TS;
  __shared__ __attribute__((aligned(16))) uint8_t smem[C::kLds > N::kLds ? C::kLds : N::kLds];
  __shared__ __attribute__((aligned(16))) float s_ks[C::kScales ? kTokens : 4], s_log_vs[C::kScales ? kTokens : 4], s_inv_vs[C::kScales ? kTokens : 4];
  __shared__ float s_m[C::kWaves][32], s_l[C::kWaves][32];
  __shared__ uint32_t s_bad[2][8];
  const KvView& kv = a.kv;
  const int tid = threadIdx.x, lane = tid & 63;

  const Share share(kv.batch, a.ranges, a.few, a.tiles8, nullptr,
                    [&](int r) { return steps_of<C, N>(a, Request(a, r)).units() * kv.num_kv_heads; }, [&](int c) {
    // requests without a token in the cache have no unit: their rows are shared out among the workgroups
    for (uint64_t none = __ballot(c + lane < kv.batch && kv.seq_lens[min(c + lane, kv.batch - 1)] <= 0); none; none &= none - 1) {
      const int r = c + __builtin_ctzll(none);
      if (r % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x)) see_nothing(a, Request(a, r));
    }
  });
  const int w = share.w, u0 = share.u0, u1 = share.u1;
  if (blockIdx.x == 0 && tid == 0) *a.total = share.total;
  if (u0 == u1) return;
  if (tid < 8) s_bad[0][tid] = 0;
  int parity = 0;              // of the stretch: the other half of s_bad is cleared meanwhile
  __syncthreads();

  // the request at work, its first unit and its units
  int b = share.b, ub = share.ub;
  Request rq(a, b);
  PromptSteps plan = steps_of<C, N>(a, rq);
  int per_head = plan.units();
  for (int u = u0; u < u1;) {
    while (u >= ub + per_head * kv.num_kv_heads) {       // (requests without units among them)
      ub += per_head * kv.num_kv_heads;
      b = __builtin_amdgcn_readfirstlane(b + 1);
      rq = Request(a, b);
      plan = steps_of<C, N>(a, rq);
      per_head = plan.units();
    }
    Stretch st;
    const int rel = u - ub, in_head = rel % per_head;
    const int tile = __builtin_amdgcn_readfirstlane(plan.tile_of(in_head));
    const int steps = plan.steps(tile), idx = in_head - plan.before(tile), units = steps + a.setup;
    st.b = b;
    st.g = rel / per_head;
    st.s0 = max(0, idx - a.setup);
    st.s1 = min(units, idx + (u1 - u)) - a.setup;        // (0 or less: the range ends before the tile's first step)
    st.whole = st.s0 == 0 && st.s1 == steps;
    st.slot = 2 * w + (u == u0 ? 0 : 1);
    st.i0 = tile << a.q_shift;
    st.rows = min(rq.n - st.i0, 1 << a.q_shift) * a.group;
    if (u == u0 && tid == 0) {
      Cut cut{};
      cut.first = u - idx;
      cut.steps = steps;
      cut.row = rq.row0 + st.i0;
      cut.rows = st.rows;
      cut.head = st.g * a.group;
      a.cuts[w] = cut;
    }
    u += min(units - idx, u1 - u);
    if (st.s1 <= 0) break;
    if constexpr (std::is_same_v<C, N>) do_stretch<C>(a, st, rq, PassLds<C>{smem, s_ks, s_log_vs, s_inv_vs, s_m, s_l, s_bad}, parity);
    else if (is_narrow(a, rq)) do_stretch<N>(a, st, rq, PassLds<N>{smem, s_ks, s_log_vs, s_inv_vs, s_m, s_l, s_bad}, parity);
    else do_stretch<C>(a, st, rq, PassLds<C>{smem, s_ks, s_log_vs, s_inv_vs, s_m, s_l, s_bad}, parity);
    parity ^= 1;
  }
}

// ---- joins what several ranges left of a tile.  A tile is cut where a range begins inside it, so there is a row of workgroups for each range, which
// do nothing unless theirs is the first to begin inside its tile.  A row has D/4 lanes: they fetch (m, l) of as many partials side by
// side, and the partials of O kAhead at a time. ----
template <int D, int RT, int kAhead>
__global__ __launch_bounds__(128) void prompt_merge(PromptParams a) {
  constexpr int kLanes = D / 4, kRows = 128 / kLanes;
  const int part = threadIdx.x % kLanes;
  const int w = blockIdx.x + 1;
  const Ranges ranges(*a.total, a.ranges, a.few, a.tiles8);
  if (w >= ranges.n) return;
  const Cut cut = a.cuts[w];
  // (the tile's first `setup` units are no steps: a range that has none but those leaves nothing)
  const int first = cut.first + a.setup, w0 = ranges.of(first), w1 = ranges.of(first + cut.steps - 1);
  if (w0 != w - 1) return;                               // the range begins with the tile, or is not the second of its ranges
  const int first_slot = 2 * w0 + (ranges.begin(w0) < cut.first ? 1 : 0);      // the others begin their range
  const int rows = cut.rows;
  const int count = w1 - w0 + 1;
  for (int r = blockIdx.y * kRows + threadIdx.x / kLanes; r < rows; r += gridDim.y * kRows) {
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
    const int64_t to = static_cast<int64_t>(cut.row + r / a.group) * a.kv.num_q_heads + cut.head + r % a.group;
    if (part == 0 && a.lse) a.lse[to] = (l == 0.f ? -INFINITY : m + log2f(l)) * kLn2;
    store_four(a, to * D + 4 * part, x * (l == 0.f ? 0.f : 1.f / l));
  }
}

// ------------------------------------------------------------------ host --
struct PromptPlan {
  int rt, ts, q_shift, ranges, setup;
  int64_t tiles, units, slots; // (request, head, tile of rows) and units there may be; partial results
  bool bypass;                 // rows of the cache are read once: they bypass the Infinity Cache
};

// Wavefronts side by side on the rows: as many groups of 32 as a request may have rows, up to 8; the others of a workgroup of four take other tokens.
PromptPlan plan_of(const KvView& kv, int total_rows, int max_new, bool f32) {
  PromptPlan p;
  const int group = kv.num_q_heads / kv.num_kv_heads;
  const int64_t groups = (static_cast<int64_t>(max_new) * group + 31) / 32;
  auto tiles_of = [&](int rt) {
    return kv.num_kv_heads * (kv.batch + (static_cast<int64_t>(total_rows) >> tile_tokens_shift(rt, group)));
  };
  int per_cu;
  if (f32) {
    p.rt = groups <= 1 ? 32 : groups <= 2 ? 64 : 128;
    p.ts = groups <= 1 ? 128 : 64;
    per_cu = kv.head_dim == 64 ? 2 : 1;
  } else {
    const bool many = tiles_of(256) * ((kv.max_seq_len + 63) / 64) >= 16 * static_cast<int64_t>(num_cus());
    p.rt = groups <= 1 ? 32 : groups <= 2 ? 64 : groups <= 4 || !many ? 128 : 256;
    p.ts = groups <= 1 ? 128 : 64;
    per_cu = p.rt <= 128 ? 2 : 1;
  }
  // Beginning and ending a tile (its place, queries, first rows of the cache, results) takes about as long as four steps of 128 or 256 rows, so it counts for
  // that many in the cutting of the ranges: else ranges of many short tiles, as the first ones of a prompt are, end last.  Counted as none / 2 / 4 / 6 / 8 steps:
  // 4 prompts of 8 K tokens 2660 / 2593 / 2513 / 2514 / 2513 us, one of 2 K 112 / 80 / 73 / 78 / 79, short ones over fp8 74 / 63 / 62 / 68 / 73.  Tiles of
  // single tokens: none / 1 / 2 / 4: 64 contexts of 1-8 K 190 / 189 / 191 / 196.
  p.setup = p.rt >= 128 ? 4 : 1;
  p.q_shift = tile_tokens_shift(p.rt, group);
  p.tiles = tiles_of(p.rt);
  p.units = p.tiles * ((kv.max_seq_len + p.ts - 1) / p.ts + p.setup);
  p.bypass = p.rt == 32 && tree_bypasses(static_cast<int64_t>(kv.batch) * kv.num_kv_heads * kv.max_seq_len * 4 * kv.head_dim);
  p.ranges = static_cast<int>(std::min<int64_t>(p.units, static_cast<int64_t>(per_cu) * num_cus()));
  p.slots = 2 * static_cast<int64_t>(p.ranges);
  return p;
}

struct PromptWs {
  size_t ml, o, bytes;
};
PromptWs carve(const KvView& kv, int64_t slots, int rt) {
  PromptWs w;
  size_t at = align_up(256 + static_cast<size_t>(slots / 2) * sizeof(Cut), 256);
  w.ml = at;
  at = align_up(at + static_cast<size_t>(slots) * rt * 8, 256);
  w.o = at;
  w.bytes = align_up(at + static_cast<size_t>(slots) * rt * kv.head_dim * 4, 256);
  return w;
}

template <typename C, typename N>
hipError_t launch_as(const PromptParams& p, const PromptPlan& plan, hipStream_t s) {
  static_assert((C::kLds > N::kLds ? C::kLds : N::kLds) + 12 * (C::TS > N::TS ? C::TS : N::TS) + 64 * C::kWaves * 4 + 64 <= 160 * 1024, "");
  {
    KernelTimer timer("prompt_pass", s);
    hipLaunchKernelGGL((prompt_pass<C, N>), dim3(p.ranges), dim3(C::kThreads), 0, s, p);
  }
  if (p.ranges > 1) {
    KernelTimer timer("prompt_merge", s);
    constexpr int kThreads = 128, kRows = kThreads / (C::D / 4);
    const int rows = (1 << p.q_shift) * p.group;
    const int64_t busy = std::min<int64_t>(p.ranges - 1, plan.tiles);
    const int room = static_cast<int>(std::max<int64_t>(1, 16 * num_cus() / busy));
    const dim3 grid(p.ranges - 1, std::min(room, (rows + kRows - 1) / kRows));
    if (p.ranges > 4 * plan.tiles) hipLaunchKernelGGL((prompt_merge<C::D, C::RT, 16>), grid, dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((prompt_merge<C::D, C::RT, 4>), grid, dim3(kThreads), 0, s, p);
  }
  return hipGetLastError();
}

template <int D, int KV>
hipError_t launch_bf16(const PromptParams& p, const PromptPlan& plan, hipStream_t s) {
  using N4 = Cfg<D, KV, false, 1, 4, 1, false>;
  using N2 = Cfg<D, KV, false, 2, 2, 1, false>;
  switch (plan.rt) {
    case 32:
      if (plan.bypass) return launch_as<Cfg<D, KV, false, 1, 4, 1, true>, Cfg<D, KV, false, 1, 4, 1, true>>(p, plan, s);
      return launch_as<N4, N4>(p, plan, s);
    case 64: return launch_as<N2, N2>(p, plan, s);
    case 128: return launch_as<Cfg<D, KV, false, 4, 1, 2, false>, N2>(p, plan, s);
    default: return launch_as<Cfg<D, KV, false, 8, 1, 2, false>, Cfg<D, KV, false, 2, 4, 1, false>>(p, plan, s);
  }
}
template <int D, int KV>
hipError_t launch_f32(const PromptParams& p, const PromptPlan& plan, hipStream_t s) {
  using N4 = Cfg<D, KV, true, 1, 4, 1, false>;
  if (plan.rt == 32) return launch_as<N4, N4>(p, plan, s);
  if (plan.rt == 64) return launch_as<Cfg<D, KV, true, 2, 2, 1, false>, Cfg<D, KV, true, 2, 2, 1, false>>(p, plan, s);
  return launch_as<Cfg<D, KV, true, 4, 1, 2, false>, Cfg<D, KV, true, 4, 1, 2, false>>(p, plan, s);
}

}  // namespace

// Whatever a smaller call is planned as, it has no more partial results than the chip holds workgroups, and no more than 256 rows to each.
size_t prompt_workspace(const KvView& kv, int, int) {
  return std::max(carve(kv, 2 * static_cast<int64_t>(num_cus()), 256).bytes, carve(kv, 4 * static_cast<int64_t>(num_cus()), 128).bytes);
}

// units are counted in 32 bits
bool prompt_counts(const KvView& kv, int total_rows, int max_new) {
  return plan_of(kv, total_rows, max_new, false).units < (int64_t{1} << 30) && plan_of(kv, total_rows, max_new, true).units < (int64_t{1} << 30);
}

hipError_t launch_prompt(const PromptArgs& t, hipStream_t s) {
  const KvView& kv = t.kv;
  const bool dense = ((reinterpret_cast<uintptr_t>(t.q) | reinterpret_cast<uintptr_t>(t.out)) & 15u) == 0;
  const bool f32 = t.generic || t.q_dtype != PILLAR_BF16 || t.kv_dtype == PILLAR_F32 || !rows_aligned(kv, t.kv_dtype) || !strides_fit(kv, t.kv_dtype) || !dense;
  const PromptPlan plan = plan_of(kv, t.total_rows, t.max_new, f32);
  const PromptWs w = carve(kv, plan.slots, plan.rt);
  char* ws = static_cast<char*>(t.workspace);
  PromptParams p;
  p.kv = kv;
  p.q = t.q;
  p.starts = t.starts;
  p.out = t.out;
  p.lse = t.lse;
  p.total_rows = t.total_rows;
  p.max_new = t.max_new;
  p.group = kv.num_q_heads / kv.num_kv_heads;
  p.q_dtype = t.q_dtype;
  p.q_shift = plan.q_shift;
  p.setup = plan.setup;
  p.part_rows = plan.rt;
  p.aligned = rows_aligned(kv, t.kv_dtype);
  p.dense = dense;
  p.total = reinterpret_cast<int32_t*>(ws);
  p.cuts = reinterpret_cast<Cut*>(ws + 256);
  p.part_ml = reinterpret_cast<float*>(ws + w.ml);
  p.part_o = reinterpret_cast<float*>(ws + w.o);
  p.ranges = plan.ranges;
  p.few = std::min(plan.ranges, num_cus());
  p.tiles8 = f32 ? INT32_MAX : static_cast<int32_t>(std::min<int64_t>(8 * plan.tiles, INT32_MAX));
  const bool wide = kv.head_dim == 128;
  if (!f32) {
    if (t.kv_dtype == PILLAR_BF16) return wide ? launch_bf16<128, PILLAR_BF16>(p, plan, s) : launch_bf16<64, PILLAR_BF16>(p, plan, s);
    return wide ? launch_bf16<128, PILLAR_FP8_E4M3>(p, plan, s) : launch_bf16<64, PILLAR_FP8_E4M3>(p, plan, s);
  }
  switch (t.kv_dtype) {
    case PILLAR_F32: return wide ? launch_f32<128, PILLAR_F32>(p, plan, s) : launch_f32<64, PILLAR_F32>(p, plan, s);
    case PILLAR_BF16: return wide ? launch_f32<128, PILLAR_BF16>(p, plan, s) : launch_f32<64, PILLAR_BF16>(p, plan, s);
    default: return wide ? launch_f32<128, PILLAR_FP8_E4M3>(p, plan, s) : launch_f32<64, PILLAR_FP8_E4M3>(p, plan, s);
  }
}

}  // namespace pillar

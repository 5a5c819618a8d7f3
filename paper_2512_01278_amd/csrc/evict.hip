// Eviction from the cache by accumulated attention weight.
//
// Every token of a (request, KV head) has a weight w: w <- decay w + score at every call, a new token's is its score.  Of L tokens K' =
// min(budget, L) stay: those that are protected (the first positions, and the most recent ones), then those of largest weight, equal
// weights resolved towards the lower slot.
//
// Attention does not ask for the order of the rows, so what stays below slot K' stays where it is, and what stays beyond K' moves into the
// holes below it, the i-th into the i-th.  There are as many of either (K' minus the kept ones below K').  Sources and destinations are
// disjoint, so all rows move at once, in place, and no fewer could: at five new tokens a step at most five rows of a head move where
// closing the gaps would move the whole cache.  Positions travel with the rows, as a slot no longer says how old a token is.
//
// One or two launches:
//   evict_select  one workgroup per (request, KV head): the weights, a radix select of the K'-th key, the list of holes and sources in
//                 order, the moves within weights and positions, and the rows of K and V, unless few workgroups would have many to move:
//   evict_move    then, workgroups of their own.
//
// A step at the budget moves a few rows: it is as long as a chain of loads (lengths, state, page ids, rows), two histograms and their
// barriers.  So the keys stay in registers from one load on, and a digit of the K'-th key that all its keys survive ends the search (the
// second of three, unless weights agree in 22 bits).
#include <algorithm>
#include <type_traits>

#include "launch.hpp"
#include "page_scale.hpp"

namespace pillar {
namespace {

constexpr int kMoveThreads = 256;
constexpr int kMoveList = 1024;          // moves whose list is kept in LDS
constexpr uint32_t kProtected = 0xffffffffu;

struct MoveWs {
  int32_t* moves;              // [pairs] rows to move
  int32_t* kept;               // [pairs] K'
  float* edge;                 // [pairs][2] scales of the page that has slot K', before any row moved
  int32_t* list;               // [pairs][max_seq_len] holes, then sources
};

// A weight orders as the pattern of its bits; what is negative or no number counts as 0.
__device__ __forceinline__ uint32_t weight_key(float w) { return w > 0.f ? __float_as_uint(w) : 0u; }

// two roundings, as the formula is written
__device__ __forceinline__ float accumulate(float weight, float decay, float score) {
#pragma clang fp contract(off)
  return weight * decay + score;
}

// Rows are read several at a time before any is written: the compiler cannot know that no load depends on a store before it.
constexpr int kBatch = 2;

// ---- rows of K and V into the holes: worker `me` of `workers` threads (fp8: wavefronts) ----
template <typename Hole, typename Source>
__device__ __forceinline__ void copy_rows(const RowPlace& at, int pieces, int moves, Hole hole, Source source, int me, int workers) {
  const int shift = __builtin_ctz(pieces), piece = 16 * (me & (pieces - 1)), step = workers >> shift;
  for (int i = me >> shift; i < moves; i += kBatch * step) {
    u32x4 k[kBatch], v[kBatch];
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      if (i + n * step >= moves) break;
      const int64_t from = at.at(source(i + n * step)) + piece;
      k[n] = *reinterpret_cast<const u32x4*>(at.k + from);
      v[n] = *reinterpret_cast<const u32x4*>(at.v + from);
    }
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      if (i + n * step >= moves) break;
      const int64_t to = at.at(hole(i + n * step)) + piece;
      *reinterpret_cast<u32x4*>(at.k + to) = k[n];
      *reinterpret_cast<u32x4*>(at.v + to) = v[n];
    }
  }
}

// fp8: LANES lanes take the page that hole h0 is the first one of (holes ascending), as its scale is a matter of all its rows.
template <int LANES, typename Hole, typename Source>
__device__ __forceinline__ void recode_page(const KvView& kv, const RowPlace& at, int g, int keep, const float (&edge_scale)[2], int moves, Hole hole, Source source,
                                            int h0) {
  const int lane = threadIdx.x & (LANES - 1), mine = threadIdx.x & 63 & ~(LANES - 1);
  auto vote = [&](bool x) { return __ballot(x) >> mine & (~0ull >> (64 - LANES)); };
  float* k_scale = const_cast<float*>(kv.k_scale) + g;
  float* v_scale = const_cast<float*>(kv.v_scale) + g;
  const int pieces = kv.head_dim / 16, shift = __builtin_ctz(pieces), rows = LANES >> shift;
  const int piece = 16 * (lane & (pieces - 1)), r = lane >> shift;
  const int edge = keep >> at.shift;                     // the one page that may have rows of both kinds: its scales are those it had
  auto scales_of = [&](int t, int page, float& ks, float& vs) {
    const int64_t s = static_cast<int64_t>(page) * kv.num_kv_heads;
    const bool there = (t >> at.shift) == edge;
    ks = there ? edge_scale[0] : k_scale[s];
    vs = there ? edge_scale[1] : v_scale[s];
  };
  const int t0 = hole(h0) & ~at.mask, live = min(at.mask + 1, keep - t0);
  const int page = at.page(t0);
  const float ko = k_scale[static_cast<int64_t>(page) * kv.num_kv_heads], vo = v_scale[static_cast<int64_t>(page) * kv.num_kv_heads];
  int h1 = h0;                                       // past the page's last hole
  float kn = 0.f, vn = 0.f;
  for (uint64_t in = ~0ull; in >> (LANES - 1) & 1;) {
    const int h = h1 + lane;
    const bool here = h < moves && hole(min(h, moves - 1)) - t0 < live;
    if (here) {
      const int from = source(h);
      float ks, vs;
      scales_of(from, at.page(from), ks, vs);
      kn = fmaxf(kn, ks);
      vn = fmaxf(vn, vs);
    }
    in = vote(here);
    h1 += __popcll(in);
  }
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    kn = fmaxf(kn, __shfl_xor(kn, o, LANES));
    vn = fmaxf(vn, __shfl_xor(vn, o, LANES));
  }
  if (h1 - h0 < live) {                              // some rows stay
    kn = fmaxf(kn, ko);
    vn = fmaxf(vn, vo);
    const float kr = scale_ratio(ko, kn), vr = scale_ratio(vo, vn);
    auto is_hole = [&](int t) {
      int lo = h0, hi = h1;
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (hole(mid) < t) lo = mid + 1;
        else hi = mid;
      }
      return lo < h1 && hole(lo) == t;
    };
    if (kr != 1.f || vr != 1.f) {
      for (int r0 = r; r0 < live; r0 += kBatch * rows) {
        u32x4 k[kBatch], v[kBatch];
        uint32_t stay = 0;
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
          const int row = r0 + n * rows;
          if (row >= live || is_hole(t0 + row)) continue;
          const int64_t to = at.at(page, t0 + row) + piece;
          stay |= 1u << n;
          k[n] = *reinterpret_cast<const u32x4*>(at.k + to);
          v[n] = *reinterpret_cast<const u32x4*>(at.v + to);
        }
#pragma unroll
        for (int n = 0; n < kBatch; ++n) {
          if (!(stay >> n & 1u)) continue;
          const int64_t to = at.at(page, t0 + r0 + n * rows) + piece;
          *reinterpret_cast<u32x4*>(at.k + to) = rescale_codes(k[n], kr);
          *reinterpret_cast<u32x4*>(at.v + to) = rescale_codes(v[n], vr);
        }
      }
    }
  }
  for (int h = h0 + r; h < h1; h += kBatch * rows) {
    u32x4 k[kBatch], v[kBatch];
    float kr[kBatch], vr[kBatch];
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      if (h + n * rows >= h1) break;
      const int from = source(h + n * rows), src_page = at.page(from);
      float ks, vs;
      scales_of(from, src_page, ks, vs);
      kr[n] = scale_ratio(ks, kn);
      vr[n] = scale_ratio(vs, vn);
      const int64_t src = at.at(src_page, from) + piece;
      k[n] = *reinterpret_cast<const u32x4*>(at.k + src);
      v[n] = *reinterpret_cast<const u32x4*>(at.v + src);
    }
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      if (h + n * rows >= h1) break;
      const int64_t to = at.at(page, hole(h + n * rows)) + piece;
      *reinterpret_cast<u32x4*>(at.k + to) = rescale_codes(k[n], kr[n]);
      *reinterpret_cast<u32x4*>(at.v + to) = rescale_codes(v[n], vr[n]);
    }
  }
  // (all lanes of the page have read its old scale)
  if (lane == 0) {
    k_scale[static_cast<int64_t>(page) * kv.num_kv_heads] = kn;
    v_scale[static_cast<int64_t>(page) * kv.num_kv_heads] = vn;
  }
}

// The pages of a (request, head), LANES lanes to each, so many side by side in each of the `workers` wavefronts.
template <int LANES, typename Hole, typename Source>
__device__ __forceinline__ void recode_all(const KvView& kv, const RowPlace& at, int g, int keep, int pages, const float (&edge_scale)[2], int moves, Hole hole, Source source,
                                           int me, int workers) {
  for (int p = me * (64 / LANES) + (threadIdx.x & 63) / LANES; p < pages; p += workers * (64 / LANES)) {
    int lo = 0, hi = moves;                              // the page's first hole
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (hole(mid) < p << at.shift) lo = mid + 1;
      else hi = mid;
    }
    if (lo < moves && hole(lo) >> at.shift == p) recode_page<LANES>(kv, at, g, keep, edge_scale, moves, hole, source, lo);
  }
}

// Worker `me` of `workers` wavefronts.  A page is a chain of six loads and little else.  Where there are fewer holes than pages (a step at the budget:
// a few rows in as many pages) the holes are dealt out, a wavefront to each, which has a page of 16 rows in one turn; else the
// pages, sixteen lanes to each, four chains side by side, or from 32 rows on a wavefront, as the rows to write anew are what takes time.  Both sides on caches
// restored before each pass, whose pages have scales of their own (us): 64 requests, budget 4096, five new tokens, holes to 16 lanes 50, to wavefronts 40; 32
// prompts of 8 K, pages of 4, 8, 16, 32, 64, 128 rows to 16 lanes 178, 166, 160, 166, 241, 372, to wavefronts 327, 203, 176, 162, 154, 163; 64 of 4 K
// 231, 211, 214, 222, 351, 361 and 412, 251, 218, 188, 182, 207; 16 of 32 K, pages of 16, 32, 64, 176, 277, 490 and 211, 190, 178.
template <typename Hole, typename Source>
__device__ __forceinline__ void recode_pages(const KvView& kv, const RowPlace& at, int g, int keep, const float (&edge_scale)[2], int moves, Hole hole, Source source,
                                             int me, int workers) {
  const int pages = (keep + at.mask) >> at.shift;
  if (moves < pages) {
    for (int h = me; h < moves; h += workers)
      if (h == 0 || hole(h) >> at.shift != hole(h - 1) >> at.shift) recode_page<64>(kv, at, g, keep, edge_scale, moves, hole, source, h);
  } else if (at.mask < 31) {
    recode_all<16>(kv, at, g, keep, pages, edge_scale, moves, hole, source, me, workers);
  } else {
    recode_all<64>(kv, at, g, keep, pages, edge_scale, moves, hole, source, me, workers);
  }
}

// THREADS: a thread has NQ times four neighbouring tokens in registers.  MANY: rows longer than that are walked in blocks, their keys worked
// out anew each time.
template <int THREADS, int NQ, bool MANY, bool FP8>
__global__ __launch_bounds__(THREADS, THREADS < 1024 ? 1 : NQ <= 2 && !FP8 ? 8 : 4) void evict_select(EvictArgs a, MoveWs ws, int esz, bool wide, bool moves_rows) {
  constexpr int kWaves = THREADS / 64, kSpan = 4 * THREADS, kBlock = NQ * kSpan;
  constexpr bool kHold = NQ <= 2;        // weights and positions stay in registers beside the keys
  static_assert(NQ * kWaves <= 128, "");
  __shared__ uint32_t hist[3][2048];
  __shared__ int s_tot[2][NQ * kWaves];
  __shared__ uint32_t s_sum[kWaves];
  __shared__ int s_last[kWaves];
  __shared__ uint32_t s_digit[3], s_above[3];
  __shared__ int s_hole[kMoveList], s_from[kMoveList], s_pos[kMoveList];
  __shared__ float s_w[kMoveList];
  const KvView& kv = a.kv;
  const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t pair = static_cast<int64_t>(b) * kv.num_kv_heads + g;
  const int len = min(max(kv.seq_lens[b], 0), kv.max_seq_len);
  const int old = min(max(a.old_lens[b], 0), len), keep = min(max(a.budgets[b], 0), len);
  float* weights = a.weights + pair * a.state_stride;
  int32_t* positions = a.positions + pair * a.state_stride;
  const float* scores = a.scores ? a.scores + pair * a.score_stride : nullptr;
  for (int i = tid; i < 3 * 2048; i += THREADS) (&hist[0][0])[i] = 0;

  auto read4 = [&](const auto* p, int t, auto (&x)[4]) { // p[t .. t+3], those that are tokens
    typedef std::remove_reference_t<decltype(x[0])> T;
    typedef T vec __attribute__((ext_vector_type(4)));
    if (wide && t + 4 <= len) {
      const vec y = *reinterpret_cast<const vec*>(p + t);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = y[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = t + j < len ? p[t + j] : T(0);
    }
  };
  auto first_of = [&](int block, int q) { return block * kBlock + q * kSpan + 4 * tid; };
  auto weights_at = [&](int t, float (&w)[4]) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (scores) read4(scores, t, s);
    if (t < old) {
      read4(weights, t, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = t + j >= old ? s[j] : scores ? accumulate(w[j], a.decay, s[j]) : w[j];
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = s[j];
    }
  };
  const int blocks = MANY ? (len + kBlock - 1) / kBlock : 1;

  // ---- what is there, and the newest position so far ----
  float w[kHold ? NQ : 1][4];
  int pos[kHold ? NQ : 1][4];
  int last = -1;
  for (int block = 0; block < blocks; ++block) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int t = first_of(block, q), at = kHold ? q : 0;
      if (kHold) weights_at(t, w[at]);
#pragma unroll
      for (int j = 0; j < 4; ++j) pos[at][j] = -1;
      if (t < old) {
        read4(positions, t, pos[at]);
#pragma unroll
        for (int j = 0; j < 4; ++j) last = t + j < old ? max(last, pos[at][j]) : last;
      }
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) last = max(last, __shfl_xor(last, o, 64));
  if (lane == 0) s_last[wave] = last;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) last = max(last, s_last[i]);
  const int64_t recent_from = static_cast<int64_t>(last) + (len - old) - a.recent_tokens;      // positions beyond it are protected
  auto numbered = [&](int t, int p) { return t < old ? p : last + 1 + (t - old); };
  auto key_of = [&](int p, float weight) { return p < a.sink_tokens || p > recent_from ? kProtected : weight_key(weight); };

  uint32_t key[NQ][4];
  auto load_keys = [&](int block) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int t = first_of(block, q), at = kHold ? q : 0;
      if (!kHold || MANY) {
        weights_at(t, w[at]);
        if (t < old) read4(positions, t, pos[at]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) key[q][j] = key_of(numbered(t + j, pos[at][j]), w[at][j]);
    }
  };
  load_keys(0);

  // ---- the K'-th largest key, from the top: 11, 11 and 10 bits ----
  int shift = 32;
  uint32_t prefix = 0, want = keep, equal = 0;           // keys whose bits from `shift` on are `prefix`: `equal` of them, `want` stay
  if (keep > 0 && keep < len) {
    for (int pass = 0; pass < 3; ++pass) {
      const int bits = pass == 2 ? 10 : 11, above_shift = shift;
      const uint32_t bins = 1u << bits;
      shift -= bits;
      for (int block = 0; block < blocks; ++block) {
        if (MANY && (pass > 0 || block > 0)) load_keys(block);
#pragma unroll
        for (int q = 0; q < NQ; ++q)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (first_of(block, q) + j < len && (pass == 0 || key[q][j] >> above_shift == prefix)) atomicAdd(&hist[pass][key[q][j] >> shift & (bins - 1)], 1u);
      }
      __syncthreads();
      constexpr int kMost = 2048 / THREADS;              // bins of a thread, from the top
      const int per = pass == 2 ? (kMost + 1) / 2 : kMost;
      int mine = 0;
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        const int bin = static_cast<int>(bins) - 1 - (tid * per + i);
        if (i < per && bin >= 0) mine += hist[pass][bin];
      }
      int upto = wave_inclusive(mine);
      if (lane == 63) s_sum[wave] = upto;
      __syncthreads();
      for (int i = 0; i < wave; ++i) upto += s_sum[i];
      if (upto >= static_cast<int>(want) && upto - mine < static_cast<int>(want)) {
        uint32_t above = upto - mine;
        for (int i = 0; i < per; ++i) {
          const int bin = static_cast<int>(bins) - 1 - (tid * per + i);
          if (above + hist[pass][bin] >= want) {
            s_digit[pass] = bin;
            s_above[pass] = above;
            break;
          }
          above += hist[pass][bin];
        }
      }
      __syncthreads();
      prefix = prefix << bits | s_digit[pass];
      equal = hist[pass][s_digit[pass]];
      want -= s_above[pass];
      if (want == equal) break;
    }
  }
  const bool ties = want < equal;                        // (all bits told apart)
  auto stays_of = [&](uint32_t k) { return keep == len || (keep > 0 && (k >> shift > prefix || (k >> shift == prefix && !ties))); };
  auto ties_of = [&](uint32_t k) { return ties && k >> shift == prefix; };

  // ---- in order of the slots: ranks of flagged tokens ----
  // flags[q]: four bits; rank[q]: flagged tokens before this thread's of quad q, in this block and `base` before; returns base and all of the block
  auto ranks = [&](const uint32_t (&flags)[NQ], int (&rank)[NQ], int base, int* totals) {
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int mine = __popc(flags[q]), upto = wave_inclusive(mine);
      if (lane == 63) totals[q * kWaves + wave] = upto;
      rank[q] = upto - mine;
    }
    __syncthreads();
    int x0 = lane < NQ * kWaves ? totals[lane] : 0, x1 = 64 + lane < NQ * kWaves ? totals[64 + lane] : 0;
    const int i0 = wave_inclusive(x0), half = __builtin_amdgcn_readlane(i0, 63), i1 = wave_inclusive(x1) + half;
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int e = q * kWaves + wave;
      rank[q] += base + (e < 64 ? __builtin_amdgcn_readlane(i0 - x0, e & 63) : __builtin_amdgcn_readlane(i1 - x1, e & 63));
    }
    return base + __builtin_amdgcn_readlane(i1, 63);
  };

  int32_t* list = ws.list + pair * kv.max_seq_len;
  int ties_before = 0, flagged = 0;
  for (int block = 0; block < blocks; ++block) {
    if (MANY) load_keys(block);
    uint32_t stays[NQ], moves[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      stays[q] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) stays[q] |= static_cast<uint32_t>(first_of(block, q) + j < len && stays_of(key[q][j])) << j;
    }
    if (ties) {
      uint32_t equals[NQ];
      int rank[NQ];
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        equals[q] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) equals[q] |= static_cast<uint32_t>(first_of(block, q) + j < len && ties_of(key[q][j])) << j;
      }
      ties_before = ranks(equals, rank, ties_before, s_tot[0]);
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (equals[q] >> j & 1u) stays[q] |= static_cast<uint32_t>(rank[q] + __popc(equals[q] & ((1u << j) - 1)) < static_cast<int>(want)) << j;
    }
    int rank[NQ];
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      moves[q] = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = first_of(block, q) + j;
        moves[q] |= static_cast<uint32_t>(t < len && (t < keep) != (stays[q] >> j & 1u)) << j;
      }
    }
    flagged = ranks(moves, rank, flagged, s_tot[1]);
    const int holes = flagged / 2;                       // (of a row in one block: as many sources as holes, all holes first)
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      const int t0 = first_of(block, q), at = kHold ? q : 0;
      if (t0 >= len) continue;
      if (!kHold) {
        weights_at(t0, w[at]);
        if (t0 < old) read4(positions, t0, pos[at]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = t0 + j;
        if (moves[q] >> j & 1u) {
          const int r = rank[q] + __popc(moves[q] & ((1u << j) - 1));
          list[r] = t;
          if (!MANY && t < keep && r < kMoveList) s_hole[r] = t;
          if (!MANY && t >= keep && r - holes < kMoveList) {
            s_from[r - holes] = t;
            s_w[r - holes] = w[at][j];
            s_pos[r - holes] = numbered(t, pos[at][j]);
          }
        } else if (t < keep) {
          if (t >= old || scores) weights[t] = w[at][j];
          if (t >= old) positions[t] = numbered(t, pos[at][j]);
        }
      }
    }
    if (MANY) __syncthreads();                           // (s_tot is written again)
  }
  __syncthreads();                                       // the list is complete; weights and positions beyond K' are as they were
  const int holes = flagged / 2;
  auto hole = [&](int i) { return !MANY && i < kMoveList ? s_hole[i] : list[i]; };
  auto source = [&](int i) { return !MANY && i < kMoveList ? s_from[i] : list[holes + i]; };
  for (int i = tid; i < holes; i += THREADS) {
    const int to = hole(i);
    if (!MANY && i < kMoveList) {
      weights[to] = s_w[i];
      positions[to] = s_pos[i];
    } else {
      const int t = list[holes + i];
      const float s = scores ? scores[t] : 0.f;
      weights[to] = t >= old ? s : scores ? accumulate(weights[t], a.decay, s) : weights[t];
      positions[to] = numbered(t, positions[t]);
    }
  }
  float edge[2] = {0.f, 0.f};
  if (FP8 && holes) {
    const int64_t at = static_cast<int64_t>(kv.block_table[static_cast<int64_t>(b) * kv.block_table_stride + (keep >> kv.page_shift)]) * kv.num_kv_heads + g;
    edge[0] = kv.k_scale[at];
    edge[1] = kv.v_scale[at];
  }
  if (!moves_rows) {
    if (tid == 0) {
      ws.moves[pair] = holes;
      ws.kept[pair] = keep;
      ws.edge[2 * pair] = edge[0];
      ws.edge[2 * pair + 1] = edge[1];
    }
    return;
  }
  if (g == 0 && tid == 0) a.new_lens[b] = keep;
  const RowPlace at(kv, b, g, esz);
  if constexpr (FP8) {
    __syncthreads();                                     // all have read the scales of the page at K'
    recode_pages(kv, at, g, keep, edge, holes, hole, source, wave, kWaves);
  } else {
    copy_rows(at, kv.head_dim * esz / 16, holes, hole, source, tid, THREADS);
  }
}

template <bool FP8>
__global__ __launch_bounds__(kMoveThreads) void evict_move(EvictArgs a, MoveWs ws, int esz) {
  const KvView& kv = a.kv;
  const int g = blockIdx.y, b = blockIdx.z;
  const int64_t pair = static_cast<int64_t>(b) * kv.num_kv_heads + g;
  const int keep = ws.kept[pair], moves = ws.moves[pair];
  if (g == 0 && blockIdx.x == 0 && threadIdx.x == 0) a.new_lens[b] = keep;
  const int32_t* list = ws.list + pair * kv.max_seq_len;
  auto hole = [&](int i) { return list[i]; };
  auto source = [&](int i) { return list[moves + i]; };
  const RowPlace at(kv, b, g, esz);
  const int me = blockIdx.x * kMoveThreads + threadIdx.x, workers = gridDim.x * kMoveThreads;
  if constexpr (FP8) {
    const float edge[2] = {ws.edge[2 * pair], ws.edge[2 * pair + 1]};
    recode_pages(kv, at, g, keep, edge, moves, hole, source, me >> 6, workers >> 6);
  } else {
    copy_rows(at, kv.head_dim * esz / 16, moves, hole, source, me, workers);
  }
}

struct EvictWs {
  size_t kept, edge, list, bytes;
};
EvictWs carve(const KvView& kv) {
  const size_t pairs = static_cast<size_t>(kv.batch) * kv.num_kv_heads;
  EvictWs w;
  w.kept = align_up(pairs * 4, 256);
  w.edge = align_up(w.kept + pairs * 4, 256);
  w.list = align_up(w.edge + pairs * 8, 256);
  w.bytes = align_up(w.list + pairs * kv.max_seq_len * 4, 256);
  return w;
}

}  // namespace

size_t evict_workspace(const KvView& kv) { return carve(kv).bytes; }

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
  const EvictWs w = carve(a.kv);
  char* p = static_cast<char*>(a.workspace);
  MoveWs ws;
  ws.moves = reinterpret_cast<int32_t*>(p);
  ws.kept = reinterpret_cast<int32_t*>(p + w.kept);
  ws.edge = reinterpret_cast<float*>(p + w.edge);
  ws.list = reinterpret_cast<int32_t*>(p + w.list);
  const int64_t pairs = static_cast<int64_t>(a.kv.batch) * a.kv.num_kv_heads;
  const int esz = a.kv_dtype == PILLAR_F32 ? 4 : a.kv_dtype == PILLAR_BF16 ? 2 : 1;
  const bool wide = a.state_stride % 4 == 0 && (!a.scores || a.score_stride % 4 == 0) &&
                    ((reinterpret_cast<uintptr_t>(a.weights) | reinterpret_cast<uintptr_t>(a.positions) | reinterpret_cast<uintptr_t>(a.scores)) & 15u) == 0;
  // One launch, in which the workgroup that selects moves its rows too, where that fills the chip or the rows are short.  The host does not know how many rows
  // will move, and a step at the budget moves few.  Two / one, on caches restored before each pass (us): steps, one request, 2 of 2050 11.4 / 9.6, 8, 4
  // of 4004 14.4 / 11.9, 31, 16 of 8016 22 / 19, 64, 5 of 4101 24 / 20; fp8 17 / 15.5, 30 / 18, 37 / 30.5, 47 / 40.  The first eviction of a prompt
  // loses by it where there are few pairs: one of 4096 to 2048 14.6 / 24, fp8 65 / 106, 8 of 8192 36 / 75, 124 / 133, 31 105 / 101, 152 / 158; steps are
  // hundreds to a prompt.  Beyond 8192 tokens it would lose more than steps gain: one of 32 K to 4096 43 / 111, fp8 122 / 259, one of
  // 21000 to 20000 41 / 50, 56 / 358; steps of 16000 33 / 31, 45 / 39.  (Not where the new lengths replace what the workgroups of other heads read.)
  auto apart = [&](const int32_t* p) { return a.new_lens + a.kv.batch <= p || p + a.kv.batch <= a.new_lens; };
  const bool moves_rows = (pairs >= num_cus() || a.kv.max_seq_len <= 8192) && apart(a.kv.seq_lens) && apart(a.old_lens) && apart(a.budgets);
  const bool fp8 = a.kv_dtype == PILLAR_FP8_E4M3;
  {
    KernelTimer timer("evict_select", s);
    const dim3 grid(a.kv.num_kv_heads, a.kv.batch);
    const int n = a.kv.max_seq_len;
#define PILLAR_EVICT(threads, quads, many)                                                                                                             \
  do {                                                                                                                                                 \
    if (fp8) hipLaunchKernelGGL((evict_select<threads, quads, many, true>), grid, dim3(threads), 0, s, a, ws, esz, wide, moves_rows);                    \
    else hipLaunchKernelGGL((evict_select<threads, quads, many, false>), grid, dim3(threads), 0, s, a, ws, esz, wide, moves_rows);                       \
  } while (0)
    if (n <= 1024) PILLAR_EVICT(256, 1, false);
    else if (n <= 4096) PILLAR_EVICT(1024, 1, false);
    else if (n <= 8192) PILLAR_EVICT(1024, 2, false);
    else if (n <= 32768) PILLAR_EVICT(1024, 8, false);
    else PILLAR_EVICT(1024, 8, true);
#undef PILLAR_EVICT
  }
  if (!moves_rows) {
    KernelTimer timer("evict_move", s);
    // at most half of the rows move; as many workgroups as that gives work, and no more than eight per compute unit
    const int most = (a.kv.max_seq_len / 2 + 15) / 16;
    const int blocks = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(most, (8 * num_cus() + pairs - 1) / pairs)));
    const dim3 grid(blocks, a.kv.num_kv_heads, a.kv.batch);
    if (fp8) hipLaunchKernelGGL(evict_move<true>, grid, dim3(kMoveThreads), 0, s, a, ws, esz);
    else hipLaunchKernelGGL(evict_move<false>, grid, dim3(kMoveThreads), 0, s, a, ws, esz);
  }
  return hipGetLastError();
}

}  // namespace pillar

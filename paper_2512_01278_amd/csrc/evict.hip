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
// Two launches:
//   evict_select  one workgroup per (request, KV head): the weights, a radix select of the K'-th key, the list of holes and sources
//                 in order, and the moves within weights and positions;
//   evict_move    the rows of K and V.
#include <algorithm>

#include "launch.hpp"
#include "page_scale.hpp"

namespace pillar {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kMoveThreads = 256;
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

__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs a, MoveWs ws) {
  __shared__ uint32_t hist[2048];
  __shared__ uint32_t s_scan[2][kSelWaves];
  __shared__ int s_last[kSelWaves];
  __shared__ uint32_t s_digit, s_above;
  const KvView& kv = a.kv;
  const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t pair = static_cast<int64_t>(b) * kv.num_kv_heads + g;
  const int len = min(max(kv.seq_lens[b], 0), kv.max_seq_len);
  const int old = min(max(a.old_lens[b], 0), len), keep = min(max(a.budgets[b], 0), len);
  float* weights = a.weights + pair * a.state_stride;
  int32_t* positions = a.positions + pair * a.state_stride;
  const float* scores = a.scores ? a.scores + pair * a.score_stride : nullptr;

  // ---- the newest position so far ----
  int last = -1;
  for (int t = tid; t < old; t += kSelThreads) last = max(last, positions[t]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) last = max(last, __shfl_xor(last, o, 64));
  if (lane == 0) s_last[wave] = last;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSelWaves; ++i) last = max(last, s_last[i]);
  const int64_t recent_from = static_cast<int64_t>(last) + (len - old) - a.recent_tokens;      // positions beyond it are protected

  auto weight_of = [&](int t) {
    const float s = scores ? scores[t] : 0.f;
    if (t >= old) return s;
    return scores ? accumulate(weights[t], a.decay, s) : weights[t];
  };
  auto position_of = [&](int t) { return t < old ? positions[t] : last + 1 + (t - old); };
  auto key_of = [&](int t) {
    const int pos = position_of(t);
    return pos < a.sink_tokens || pos > recent_from ? kProtected : weight_key(weight_of(t));
  };

  // ---- the K'-th largest key, by digits of 11, 11 and 10 bits; `need`: how many of the keys equal to it stay ----
  uint32_t kth = 0, need = 0, equal = 0;
  if (keep > 0 && keep < len) {
    uint32_t prefix = 0, want = keep;
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : 2048;
      for (int i = tid; i < bins; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      for (int t = tid; t < len; t += kSelThreads) {
        const uint32_t k = key_of(t);
        if (pass == 0 || (k >> (shift + (pass == 1 ? 11 : 10))) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
      }
      __syncthreads();
      // from the top: each thread has `per` bins; the digit is where the running count reaches `want`
      const int per = bins / kSelThreads;
      uint32_t mine = 0;
      for (int i = 0; i < per; ++i) mine += hist[bins - 1 - (tid * per + i)];
      uint32_t upto = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(upto, o, 64);
        if (lane >= o) upto += x;
      }
      if (lane == 63) s_scan[0][wave] = upto;
      __syncthreads();
      for (int i = 0; i < wave; ++i) upto += s_scan[0][i];
      if (upto >= want && upto - mine < want) {
        uint32_t above = upto - mine;
        for (int i = 0; i < per; ++i) {
          const int bin = bins - 1 - (tid * per + i);
          if (above + hist[bin] >= want) {
            s_digit = bin;
            s_above = above;
            break;
          }
          above += hist[bin];
        }
      }
      __syncthreads();
      prefix = prefix << (pass == 2 ? 10 : 11) | s_digit;
      equal = hist[s_digit];
      want -= s_above;
      __syncthreads();
    }
    kth = prefix;
    need = want;
  } else if (keep == len) {
    need = equal = 0x7fffffffu;                          // everything stays: every key is >= 0
  } else {
    kth = kProtected;                                    // nothing does
  }
  const bool ties = need < equal;

  // ---- in order of the slots: weights and positions of what stays, and the list of holes and sources ----
  int32_t* list = ws.list + pair * kv.max_seq_len;
  uint32_t base_eq = 0, base_move = 0, holes = 0;
  for (int t0 = 0; t0 < len; t0 += kSelThreads) {
    const int t = t0 + tid;
    const bool there = t < len;
    const uint32_t k = there ? key_of(t) : 0;
    bool stays = there && (keep == len || k > kth);
    const bool eq = there && keep < len && k == kth;
    if (ties) {
      const uint64_t bits = __ballot(eq);
      if (lane == 0) s_scan[0][wave] = __popcll(bits);
      __syncthreads();
      uint32_t before = base_eq, all = 0;
      for (int i = 0; i < kSelWaves; ++i) {
        before += i < wave ? s_scan[0][i] : 0;
        all += s_scan[0][i];
      }
      stays |= eq && before + __popcll(bits & ((1ull << lane) - 1)) < need;
      base_eq += all;
    } else {
      stays |= eq && need > 0;
    }
    const bool moves = there && (t < keep ? !stays : stays);
    const uint64_t bits = __ballot(moves);
    if (lane == 0) s_scan[1][wave] = __popcll(bits);
    __syncthreads();
    uint32_t before = base_move, all = 0;
    for (int i = 0; i < kSelWaves; ++i) {
      before += i < wave ? s_scan[1][i] : 0;
      all += s_scan[1][i];
    }
    if (moves) list[before + __popcll(bits & ((1ull << lane) - 1))] = t;
    base_move += all;
    if (t < keep && stays) {
      if (t >= old || scores) weights[t] = weight_of(t);
      if (t >= old) positions[t] = position_of(t);
    }
    __syncthreads();
  }
  holes = base_move / 2;                                 // as many sources as holes, and all holes come first
  // (weights and positions beyond K' are as they were, the list is complete: the barriers above)
  for (uint32_t i = tid; i < holes; i += kSelThreads) {
    const int from = list[holes + i], to = list[i];
    weights[to] = weight_of(from);
    positions[to] = position_of(from);
  }
  if (tid == 0) {
    ws.moves[pair] = holes;
    ws.kept[pair] = keep;
    if (kv.k_scale && holes) {
      const int64_t at = static_cast<int64_t>(kv.block_table[static_cast<int64_t>(b) * kv.block_table_stride + (keep >> kv.page_shift)]) * kv.num_kv_heads + g;
      ws.edge[2 * pair] = kv.k_scale[at];
      ws.edge[2 * pair + 1] = kv.v_scale[at];
    }
  }
}

// ---- rows of 16-byte pieces, copied ----
__global__ __launch_bounds__(kMoveThreads) void evict_move(EvictArgs a, MoveWs ws, int esz) {
  const KvView& kv = a.kv;
  const int g = blockIdx.y, b = blockIdx.z;
  const int64_t pair = static_cast<int64_t>(b) * kv.num_kv_heads + g;
  if (g == 0 && blockIdx.x == 0 && threadIdx.x == 0) a.new_lens[b] = ws.kept[pair];
  const int moves = ws.moves[pair];
  const int32_t* list = ws.list + pair * kv.max_seq_len;
  const RowPlace at(kv, b, g, esz);
  const int pieces = kv.head_dim * esz / 16, shift = __builtin_ctz(pieces), rows = kMoveThreads >> shift;
  const int piece = 16 * (threadIdx.x & (pieces - 1));
#pragma unroll 2
  for (int i = blockIdx.x * rows + (threadIdx.x >> shift); i < moves; i += gridDim.x * rows) {
    const int64_t from = at.at(list[moves + i]) + piece, to = at.at(list[i]) + piece;
    const u32x4 k = *reinterpret_cast<const u32x4*>(at.k + from), v = *reinterpret_cast<const u32x4*>(at.v + from);
    *reinterpret_cast<u32x4*>(at.k + to) = k;
    *reinterpret_cast<u32x4*>(at.v + to) = v;
  }
}

// ---- fp8: a wavefront per page that has holes ----
__global__ __launch_bounds__(kMoveThreads) void evict_move_fp8(EvictArgs a, MoveWs ws) {
  const KvView& kv = a.kv;
  const int g = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63;
  const int64_t pair = static_cast<int64_t>(b) * kv.num_kv_heads + g;
  const int keep = ws.kept[pair], moves = ws.moves[pair];
  if (g == 0 && blockIdx.x == 0 && threadIdx.x == 0) a.new_lens[b] = keep;
  if (moves == 0) return;
  const int32_t* holes = ws.list + pair * kv.max_seq_len;
  const int32_t* sources = holes + moves;
  const RowPlace at(kv, b, g, 1);
  float* k_scale = const_cast<float*>(kv.k_scale) + g;
  float* v_scale = const_cast<float*>(kv.v_scale) + g;
  const int pieces = kv.head_dim / 16, shift = __builtin_ctz(pieces), rows = 64 >> shift;
  const int piece = 16 * (lane & (pieces - 1));
  const int edge = keep >> at.shift;                     // the one page that may have rows of both kinds: its scales are read from the workspace
  auto scales_of = [&](int t, float& ks, float& vs) {
    if ((t >> at.shift) == edge) {
      ks = ws.edge[2 * pair];
      vs = ws.edge[2 * pair + 1];
    } else {
      const int64_t s = static_cast<int64_t>(at.page(t)) * kv.num_kv_heads;
      ks = k_scale[s];
      vs = v_scale[s];
    }
  };
  auto hole_at_or_after = [&](int t) {
    int lo = 0, hi = moves;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (holes[mid] < t) lo = mid + 1;
      else hi = mid;
    }
    return lo;
  };
  const int pages = (keep + at.mask) >> at.shift, waves = kMoveThreads / 64;
  for (int p = blockIdx.x * waves + (threadIdx.x >> 6); p < pages; p += gridDim.x * waves) {
    const int t0 = p << at.shift, live = min(at.mask + 1, keep - t0);
    const int h0 = hole_at_or_after(t0), h1 = hole_at_or_after(t0 + live);
    if (h0 == h1) continue;
    const int page = at.page(t0);
    float kn = 0.f, vn = 0.f;
    for (int h = h0 + lane; h < h1; h += 64) {
      float ks, vs;
      scales_of(sources[h], ks, vs);
      kn = fmaxf(kn, ks);
      vn = fmaxf(vn, vs);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      kn = fmaxf(kn, __shfl_xor(kn, o, 64));
      vn = fmaxf(vn, __shfl_xor(vn, o, 64));
    }
    const float ko = k_scale[static_cast<int64_t>(page) * kv.num_kv_heads], vo = v_scale[static_cast<int64_t>(page) * kv.num_kv_heads];
    if (h1 - h0 < live) {                                // some rows stay
      kn = fmaxf(kn, ko);
      vn = fmaxf(vn, vo);
      const float kr = scale_ratio(ko, kn), vr = scale_ratio(vo, vn);
      if (kr != 1.f || vr != 1.f) {
        for (int i = lane >> shift; i < live; i += rows) {
          bool hole = false;
          const int at_or_after = hole_at_or_after(t0 + i);
          if (at_or_after < h1) hole = holes[at_or_after] == t0 + i;
          if (hole) continue;
          const int64_t to = at.at(page, t0 + i) + piece;
          u32x4* kp = reinterpret_cast<u32x4*>(at.k + to);
          u32x4* vp = reinterpret_cast<u32x4*>(at.v + to);
          *kp = rescale_codes(*kp, kr);
          *vp = rescale_codes(*vp, vr);
        }
      }
    }
    for (int h = h0 + (lane >> shift); h < h1; h += rows) {
      const int from = sources[h];
      float ks, vs;
      scales_of(from, ks, vs);
      const int64_t src = at.at(from) + piece, to = at.at(page, holes[h]) + piece;
      const u32x4 k = *reinterpret_cast<const u32x4*>(at.k + src), v = *reinterpret_cast<const u32x4*>(at.v + src);
      *reinterpret_cast<u32x4*>(at.k + to) = rescale_codes(k, scale_ratio(ks, kn));
      *reinterpret_cast<u32x4*>(at.v + to) = rescale_codes(v, scale_ratio(vs, vn));
    }
    // (every lane has read the old scale: the reads above are in program order for the whole wavefront)
    if (lane == 0) {
      k_scale[static_cast<int64_t>(page) * kv.num_kv_heads] = kn;
      v_scale[static_cast<int64_t>(page) * kv.num_kv_heads] = vn;
    }
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
  {
    KernelTimer timer("evict_select", s);
    hipLaunchKernelGGL(evict_select, dim3(a.kv.num_kv_heads, a.kv.batch), dim3(kSelThreads), 0, s, a, ws);
  }
  KernelTimer timer("evict_move", s);
  const int pairs = a.kv.batch * a.kv.num_kv_heads, esz = a.kv_dtype == PILLAR_F32 ? 4 : a.kv_dtype == PILLAR_BF16 ? 2 : 1;
  // at most half of the rows move; as many workgroups as that gives work, and no more than eight per compute unit
  const int most = a.kv_dtype == PILLAR_FP8_E4M3 ? ((a.kv.max_seq_len + a.kv.page_size - 1) / a.kv.page_size + 3) / 4
                                                 : (a.kv.max_seq_len / 2 + 15) / 16;
  const int blocks = std::max(1, std::min(most, (8 * num_cus() + pairs - 1) / pairs));
  const dim3 grid(blocks, a.kv.num_kv_heads, a.kv.batch);
  if (a.kv_dtype == PILLAR_FP8_E4M3) hipLaunchKernelGGL(evict_move_fp8, grid, dim3(kMoveThreads), 0, s, a, ws);
  else hipLaunchKernelGGL(evict_move, grid, dim3(kMoveThreads), 0, s, a, ws, esz);
  return hipGetLastError();
}

}  // namespace pillar

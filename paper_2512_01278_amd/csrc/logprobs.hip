// What rows of logits say about given tokens: log-sum-exp, log probabilities, entropy, the tokens of largest logit.
//
// With c = scale log2 e and m the largest logit so far, y = (x - m) c:   S = sum 2^y,  A = sum 2^y y,
//   lse = scale m + ln 2 log2 S,  log p = scale (x - m) - ln 2 log2 S,  entropy = ln 2 (log2 S - A / S)
// so one pass over the row does (when m moves, S and A are carried over: with d = (m - m') c, S' = 2^d S, A' = 2^d (A + d S)).  Everything is a
// difference against the row's own maximum and loses nothing to its size: a row of nothing but -3e38, as masks have it, is as any other row of equal logits.
//
//   logprob_pass   a workgroup per (row, part of the row): (M, S, A) and the `top` largest of the part
//   logprob_join   a workgroup per row: joins the parts, looks the given tokens up
//
// The largest logits are kept by each wavefront as one sorted list over its 64 lanes.  A logit gets in when it is larger than the list's last, which after
// a few hundred logits is rare; the maximum of a lane's batch of logits, needed for the reference anyway, says whether to look.
#include <algorithm>

#include "launch.hpp"
#include "rope.hpp"

namespace pillar {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kNoId = INT32_MAX;

struct Params {
  LogprobArgs a;
  float c;                     // scale * log2 e
  int32_t parts, each;         // parts of a row, logits of a part (a multiple of 16)
  float* msa;                  // [rows][parts][4]
  float2* lists;               // [rows][parts][top]: logit, id (as bits)
};

struct Sums {
  float m, s, a;               // m = -inf: nothing but -inf so far
  // moves the maximum up to `to`
  __device__ __forceinline__ void move(float to, float c) {
    if (m == to) return;                                 // (also: both -inf)
    const float d = (m - to) * c;                        // -inf: nothing there
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(d);
    a = f == 0.f ? 0.f : f * (a + d * s);
    s = f == 0.f && !(s != s) ? 0.f : f * s;
    m = to;
  }
  __device__ __forceinline__ void add(Sums o, float c) {
    const float top = fmaxf(m, o.m);
    move(top, c);
    o.move(top, c);
    s += o.s;
    a += o.a;
  }
};

// larger logit, or the same one earlier
__device__ __forceinline__ bool before(float x, int i, float y, int j) { return x > y || (x == y && i < j); }

// A sorted list over the lanes of a wavefront: lane 0 has the largest.
struct List {
  float x;
  int id;
  __device__ __forceinline__ void clear() { x = -INFINITY; id = kNoId; }
  __device__ __forceinline__ void insert(float nx, int nid) {            // (the same in all lanes)
    const bool mine = before(x, id, nx, nid);
    const int at = __builtin_popcountll(__ballot(mine));
    const int lane = threadIdx.x & 63;
    const float ux = __shfl_up(x, 1);
    const int uid = __shfl_up(id, 1);
    if (!mine) {
      x = lane == at ? nx : ux;
      id = lane == at ? nid : uid;
    }
  }
  // the best 64 of both, sorted
  __device__ __forceinline__ void merge(float ox, int oid) {
    const int lane = threadIdx.x & 63;
    const float rx = __shfl(ox, 63 - lane);
    const int rid = __shfl(oid, 63 - lane);
    if (before(rx, rid, x, id)) { x = rx; id = rid; }    // a sequence that rises and falls, of the best 64
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float px = __shfl_xor(x, o);
      const int pid = __shfl_xor(id, o);
      const bool take = (lane & o) ? before(x, id, px, pid) : before(px, pid, x, id);
      if (take) { x = px; id = pid; }
    }
  }
};

template <int DT>
__device__ __forceinline__ float logit(const void* p, int64_t i) { return Storage<DT>::load(p, i); }

// TOP: a list is wanted
template <int DT, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_pass(Params p) {
  constexpr int V = DT == PILLAR_F32 ? 4 : 8;
  __shared__ Sums s_sums[kWaves];
  __shared__ float s_x[kWaves][64];
  __shared__ int s_id[kWaves][64];
  const LogprobArgs& a = p.a;
  const int r = blockIdx.x / p.parts, part = blockIdx.x - r * p.parts, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = r * a.row_stride;
  const int begin = part * p.each, end = min(a.vocab, begin + p.each);
  Sums sums{-INFINITY, 0.f, 0.f};
  List list;
  list.clear();
  float least = -INFINITY;                               // the list's last of `top`
  for (int i0 = begin + wave * 64; i0 < end; i0 += kThreads) {
    const int i = i0 + lane;
    const float x = i < end ? logit<DT>(a.logits, row + i) : -INFINITY;
    if (x > sums.m) sums.move(x, p.c);
    const float y = (x - (sums.m == -INFINITY ? 0.f : sums.m)) * p.c;
    const float e = __builtin_amdgcn_exp2f(y);
    sums.s += e;
    sums.a = __builtin_fmaf(e, fmaxf(y, -200.f), sums.a);
    if (TOP) {
      for (uint64_t over = __ballot(x > least); over; over &= over - 1) {
        const int from = __builtin_ctzll(over);
        list.insert(__shfl(x, from), i0 + from);
      }
      least = __shfl(list.x, a.top - 1);
    }
  }
  (void)V;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sums.add(Sums{__shfl_xor(sums.m, o), __shfl_xor(sums.s, o), __shfl_xor(sums.a, o)}, p.c);
  if (lane == 0) s_sums[wave] = sums;
  if (TOP) { s_x[wave][lane] = list.x; s_id[wave][lane] = list.id; }
  __syncthreads();
  if (wave > 0) return;
  const int64_t slot = static_cast<int64_t>(r) * p.parts + part;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    sums.add(s_sums[w], p.c);
    if (TOP) list.merge(s_x[w][lane], s_id[w][lane]);
  }
  if (lane == 0) *reinterpret_cast<f32x4_t*>(p.msa + 4 * slot) = f32x4_t{sums.m, sums.s, sums.a, 0.f};
  if (TOP && lane < a.top) p.lists[slot * a.top + lane] = make_float2(list.x, __int_as_float(list.id));
}

template <int DT, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_join(Params p) {
  __shared__ Sums s_sums[kWaves];
  __shared__ float s_x[kWaves][64];
  __shared__ int s_id[kWaves][64];
  const LogprobArgs& a = p.a;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t row = r * a.row_stride, slot = static_cast<int64_t>(r) * p.parts;
  Sums sums{-INFINITY, 0.f, 0.f};
  for (int i = tid; i < p.parts; i += kThreads) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p.msa + 4 * (slot + i));
    sums.add(Sums{v[0], v[1], v[2]}, p.c);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sums.add(Sums{__shfl_xor(sums.m, o), __shfl_xor(sums.s, o), __shfl_xor(sums.a, o)}, p.c);
  if (lane == 0) s_sums[wave] = sums;
  List list;
  list.clear();
  if (TOP) {
    for (int i = wave; i < p.parts; i += kWaves) {
      float2 v = make_float2(-INFINITY, __int_as_float(kNoId));
      if (lane < a.top) v = p.lists[(slot + i) * a.top + lane];
      list.merge(v.x, __float_as_int(v.y));
    }
    s_x[wave][lane] = list.x;
    s_id[wave][lane] = list.id;
  }
  __syncthreads();
  sums = s_sums[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) sums.add(s_sums[w], p.c);
  // m = -inf: nothing but -inf (and NaN); +inf: the sum is NaN, from inf - inf, and whether the row has NaN too has to be looked up
  const float log_s = log2f(sums.s);
  const bool endless = sums.m == INFINITY, empty = sums.m == -INFINITY;
  bool nan = sums.s != sums.s;
  if (endless) {
    bool mine = false;
    for (int i = tid; i < a.vocab; i += kThreads) {
      const float x = logit<DT>(a.logits, row + i);
      mine |= x != x;
    }
    nan = __syncthreads_or(mine);
  }
  auto log_prob = [&](float x) {
    if (nan) return NAN;
    if (empty) return -INFINITY;
    if (endless) return x < INFINITY ? -INFINITY : NAN;
    return __builtin_fmaf(x - sums.m, a.scale, -kLn2 * log_s);
  };
  if (tid == 0) {
    if (a.lse) a.lse[r] = nan ? NAN : empty ? -INFINITY : endless ? INFINITY : __builtin_fmaf(a.scale, sums.m, kLn2 * log_s);
    if (a.entropy) a.entropy[r] = nan || endless ? NAN : empty ? 0.f : kLn2 * (log_s - sums.a / sums.s);
  }
  for (int j = tid; j < a.num_tokens; j += kThreads) {
    const int id = a.tokens[static_cast<int64_t>(r) * a.num_tokens + j];
    a.logprobs[static_cast<int64_t>(r) * a.num_tokens + j] = id >= 0 && id < a.vocab ? log_prob(logit<DT>(a.logits, row + id)) : -INFINITY;
  }
  if (!TOP || wave > 0) return;
#pragma unroll
  for (int w = 1; w < kWaves; ++w) list.merge(s_x[w][lane], s_id[w][lane]);
  // Fewer numbers above -inf than wanted: the first of -inf, then the first that are none at all.
  int have = __builtin_popcountll(__ballot(list.x > -INFINITY));
  for (int nan = 0; nan < 2 && have < a.top; ++nan)
    for (int i0 = 0; i0 < a.vocab && have < a.top; i0 += 64) {
      const float x = i0 + lane < a.vocab ? logit<DT>(a.logits, row + i0 + lane) : 0.f;
      for (uint64_t some = __ballot(nan ? x != x : x == -INFINITY); some && have < a.top; some &= some - 1, ++have) {
        const int from = __builtin_ctzll(some);
        if (lane == have) { list.x = nan ? NAN : -INFINITY; list.id = i0 + from; }
      }
    }
  if (lane < a.top) {
    const int64_t to = static_cast<int64_t>(r) * a.top + lane;
    a.top_ids[to] = lane < have ? list.id : -1;
    a.top_logprobs[to] = lane < have ? log_prob(list.x) : -INFINITY;
  }
}

struct Plan {
  int parts, each;
};
Plan plan_of(int rows, int vocab) {
  const int64_t wanted = (4 * 256 + rows - 1) / std::max(rows, 1);
  const int most = (vocab + 4095) / 4096;
  Plan p;
  p.parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(wanted, most)));
  p.each = (((vocab + p.parts - 1) / p.parts) + 15) / 16 * 16;
  p.parts = (vocab + p.each - 1) / p.each;
  return p;
}

template <int DT, bool TOP>
hipError_t launch(const Params& p, hipStream_t s) {
  {
    KernelTimer timer("logprob_pass", s);
    hipLaunchKernelGGL((logprob_pass<DT, TOP>), dim3(static_cast<unsigned>(p.parts) * p.a.rows), dim3(kThreads), 0, s, p);
  }
  KernelTimer timer("logprob_join", s);
  hipLaunchKernelGGL((logprob_join<DT, TOP>), dim3(p.a.rows), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

size_t logprobs_workspace(int rows, int vocab, int top) {
  const Plan p = plan_of(rows, vocab);
  return align_up(static_cast<size_t>(rows) * p.parts * 16, 256) + static_cast<size_t>(rows) * p.parts * top * 8;
}

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t s) {
  const Plan plan = plan_of(a.rows, a.vocab);
  Params p;
  p.a = a;
  p.c = static_cast<float>(static_cast<double>(a.scale) * 1.4426950408889634);
  p.parts = plan.parts;
  p.each = plan.each;
  p.msa = static_cast<float*>(a.workspace);
  p.lists = reinterpret_cast<float2*>(static_cast<char*>(a.workspace) + align_up(static_cast<size_t>(a.rows) * plan.parts * 16, 256));
  if (a.dtype == PILLAR_F32) return a.top ? launch<PILLAR_F32, true>(p, s) : launch<PILLAR_F32, false>(p, s);
  return a.top ? launch<PILLAR_BF16, true>(p, s) : launch<PILLAR_BF16, false>(p, s);
}

}  // namespace pillar

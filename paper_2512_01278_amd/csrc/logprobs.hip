// What rows of logits say about given tokens: log-sum-exp, log probabilities, entropy, the tokens of largest logit.
//
// With c = scale log2 e, m one of the largest logits so far, y = (x - m) c:   R = sum of 2^y over all others,  A = sum of 2^y y over them,
//   lse = scale m + log(1 + R),  log p = scale (x - m) - log(1 + R),  entropy = log(1 + R) - ln 2 A / (1 + R)
// so one pass over the row does (when m moves to m', with d = (m - m') c:  R' = 2^d (1 + R),  A' = 2^d (A + d (1 + R)), and the new m stays out).  Everything is a
// difference against a logit of the row and loses nothing to its size: a row of nothing but -3e38, as masks have it, is as any other row of equal logits.
//
// The 1 of m is never added to the rest.  Of a token that is nearly certain, 1 + R would keep what of R lies above 2^-24, while log(1 + R) and the entropy are
// hardly more than R: 10^-4 of themselves off at 1 - p = 10^-3.  Apart from it they are exact to 10^-5 of themselves, however small.
//
//   logprob_pass   a workgroup per (row, part of the row): (m, R, A) and the `top` largest of the part
//   logprob_join   a workgroup per row: joins the parts, looks the given tokens up
//
// The largest logits are kept by each wavefront as one sorted list over its 64 lanes.  A logit gets in when it comes before the list's last, which after
// a few batches is rare; the maximum of a lane's batch, needed for m anyway, says whether to look.
//
// What bounds it: the rows at 4.8 TB/s (640 rows of 150000 bf16 logits: 40 us without alternatives, read alone 28), with two or three rows to a compute unit, and what
// the lists cost, 7 us with one alternative, 19 with eight.  Branches by what a wavefront is have to be scalar ones (readfirstlane): as lanes of a mask, the loop waited for
// every load before its next turn.  A key is one whole number, because comparisons of two parts became branches, at every step of a sort.
// More wavefronts to a row, or more parts, make more lists to fill (512 threads 52 us with one alternative, 256 49; 240 rows of 50001 fp32 with twenty 32 and
// 28), deeper prefetch gains nothing (three batches 48.4, four 48.7).
#include <algorithm>

#include "lanes.hpp"
#include "launch.hpp"
#include "rope.hpp"

namespace pillar {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// No logit is further (log2) above the reference m than this.  A first token of more than p = 4/5 is the reference, then; with less, R is 1/4 and more and
// nothing is lost in 1 + R.  A move takes a wavefront as long as a batch does: with every new largest 640 rows of 150000 took 50.8 us, so 46.5.  (Rows that rise from
// their first logit to their last move in every second batch: 53 us without alternatives instead of 43.)
constexpr float kRoom = 2.f;

// Half of x - m, which itself may be more than fp32 holds (logits of either sign near the type's end, under a small scale); factors on it are doubled.
__device__ __forceinline__ float half_apart(float x, float m) { return __builtin_fmaf(x, 0.5f, -0.5f * m); }

struct Sums {
  float m, s, a;               // reference (-inf: none so far), R (NaN: there was one), A
  // Those with the smaller reference come over with it, whose share is 1.
  __device__ __forceinline__ void add(Sums o, float c) {
    const bool mine = m >= o.m;
    const float top = mine ? m : o.m, low = mine ? o.m : m;
    const float d = top == low ? 0.f : half_apart(low, top) * (2.f * c), f = low == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(d);
    const float t = (low == -INFINITY ? 0.f : 1.f) + (mine ? o.s : s);
    s = __builtin_fmaf(f, t, mine ? s : o.s);
    a = (mine ? a : o.a) + (f == 0.f ? 0.f : f * __builtin_fmaf(d, t, mine ? o.a : a));
    m = top;
  }
};

// A logit and its number as one whole number that grows with the logit and, among equal ones (zeros of either sign are equal), towards the lower number.  0: none.
typedef uint64_t Key;
__device__ __forceinline__ Key key_of(float x, int id) {
  const uint32_t u = __float_as_uint(x + 0.f), o = u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
  return static_cast<Key>(o) << 32 | ~static_cast<uint32_t>(id);
}
__device__ __forceinline__ float logit_of(Key k) {
  const uint32_t o = static_cast<uint32_t>(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ int id_of(Key k) { return static_cast<int>(~static_cast<uint32_t>(k)); }
__device__ __forceinline__ Key of_lane(Key k, int lane) {
  return static_cast<Key>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(k >> 32), lane))) << 32 |
         static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(k), lane));
}

struct Params {
  LogprobArgs a;
  float c;                     // scale * log2 e
  int32_t parts, each;         // parts of a row, vectors of 16 bytes of a part
  float* msa;                  // [rows][parts][4]
  Key* lists;                  // [rows][parts][top]
};

// A sorted list over the lanes of a wavefront: lane 0 has the largest.
struct List {
  Key key = 0;
  __device__ __forceinline__ void insert(Key k) {        // (the same in all lanes)
    const bool before = key > k;
    const int at = __builtin_popcountll(__ballot(before)), lane = threadIdx.x & 63;
    const Key up = lane_before(key), other = lane == at ? k : up;
    key = before ? key : other;
  }
  // the best 64 of both, sorted
  __device__ __forceinline__ void merge(Key o) {
    const Key r = lane_reversed(o);
    key = key > r ? key : r;                             // a sequence that rises and falls, of the best 64
    steps<64, 32>();
  }
  template <int K = 2>
  __device__ __forceinline__ void sort() {
    steps<K, K / 2>();
    if constexpr (K < 64) sort<2 * K>();
  }

 private:
  // stretches of K lanes that rise and fall, or fall and rise, into order, every second one backwards
  template <int K, int O>
  __device__ __forceinline__ void steps() {
    const Key other = lane_xor<O>(key);
    const bool larger = ((threadIdx.x & O) == 0) == (K == 64 || (threadIdx.x & K) == 0);
    key = (key > other) == larger ? key : other;
    if constexpr (O > 1) steps<K, O / 2>();
  }
};

// (the same in all lanes)
template <int O = 32>
__device__ __forceinline__ float over_lanes_max(float x) {
  x = fmaxf(x, lane_xor<O>(x));
  if constexpr (O > 1) return over_lanes_max<O / 2>(x);
  else return __uint_as_float(__builtin_amdgcn_readfirstlane(static_cast<int>(__float_as_uint(x))));
}
template <int O = 32>
__device__ __forceinline__ float over_lanes_sum(float x) {
  x += lane_xor<O>(x);
  if constexpr (O > 1) return over_lanes_sum<O / 2>(x);
  else return x;
}

template <int DT>
__device__ __forceinline__ float logit(const void* p, int64_t i) { return Storage<DT>::load(p, i); }

constexpr int kLoads = 2, kAhead = 2;                    // 16-byte loads of a lane in a batch, batches on their way
constexpr int kFew = 8;                                  // what is put into a list one by one rather than sorted

// One wavefront's share of a row.  (m: the same in all its lanes, so that the one that stays out is the wavefront's.)
template <int DT, bool TOP>
struct Scan {
  static constexpr int V = DT == PILLAR_F32 ? 4 : 8, kBatch = kLoads * V;
  Sums sums;                   // m: the same in all lanes; s, a: of this lane
  float limit, room;           // what a logit has to exceed to become the reference; how far above that this is
  List list;
  float least;                 // the list's last of `top`
  Key least_key;
  float c;
  int top, lane;

  __device__ __forceinline__ Scan(float c_, int top_) : sums{-INFINITY, 0.f, 0.f}, limit(-INFINITY), room(fminf(kRoom / c_, 1e37f)), least(-INFINITY), least_key(0), c(c_), top(top_), lane(threadIdx.x & 63) {}

  // What of N logits of every lane gets into the list.  Each lane brings its best (`most`), then its next best as long as some get in: one by one where
  // they are few, else sorted and merged at once.
  template <int N, typename Id>
  __device__ __forceinline__ void enter(float (&x)[N], Id id, float most) {
    while (true) {
      int at = 0;
#pragma unroll
      for (int i = N - 1; i > 0; --i) at = x[i] == most ? i : at;
      if (x[0] == most) at = 0;
      const Key mine = most >= least && most > -INFINITY ? key_of(most, id(at)) : 0;
      uint64_t some = __ballot(mine > least_key);
      if (!some) return;                                 // (a logit equal to the list's last gets in where its number is lower)
      if (__builtin_popcountll(some) > kFew) {
        List sorted;
        sorted.key = mine;
        sorted.sort();
        list.merge(sorted.key);
        least_key = of_lane(list.key, top - 1);
      } else {
        while (some) {
          const int from = __builtin_ctzll(some);
          list.insert(of_lane(mine, from));
          least_key = of_lane(list.key, top - 1);
          some &= some - 1;
          some &= __ballot(mine > least_key);
        }
      }
      least = least_key ? logit_of(least_key) : -INFINITY;
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = i == at ? -INFINITY : x[i];
      most = x[0];
#pragma unroll
      for (int i = 1; i < N; ++i) most = fmaxf(most, x[i]);
    }
  }

  // logits into the sums
  template <int N>
  __device__ __forceinline__ void weigh(const float (&x)[N]) {
    const float m = sums.m == -INFINITY ? 0.f : sums.m;
    float s[2] = {0.f, 0.f}, a[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = half_apart(x[i], m) * (2.f * c), e = __builtin_amdgcn_exp2f(y);
      s[i & 1] += e;
      a[i & 1] = __builtin_fmaf(e, fmaxf(y, -200.f), a[i & 1]);          // (-inf: 0 * -200)
    }
    sums.s += s[0] + s[1];
    sums.a += a[0] + a[1];
  }

  // N logits of every lane, -inf where there is none; id(i): the number of a lane's i-th.  LATER: all of them higher than those before.
  template <bool LATER, int N, typename Id>
  __device__ __forceinline__ void take(float (&x)[N], Id id) {
    float most = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) most = fmaxf(most, x[i]);
    // A logit far enough above the reference becomes it (rare after a few batches): it stays out of the sums, and the one before goes into them, in lane 0.
    if (__any(most > limit)) {
      const float to = over_lanes_max(most), d = half_apart(sums.m, to) * (2.f * c), f = sums.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(d);
      const float t = sums.s + (lane == 0 && f > 0.f ? 1.f : 0.f);
      sums.a = f == 0.f ? 0.f : f * __builtin_fmaf(d, t, sums.a);
      sums.s = f * t;
      sums.m = to;
      limit = to + room;
      const bool mine = lane == __builtin_ctzll(__ballot(most == to));
      float equal = mine ? -1.f : 0.f;                   // others of the lane that are as large
      float rest[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const bool same = mine && x[i] == to;
        rest[i] = same ? -INFINITY : x[i];
        equal += same ? 1.f : 0.f;
      }
      sums.s += equal;
      weigh(rest);
    } else {
      weigh(x);
    }
    if constexpr (TOP) {
      if (__any(LATER ? most > least : most >= least)) enter(x, id, most);
    }
  }

  static __device__ __forceinline__ void unpack(const u32x4 (&raw)[kLoads], float (&x)[kBatch]) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
#pragma unroll
      for (int j = 0; j < V; ++j)
        x[u * V + j] = DT == PILLAR_F32 ? __uint_as_float(raw[u][j & 3]) : __uint_as_float((j & 1) ? raw[u][(j >> 1) & 3] & 0xffff0000u : raw[u][(j >> 1) & 3] << 16);
  }

  // vectors v0 .. v1 - 1 of 16 bytes, kWaves wavefronts in turn; the first logit of vector 0 is number `first`.  kAhead batches are on their way.
  __device__ __forceinline__ void vectors(const u32x4* p, int v0, int v1, int first, int wave) {
    constexpr int kStep = 64 * kLoads, kNext = kWaves * kStep;
    int v = v0 + wave * kStep;
    if (v >= v1) return;
    u32x4 raw[kAhead][kLoads];
    auto fetch = [&](u32x4 (&to)[kLoads], int from) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) to[u] = __builtin_nontemporal_load(p + min(from + 64 * u + lane, v1 - 1));
    };
#pragma unroll
    for (int k = 0; k < kAhead; ++k) fetch(raw[k], v + k * kNext);
    while (true) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        float x[kBatch];
        unpack(raw[k], x);
        if (v + kAhead * kNext < v1) fetch(raw[k], v + kAhead * kNext);
        if (v + kStep > v1) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) x[i] = v + 64 * (i / V) + lane < v1 ? x[i] : -INFINITY;
        }
        take<true>(x, [&](int i) { return first + (v + 64 * (i / V) + lane) * V + i % V; });          // (V is a power of two)
        v += kNext;
        if (v >= v1) return;
      }
    }
  }
};

// What a row says, once its sums are known.
template <int DT>
struct Row {
  const LogprobArgs& a;
  int r;
  int64_t at;                  // its first element
  Sums sums;
  float log_s;                 // log(1 + R), in natural units
  bool nan, empty, endless;

  __device__ __forceinline__ Row(const LogprobArgs& a_, int r_) : a(a_), r(r_), at(r_ * a_.row_stride) {}
  // (all threads of a workgroup) m = -inf: nothing but -inf (and NaN); +inf: the sum may be NaN from inf - inf, and whether the row has NaN too has to be looked up
  __device__ __forceinline__ void settle(Sums s) {
    sums = s;
    log_s = log1pf(s.s);
    endless = s.m == INFINITY, empty = s.m == -INFINITY;
    nan = s.s != s.s;
    if (endless) {
      bool mine = false;
      for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
        const float x = logit<DT>(a.logits, at + i);
        mine |= x != x;
      }
      nan = __syncthreads_or(mine);
    }
  }
  __device__ __forceinline__ float log_prob(float x) const {
    if (nan) return NAN;
    if (empty) return -INFINITY;
    if (endless) return x < INFINITY ? -INFINITY : NAN;
    return __builtin_fmaf(half_apart(x, sums.m), 2.f * a.scale, -log_s);
  }
  // the j-th given token: its logit, or NaN where there is no such token
  __device__ __forceinline__ bool given(int j, float& x) const {
    const int id = a.tokens[static_cast<int64_t>(r) * a.num_tokens + j];
    const bool there = id >= 0 && id < a.vocab;
    x = there ? logit<DT>(a.logits, at + id) : 0.f;
    return there;
  }
  __device__ __forceinline__ void put(int j, bool there, float x) const {
    a.logprobs[static_cast<int64_t>(r) * a.num_tokens + j] = there ? log_prob(x) : -INFINITY;
  }
  __device__ __forceinline__ void put_sums() const {
    if (a.lse) a.lse[r] = nan ? NAN : empty ? -INFINITY : endless ? INFINITY : __builtin_fmaf(a.scale, sums.m, log_s);
    if (a.entropy) a.entropy[r] = nan || endless ? NAN : empty ? 0.f : log_s - kLn2 * (sums.a / (1.f + sums.s));        // (a sum: A is not positive)
  }
  // (one wavefront) Fewer numbers above -inf than wanted: the first of -inf, then the first that are none at all.
  __device__ __forceinline__ void put_list(List list) const {
    const int lane = threadIdx.x & 63;
    float x = logit_of(list.key);
    int id = id_of(list.key), have = __builtin_popcountll(__ballot(list.key != 0));
    for (int none = 0; none < 2 && have < a.top; ++none)
      for (int i0 = 0; i0 < a.vocab && have < a.top; i0 += 64) {
        const float y = i0 + lane < a.vocab ? logit<DT>(a.logits, at + i0 + lane) : 0.f;
        for (uint64_t some = __ballot(none ? y != y : y == -INFINITY); some && have < a.top; some &= some - 1, ++have) {
          if (lane == have) { x = none ? NAN : -INFINITY; id = i0 + __builtin_ctzll(some); }
        }
      }
    if (lane < a.top) {
      const int64_t to = static_cast<int64_t>(r) * a.top + lane;
      a.top_ids[to] = lane < have ? id : -1;
      a.top_logprobs[to] = lane < have ? log_prob(x) : -INFINITY;
    }
  }
};

// The lists of a workgroup's wavefronts into the first one's.
__device__ __forceinline__ void merge_lists(List& list, Key (&s_key)[kWaves][64], int wave, int lane) {
  s_key[wave][lane] = list.key;
#pragma unroll
  for (int half = kWaves / 2; half > 0; half >>= 1) {
    __syncthreads();
    if (wave < half) {
      list.merge(s_key[wave + half][lane]);
      s_key[wave][lane] = list.key;
    }
  }
}

template <int O = 32>
__device__ __forceinline__ Sums over_lanes(Sums s, float c) {
  s.add(Sums{lane_xor<O>(s.m), lane_xor<O>(s.s), lane_xor<O>(s.a)}, c);
  if constexpr (O > 1) return over_lanes<O / 2>(s, c);
  else return s;
}

// TOP: a list is wanted.  Rows of one part are done here.
template <int DT, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_pass(Params p) {
  using S = Scan<DT, TOP>;
  constexpr int V = S::V, kSize = DT == PILLAR_F32 ? 4 : 2;
  __shared__ Sums s_sums[kWaves];
  __shared__ Key s_key[kWaves][64];
  const LogprobArgs& a = p.a;
  const int r = blockIdx.x / p.parts, part = blockIdx.x - r * p.parts, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Row<DT> row(a, r);
  float given = 0.f;
  bool is_given = false;
  if (p.parts == 1 && tid < a.num_tokens) is_given = row.given(tid, given);                  // (on its way beside the row)
  // the row up to the first multiple of 16 bytes, vectors of 16 bytes, the rest
  const char* const base = static_cast<const char*>(a.logits) + row.at * kSize;
  const int head = min(a.vocab, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(base) & 15u)) & 15u) / kSize);
  const int whole = (a.vocab - head) / V, rest = a.vocab - head - whole * V;
  S scan(p.c, a.top);
  scan.vectors(reinterpret_cast<const u32x4*>(base + head * kSize), part * p.each, min(whole, (part + 1) * p.each), head, wave);
  if (part == 0 && wave == kWaves - 1) {                 // what is left of the row at both ends, less than 16 logits
    const int id = lane < head ? lane : a.vocab - rest + lane - head;
    float x[1] = {lane < head + rest ? logit<DT>(a.logits, row.at + id) : -INFINITY};
    scan.template take<false>(x, [&](int) { return id; });
  }
  const Sums sums{scan.sums.m, over_lanes_sum(scan.sums.s), over_lanes_sum(scan.sums.a)};
  if (lane == 0) s_sums[wave] = sums;
  List list = scan.list;
  if (TOP) merge_lists(list, s_key, wave, lane);
  else __syncthreads();
  Sums all = s_sums[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) all.add(s_sums[w], p.c);
  if (p.parts > 1) {
    const int64_t slot = static_cast<int64_t>(r) * p.parts + part;
    if (tid == 0) *reinterpret_cast<f32x4_t*>(p.msa + 4 * slot) = f32x4_t{all.m, all.s, all.a, 0.f};
    if (TOP && wave == 0 && lane < a.top) p.lists[slot * a.top + lane] = list.key;
    return;
  }
  row.settle(all);
  if (tid == 0) row.put_sums();
  if (tid < a.num_tokens) row.put(tid, is_given, given);
  for (int j = tid + kThreads; j < a.num_tokens; j += kThreads) {
    is_given = row.given(j, given);
    row.put(j, is_given, given);
  }
  if (TOP && wave == 0) row.put_list(list);
}

template <int DT, bool TOP>
__global__ __launch_bounds__(kThreads) void logprob_join(Params p) {
  __shared__ Sums s_sums[kWaves];
  __shared__ Key s_key[kWaves][64];
  const LogprobArgs& a = p.a;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t slot = static_cast<int64_t>(r) * p.parts;
  Row<DT> row(a, r);
  float given = 0.f;
  bool is_given = false;
  if (tid < a.num_tokens) is_given = row.given(tid, given);
  Sums sums{-INFINITY, 0.f, 0.f};
  for (int i = tid; i < p.parts; i += kThreads) {
    const f32x4_t v = *reinterpret_cast<const f32x4_t*>(p.msa + 4 * (slot + i));
    sums.add(Sums{v[0], v[1], v[2]}, p.c);
  }
  sums = over_lanes(sums, p.c);
  if (lane == 0) s_sums[wave] = sums;
  List list;
  if (TOP) {
    constexpr int kLists = 8;                            // lists on their way at once
    for (int i = wave; i < p.parts; i += kLists * kWaves) {
      Key v[kLists];
#pragma unroll
      for (int k = 0; k < kLists; ++k) {
        v[k] = 0;
        if (i + k * kWaves < p.parts && lane < a.top) v[k] = p.lists[(slot + i + k * kWaves) * a.top + lane];
      }
#pragma unroll 1
      for (int k = 0; k < kLists && i + k * kWaves < p.parts; ++k) {     // (one copy of the code)
        list.merge(v[0]);
#pragma unroll
        for (int l = 0; l + 1 < kLists; ++l) v[l] = v[l + 1];
      }
    }
    merge_lists(list, s_key, wave, lane);
  } else {
    __syncthreads();
  }
  sums = s_sums[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) sums.add(s_sums[w], p.c);
  row.settle(sums);
  if (tid == 0) row.put_sums();
  if (tid < a.num_tokens) row.put(tid, is_given, given);
  for (int j = tid + kThreads; j < a.num_tokens; j += kThreads) {
    is_given = row.given(j, given);
    row.put(j, is_given, given);
  }
  if (TOP && wave == 0) row.put_list(list);
}

struct Plan {
  int parts, each;
};
// Two workgroups to a compute unit, in parts of 4096 bf16 or 2048 fp32 logits at the least: shorter parts are more lists to join, longer ones take longer.  One row of
// 150000 bf16 logits with eight alternatives, parts of 2048 / 4096 / 8192 / 16384: 16.4 / 13.5 / 13.5 / 15.2 us, of 32000 12.1 / 12.4 / 13.2 / 14.3.
int64_t wanted_workgroups() { return 2 * static_cast<int64_t>(num_cus()); }
Plan plan_of(int rows, int vocab, int dtype) {
  const int per = dtype == PILLAR_F32 ? 4 : 8, vectors = vocab / per;
  const int64_t wanted = (wanted_workgroups() + rows - 1) / std::max(rows, 1);
  const int most = (vectors + 511) / 512;
  Plan p;
  p.parts = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(wanted, most)));
  p.each = std::max(1, (vectors + p.parts - 1) / p.parts);
  p.parts = std::max(1, (vectors + p.each - 1) / p.each);
  return p;
}

template <int DT, bool TOP>
hipError_t launch(const Params& p, hipStream_t s) {
  {
    KernelTimer timer("logprob_pass", s);
    hipLaunchKernelGGL((logprob_pass<DT, TOP>), dim3(static_cast<unsigned>(p.parts) * p.a.rows), dim3(kThreads), 0, s, p);
  }
  if (p.parts == 1) return hipGetLastError();
  KernelTimer timer("logprob_join", s);
  hipLaunchKernelGGL((logprob_join<DT, TOP>), dim3(p.a.rows), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace

// Whatever the type, and enough for any smaller call: r rows have at most r * most parts, and fewer than the wanted workgroups and one more for each row; as many
// rows as workgroups are wanted have one part each, which leaves nothing.
size_t logprobs_workspace(int rows, int vocab, int top) {
  const int64_t most = (vocab / 4 + 511) / 512, few = std::min<int64_t>(rows, wanted_workgroups() - 1);
  const size_t slots = most > 1 ? std::min(few * most, wanted_workgroups() + few - 1) : 0;
  return align_up(slots * 16, 256) + slots * top * 8;
}

hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t s) {
  const Plan plan = plan_of(a.rows, a.vocab, a.dtype);
  Params p;
  p.a = a;
  p.c = static_cast<float>(static_cast<double>(a.scale) * 1.4426950408889634);
  p.parts = plan.parts;
  p.each = plan.each;
  p.msa = static_cast<float*>(a.workspace);
  p.lists = reinterpret_cast<Key*>(static_cast<char*>(a.workspace) + align_up(static_cast<size_t>(a.rows) * plan.parts * 16, 256));
  if (a.dtype == PILLAR_F32) return a.top ? launch<PILLAR_F32, true>(p, s) : launch<PILLAR_F32, false>(p, s);
  return a.top ? launch<PILLAR_BF16, true>(p, s) : launch<PILLAR_BF16, false>(p, s);
}

}  // namespace pillar

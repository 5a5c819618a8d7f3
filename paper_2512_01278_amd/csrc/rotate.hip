// Rotary positions of rows, and the write of new tokens into the paged cache with the rotation on the way.
//
//   rotate_rows    heads of given rows (pillar_rotate), queries of an append into an fp8 cache
//   append_rows    queries, keys and values of new tokens, into a bf16 or fp32 cache: every element is read once and written once
//   append_pages   keys and values of new tokens into an fp8 cache, by (page, KV head), because a page's scale is that of all its rows
#include <algorithm>

#include "launch.hpp"
#include "page_scale.hpp"
#include "rope.hpp"

namespace pillar {
namespace {

constexpr int kThreads = 256;
constexpr int kMostHalf = 256;                           // pairs of a head of 512
constexpr float kLeastMax = 0x1p-90f;                    // rows of nothing larger count as zeros: 1 / scale stays finite

// Request and number of a packed row; false: no such row.  (Every wavefront for itself: 64 ends at a time.)
struct Row {
  int b, n, i, len;            // its request, that request's new rows, the row among them, tokens in the cache
  __device__ __forceinline__ bool find(const AppendArgs& a, int t) {
    if (!a.starts) {
      b = t / a.max_new;
      n = a.max_new;
      i = t - b * n;
    } else {
      const int lane = threadIdx.x & 63;
      b = 0;
      for (int c = 0; c < a.kv.batch; c += 64) {
        const uint64_t over = __ballot(c + lane < a.kv.batch && a.starts[c + lane + 1] <= t);
        b += __builtin_popcountll(over);
        if (over != ~0ull) break;
      }
      if (b >= a.kv.batch) return false;
      const int first = a.starts[b];
      n = a.starts[b + 1] - first;
      i = t - first;
      if (i < 0) return false;
    }
    len = min(a.kv.seq_lens[b], a.kv.max_seq_len);
    return true;
  }
  __device__ __forceinline__ int token() const { return len - n + i; }
};

template <int DT, int V>
__global__ __launch_bounds__(kThreads) void rotate_rows(RotateArgs a) {
  __shared__ float2 s_turn[kMostHalf];
  const int t = blockIdx.x, tid = threadIdx.x;
  const int position = a.positions[t];
  for (int i = tid; i < a.rope.half; i += kThreads) s_turn[i] = turned(position, a.rope.frequencies[i], a.rope.amplitude);
  __syncthreads();
  const int pieces = pieces_of_head<V>(a.rope, a.head_dim);
  const int64_t from = t * a.x_stride, to = t * a.out_stride;
  for (int e = tid; e < a.heads * pieces; e += kThreads) {
    const int h = e / pieces;
    const Piece p = piece_of<V>(a.rope, e - h * pieces);
    const int64_t head = static_cast<int64_t>(h) * a.head_dim;
    float x[V], y[V];
    load_elems<DT, V>(a.x, from + head + p.lo, x);
    if (p.hi >= 0) load_elems<DT, V>(a.x, from + head + p.hi, y);
    turn_piece<V>(p, x, y, [&](int j) { return s_turn[p.pair + j]; });
    store_elems<DT, V>(a.out, to + head + p.lo, x);
    if (p.hi >= 0) store_elems<DT, V>(a.out, to + head + p.hi, y);
  }
}

// KV < 0: queries alone (the cache is written by another kernel)
template <int DT, int KV, int V>
__global__ __launch_bounds__(kThreads) void append_rows(AppendArgs a) {
  __shared__ float2 s_turn[kMostHalf];
  const int t = blockIdx.x, tid = threadIdx.x, D = a.kv.head_dim;
  Row row;
  if (!row.find(a, t)) return;
  const int token = row.token();
  const int position = a.positions ? a.positions[t] : token;
  for (int i = tid; i < a.rope.half; i += kThreads) s_turn[i] = turned(position, a.rope.frequencies[i], a.rope.amplitude);
  __syncthreads();
  const int pieces = pieces_of_head<V>(a.rope, D);
  auto head = [&](const void* src, int64_t from, int c, auto store) {
    const Piece p = piece_of<V>(a.rope, c);
    float x[V], y[V];
    load_elems<DT, V>(src, from + p.lo, x);
    if (p.hi >= 0) load_elems<DT, V>(src, from + p.hi, y);
    turn_piece<V>(p, x, y, [&](int j) { return s_turn[p.pair + j]; });
    store(p.lo, x);
    if (p.hi >= 0) store(p.hi, y);
  };
  if (a.q)
    for (int e = tid; e < a.kv.num_q_heads * pieces; e += kThreads) {
      const int h = e / pieces;
      const int64_t to = (static_cast<int64_t>(t) * a.kv.num_q_heads + h) * D;
      head(a.q, t * a.q_stride + static_cast<int64_t>(h) * D, e - h * pieces, [&](int dim, const float (&x)[V]) { store_elems<DT, V>(a.q_out, to + dim, x); });
    }
  if constexpr (KV >= 0) {
    if (token < 0) return;
    int page;
    for (int e = tid; e < a.kv.num_kv_heads * pieces; e += kThreads) {
      const int g = e / pieces;
      const int64_t to = row_offset(a.kv, row.b, g, token, &page);
      head(a.k_new, t * a.k_stride + static_cast<int64_t>(g) * D, e - g * pieces,
           [&](int dim, const float (&x)[V]) { store_elems<KV, V>(const_cast<void*>(a.kv.k_pool), to + dim, x); });
    }
    for (int e = tid; e < a.kv.num_kv_heads * (D / V); e += kThreads) {
      const int g = e / (D / V), dim = (e - g * (D / V)) * V;
      float x[V];
      load_elems<DT, V>(a.v_new, t * a.v_stride + static_cast<int64_t>(g) * D + dim, x);
      store_elems<KV, V>(const_cast<void*>(a.kv.v_pool), row_offset(a.kv, row.b, g, token, &page) + dim, x);
    }
  }
}

__device__ __forceinline__ float finite_magnitude(float x) {
  const float m = fabsf(x);
  return m < INFINITY ? m : 0.f;                         // (NaN too)
}
// one code: nearest, infinities to the largest; NaN stays
__device__ __forceinline__ uint8_t code_of(float x) {
  const float y = fabsf(x) > 448.f ? copysignf(448.f, x) : x;
  return static_cast<uint8_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y, y, 0, false));
}

// One workgroup per (page of a request that receives rows, KV head): the largest value among the new rows, the page's scale from it, the codes.
template <int DT, int V>
__global__ __launch_bounds__(kThreads) void append_pages(AppendArgs a, int pages_each) {
  __shared__ float s_max[2][kThreads / 64];
  const int b = blockIdx.x / pages_each, nth = blockIdx.x - b * pages_each, g = blockIdx.y, tid = threadIdx.x;
  const KvView& kv = a.kv;
  const int D = kv.head_dim;
  const int first = a.starts ? a.starts[b] : b * a.max_new, n = a.starts ? a.starts[b + 1] - first : a.max_new;
  const int len = min(kv.seq_lens[b], kv.max_seq_len), begin = max(0, len - n);              // new tokens begin .. len - 1
  const int index = (begin >> kv.page_shift) + nth, page0 = index << kv.page_shift;
  const int t0 = max(begin, page0), t1 = min(len, page0 + kv.page_size);                     // those in this page
  if (t0 >= t1) return;
  const int page = kv.block_table[static_cast<int64_t>(b) * kv.block_table_stride + index];
  const int64_t at_scale = static_cast<int64_t>(page) * kv.num_kv_heads + g;
  const int64_t head = static_cast<int64_t>(page) * kv.stride_page + static_cast<int64_t>(g) * kv.stride_head;
  const int older = t0 - page0;                                                              // tokens of the page that were there
  const int row0 = first + n - len;                                                          // packed row of token t: row0 + t
  const int pieces = pieces_of_head<V>(a.rope, D);
  auto each_k = [&](auto use) {
    for (int e = tid; e < (t1 - t0) * pieces; e += kThreads) {
      const int i = e / pieces, t = t0 + i;
      const int64_t r = row0 + t;
      const Piece p = piece_of<V>(a.rope, e - i * pieces);
      const int64_t from = r * a.k_stride + static_cast<int64_t>(g) * D;
      float x[V], y[V];
      load_elems<DT, V>(a.k_new, from + p.lo, x);
      if (p.hi >= 0) load_elems<DT, V>(a.k_new, from + p.hi, y);
      if (p.pair >= 0) {
        const int position = a.positions ? a.positions[r] : t;
        turn_piece<V>(p, x, y, [&](int j) { return turned(position, a.rope.frequencies[p.pair + j], a.rope.amplitude); });
      }
      use(t, p.lo, x);
      if (p.hi >= 0) use(t, p.hi, y);
    }
  };
  auto each_v = [&](auto use) {
    for (int e = tid; e < (t1 - t0) * (D / V); e += kThreads) {
      const int i = e / (D / V), dim = (e - i * (D / V)) * V, t = t0 + i;
      float x[V];
      load_elems<DT, V>(a.v_new, (row0 + static_cast<int64_t>(t)) * a.v_stride + static_cast<int64_t>(g) * D + dim, x);
      use(t, dim, x);
    }
  };
  float top[2] = {0.f, 0.f};
  each_k([&](int, int, const float (&x)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) top[0] = fmaxf(top[0], finite_magnitude(x[j]));
  });
  each_v([&](int, int, const float (&x)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) top[1] = fmaxf(top[1], finite_magnitude(x[j]));
  });
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    top[w] = wave_max(top[w]);
    if ((tid & 63) == 0) s_max[w][tid >> 6] = top[w];
  }
  const float had[2] = {kv.k_scale[at_scale], kv.v_scale[at_scale]};
  __syncthreads();                                       // (the old scales have been read by everybody, too)
  float now[2], inv[2];
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) most = fmaxf(most, s_max[w][i]);
    const float fresh = most < kLeastMax ? 0.f : most / 448.f;
    now[w] = older > 0 ? fmaxf(had[w], fresh) : fresh;
    inv[w] = now[w] > 0.f ? 1.f / now[w] : 0.f;
  }
  if (tid == 0) {
    const_cast<float*>(kv.k_scale)[at_scale] = now[0];
    const_cast<float*>(kv.v_scale)[at_scale] = now[1];
  }
  uint8_t* const pools[2] = {static_cast<uint8_t*>(const_cast<void*>(kv.k_pool)) + head, static_cast<uint8_t*>(const_cast<void*>(kv.v_pool)) + head};
  const int chunks = D / 16;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const float ratio = scale_ratio(had[w], now[w]);
    if (ratio == 1.f) continue;
    for (int e = tid; e < older * chunks; e += kThreads) {
      const int i = e / chunks;
      u32x4* const c = reinterpret_cast<u32x4*>(pools[w] + i * kv.stride_slot + 16 * (e - i * chunks));
      *c = rescale_codes(*c, ratio);
    }
  }
  auto put = [&](int w, int t, int dim, const float (&x)[V]) {
    uint8_t* const to = pools[w] + static_cast<int64_t>(t - page0) * kv.stride_slot + dim;
#pragma unroll
    for (int j = 0; j < V; ++j) to[j] = code_of(x[j] * inv[w]);
  };
  each_k([&](int t, int dim, const float (&x)[V]) { put(0, t, dim, x); });
  each_v([&](int t, int dim, const float (&x)[V]) { put(1, t, dim, x); });
}

template <int DT, int V>
hipError_t rotate(const RotateArgs& a, hipStream_t s) {
  KernelTimer timer("rotate_rows", s);
  hipLaunchKernelGGL((rotate_rows<DT, V>), dim3(a.tokens), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <int DT, int V>
hipError_t append(const AppendArgs& a, hipStream_t s) {
  if (a.kv_dtype == PILLAR_FP8_E4M3) {
    if (a.q) {
      KernelTimer timer("append_rows", s);
      hipLaunchKernelGGL((append_rows<DT, -1, V>), dim3(a.total_rows), dim3(kThreads), 0, s, a);
    }
    KernelTimer timer("append_pages", s);
    const int64_t pages_each = (std::min<int64_t>(a.max_new, a.kv.max_seq_len) + 2 * a.kv.page_size - 2) / a.kv.page_size;      // n rows lie in that many pages at most
    hipLaunchKernelGGL((append_pages<DT, V>), dim3(static_cast<unsigned>(pages_each * a.kv.batch), a.kv.num_kv_heads), dim3(kThreads), 0, s, a, static_cast<int>(pages_each));
    return hipGetLastError();
  }
  KernelTimer timer("append_rows", s);
  if (a.kv_dtype == PILLAR_F32) hipLaunchKernelGGL((append_rows<DT, PILLAR_F32, V>), dim3(a.total_rows), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((append_rows<DT, PILLAR_BF16, V>), dim3(a.total_rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

bool multiple_of_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t s) {
  const int per = a.dtype == PILLAR_F32 ? 4 : 8;
  const bool pieces = rope_in_pieces(a.rope, a.head_dim, per) && multiple_of_16(a.x) && multiple_of_16(a.out) && a.x_stride % per == 0 && a.out_stride % per == 0;
  if (a.dtype == PILLAR_F32) return pieces ? rotate<PILLAR_F32, 4>(a, s) : rotate<PILLAR_F32, 1>(a, s);
  return pieces ? rotate<PILLAR_BF16, 8>(a, s) : rotate<PILLAR_BF16, 1>(a, s);
}

hipError_t launch_append_rotated(const AppendArgs& a, hipStream_t s) {
  const bool pieces = rope_in_pieces(a.rope, a.kv.head_dim, a.q_dtype == PILLAR_F32 ? 4 : 8);
  if (a.q_dtype == PILLAR_F32) return pieces ? append<PILLAR_F32, 4>(a, s) : append<PILLAR_F32, 1>(a, s);
  return pieces ? append<PILLAR_BF16, 8>(a, s) : append<PILLAR_BF16, 1>(a, s);
}

}  // namespace pillar

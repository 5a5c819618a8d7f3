// Rotary positions of rows, and the write of new tokens into the paged cache with the rotation on the way.
//
//   rotate_rows    heads of given rows (pillar_rotate)
//   append_rows    queries, keys and values of new tokens, into a bf16 or fp32 cache, a workgroup per row
//   append_pages   the same into an fp8 cache, keys and values by (page, KV head), because a page's scale is that of all its rows
//
// Bound by memory where there is much to move: every element is read once and written once, 32768 tokens of 32 heads (537 MB) in 108 us, 25 K tokens of 32 + 2 x 8 heads
// with keys and values into their pages (638 MB) in 132 us, 5.0 and 4.8 TB/s: nine tenths of what copies of as many bytes run at (98 and 119 us).  Turns are worked out
// once per row, into LDS, for all its heads.
// Where there is little, by the launch: one token 4.7 us, of which the chain starts, lengths, page id, rows is the most.
#include <algorithm>
#include <type_traits>

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
  for (HeadPiece at(pieces, kThreads); at.h < a.heads; at.next()) {
    const Piece p = piece_of<V>(a.rope, at.c);
    const int64_t head = static_cast<int64_t>(at.h) * a.head_dim;
    float x[V], y[V] = {};
    load_elems<DT, V>(a.x, from + head + p.lo, x);
    if (p.hi >= 0) load_elems<DT, V>(a.x, from + head + p.hi, y);
    turn_piece<V>(p, x, y, [&](int j) { return s_turn[p.pair + j]; });
    store_elems<DT, V>(a.out, to + head + p.lo, x);
    if (p.hi >= 0) store_elems<DT, V>(a.out, to + head + p.hi, y);
  }
}

// a piece of a head on its way: store(dim, values)
template <int DT, int V, typename Store>
__device__ __forceinline__ void turn_and_store(const RopeView& rope, const void* src, int64_t from, int c, const float2* s_turn, Store store) {
  const Piece p = piece_of<V>(rope, c);
  float x[V], y[V] = {};
  load_elems<DT, V>(src, from + p.lo, x);
  if (p.hi >= 0) load_elems<DT, V>(src, from + p.hi, y);
  turn_piece<V>(p, x, y, [&](int j) { return s_turn[p.pair + j]; });
  store(p.lo, x);
  if (p.hi >= 0) store(p.hi, y);
}

// A row's place, and the turns of its position in LDS.  false: no such row
__device__ __forceinline__ bool begin_row(const AppendArgs& a, int t, Row& row, float2* s_turn) {
  if (!row.find(a, t)) return false;
  const int position = a.positions ? a.positions[t] : row.token();
  for (int i = threadIdx.x; i < a.rope.half; i += kThreads) s_turn[i] = turned(position, a.rope.frequencies[i], a.rope.amplitude);
  __syncthreads();
  return true;
}

template <int DT, int V>
__device__ __forceinline__ void turn_queries(const AppendArgs& a, int t, const float2* s_turn) {
  const int D = a.kv.head_dim, pieces = pieces_of_head<V>(a.rope, D);
  for (HeadPiece at(pieces, kThreads); at.h < a.kv.num_q_heads; at.next()) {
    const int64_t to = (static_cast<int64_t>(t) * a.kv.num_q_heads + at.h) * D;
    turn_and_store<DT, V>(a.rope, a.q, t * a.q_stride + static_cast<int64_t>(at.h) * D, at.c, s_turn,
                          [&](int dim, const float (&x)[V]) { store_elems<DT, V>(a.q_out, to + dim, x); });
  }
}
template <int DT, int V>
__device__ __forceinline__ void queries(const AppendArgs& a, int t, float2* s_turn) {
  Row row;
  if (begin_row(a, t, row, s_turn)) turn_queries<DT, V>(a, t, s_turn);
}

template <int DT, int KV, int V>
__global__ __launch_bounds__(kThreads) void append_rows(AppendArgs a) {
  __shared__ float2 s_turn[kMostHalf];
  const int t = blockIdx.x, tid = threadIdx.x, D = a.kv.head_dim;
  Row row;
  if (!begin_row(a, t, row, s_turn)) return;
  const int pieces = pieces_of_head<V>(a.rope, D), token = row.token();
  if (a.q) turn_queries<DT, V>(a, t, s_turn);
  if (token < 0) return;
  int page;
  for (HeadPiece at(pieces, kThreads); at.h < a.kv.num_kv_heads; at.next()) {
    const int64_t to = row_offset(a.kv, row.b, at.h, token, &page);
    turn_and_store<DT, V>(a.rope, a.k_new, t * a.k_stride + static_cast<int64_t>(at.h) * D, at.c, s_turn,
                          [&](int dim, const float (&x)[V]) { store_elems<KV, V>(const_cast<void*>(a.kv.k_pool), to + dim, x); });
  }
  constexpr int W = DT == PILLAR_F32 ? 4 : 8;            // (values are not turned: in 16 bytes whatever V is)
  for (HeadPiece at(D / W, kThreads); at.h < a.kv.num_kv_heads; at.next()) {
    float x[W];
    load_elems<DT, W>(a.v_new, t * a.v_stride + static_cast<int64_t>(at.h) * D + at.c * W, x);
    store_elems<KV, W>(const_cast<void*>(a.kv.v_pool), row_offset(a.kv, row.b, at.h, token, &page) + at.c * W, x);
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

// The n-th page that receives rows, of the launch: its request, and which of the pages that hold the request's new rows it is.  (Every wavefront for itself: 64
// requests at a time, a request per lane.)
struct PageOf {
  int b, nth;
  __device__ __forceinline__ bool find(const AppendArgs& a, int unit, int pages_each) {
    if (!a.starts) {
      b = unit / pages_each;
      nth = unit - b * pages_each;
      return true;
    }
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int c = 0; c < a.kv.batch; c += 64) {
      int mine = 0;
      if (c + lane < a.kv.batch) {
        const int n = a.starts[c + lane + 1] - a.starts[c + lane], len = min(a.kv.seq_lens[c + lane], a.kv.max_seq_len), begin = max(0, len - n);
        if (n > 0 && len > 0) mine = ((len - 1) >> a.kv.page_shift) - (begin >> a.kv.page_shift) + 1;
      }
      const int upto = before + wave_inclusive(mine);
      const uint64_t after = __ballot(upto > unit);
      if (after) {
        const int at = __builtin_ctzll(after);
        b = __builtin_amdgcn_readfirstlane(c + at);
        nth = __builtin_amdgcn_readfirstlane(unit - __builtin_amdgcn_readlane(upto - mine, at));
        return true;
      }
      before = __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
  }
};

// V codes, one behind the other
template <int V>
__device__ __forceinline__ void store_codes(uint8_t* to, const float (&x)[V], float inv) {
  if constexpr (V < 4) {
#pragma unroll
    for (int j = 0; j < V; ++j) to[j] = code_of(x[j] * inv);
  } else {
    uint32_t w[V / 4];
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      float y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float v = x[j + k] * inv;
        y[k] = fabsf(v) > 448.f ? copysignf(448.f, v) : v;
      }
      const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      w[j / 4] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true));
    }
    if constexpr (V == 8) *reinterpret_cast<u32x2*>(to) = u32x2{w[0], w[1]};
    else *reinterpret_cast<uint32_t*>(to) = w[0];
  }
}

// A workgroup per (page that receives rows, KV head): the largest value among the new rows, the page's scale from it, the codes.  Rows whose pieces are
// at hand in one turn of the workgroup (pages of up to 16 tokens) stay in registers between the two; of larger pages they are read and turned again,
// from the caches.  Behind those workgroups, one per row for the queries.
template <int DT, int V>
__global__ __launch_bounds__(kThreads) void append_pages(AppendArgs a, int pages_each, int pages) {
  __shared__ float s_max[2][kThreads / 64];
  __shared__ float2 s_turn[kMostHalf];
  const int tid = threadIdx.x;
  const KvView& kv = a.kv;
  const int D = kv.head_dim;
  if (static_cast<int>(blockIdx.x) >= pages * kv.num_kv_heads) {
    queries<DT, V>(a, blockIdx.x - pages * kv.num_kv_heads, s_turn);
    return;
  }
  const int unit = blockIdx.x / kv.num_kv_heads, g = blockIdx.x - unit * kv.num_kv_heads;
  PageOf of;
  if (!of.find(a, unit, pages_each)) return;
  const int b = of.b;
  const int first = a.starts ? a.starts[b] : b * a.max_new, n = a.starts ? a.starts[b + 1] - first : a.max_new;
  const int len = min(kv.seq_lens[b], kv.max_seq_len), begin = max(0, len - n);              // new tokens begin .. len - 1
  const int index = (begin >> kv.page_shift) + of.nth, page0 = index << kv.page_shift;
  const int t0 = max(begin, page0), t1 = min(len, page0 + kv.page_size);                     // those in this page
  if (t0 >= t1) return;
  const int page = kv.block_table[static_cast<int64_t>(b) * kv.block_table_stride + index];
  const int64_t at_scale = static_cast<int64_t>(page) * kv.num_kv_heads + g;
  const int64_t head = static_cast<int64_t>(page) * kv.stride_page + static_cast<int64_t>(g) * kv.stride_head;
  const int older = t0 - page0;                                                              // tokens of the page that were there
  const int row0 = first + n - len;                                                          // packed row of token t: row0 + t
  const int pieces = pieces_of_head<V>(a.rope, D), chunks = D / V;
  const int k_items = (t1 - t0) * pieces, v_items = (t1 - t0) * chunks;

  // piece e of K's new rows, turned; chunk e of V's
  auto take_k = [&](int e, int& t, Piece& p, float (&x)[V], float (&y)[V]) {
    const int i = e / pieces;
    t = t0 + i;
    p = piece_of<V>(a.rope, e - i * pieces);
    const int64_t r = row0 + t, from = r * a.k_stride + static_cast<int64_t>(g) * D;
    load_elems<DT, V>(a.k_new, from + p.lo, x);
    if (p.hi >= 0) load_elems<DT, V>(a.k_new, from + p.hi, y);
    if (p.pair >= 0) {
      const int position = a.positions ? a.positions[r] : t;
      turn_piece<V>(p, x, y, [&](int j) { return turned(position, a.rope.frequencies[p.pair + j], a.rope.amplitude); });
    }
  };
  auto take_v = [&](int e, int& t, int& dim, float (&x)[V]) {
    const int i = e / chunks;
    t = t0 + i;
    dim = (e - i * chunks) * V;
    load_elems<DT, V>(a.v_new, (row0 + static_cast<int64_t>(t)) * a.v_stride + static_cast<int64_t>(g) * D + dim, x);
  };
  auto largest = [](float top, const float (&x)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) top = fmaxf(top, finite_magnitude(x[j]));
    return top;
  };

  const bool at_hand = k_items <= kThreads && v_items <= kThreads;
  float top[2] = {0.f, 0.f};
  float kx[V] = {}, ky[V] = {}, vx[V] = {};
  Piece kp{0, -1, -1};
  int kt = t0, vt = t0, vdim = 0;
  if (at_hand) {
    if (tid < v_items) take_v(tid, vt, vdim, vx);
    if (tid < k_items) take_k(tid, kt, kp, kx, ky);
    top[0] = largest(largest(0.f, kx), ky);
    top[1] = largest(0.f, vx);
  } else {
    for (int e = tid; e < k_items; e += kThreads) {
      float x[V] = {}, y[V] = {};
      take_k(e, kt, kp, x, y);
      top[0] = largest(largest(top[0], x), y);
    }
    for (int e = tid; e < v_items; e += kThreads) {
      float x[V];
      take_v(e, vt, vdim, x);
      top[1] = largest(top[1], x);
    }
  }
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
    inv[w] = now[w] < kLeastMax / 448.f ? 0.f : 1.f / now[w];            // (older tokens next to nothing: the new ones, which are no larger, are zeros)
  }
  if (tid == 0) {
    const_cast<float*>(kv.k_scale)[at_scale] = now[0];
    const_cast<float*>(kv.v_scale)[at_scale] = now[1];
  }
  uint8_t* const pools[2] = {static_cast<uint8_t*>(const_cast<void*>(kv.k_pool)) + head, static_cast<uint8_t*>(const_cast<void*>(kv.v_pool)) + head};
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    const float ratio = scale_ratio(had[w], now[w]);
    if (ratio == 1.f) continue;
    for (int e = tid; e < older * (D / 16); e += kThreads) {
      const int i = e / (D / 16);
      u32x4* const c = reinterpret_cast<u32x4*>(pools[w] + i * kv.stride_slot + 16 * (e - i * (D / 16)));
      *c = rescale_codes(*c, ratio);
    }
  }
  auto put = [&](int w, int t, int dim, const float (&x)[V]) { store_codes<V>(pools[w] + static_cast<int64_t>(t - page0) * kv.stride_slot + dim, x, inv[w]); };
  if (at_hand) {
    if (tid < k_items) {
      put(0, kt, kp.lo, kx);
      if (kp.hi >= 0) put(0, kt, kp.hi, ky);
    }
    if (tid < v_items) put(1, vt, vdim, vx);
    return;
  }
  for (int e = tid; e < k_items; e += kThreads) {
    float x[V] = {}, y[V] = {};
    take_k(e, kt, kp, x, y);
    put(0, kt, kp.lo, x);
    if (kp.hi >= 0) put(0, kt, kp.hi, y);
  }
  for (int e = tid; e < v_items; e += kThreads) {
    float x[V];
    take_v(e, vt, vdim, x);
    put(1, vt, vdim, x);
  }
}

// Pages that may receive rows: n rows lie in (n - 2) / page_size + 2 pages at most; all of them in no more than total_rows / page_size and two for each request.
struct Pages {
  int64_t each, all, workgroups;
};
Pages pages_of(const AppendArgs& a) {
  Pages p;
  p.each = (std::min<int64_t>(a.max_new, a.kv.max_seq_len) + 2 * a.kv.page_size - 2) / a.kv.page_size;
  p.all = p.each * a.kv.batch;
  if (a.starts) p.all = std::min<int64_t>(p.all, a.total_rows / a.kv.page_size + 2 * static_cast<int64_t>(a.kv.batch));
  p.workgroups = p.all * a.kv.num_kv_heads + (a.q ? a.total_rows : 0);
  return p;
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
    KernelTimer timer("append_pages", s);
    const Pages p = pages_of(a);
    hipLaunchKernelGGL((append_pages<DT, V>), dim3(static_cast<unsigned>(p.workgroups)), dim3(kThreads), 0, s, a, static_cast<int>(p.each), static_cast<int>(p.all));
    return hipGetLastError();
  }
  KernelTimer timer("append_rows", s);
  if (a.kv_dtype == PILLAR_F32) hipLaunchKernelGGL((append_rows<DT, PILLAR_F32, V>), dim3(a.total_rows), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((append_rows<DT, PILLAR_BF16, V>), dim3(a.total_rows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// calls f with the largest pieces that will do: 16 bytes, half of that, and so on
template <int DT, typename Will, typename F>
hipError_t by_piece(Will will, F f) {
  if constexpr (DT == PILLAR_BF16) {
    if (will(8)) return f(std::integral_constant<int, 8>());
  }
  if (will(4)) return f(std::integral_constant<int, 4>());
  if (will(2)) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}

template <int DT>
hipError_t rotate_as(const RotateArgs& a, hipStream_t s) {
  const int esz = DT == PILLAR_F32 ? 4 : 2;
  auto will = [&](int V) {
    return rope_in_pieces(a.rope, a.head_dim, V) && ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.out)) % (V * esz)) == 0 &&
           a.x_stride % V == 0 && a.out_stride % V == 0;
  };
  return by_piece<DT>(will, [&](auto V) { return rotate<DT, V.value>(a, s); });
}
template <int DT>
hipError_t append_as(const AppendArgs& a, hipStream_t s) {
  return by_piece<DT>([&](int V) { return rope_in_pieces(a.rope, a.kv.head_dim, V); }, [&](auto V) { return append<DT, V.value>(a, s); });
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, hipStream_t s) { return a.dtype == PILLAR_F32 ? rotate_as<PILLAR_F32>(a, s) : rotate_as<PILLAR_BF16>(a, s); }

bool append_fits_a_grid(const AppendArgs& a) { return (a.kv_dtype == PILLAR_FP8_E4M3 ? pages_of(a).workgroups : a.total_rows) <= kMostGroups; }

hipError_t launch_append_rotated(const AppendArgs& a, hipStream_t s) {
  return a.q_dtype == PILLAR_F32 ? append_as<PILLAR_F32>(a, s) : append_as<PILLAR_BF16>(a, s);
}

}  // namespace pillar

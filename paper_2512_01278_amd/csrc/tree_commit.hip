// The accepted path of a verified tree becomes the end of the context: rows first + path[i] of K, V and the statistic go to first + i
// (first: the token of node 0).
//
// One workgroup per (request, KV head) reads all rows of the path before it writes any, so a path may name nodes in any order and
// a row may be overwritten by one before it.  A path is at most 64 rows (32 KB of bf16 K and V): the kernel is a chain of four
// loads (lengths, path, page ids, rows) and as long as that.
#include "launch.hpp"
#include "page_scale.hpp"

namespace pillar {
namespace {

constexpr int kThreads = 256, kMaxPath = 64;

template <int KV>
__global__ __launch_bounds__(kThreads) void tree_commit(CommitArgs a) {
  constexpr int esz = KV == PILLAR_F32 ? 4 : KV == PILLAR_BF16 ? 2 : 1;
  constexpr int kCarry = kMaxPath * (128 * esz / 16) / kThreads;             // pieces of K, and of V, per thread at most
  __shared__ int s_path[kMaxPath];
  __shared__ float s_ks[kMaxPath], s_vs[kMaxPath], s_kr[kMaxPath], s_vr[kMaxPath];
  __shared__ float s_stay[2];
  const KvView& kv = a.kv;
  const int g = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int len = min(max(kv.seq_lens[b], 0), kv.max_seq_len);
  const int nodes = a.tree_sizes ? min(max(a.tree_sizes[b], 0), a.max_nodes) : a.max_nodes;
  const int first = len - nodes;
  // the path ends at its first entry that is no node
  const int node = lane < a.max_path ? a.path[static_cast<int64_t>(b) * a.max_path + lane] : -1;
  const bool fine = first >= 0 && lane < min(a.path_lens[b], a.max_path) && node >= 0 && node < nodes;
  const uint64_t bad = ~__ballot(fine);
  const int count = bad ? __builtin_ctzll(bad) : 64;
  if (g == 0 && tid == 0) a.new_lens[b] = max(first, 0) + count;
  if (count == 0) return;
  if (tid < kMaxPath) s_path[tid] = node;
  __syncthreads();

  // ---- read ----
  const RowPlace at(kv, b, g, esz);
  const int pieces = kv.head_dim * esz / 16, shift = __builtin_ctz(pieces);
  u32x4 k[kCarry], v[kCarry];
#pragma unroll
  for (int u = 0; u < kCarry; ++u) {
    const int e = tid + u * kThreads, i = e >> shift;
    if (i < count) {
      const int64_t from = at.at(first + s_path[i]) + 16 * (e & (pieces - 1));
      k[u] = *reinterpret_cast<const u32x4*>(at.k + from);
      v[u] = *reinterpret_cast<const u32x4*>(at.v + from);
    }
  }
  float* score = a.scores ? a.scores + (static_cast<int64_t>(b) * kv.num_kv_heads + g) * a.score_stride + first : nullptr;
  float moved_score = 0.f;
  if (score && tid < count) moved_score = score[s_path[tid]];
  if constexpr (KV == PILLAR_FP8_E4M3) {
    if (tid < count) {
      const int64_t sc = static_cast<int64_t>(at.page(first + s_path[tid])) * kv.num_kv_heads + g;
      s_ks[tid] = kv.k_scale[sc];
      s_vs[tid] = kv.v_scale[sc];
    }
  }
  __syncthreads();

  // ---- the pages' new scales: those of the rows that end up there, arriving and staying ----
  if constexpr (KV == PILLAR_FP8_E4M3) {
    int64_t scale_at = 0;
    float kn = 0.f, vn = 0.f;
    bool sets = false;
    if (tid < count) {
      const int t = first + tid, lo = max(first, t & ~at.mask) - first, hi = min(count, (t | at.mask) + 1 - first);
      scale_at = static_cast<int64_t>(at.page(t)) * kv.num_kv_heads + g;
      sets = tid == lo;                                  // the page's first arriving row
      kn = s_ks[lo];
      vn = s_vs[lo];
      for (int i = lo + 1; i < hi; ++i) {
        kn = fmaxf(kn, s_ks[i]);
        vn = fmaxf(vn, s_vs[i]);
      }
      if (lo == 0 && (first & at.mask) != 0) {           // the last rows before the tree are in this page
        const float ko = kv.k_scale[scale_at], vo = kv.v_scale[scale_at];
        kn = fmaxf(kn, ko);
        vn = fmaxf(vn, vo);
        if (tid == 0) {
          s_stay[0] = scale_ratio(ko, kn);
          s_stay[1] = scale_ratio(vo, vn);
        }
      }
      s_kr[tid] = scale_ratio(s_ks[tid], kn);
      s_vr[tid] = scale_ratio(s_vs[tid], vn);
    }
    __syncthreads();                                     // all have read the old scales
    if (sets) {
      const_cast<float*>(kv.k_scale)[scale_at] = kn;
      const_cast<float*>(kv.v_scale)[scale_at] = vn;
    }
    const int stay = first & at.mask;
    if (stay != 0 && (s_stay[0] != 1.f || s_stay[1] != 1.f)) {
      const int64_t page = at.at(first - stay);
      for (int e = tid; e < stay * pieces; e += kThreads) {
        const int64_t to = page + static_cast<int64_t>(e >> shift) * at.slot_bytes + 16 * (e & (pieces - 1));
        u32x4* kp = reinterpret_cast<u32x4*>(at.k + to);
        u32x4* vp = reinterpret_cast<u32x4*>(at.v + to);
        *kp = rescale_codes(*kp, s_stay[0]);
        *vp = rescale_codes(*vp, s_stay[1]);
      }
    }
  }

  // ---- write ----
  if (score && tid < count) score[tid] = moved_score;
#pragma unroll
  for (int u = 0; u < kCarry; ++u) {
    const int e = tid + u * kThreads, i = e >> shift;
    if (i < count) {
      const int64_t to = at.at(first + i) + 16 * (e & (pieces - 1));
      if constexpr (KV == PILLAR_FP8_E4M3) {
        k[u] = rescale_codes(k[u], s_kr[i]);
        v[u] = rescale_codes(v[u], s_vr[i]);
      }
      *reinterpret_cast<u32x4*>(at.k + to) = k[u];
      *reinterpret_cast<u32x4*>(at.v + to) = v[u];
    }
  }
}

}  // namespace

hipError_t launch_tree_commit(const CommitArgs& a, hipStream_t s) {
  KernelTimer timer("tree_commit", s);
  const dim3 grid(a.kv.num_kv_heads, a.kv.batch), block(kThreads);
  switch (a.kv_dtype) {
    case PILLAR_F32: hipLaunchKernelGGL(tree_commit<PILLAR_F32>, grid, block, 0, s, a); break;
    case PILLAR_BF16: hipLaunchKernelGGL(tree_commit<PILLAR_BF16>, grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL(tree_commit<PILLAR_FP8_E4M3>, grid, block, 0, s, a); break;
  }
  return hipGetLastError();
}

}  // namespace pillar

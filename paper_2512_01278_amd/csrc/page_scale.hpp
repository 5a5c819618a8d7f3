// Rows that move between the pages of a cache (gfx950).
//
// bf16 and fp32 rows are copied.  An fp8 page has one scale per KV head, so a row that arrives, and those that stay, are written anew against
// the page's new scale: the largest that any of its live rows had before.  With r = old scale / new scale <= 1 a code c becomes the fp8
// number nearest to c r (at most half a step, 2^-4 of the value, or 2^-10 below the smallest normal): nothing overflows, and where
// the scales are equal the bytes stay as they are.
#pragma once

#include "common.hpp"

namespace pillar {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// (0 / 0: a page of zeros)
__device__ __forceinline__ float scale_ratio(float had, float now) { return had == now ? 1.f : had / now; }

// sixteen codes times ratio, rounded to nearest even
__device__ __forceinline__ u32x4 rescale_codes(u32x4 c, float ratio) {
  if (ratio == 1.f) return c;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t x = c[w];
    float f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = e4m3_to_f32(static_cast<uint8_t>(x >> (8 * j))) * ratio;
    int y = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    y = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], y, true);
    c[w] = static_cast<uint32_t>(y);
  }
  return c;
}

// where one request's rows of one KV head lie, in bytes; pools are written through these
struct RowPlace {
  uint8_t* k;
  uint8_t* v;
  const int32_t* table;
  int64_t page_bytes, slot_bytes;
  int shift, mask;
  __device__ __forceinline__ RowPlace(const KvView& kv, int b, int g, int esz)
      : k(static_cast<uint8_t*>(const_cast<void*>(kv.k_pool)) + static_cast<int64_t>(g) * kv.stride_head * esz),
        v(static_cast<uint8_t*>(const_cast<void*>(kv.v_pool)) + static_cast<int64_t>(g) * kv.stride_head * esz),
        table(kv.block_table + static_cast<int64_t>(b) * kv.block_table_stride), page_bytes(kv.stride_page * esz),
        slot_bytes(kv.stride_slot * esz), shift(kv.page_shift), mask(kv.page_size - 1) {}
  __device__ __forceinline__ int page(int t) const { return table[t >> shift]; }
  __device__ __forceinline__ int64_t at(int page, int t) const { return static_cast<int64_t>(page) * page_bytes + static_cast<int64_t>(t & mask) * slot_bytes; }
  __device__ __forceinline__ int64_t at(int t) const { return at(page(t), t); }
};

}  // namespace pillar

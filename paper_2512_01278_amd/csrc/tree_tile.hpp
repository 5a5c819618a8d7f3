// Tile arithmetic of the tree verification (gfx950): 32 query rows of one wavefront against 32 tokens.
//
//   S^T[token, row] = K[token, :] . Q[row, :]          A = K   (32 tokens), B = Q^T (32 rows)
//   O^T[dim, row]  += V[token, dim] * P[row, token]    A = V^T (32 dims),   B = P^T (32 rows)
//
// With 32 x 32 products a lane owns ONE row (n = lane % 32) and half of the tokens (g = lane / 32): element i of an accumulator is
// token (or dim) 8 (i/4) + 4 g + i%4 of the 32.  So a row's maximum and sum need one exchange, between a lane and lane ^ 32, and the
// accumulator of S^T is the B operand of the second product as it stands, once V's tokens are taken in the same order.  32 rows to a
// wavefront because every wavefront reads the whole K and V tile from LDS: 16 KB per 32 tokens and 2 x 32 x 32 x 128 x 2 operations, 128
// cycles of LDS against 128 of its share of the matrix cores; 16 rows would double the reads.
//
// Two engines share the code around them:
//   EngineBf16   bf16 queries, bf16 or fp8 cache: v_mfma_f32_32x32x16_bf16; fp8 rows are widened (exactly) on the way into LDS, their page
//                scales are applied in fp32, v_scale as a summand of the logits in log2.  P is rounded to bf16 (at most 2^-8 of each
//                probability), as the matrix cores take it; sums of P are those of the unrounded values.
//   EngineF32    anything: rows become fp32 in LDS (fp8 times its scale), v_mfma_f32_32x32x2_f32.
//
// LDS rows are padded: K by 16 bytes, so that the 16-byte pieces that 16 rows hold at one place cover all banks; V so that the four rows of a
// transposing read lie 16 banks apart and fill all 64 with 32 dims each (bf16), or that two rows read together, four apart, lie 32 banks apart (fp32).
#pragma once

#include "common.hpp"
#include "mfma_tile.hpp"

namespace pillar {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int KV> constexpr int kv_bytes() { return KV == PILLAR_F32 ? 4 : KV == PILLAR_BF16 ? 2 : 1; }

// a lane's half of a row <-> the other half's
__device__ __forceinline__ float other_half_max(float v) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float other_half_sum(float v) {
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// token (or dim) within 32 of accumulator element i
__device__ __forceinline__ constexpr int elem_of(int i, int g) { return 8 * (i >> 2) + 4 * g + (i & 3); }

// Zeroes what is not finite in eight bf16 and says whether there was any.
__device__ __forceinline__ bool drop_nonfinite(u32x4& c) {
  bool any = false;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t x = c[w];
    if ((x & 0x7f80u) == 0x7f80u) { x &= 0xffff0000u; any = true; }
    if ((x & 0x7f800000u) == 0x7f800000u) { x &= 0xffffu; any = true; }
    c[w] = x;
  }
  return any;
}
__device__ __forceinline__ bool drop_nonfinite(float& f) {
  if ((__float_as_uint(f) & 0x7f800000u) != 0x7f800000u) return false;
  f = 0.f;
  return true;
}

template <int D>
struct EngineBf16 {
  static constexpr bool kF32 = false;
  static constexpr int kKPitch = 2 * D + 16, kVPitch = 2 * D + 64;          // bytes of an LDS row
  struct Query { bf16x8 q[D / 16]; };

  // rows: Q[row][0..D-1] of this lane's row, or null (zeros)
  static __device__ __forceinline__ void load_query(Query& f, const void* q, int64_t row, bool there, int, bool, int g) {
    const uint16_t* p = static_cast<const uint16_t*>(q) + row * D + 8 * g;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) f.q[s] = as_bf16x8(there ? *reinterpret_cast<const u32x4*>(p + 16 * s) : u32x4{0, 0, 0, 0});
  }
  static __device__ __forceinline__ f32x16 qk(const uint8_t* k, const Query& f, int lane) {
    const uint8_t* p = k + (lane & 31) * kKPitch + ((lane >> 5) << 4);
    f32x16 acc = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*reinterpret_cast<const u32x4*>(p + 32 * s)), f.q[s], acc, 0, 0, 0);
    return acc;
  }
  // the same with the roles exchanged: element i is row elem_of(i, g), and a lane's column is a token
  static __device__ __forceinline__ f32x16 qk_token(const uint8_t* k, const Query& f, int lane) {
    const uint8_t* p = k + (lane & 31) * kKPitch + ((lane >> 5) << 4);
    f32x16 acc = {};
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.q[s], as_bf16x8(*reinterpret_cast<const u32x4*>(p + 32 * s)), acc, 0, 0, 0);
    return acc;
  }
  // ds_read_b64_tr_b16: within 16 lanes, lane 4k+a gives the address of 4 dims of token k, and lane m receives dim m of the four tokens
  static __device__ __forceinline__ void pv(const uint8_t* v, const f32x16& p, f32x16 (&o)[D / 32], int lane) {
    const int j = lane & 15, h = (lane >> 4) & 1, g = lane >> 5;
    const uint8_t* src = v + (4 * g + (j >> 2)) * kVPitch + 32 * h + 8 * (j & 3);
    bf16x8 pb[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) pb[u][e] = static_cast<__bf16>(p[8 * u + e]);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(src + 64 * db + 16 * u * kVPitch));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(src + 64 * db + (16 * u + 8) * kVPitch));
        const bf16x8 a = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[u], o[db], 0, 0, 0);
      }
  }
};

template <int D>
struct EngineF32 {
  static constexpr bool kF32 = true;
  static constexpr int kKPitch = 4 * (D + 4), kVPitch = 4 * (D + 8);
  struct Query { f32x4 q[D / 8]; };

  // dense: rows of q are multiples of 16 bytes
  static __device__ __forceinline__ void load_query(Query& f, const void* q, int64_t row, bool there, int q_dtype, bool dense, int g) {
    const int64_t first = row * D + 4 * g;
    if (!there) {
#pragma unroll
      for (int s = 0; s < D / 8; ++s) f.q[s] = f32x4{0.f, 0.f, 0.f, 0.f};
    } else if (q_dtype == PILLAR_F32 && dense) {
#pragma unroll
      for (int s = 0; s < D / 8; ++s) f.q[s] = *reinterpret_cast<const f32x4*>(static_cast<const float*>(q) + first + 8 * s);
    } else {
#pragma unroll
      for (int s = 0; s < D / 8; ++s)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          f.q[s][c] = q_dtype == PILLAR_F32 ? Storage<PILLAR_F32>::load(q, first + 8 * s + c) : Storage<PILLAR_BF16>::load(q, first + 8 * s + c);
    }
  }
  static __device__ __forceinline__ f32x16 qk(const uint8_t* k, const Query& f, int lane) {
    const uint8_t* p = k + (lane & 31) * kKPitch + ((lane >> 5) << 4);
    f32x16 acc[2] = {};                          // two short sums: less rounding than one long one
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(p + 32 * s);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c & 1] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[c], f.q[s][c], acc[c & 1], 0, 0, 0);
    }
    return acc[0] + acc[1];
  }
  static __device__ __forceinline__ f32x16 qk_token(const uint8_t* k, const Query& f, int lane) {
    const uint8_t* p = k + (lane & 31) * kKPitch + ((lane >> 5) << 4);
    f32x16 acc[2] = {};
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(p + 32 * s);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c & 1] = __builtin_amdgcn_mfma_f32_32x32x2f32(f.q[s][c], a[c], acc[c & 1], 0, 0, 0);
    }
    return acc[0] + acc[1];
  }
  static __device__ __forceinline__ void pv(const uint8_t* v, const f32x16& p, f32x16 (&o)[D / 32], int lane) {
    const uint8_t* src = v + 4 * (lane >> 5) * kVPitch + 4 * (lane & 31);
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float a = *reinterpret_cast<const float*>(src + (8 * (i >> 2) + (i & 3)) * kVPitch + 128 * db);
        o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[i], o[db], 0, 0, 0);
      }
  }
};

// ---- rows of the cache on their way into LDS ----

// one 16-byte piece of a row; `aligned`: the pool's base and strides are multiples of 16 bytes, else element by element
template <int KV>
__device__ __forceinline__ u32x4 load_piece(const void* pool, int64_t elem, bool aligned) {
  const uint8_t* p = static_cast<const uint8_t*>(pool) + elem * kv_bytes<KV>();
  if (aligned) return *reinterpret_cast<const u32x4*>(p);
  u32x4 r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if constexpr (KV == PILLAR_F32) {
      r[w] = reinterpret_cast<const uint32_t*>(p)[w];
    } else if constexpr (KV == PILLAR_BF16) {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p) + 2 * w;
      r[w] = h[0] | static_cast<uint32_t>(h[1]) << 16;
    } else {
      r[w] = p[4 * w] | p[4 * w + 1] << 8 | p[4 * w + 2] << 16 | static_cast<uint32_t>(p[4 * w + 3]) << 24;
    }
  }
  return r;
}

// Element e of a piece as fp32.
template <int KV>
__device__ __forceinline__ float piece_elem(const u32x4& c, int e) {
  if constexpr (KV == PILLAR_F32) return __uint_as_float(c[e]);
  else if constexpr (KV == PILLAR_BF16) return __uint_as_float((e & 1) ? c[e >> 1] & 0xffff0000u : c[e >> 1] << 16);
  else return e4m3_to_f32(static_cast<uint8_t>(c[e >> 2] >> (8 * (e & 3))));
}

// Parks a piece in LDS at `row`, the row's element 16 / esz * piece on.  CLEAN: what is not finite becomes zero; returns whether there was any.
template <typename E, int KV, bool CLEAN>
__device__ __forceinline__ bool park_piece(u32x4 c, float scale, uint8_t* row, int piece) {
  bool bad = false;
  if constexpr (!E::kF32) {
    if constexpr (KV == PILLAR_BF16) {
      if (CLEAN) bad = drop_nonfinite(c);
      *reinterpret_cast<u32x4*>(row + 16 * piece) = c;
    } else {
      u32x4 lo, hi;
      widen_fp8x16(c, lo, hi);
      if (CLEAN) { bad = drop_nonfinite(lo); bad |= drop_nonfinite(hi); }
      *reinterpret_cast<u32x4*>(row + 32 * piece) = lo;
      *reinterpret_cast<u32x4*>(row + 32 * piece + 16) = hi;
    }
  } else {
    constexpr int kElems = 16 / kv_bytes<KV>();
    float* out = reinterpret_cast<float*>(row) + kElems * piece;
#pragma unroll
    for (int e = 0; e < kElems; e += 4) {
      f32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = piece_elem<KV>(c, e + j);
        if constexpr (KV == PILLAR_FP8_E4M3) x[j] *= scale;
        if (CLEAN) { float y = x[j]; bad |= drop_nonfinite(y); x[j] = y; }
      }
      *reinterpret_cast<f32x4*>(out + e) = x;
    }
  }
  return bad;
}

}  // namespace pillar

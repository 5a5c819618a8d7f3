// Rotary positions (gfx950): angles, and pieces of a head that are loaded, turned and stored together.
//
//   y1 = a (x1 cos t - x2 sin t),  y2 = a (x2 cos t + x1 sin t),  t = position * frequency of the pair
//
// A float cannot hold the angle of a far position (position 10^6 at frequency 1: the fraction of a turn to 2^-5), and 64 bits hold that of the farthest to 2^-23
// of a turn, so it is worked out in turns, in 64 bits and what their roundings leave.  The whole turns and then the quarters are taken off there,
// and what is left, at most an eighth of a turn either way, goes through the power series of sine and cosine in fp32 (up to x^9 and x^10: within 2^-29 of either).
#pragma once

#include "common.hpp"
#include "launch.hpp"

namespace pillar {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// cosine and sine of position * frequency, times amplitude
__device__ __forceinline__ float2 turned(int position, double frequency, float amplitude) {
  constexpr double kTurnsPerRadian = 0x1.45f306dc9c883p-3, kTurnsPerRadianLow = -0x1.6b01ec5417056p-57;        // 1 / 2 pi
  const double p = static_cast<double>(position);
  const double each = frequency * kTurnsPerRadian, each_low = __builtin_fma(frequency, kTurnsPerRadian, -each) + frequency * kTurnsPerRadianLow;
  double part = __builtin_fma(p, each, -__builtin_rint(p * each)) + p * each_low;           // (the product is not rounded)
  part -= __builtin_rint(part);                                          // -1/2 .. 1/2
  const double quarters = __builtin_rint(4.0 * part);                    // -2 .. 2
  const float x = static_cast<float>(__builtin_fma(quarters, -0.25, part)) * 6.28318530717958647692f;
  const int k = static_cast<int>(quarters);
  const float z = x * x;
  auto fma = [](float p, float q, float r) { return __builtin_fmaf(p, q, r); };
  const float s = fma(x * z, fma(z, fma(z, fma(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float c = fma(z, fma(z, fma(z, fma(z, fma(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  float cosine = (k & 1) ? s : c, sine = (k & 1) ? c : s;
  if ((k + 1) & 2) cosine = -cosine;                                     // quarters 1 and 2 (and -2, -3)
  if (k & 2) sine = -sine;                                               // quarters 2 and 3 (and -1, -2)
  return make_float2(cosine * amplitude, sine * amplitude);
}

// V elements as fp32, V of 1, 2, 4, 8 (bf16) in one load
template <int DT, int V>
__device__ __forceinline__ void load_elems(const void* p, int64_t at, float (&x)[V]) {
  if constexpr (V == 1) {
    x[0] = Storage<DT>::load(p, at);
  } else if constexpr (DT == PILLAR_F32) {
    typedef float Vec __attribute__((ext_vector_type(V)));
    const Vec v = *reinterpret_cast<const Vec*>(static_cast<const float*>(p) + at);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = v[j];
  } else {
    typedef uint16_t Vec __attribute__((ext_vector_type(V)));
    const Vec v = *reinterpret_cast<const Vec*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = bf16_to_f32(v[j]);
  }
}

// V elements from fp32, rounded to nearest even
template <int DT, int V>
__device__ __forceinline__ void store_elems(void* p, int64_t at, const float (&x)[V]) {
  if constexpr (V == 1) {
    Storage<DT>::store(p, at, x[0]);
  } else if constexpr (DT == PILLAR_F32) {
    constexpr int W = V < 4 ? V : 4;
    typedef float Vec __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int j = 0; j < V; j += W) {
      Vec y;
#pragma unroll
      for (int k = 0; k < W; ++k) y[k] = x[j + k];
      *reinterpret_cast<Vec*>(static_cast<float*>(p) + at + j) = y;
    }
  } else {
    typedef __bf16 Vec __attribute__((ext_vector_type(V)));
    Vec y;
#pragma unroll
    for (int j = 0; j < V; ++j) y[j] = static_cast<__bf16>(x[j]);
    *reinterpret_cast<Vec*>(static_cast<uint16_t*>(p) + at) = y;
  }
}

// A head is cut into pieces of V elements that one load takes, each with its partner: piece c of a head of D dims, of which 2 * half are rotated.
//   halves       dims c V .. and half + c V ..; pairs c V ..
//   interleaved  dims c V .., which are pairs c V / 2 ..; one element at a time: dims 2 c and 2 c + 1
//   the rest     dims as they are
// V > 1 wants half (halves) or 2 half (interleaved), and D, to be multiples of V.
struct Piece {
  int lo, hi;                  // first dims; hi < 0: none
  int pair;                    // first pair, or -1: not rotated
};
template <int V>
__device__ __forceinline__ Piece piece_of(const RopeView& rope, int c) {
  const int turning = V > 1 && rope.interleaved ? 2 * rope.half / V : rope.half / V;
  if (c >= turning) return Piece{2 * rope.half + (c - turning) * V, -1, -1};
  if (!rope.interleaved) return Piece{c * V, rope.half + c * V, c * V};
  if (V > 1) return Piece{c * V, -1, c * V / 2};
  return Piece{2 * c, 2 * c + 1, c};
}
template <int V>
__host__ __device__ __forceinline__ int pieces_of_head(const RopeView& rope, int D) {
  const int turning = V > 1 && rope.interleaved ? 2 * rope.half / V : rope.half / V;
  return turning + (D - 2 * rope.half) / V;
}
// whether pieces of V elements will do
inline bool rope_in_pieces(const RopeView& rope, int D, int V) {
  return D % V == 0 && (rope.interleaved ? 2 * rope.half : rope.half) % V == 0;
}

// Head and piece of a thread, turn by turn, without a division in each.
struct HeadPiece {
  int h, c;
  int pieces, heads_on, pieces_on;
  __device__ __forceinline__ HeadPiece(int pieces_, int threads) : pieces(pieces_) {
    h = static_cast<int>(threadIdx.x) / pieces;
    c = static_cast<int>(threadIdx.x) - h * pieces;
    heads_on = threads / pieces;
    pieces_on = threads - heads_on * pieces;
  }
  __device__ __forceinline__ void next() {
    h += heads_on;
    c += pieces_on;
    if (c >= pieces) { c -= pieces; ++h; }
  }
};

// turns a piece (in the same operations whatever V is: the same bits); angle(i): cosine and sine of its i-th pair
template <int V, typename Angle>
__device__ __forceinline__ void turn_piece(const Piece& p, float (&a)[V], float (&b)[V], Angle angle) {
  if (p.pair < 0) return;
  if (p.hi >= 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 t = angle(j);
      const float x = a[j], y = b[j];
      a[j] = __builtin_fmaf(x, t.x, -(y * t.y));
      b[j] = __builtin_fmaf(y, t.x, x * t.y);
    }
  } else if constexpr (V > 1) {
#pragma unroll
    for (int j = 0; j < V; j += 2) {
      const float2 t = angle(j >> 1);
      const float x = a[j], y = a[j + 1];
      a[j] = __builtin_fmaf(x, t.x, -(y * t.y));
      a[j + 1] = __builtin_fmaf(y, t.x, x * t.y);
    }
  }
}

}  // namespace pillar

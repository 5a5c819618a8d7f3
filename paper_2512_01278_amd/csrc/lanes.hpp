// Values of other lanes without a trip through LDS (gfx950): what a shuffle does through the LDS crossbar in some hundred cycles, the vector ALU does in one or two
// instructions for the patterns below.
#pragma once

#include "common.hpp"

namespace pillar {

// the value of lane ^ O
template <int O>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  static_assert(O == 1 || O == 2 || O == 4 || O == 8 || O == 16 || O == 32, "");
  typedef unsigned u2 __attribute__((ext_vector_type(2)));
  const int x = static_cast<int>(v);
  if constexpr (O == 1) return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, true));      // quad_perm [1,0,3,2]
  else if constexpr (O == 2) return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, true)); // quad_perm [2,3,0,1]
  else if constexpr (O == 4) {                             // eight lanes reversed, then every four of them
    const int r = __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, true);
    return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, r, 0x1B, 0xF, 0xF, true));
  } else if constexpr (O == 8) return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, true));      // row_ror 8: 16 lanes turned by half
  else {
    // with both operands the same, one result has rows 0 and 2 (lanes 0 to 31) twice, the other rows 1 and 3 (lanes 32 to 63)
    u2 r;
    if constexpr (O == 16) r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    else r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & O) ? r.x : r.y;
  }
}
template <int O> __device__ __forceinline__ float lane_xor(float v) { return __uint_as_float(lane_xor<O>(__float_as_uint(v))); }
template <int O> __device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
  return static_cast<uint64_t>(lane_xor<O>(static_cast<uint32_t>(v >> 32))) << 32 | lane_xor<O>(static_cast<uint32_t>(v));
}

// the value of the lane before; lane 0 keeps its own
__device__ __forceinline__ uint32_t lane_before(uint32_t v) {
  return static_cast<uint32_t>(__builtin_amdgcn_update_dpp(static_cast<int>(v), static_cast<int>(v), 0x138, 0xF, 0xF, false));     // wave_shr 1
}
__device__ __forceinline__ uint64_t lane_before(uint64_t v) {
  return static_cast<uint64_t>(lane_before(static_cast<uint32_t>(v >> 32))) << 32 | lane_before(static_cast<uint32_t>(v));
}

// 64 lanes in reverse order
__device__ __forceinline__ uint32_t lane_reversed(uint32_t v) {
  v = static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), 0x140, 0xF, 0xF, true));                            // row_mirror: 16 lanes
  return lane_xor<32>(lane_xor<16>(v));
}
__device__ __forceinline__ uint64_t lane_reversed(uint64_t v) {
  return static_cast<uint64_t>(lane_reversed(static_cast<uint32_t>(v >> 32))) << 32 | lane_reversed(static_cast<uint32_t>(v));
}

}  // namespace pillar

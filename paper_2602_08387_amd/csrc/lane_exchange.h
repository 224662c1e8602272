// The value of lane l ^ M, for M a power of two, in the register file: lanes of a row of 16 by DPP, rows by permlane swaps.  A shuffle through LDS takes some 60
// cycles; these take one or two instructions.
#pragma once
#include "common.h"

namespace dl {

template <int M>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
  static_assert(M == 1 || M == 2 || M == 4 || M == 8 || M == 16 || M == 32, "a power of two below 64");
  const int v = (int)x;
  if constexpr (M == 1) return (uint32_t)__builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);        // quad_perm 1, 0, 3, 2
  else if constexpr (M == 2) return (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);   // quad_perm 2, 3, 0, 1
  else if constexpr (M == 4)                                                                       // mirrored in 8 lanes, then in 4
    return (uint32_t)__builtin_amdgcn_mov_dpp(__builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true), 0x1B, 0xf, 0xf, true);
  else if constexpr (M == 8) return (uint32_t)__builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);  // rotated by 8 of 16
  else if constexpr (M == 16) {                        // rows 0 0 2 2 and 1 1 3 3
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return (__lane_id() & 16) ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (__lane_id() & 32) ? r[0] : r[1];
  }
}
template <int M>
__device__ __forceinline__ float lane_xor(float x) { return __uint_as_float(lane_xor<M>(__float_as_uint(x))); }
template <int M>
__device__ __forceinline__ uint64_t lane_xor(uint64_t x) {
  return (uint64_t)lane_xor<M>((uint32_t)(x >> 32)) << 32 | lane_xor<M>((uint32_t)x);
}

}  // namespace dl

// Sorting (value, id) keys across a wave.
#pragma once

#include "../common.hpp"

namespace respec {

// Value held by lane (lane ^ J): moves inside rows of 16 lanes for J up to 8 (4 is the quad's reversal,
// xor 3, and the mirror within 8, xor 7; 8 the mirrors within 8 and 16), row swaps above.
template <int J>
__device__ __forceinline__ int from_lane_xor(int v) {
  if constexpr (J == 1) return xchg<0>(v);
  if constexpr (J == 2) return xchg<1>(v);
  if constexpr (J == 4) return xchg<2>(__builtin_amdgcn_mov_dpp(v, 0x1B, 0xF, 0xF, false));
  if constexpr (J == 8) return xchg<3>(xchg<2>(v));
  if constexpr (J == 16) return xchg<4>(v);
  return xchg<5>(v);
}

// Bitonic sort of one key per lane, the largest into lane 0: blocks of SZ lanes are ordered, descending
// where lane & SZ is 0, by compare-exchanges at distance J = SZ/2 .. 1.
template <int SZ = 2, int J = 1>
__device__ __forceinline__ uint64_t sort_lanes_desc(uint64_t k) {
  const int lane = (int)(threadIdx.x & 63);
  const uint64_t o = ((uint64_t)(uint32_t)from_lane_xor<J>((int)(uint32_t)(k >> 32)) << 32) |
                     (uint32_t)from_lane_xor<J>((int)(uint32_t)k);
  const bool larger = ((lane & J) == 0) == ((lane & SZ) == 0);
  k = (o > k) == larger ? o : k;
  if constexpr (J > 1) return sort_lanes_desc<SZ, J / 2>(k);
  else if constexpr (SZ < 64) return sort_lanes_desc<SZ * 2, SZ>(k);
  else return k;
}

__device__ __forceinline__ uint64_t key_of_lane(uint64_t k, int l) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(k >> 32), l) << 32) |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, l);
}

}  // namespace respec

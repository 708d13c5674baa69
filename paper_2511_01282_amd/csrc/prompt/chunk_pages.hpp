// A wave's window of a sequence's page ids in LDS.
#pragma once

#include "chunk.hpp"

namespace respec {

template <int N>  // ids that it holds
struct PageIds {
  int32_t* ids;          // LDS, the wave's own
  const int32_t* table;  // the sequence's row of the page table
  uint32_t p0, p1;       // ids[0] is page p0's; ids of pages p0 .. p1 - 1 are there
  uint32_t end;          // pages of the sequence's rows that this workgroup reads end here

  // Make the ids of pages a .. b (b - a < N, a no less than before) available.
  __device__ __forceinline__ void need(uint32_t a, uint32_t b, int lane) {
    if (b < p1) return;
    p0 = a;
    p1 = min(a + (uint32_t)N, end);
    wave_lds_sync();
    for (uint32_t p = p0 + lane; p < p1; p += 64) ids[p - p0] = table[p];
    wave_lds_sync();
  }
  __device__ __forceinline__ int uniform(uint32_t p) const { return __builtin_amdgcn_readfirstlane(ids[p - p0]); }
};

}  // namespace respec

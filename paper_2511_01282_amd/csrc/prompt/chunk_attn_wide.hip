// Attention kernel of calls with long chunks, over a cache of the model's bf16: see chunk_wide.hpp.
#include "chunk_few.hpp"
#include "chunk_wide.hpp"

namespace respec {
namespace {

// MIXED: sequences of few query rows are there, too, and have workgroups of their own, of which four waves work (a
// launch for each kind, one after the other: 13 sequences of 1-90 tokens over 146-217 rows, 28 heads on 4, 32.2 us,
// like this 22.1; 9 of 1-307 over 352-564, 32 on 8, 47.3 and 38.8).
template <int D, bool MIXED>
__global__ __launch_bounds__(kAttnWideThreads, 1) void chunk_attn_wide_kernel(ChunkAttnArgs a) {
  extern __shared__ __align__(1024) unsigned char smem[];
  int x = (int)blockIdx.x;
  if (x < a.wide.items) {
    wide_rows_item<D, false>(a, x, smem);
    return;
  }
  x -= a.wide.items;
  if constexpr (MIXED) {
    if (x < a.few.items) {
      if (threadIdx.x < 256) few_rows_item<D, 1, D == 128>(a, x, smem);
      return;
    }
    x -= a.few.items;
  }
  report_status<kAttnWideThreads>(a.b, x, true);
}

template <int D, bool MIXED>
hipError_t go(bool launch, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  constexpr int kLds = MIXED && FewShape<D>::kLds > WideShape<D, false>::kLds ? FewShape<D>::kLds : WideShape<D, false>::kLds;
  if (!launch)
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&chunk_attn_wide_kernel<D, MIXED>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  const int items = a.wide.items + (MIXED ? a.few.items : 0) + (status ? a.b.batch : 0);
  hipLaunchKernelGGL((chunk_attn_wide_kernel<D, MIXED>), dim3(items), dim3(kAttnWideThreads), kLds, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn_wide(int head_dim, const ChunkAttnArgs& a, bool mixed, bool status, hipStream_t s) {
  if (mixed) return head_dim == 128 ? go<128, true>(true, a, status, s) : go<64, true>(true, a, status, s);
  return head_dim == 128 ? go<128, false>(true, a, status, s) : go<64, false>(true, a, status, s);
}
hipError_t set_chunk_attn_wide_lds_limit(int head_dim) {
  const ChunkAttnArgs none{};
  const hipError_t e = head_dim == 128 ? go<128, false>(false, none, false, nullptr) : go<64, false>(false, none, false, nullptr);
  if (e != hipSuccess) return e;
  return head_dim == 128 ? go<128, true>(false, none, false, nullptr) : go<64, true>(false, none, false, nullptr);
}

}  // namespace respec

// Attention kernel of calls whose sequences all have few query rows: see chunk_few.hpp.
#include "chunk_few.hpp"

namespace respec {
namespace {

template <int D, int GR>
__global__ __launch_bounds__(kAttnFewThreads, 1) void chunk_attn_few_kernel(ChunkAttnArgs a) {
  extern __shared__ __align__(1024) unsigned char smem[];
  if ((int)blockIdx.x >= a.few.items) {
    report_status<256>(a.b, (int)blockIdx.x - a.few.items, true);
    return;
  }
  few_rows_item<D, GR, false>(a, (int)blockIdx.x, smem);
}

template <int D, int GR>
hipError_t go(bool launch, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  if (!launch)
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&chunk_attn_few_kernel<D, GR>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, FewShape<D>::kLds);
  hipLaunchKernelGGL((chunk_attn_few_kernel<D, GR>), dim3(a.few.items + (status ? a.b.batch : 0)), dim3(kAttnFewThreads), FewShape<D>::kLds, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn_few(int head_dim, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  if (a.few.rows_per_wg == 32) return head_dim == 128 ? go<128, 1>(true, a, status, s) : go<64, 1>(true, a, status, s);
  if (a.few.rows_per_wg == 64) return head_dim == 128 ? go<128, 2>(true, a, status, s) : go<64, 2>(true, a, status, s);
  return hipErrorInvalidValue;
}
hipError_t set_chunk_attn_few_lds_limit(int head_dim) {
  const ChunkAttnArgs none{};
  const hipError_t e = head_dim == 128 ? go<128, 1>(false, none, false, nullptr) : go<64, 1>(false, none, false, nullptr);
  if (e != hipSuccess) return e;
  return head_dim == 128 ? go<128, 2>(false, none, false, nullptr) : go<64, 2>(false, none, false, nullptr);
}

}  // namespace respec

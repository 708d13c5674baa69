// Attention kernels over an 8-bit paged cache: see q8_few.hpp (few query rows) and chunk_wide.hpp (long chunks).
#include "chunk_wide.hpp"
#include "q8_few.hpp"

namespace respec {
namespace {

template <int D, int GR>
__global__ __launch_bounds__(kAttnFewThreads, GR <= 2 ? 2 : 1) void q8_attn_few_kernel(ChunkAttnArgs a) {
  extern __shared__ __align__(1024) unsigned char smem[];
  if ((int)blockIdx.x >= a.few.items) {
    report_status<kAttnFewThreads>(a.b, (int)blockIdx.x - a.few.items, true);
    return;
  }
  q8_few_rows_item<D, GR>(a, (int)blockIdx.x, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), smem);
}

// MIXED: as chunk_attn_wide_kernel's.
template <int D, bool MIXED>
__global__ __launch_bounds__(kAttnWideThreads, 1) void q8_attn_wide_kernel(ChunkAttnArgs a) {
  extern __shared__ __align__(1024) unsigned char smem[];
  int x = (int)blockIdx.x;
  if (x < a.wide.items) {
    wide_rows_item<D, true>(a, x, smem);
    return;
  }
  x -= a.wide.items;
  if constexpr (MIXED) {
    if (x < a.few.items) {
      if (threadIdx.x >= 256) return;
      const Again g = again_from(x, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
      q8_few_rows_item<D, 2>(g.a, g.x, g.wave, smem);
      return;
    }
    x -= a.few.items;
  }
  report_status<kAttnWideThreads>(a.b, x, true);
}

template <int D, int GR>
hipError_t go_few(bool launch, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  if (!launch)
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&q8_attn_few_kernel<D, GR>), hipFuncAttributeMaxDynamicSharedMemorySize,
                               Q8FewShape<D>::kLds);
  hipLaunchKernelGGL((q8_attn_few_kernel<D, GR>), dim3(a.few.items + (status ? a.b.batch : 0)), dim3(kAttnFewThreads),
                     Q8FewShape<D>::kLds, s, a);
  return hipGetLastError();
}

template <int D, bool MIXED>
hipError_t go_wide(bool launch, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  constexpr int kWide = WideShape<D, true>::kLds, kFew = Q8FewShape<D>::kLds, kLds = MIXED && kFew > kWide ? kFew : kWide;
  if (!launch)
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&q8_attn_wide_kernel<D, MIXED>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  const int items = a.wide.items + (MIXED ? a.few.items : 0) + (status ? a.b.batch : 0);
  hipLaunchKernelGGL((q8_attn_wide_kernel<D, MIXED>), dim3(items), dim3(kAttnWideThreads), kLds, s, a);
  return hipGetLastError();
}

template <int D>
hipError_t set_limits() {
  const ChunkAttnArgs none{};
  for (hipError_t e : {go_few<D, 1>(false, none, false, nullptr), go_few<D, 2>(false, none, false, nullptr), go_few<D, 4>(false, none, false, nullptr),
                       go_wide<D, false>(false, none, false, nullptr), go_wide<D, true>(false, none, false, nullptr)})
    if (e != hipSuccess) return e;
  return hipSuccess;
}

}  // namespace

hipError_t launch_q8_attn_few(int head_dim, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  if (a.few.rows_per_wg == 16) return head_dim == 128 ? go_few<128, 1>(true, a, status, s) : go_few<64, 1>(true, a, status, s);
  if (a.few.rows_per_wg == 32) return head_dim == 128 ? go_few<128, 2>(true, a, status, s) : go_few<64, 2>(true, a, status, s);
  if (a.few.rows_per_wg == 64) return head_dim == 128 ? go_few<128, 4>(true, a, status, s) : go_few<64, 4>(true, a, status, s);
  return hipErrorInvalidValue;
}
hipError_t launch_q8_attn_wide(int head_dim, const ChunkAttnArgs& a, bool mixed, bool status, hipStream_t s) {
  if (mixed) return head_dim == 128 ? go_wide<128, true>(true, a, status, s) : go_wide<64, true>(true, a, status, s);
  return head_dim == 128 ? go_wide<128, false>(true, a, status, s) : go_wide<64, false>(true, a, status, s);
}
hipError_t set_q8_attn_lds_limits(int head_dim) { return head_dim == 128 ? set_limits<128>() : set_limits<64>(); }

}  // namespace respec

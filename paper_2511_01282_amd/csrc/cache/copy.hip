// Copies of pages: page dst[i] of every plane and layer becomes its page src[i].
//
// Bytes alone: a page of a plane and layer is a row of pieces of the widest kind that its addresses allow, each
// thread moves kCopyPieces of them with all loads under way before the first store.  The host merges rows and heads that lie
// side by side into one run, so dense pages cost no division that matters.
//
// 24 pages of 64 rows in 32 layers, 8 heads of 128, bf16, K and V (201 MB read, as many written): 77 us, 5.2 TB/s.  4 pages of 16
// rows with their scales, 8 bits, 32 layers: 5.3 us, which is a launch and one round of dependent reads.
#include "cache.hpp"

namespace respec {
namespace {

template <typename T>
__device__ __forceinline__ void copy_pieces(const CopyPlane& p, int64_t src, int64_t dst, uint32_t first) {
  T x[kCopyPieces];
  int64_t at[kCopyPieces];
#pragma unroll
  for (int u = 0; u < kCopyPieces; ++u) {
    const uint32_t q = first + u * kCopyThreads;
    if (q >= p.pieces) continue;
    const uint32_t h = div_by(q, p.per_head), y = q - h * p.per_head.d, r = div_by(y, p.per_row);
    at[u] = (int64_t)h * p.head_stride + (int64_t)r * p.row_stride + (int64_t)(y - r * p.per_row.d) * (int64_t)sizeof(T);
    x[u] = *reinterpret_cast<const T*>(p.base + src + at[u]);
  }
#pragma unroll
  for (int u = 0; u < kCopyPieces; ++u)
    if (first + u * kCopyThreads < p.pieces) *reinterpret_cast<T*>(p.base + dst + at[u]) = x[u];
}

__global__ __launch_bounds__(kCopyThreads) void copy_kernel(CopyArgs a) {
  const int pair = blockIdx.z, layer = blockIdx.y;
  const int32_t src = a.src[pair], dst = a.dst[pair];
  const bool none = src == -1, bad = !none && ((uint32_t)src >= (uint32_t)a.n_pages || (uint32_t)dst >= (uint32_t)a.n_pages);
  if (a.status && blockIdx.x == 0 && layer == 0 && threadIdx.x == 0) a.status[pair] = bad ? kStPage : 0;
  if (none || bad || src == dst) return;
  int k = 0;
#pragma unroll 1
  while (k + 1 < a.n_planes && (int)blockIdx.x >= a.plane[k + 1].first_wg) ++k;
  const CopyPlane& p = a.plane[k];
  if (layer >= p.n_layers) return;
  const int64_t at = (int64_t)layer * p.layer_stride;
  const int64_t from = at + (int64_t)src * p.page_stride, to = at + (int64_t)dst * p.page_stride;
  const uint32_t first = (uint32_t)((int)blockIdx.x - p.first_wg) * (kCopyThreads * kCopyPieces) + threadIdx.x;
  switch (p.piece) {
    case 16: copy_pieces<u32x4>(p, from, to, first); break;
    case 8: copy_pieces<u32x2>(p, from, to, first); break;
    case 4: copy_pieces<uint32_t>(p, from, to, first); break;
    case 2: copy_pieces<uint16_t>(p, from, to, first); break;
    default: copy_pieces<uint8_t>(p, from, to, first); break;
  }
}

}  // namespace

hipError_t launch_copy(int wgs, int layers, int pairs, const CopyArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(copy_kernel, dim3(wgs, layers, pairs), dim3(kCopyThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace respec

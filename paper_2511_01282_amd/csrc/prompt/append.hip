// Keys and values of new tokens into the pages of a cache.
//
// K[page(L + i)][h][row] = k_new[i][h], V likewise: a copy of 2 Hkv rows of D elements per token,
// so memory alone bounds it.  A workgroup takes consecutive packed tokens as 16-byte pieces:
// consecutive threads read and write consecutive pieces of a row, eight in flight per thread.
// The reads need nothing but the token's number, so they are under way while the waves look up
// which sequence, page and row each token goes to.
//
// Measured (MI355X): five prompts, 8057 tokens of 32 KV heads of 128 bf16 (264 MB read and written), 44 us, 6.0 TB/s
// (part of the new rows is still in the memory-side cache; a copy of 8 GB reaches 4.75); 96 sequences of one token, 5.2 us, where
// the launch and the two dependent reads of a token's place are what it takes.
#include "chunk.hpp"

namespace respec {
namespace {

constexpr int kThreads = kAppendThreads, kPieces = 8;

template <int CPR>  // 16-byte pieces per row
__global__ __launch_bounds__(kThreads) void chunk_append_kernel(AppendArgs a) {
  const int tok_wgs = (int)gridDim.x - (a.b.status ? a.b.batch : 0);
  if ((int)blockIdx.x >= tok_wgs) {  // one more workgroup per sequence reports its status
    report_status<kThreads>(a.b, (int)blockIdx.x - tok_wgs, false);
    return;
  }
  __shared__ int64_t to[kAppendMaxTok];  // byte offset of each token's row within a head, or -1
  const int t0 = blockIdx.x * a.tok_per_wg, n = min(a.tok_per_wg, a.b.total_new - t0);
  const uint32_t total = (uint32_t)n * a.per_tok.d, half = a.per_tok.d / 2;
  for (uint32_t x0 = threadIdx.x; x0 - threadIdx.x < total; x0 += kThreads * kPieces) {
    u32x4 piece[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
      const uint32_t x = min(x0 + u * kThreads, total - 1);
      const uint32_t i = div_by(x, a.per_tok), y = x - i * a.per_tok.d, w = y >= half ? y - half : y;
      const int64_t t = t0 + (int)i, h = w / CPR, c = (w % CPR) * 16;
      piece[u] = ld16((y >= half ? a.v_new + t * a.v_tok + h * a.v_head : a.k_new + t * a.k_tok + h * a.k_head) + c);
    }
    if (x0 == threadIdx.x) {  // first round: the tokens' places, a wave per token
      for (int i = threadIdx.x >> 6; i < n; i += kThreads / 64) {
        int b;
        const ChunkSeq s = seq_of_token(a.b, t0 + i, b);
        if ((threadIdx.x & 63) == 0) {
          int64_t at = -1;
          if (s.n > 0) {
            const uint32_t r = (uint32_t)(s.L + (t0 + i - s.t0)), p = div_by(r, a.b.page);
            const int32_t id = a.b.table[(int64_t)b * a.b.table_stride + p];
            if ((uint32_t)id < (uint32_t)a.b.n_pages)  // (a page out of range is left out and reported)
              at = (int64_t)id * a.b.page_stride + (int64_t)((uint64_t)(r - p * a.b.page.d) * a.b.row_stride);
          }
          to[i] = at;
        }
      }
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
      const uint32_t x = x0 + u * kThreads;
      if (x >= total) continue;
      const uint32_t i = div_by(x, a.per_tok), y = x - i * a.per_tok.d, w = y >= half ? y - half : y;
      const int64_t at = to[i];
      if (at >= 0)
        *reinterpret_cast<u32x4*>((y >= half ? a.b.v : a.b.k) + at + (int64_t)(w / CPR) * a.b.head_stride + (w % CPR) * 16) =
            piece[u];
    }
  }
}

}  // namespace

hipError_t launch_chunk_append(int es, int head_dim, const AppendArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.b.total_new + a.tok_per_wg - 1) / a.tok_per_wg) + (a.b.status ? a.b.batch : 0));
  switch (head_dim * es / 16) {
    case 8: hipLaunchKernelGGL(chunk_append_kernel<8>, grid, dim3(kThreads), 0, s, a); break;
    case 16: hipLaunchKernelGGL(chunk_append_kernel<16>, grid, dim3(kThreads), 0, s, a); break;
    case 32: hipLaunchKernelGGL(chunk_append_kernel<32>, grid, dim3(kThreads), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace respec

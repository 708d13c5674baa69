// The accepted path of every verified draft tree moves to the front of its nodes' rows.
//
// Row kv_len + path[i] -> kv_len + i, i = 0 .. acc_len, of K and V, every KV head and layer.  path ascends, so path[i] >= i: no
// row is written that a later i still reads, and a thread that takes the same 16 bytes of every row, in order, moves them
// in place with nothing to wait for but its own loads.  A few rows of many heads and layers: launches and a chain of dependent
// reads (lengths and path, page ids, rows) are what it takes: 6 rows of 32 heads of 128 in 32 layers, bf16 (5 MB),
// 4.7 us; 8 sequences of up to 13 rows, 8 heads, 32 layers (18 MB) 6.2 to 6.7 us.
#include "cache.hpp"

namespace respec {
namespace {

constexpr int kStTree = 5;
constexpr int kFlight = 8;  // rows of a thread under way

// A workgroup takes 256 pieces of K and V in one layer of one sequence; where the path's rows lie within a head, from and to, is
// worked out once, in LDS.
template <int CPR>  // 16-byte pieces per row
__global__ __launch_bounds__(kKeepThreads) void keep_kernel(KeepArgs a) {
  __shared__ int64_t from[kKeepMaxPath], to[kKeepMaxPath];
  __shared__ int bad_path, bad_page;
  const int b = blockIdx.z, i = threadIdx.x;
  const ChunkBatch& c = a.b;
  if (i == 0) bad_path = bad_page = 0;
  const int acc = a.acc_len[b], L = c.kv_len[b];
  const bool in_path = i < a.path_width;
  const int32_t* path = a.path + (int64_t)b * a.path_stride;
  const int node = in_path ? path[i] : 0, before = in_path && i > 0 ? path[i - 1] : -1;  // (the first may be 0)
  __syncthreads();
  const bool known = acc >= -1 && acc < a.path_width;
  const bool mine = in_path && known && i <= acc;
  if (mine && node <= before) bad_path = 1;
  __syncthreads();
  int status = !known || bad_path ? kStTree : 0;
  if (status == 0 && (L < 0 || (acc >= 0 && (long long)L + path[acc] >= (long long)c.table_width * c.page.d))) status = kStCapacity;
  if (status == 0 && mine) {
    const int32_t* table = c.table + (int64_t)b * c.table_stride;
    const uint32_t r0 = (uint32_t)L + (uint32_t)node, r1 = (uint32_t)L + (uint32_t)i;
    const uint32_t p0 = div_by(r0, c.page), p1 = div_by(r1, c.page);
    const int32_t id0 = table[p0], id1 = table[p1];
    if ((uint32_t)id0 >= (uint32_t)c.n_pages || (uint32_t)id1 >= (uint32_t)c.n_pages) bad_page = 1;
    from[i] = id0 * c.page_stride + (int64_t)((uint64_t)(r0 - p0 * c.page.d) * c.row_stride);
    to[i] = id1 * c.page_stride + (int64_t)((uint64_t)(r1 - p1 * c.page.d) * c.row_stride);
  }
  __syncthreads();
  if (status == 0 && bad_page) status = kStPage;
  if (blockIdx.x == 0 && blockIdx.y == 0 && i == 0) {
    if (a.kv_len_out) a.kv_len_out[b] = status == 0 ? L + acc + 1 : L;
    if (c.status) c.status[b] = status;
  }
  const int piece = (int)blockIdx.x * kKeepThreads + i;
  if (status != 0 || piece >= 2 * a.pieces) return;
  const int w = piece >= a.pieces ? piece - a.pieces : piece;
  char* base = (piece >= a.pieces ? c.v : c.k) + (int64_t)blockIdx.y * a.layer_stride + (int64_t)(w / CPR) * c.head_stride + (w % CPR) * 16;
  for (int r0 = 0; r0 <= acc; r0 += kFlight) {
    u32x4 x[kFlight];
#pragma unroll
    for (int u = 0; u < kFlight; ++u)
      if (r0 + u <= acc && from[r0 + u] != to[r0 + u]) x[u] = ld16(base + from[r0 + u]);
#pragma unroll
    for (int u = 0; u < kFlight; ++u)
      if (r0 + u <= acc && from[r0 + u] != to[r0 + u]) *reinterpret_cast<u32x4*>(base + to[r0 + u]) = x[u];
  }
}

}  // namespace

hipError_t launch_keep(int head_bytes, int layers, const KeepArgs& a, hipStream_t s) {
  const dim3 grid((2 * a.pieces + kKeepThreads - 1) / kKeepThreads, layers, a.b.batch);
  switch (head_bytes / 16) {
    case 8: hipLaunchKernelGGL(keep_kernel<8>, grid, dim3(kKeepThreads), 0, s, a); break;
    case 16: hipLaunchKernelGGL(keep_kernel<16>, grid, dim3(kKeepThreads), 0, s, a); break;
    case 32: hipLaunchKernelGGL(keep_kernel<32>, grid, dim3(kKeepThreads), 0, s, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace respec

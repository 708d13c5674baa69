// Causal attention of chunks of new tokens over a paged cache.
//
// out[i][h] = sum_r p_r V[r], p = softmax over r <= L + i of scale q.K[r].
//
// A query row is a (token, head-in-group) pair: the group's heads share a KV head, so its rows are
// one matrix.  A workgroup owns rows_per_wg rows of one sequence and KV head and walks over
// (a split of) the cache rows they see, tile by tile, in one pass: S^T = K Q^T, a running maximum m
// and sum l of the softmax per row, O^T += V^T P^T.
#include "chunk.hpp"

namespace respec {
namespace {

template <int D>
__global__ __launch_bounds__(256) void chunk_attn_f32_kernel(ChunkAttnArgs a) {
  constexpr int ES = 4;
  constexpr int KC = D * ES / 64;      // 64-byte K-chunks of a head row
  constexpr int DB = D / 16;
  constexpr int TK = 32;
  constexpr int PITCH = D * ES + 16;
  constexpr int CPR = D * ES / 16;
  __shared__ __align__(16) unsigned char ks[TK * PITCH], vs[TK * PITCH];

  if ((int)blockIdx.x >= a.wide.items) {
    report_status<256>(a.b, (int)blockIdx.x - a.wide.items, true);
    return;
  }
  const ChunkGeom& ge = a.wide;
  const Item it = find_item(a.b, ge, 1, INT32_MAX, blockIdx.x);
  const ChunkSeq& sq = it.seq;
  if (sq.n == 0) return;
  const int rows = sq.n * a.b.group, row0 = it.rb * ge.rows_per_wg;
  const int limit = block_limit(a, ge, sq, it.rb);
  const int lo = it.split * ge.split_rows;
  if (lo >= limit) return;
  const bool whole = limit <= ge.split_rows;   // the block's only split
  const int hi = whole ? limit : min(limit, lo + ge.split_rows);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c16 = lane & 15, g4 = lane >> 4;
  const int row = row0 + wave * 16 + c16, rowc = min(row, rows - 1);
  const int i = (int)div_by((uint32_t)rowc, a.group), hh = rowc - i * a.b.group;
  const int vis = sq.L + i + 1;
  const int64_t t = sq.t0 + i, head = (int64_t)it.g * a.b.group + hh;
  u32x4 qf[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) qf[c] = ld16(a.q + t * a.q_tok + head * a.q_head + c * 64 + g4 * 16);
  const int32_t* table = a.b.table + (int64_t)it.b * a.b.table_stride;
  const char* kb = a.b.k + (int64_t)it.g * a.b.head_stride;
  const char* vb = a.b.v + (int64_t)it.g * a.b.head_stride;

  float m = kNegInf, l = 0.f;
  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int r0 = lo; r0 < hi; r0 += TK) {
    __syncthreads();
    for (int x = threadIdx.x; x < TK * CPR; x += 256) {
      const int r = x / CPR, c = x % CPR;
      const int64_t at = row_offset(a.b, table, (uint32_t)min(r0 + r, hi - 1)) + c * 16;
      *reinterpret_cast<u32x4*>(ks + r * PITCH + c * 16) = ld16(kb + at);
      *reinterpret_cast<u32x4*>(vs + r * PITCH + c * 16) = ld16(vb + at);
    }
    __syncthreads();
    f32x4 s[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      s[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < KC; ++c)
        s[u] = mma_k64(0.f, *reinterpret_cast<const u32x4*>(ks + (u * 16 + c16) * PITCH + c * 64 + g4 * 16), qf[c], s[u]);
    }
    const int end = min(vis, hi);
    float mx = kNegInf;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[u][e] = r0 + u * 16 + g4 * 4 + e < end ? s[u][e] * a.scale_log2 : kNegInf;
        mx = fmaxf(mx, s[u][e]);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float mn = fmaxf(m, mx), mb = mn == kNegInf ? 0.f : mn;
    const float alpha = exp2f(m - mb);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] *= alpha;
    f32x4 p[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[u][e] = exp2f(s[u][e] - mb);
        l += p[u][e];
      }
    // V^T P^T.  A masked weight is zero, and zero times a NaN or an infinity is not: in a tile that
    // some row does not see whole, values that are not finite stay out of the products and are added
    // afterwards for the rows that see them.
    const bool masked = __any(r0 + TK > end);
    bool odd = false;
    auto value = [&](int key, int d) {
      float v = Elem<float>::to_f32(vs + key * PITCH, d);
      if (masked && !(fabsf(v) < __builtin_huge_valf())) {
        odd = true;
        v = 0.f;
      }
      return v;
    };
#pragma unroll
    for (int d = 0; d < DB; ++d) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        u32x4 vf;
#pragma unroll
        for (int e = 0; e < 4; ++e) vf[e] = __float_as_uint(value(u * 16 + g4 * 4 + e, d * 16 + c16));
        o[d] = mma_k64(0.f, vf, __builtin_bit_cast(u32x4, p[u]), o[d]);
      }
    }
    if (__any(odd)) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
        for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = u * 16 + k4 * 4 + e;
            const float pk = __shfl(p[u][e], k4 * 16 + c16, 64);
            if (r0 + key >= end) continue;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const float v = Elem<float>::to_f32(vs + key * PITCH, d * 16 + g4 * 4 + x);
                if (!(fabsf(v) < __builtin_huge_valf())) o[d][x] += pk * v;
              }
          }
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (row >= rows) return;
  if (whole) {
    char* to = a.out + t * a.o_tok + head * a.o_head;
    const float inv = 1.f / l;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) Elem<float>::store(to, d * 16 + g4 * 4 + e, o[d][e] * inv);
  } else {
    const int64_t hq = (int64_t)a.b.n_kv_heads * a.b.group;
    const int64_t pr = ((int64_t)it.split * a.b.total_new + t) * hq + head;
#pragma unroll
    for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(a.part_o + pr * D + d * 16 + g4 * 4) = o[d];
    if (g4 == 0) {
      a.part_m[pr] = m;
      a.part_l[pr] = l;
    }
  }
}

// out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over a row's splits, M = max_s m_s.  A row (token
// and head) is joined by WPR waves, each a part of its splits, eight at a time; rows of one split are
// written already.
template <typename T, int D, int WPR>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkAttnArgs a) {
  constexpr int E = D / 64, RPW = 4 / WPR;  // columns per lane, rows per workgroup
  __shared__ float part[4][D];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, w = wave % WPR;
  int b;
  const ChunkSeq sq = seq_of_token(a.b, blockIdx.x, b);
  const int hq = a.b.n_kv_heads * a.b.group, h = (int)blockIdx.y * RPW + wave / WPR;
  const ChunkGeom& ge = sq.n * a.b.group <= a.few_rows ? a.few : a.wide;
  int ns = 0;
  if (sq.n > 0 && h < hq) {
    const int hh = h - (int)div_by((uint32_t)h, a.group) * a.b.group, i = (int)blockIdx.x - sq.t0;
    const int limit = block_limit(a, ge, sq, (i * a.b.group + hh) / ge.rows_per_wg);
    ns = (limit - 1) / ge.split_rows + 1;  // (at most 64)
  }
  if (WPR == 1 && ns <= 1) return;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  if (ns > 1) {
    const int64_t step = (int64_t)a.b.total_new * hq, pr = (int64_t)blockIdx.x * hq + h;
    const float ms = lane < ns ? a.part_m[lane * step + pr] : kNegInf, ls = lane < ns ? a.part_l[lane * step + pr] : 0.f;
    const float M = wave_max(ms);
    float wt = ms == kNegInf ? 0.f : exp2f(ms - M);
    const float lt = wave_sum(wt * ls);
    wt /= lt;
    const float* o = a.part_o + pr * D + lane * E;
    for (int s0 = w * 8; s0 < ns; s0 += WPR * 8) {
      float x[8][E];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float* q = o + min(s0 + u, ns - 1) * step * D;
        if constexpr (E == 2) *reinterpret_cast<float2*>(x[u]) = *reinterpret_cast<const float2*>(q);
        else x[u][0] = *q;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float ws = __shfl(wt, min(s0 + u, 63), 64);
        if (s0 + u < ns) {
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] += ws * x[u][e];
        }
      }
    }
  }
  if constexpr (WPR > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) part[wave][lane * E + e] = acc[e];
    __syncthreads();
    if (w != 0 || ns <= 1) return;
#pragma unroll
    for (int x = 1; x < WPR; ++x)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += part[wave + x][lane * E + e];
  }
  char* to = a.out + (int64_t)blockIdx.x * a.o_tok + (int64_t)h * a.o_head;
#pragma unroll
  for (int e = 0; e < E; ++e) Elem<T>::store(to, lane * E + e, acc[e]);
}

template <typename T, int D>
hipError_t go_merge(const ChunkAttnArgs& a, hipStream_t s) {
  const int hq = a.b.n_kv_heads * a.b.group;
  // many splits: a row's are read by four waves at once
  if (max(a.few.nsplit, a.wide.nsplit) > 16)
    hipLaunchKernelGGL((chunk_merge_kernel<T, D, 4>), dim3(a.b.total_new, hq), dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((chunk_merge_kernel<T, D, 1>), dim3(a.b.total_new, (hq + 3) / 4), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn_f32(int head_dim, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  const dim3 grid(a.wide.items + (status ? a.b.batch : 0));
  if (head_dim == 128) hipLaunchKernelGGL(chunk_attn_f32_kernel<128>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(chunk_attn_f32_kernel<64>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_chunk_merge(int dtype, int head_dim, const ChunkAttnArgs& a, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? go_merge<bf16_t, 128>(a, s) : go_merge<bf16_t, 64>(a, s);
  return head_dim == 128 ? go_merge<float, 128>(a, s) : go_merge<float, 64>(a, s);
}

}  // namespace respec

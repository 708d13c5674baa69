// Causal attention of chunks of new tokens over a paged cache.
//
// out[i][h] = sum_r p_r V[r], p = softmax over r <= L + i of scale q.K[r].
//
// A query row is a (token, head-in-group) pair: the group's heads share a KV head, so its rows are
// one matrix.  A workgroup owns rows_per_wg rows of one sequence and KV head and walks over
// (a split of) the cache rows they see, tile by tile, in one pass: S^T = K Q^T, a running maximum m
// and sum l of the softmax per row, O^T += V^T P^T.
#include "q8.hpp"

namespace respec {
namespace {

// float32: four waves of 16 query rows, v_mfma_f32_16x16x4 (mma_k64 in common.hpp).  S^T = K Q^T leaves, in
// lane l, the scores of row l % 16 with keys 4 (l / 16) .. + 3 of 16, which are the B operand of O^T += V^T P^T as
// they stand.  A tile of 32 cache rows is fetched into registers while the tile before is worked on, then goes to
// one of two LDS buffers, K rows as they are and V transposed.  Measured: 1500 tokens, 16 heads of 64, 68 us and 6 us for
// the merge (4.6 GFLOP: 68 TFLOP/s, where a large float32 matrix product reaches 154): the matrix cores, 32 clocks per
// product of 2048 operations, are busy 45% of the cycles; causal blocks are unequal work over one round of workgroups, and
// 40% of the LDS cycles are conflicts (see fetch).  One token of 4 heads over 512 rows, 6.9 us.
// Q8: the cache holds e4m3 values with a scale per block of rows; four of them at a time become what a piece is otherwise.
template <int D>
struct F32Shape {
  static constexpr int TK = 32;
  static constexpr int KP = D * 4 + 16;  // bytes between K rows
  static constexpr int VP = TK + 4;      // floats between V columns
};

// One pass over item x.  (Q8) V is taken in units of 2^UNIT (see kUnit in q8.hpp); in units of more than 1, the rows that the pass before
// found large, and did not store (`again`: 16 bits of each wave), are stored alone.  Returns whether this one found any.
template <int D, bool Q8, int UNIT>
__device__ __forceinline__ bool f32_rows_pass(const ChunkAttnArgs& a, int x, int lane, int wave,
                                              unsigned char (&k_lds)[2][F32Shape<D>::TK * F32Shape<D>::KP],
                                              float (&v_lds)[2][D * F32Shape<D>::VP], uint32_t (&again)[4]) {
  constexpr int KC = D / 16;           // 64-byte K-chunks of a head row
  constexpr int DB = D / 16;
  constexpr int TK = F32Shape<D>::TK, KP = F32Shape<D>::KP, VP = F32Shape<D>::VP;
  constexpr int NP = TK * D / 4 / 256;  // 16-byte pieces of a tile per thread
  const ChunkGeom& ge = a.wide;
  const Item it = find_item(a.b, ge, 1, INT32_MAX, x, lane);
  const ChunkSeq& sq = it.seq;
  if (sq.n == 0) return false;
  const int rows = sq.n * a.b.group, row0 = it.rb * ge.rows_per_wg;
  const int limit = block_limit(a, ge, sq, it.rb);
  const int lo = it.split * ge.split_rows;
  if (lo >= limit) return false;
  const bool whole = limit <= ge.split_rows;  // the block's only split
  const int hi = whole ? limit : min(limit, lo + ge.split_rows);
  const int c16 = lane & 15, g4 = lane >> 4;
  const int row = row0 + wave * 16 + c16, rowc = min(row, rows - 1);
  const int i = (int)div_by((uint32_t)rowc, a.group), hh = rowc - i * a.b.group;
  const int end = min(sq.L + i + 1, hi);  // cache rows that this lane's row sees end here, within the split
  const int64_t t = sq.t0 + i, head = (int64_t)it.g * a.b.group + hh;
  // cache rows that every row of the wave sees end here
  const int unmasked = __builtin_amdgcn_readfirstlane(
      min(sq.L + (int)div_by((uint32_t)min(row0 + wave * 16, rows - 1), a.group) + 1, hi));
  u32x4 qf[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) qf[c] = ld16(a.q + t * a.q_tok + head * a.q_head + c * 64 + g4 * 16);
  const int32_t* table = a.b.table + (int64_t)it.b * a.b.table_stride;
  const char* kb = a.b.k + (int64_t)it.g * a.b.head_stride;
  const char* vb = a.b.v + (int64_t)it.g * a.b.head_stride;

  // A thread brings every eighth 16-byte piece of one row: one address per tile for all of them.  The transposed stores of a
  // wave are of 32 rows of two columns that lie 4 VP = 144 words apart, 16 of the 64 banks, so 16 banks are met twice.  The
  // row's page id is read another tile ahead.
  const int my_row = lane % TK, my_piece = wave * (64 / TK) + lane / TK;
  u32x4 kp[NP], vp[NP];
  uint32_t k_byte = 127, v_byte = 127;  // (exponents of the row's scales)
  int32_t id = 0;
  auto row_of = [&](int r0) { return (uint32_t)min(r0 + my_row, hi - 1); };
  auto fetch_id = [&](int r0) { id = table[div_by(row_of(r0), a.b.page)]; };
  auto fetch = [&](int r0) {
    if constexpr (Q8) {
      const int64_t off = offset_in(a.b, id, row_of(r0)) + my_piece * 4;
      const int64_t at = scale_offset(a, id, row_of(r0), it.g);
      k_byte = a.q8.k[at];
      v_byte = a.q8.v[at];
#pragma unroll
      for (int x = 0; x < NP; ++x) {
        kp[x].x = *reinterpret_cast<const uint32_t*>(kb + off + x * (256 / TK * 4));
        vp[x].x = *reinterpret_cast<const uint32_t*>(vb + off + x * (256 / TK * 4));
      }
    } else {
      const int64_t off = offset_in(a.b, id, row_of(r0)) + my_piece * 16;
#pragma unroll
      for (int x = 0; x < NP; ++x) {
        kp[x] = ld16(kb + off + x * (256 / TK * 16));
        vp[x] = ld16(vb + off + x * (256 / TK * 16));
      }
    }
  };
  float m = kNegInf, l = 0.f;
  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  fetch_id(lo);
  fetch(lo);
  fetch_id(lo + TK);
  int buf = 0;
  for (int r0 = lo; r0 < hi; r0 += TK, buf ^= 1) {
    unsigned char* ks = k_lds[buf];
    float* vs = v_lds[buf];
    if constexpr (Q8) {
#pragma unroll
      for (int x = 0; x < NP; ++x) {
        kp[x] = q8_floats(kp[x].x, k_byte);
        vp[x] = q8_floats(vp[x].x, v_byte - UNIT);
      }
    }
#pragma unroll
    for (int x = 0; x < NP; ++x) {
      const int c = my_piece + x * (256 / TK);
      *reinterpret_cast<u32x4*>(ks + my_row * KP + c * 16) = kp[x];
#pragma unroll
      for (int e = 0; e < 4; ++e) vs[(c * 4 + e) * VP + my_row] = __uint_as_float(vp[x][e]);
    }
    // (one barrier per tile: a wave that is here again has seen every wave past the tile between)
    __syncthreads();
    if (r0 + TK < hi) {
      fetch(r0 + TK);
      fetch_id(r0 + 2 * TK);
    }
    // (neighbouring products are of different sums: one that waits for the product before it costs more)
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      f32x4 kf[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) kf[u] = *reinterpret_cast<const f32x4*>(ks + (u * 16 + c16) * KP + c * 64 + g4 * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          s[u] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[u][e], __uint_as_float(qf[c][e]), s[u], 0, 0, 0);
    }
    f32x4 vf[2][DB];  // (under way beside the weights)
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int d = 0; d < DB; ++d) vf[u][d] = *reinterpret_cast<const f32x4*>(vs + (d * 16 + c16) * VP + u * 16 + g4 * 4);
    const bool masked = r0 + TK > unmasked;  // (uniform) some row of the wave does not see the whole tile
    float mx = kNegInf;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s[u][e] *= a.scale_log2;
        if (masked) s[u][e] = r0 + u * 16 + g4 * 4 + e < end ? s[u][e] : kNegInf;
        mx = fmaxf(mx, s[u][e]);
      }
    mx = fmaxf(mx, xchg<4>(mx));
    mx = fmaxf(mx, xchg<5>(mx));
    const float mn = fmaxf(m, mx), mb = mn == kNegInf ? 0.f : mn;
    if (__any(mn > m)) {
      const float alpha = __builtin_amdgcn_exp2f(m - mb);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] *= alpha;
    }
    m = mn;
    f32x4 p[2];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[u][e] = __builtin_amdgcn_exp2f(s[u][e] - mb);
        l += p[u][e];
      }
    // V^T P^T.  A masked weight is zero, and zero times a NaN or an infinity is not: in a tile that
    // some row does not see whole, values that are not finite stay out of the products and are added
    // afterwards for the rows that see them.
    bool odd = false;
    if (masked) {
      uint32_t top = 0;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) top = max(top, __float_as_uint(vf[u][d][e]) & 0x7FFFFFFFu);
      odd = __any(top >= 0x7F800000u);
      if (odd) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) vf[u][d][e] = fabsf(vf[u][d][e]) < __builtin_huge_valf() ? vf[u][d][e] : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[u][d][e], p[u][e], o[d], 0, 0, 0);
    if (odd) {  // whatever the weight, they make a NaN or an infinity of the sum
      for (int key = 0; key < TK; ++key)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float v = vs[(d * 16 + g4 * 4 + e) * VP + key];
            o[d][e] += r0 + key < end && !(fabsf(v) < __builtin_huge_valf()) ? v : 0.f;
          }
    }
  }
  l += xchg<4>(l);
  l += xchg<5>(l);
  bool mine = row < rows;
  if constexpr (Q8 && UNIT == 0) {
    float size = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) add_sizes(size, o[d]);
    uint64_t large = __ballot(mine && !(size < kLarge));
    large |= large >> 32;
    if (lane == 0) again[wave] = (uint32_t)(large | large >> 16) & 0xFFFFu;
    wave_lds_sync();
  }
  if constexpr (Q8) mine = mine && (again[wave] >> c16 & 1) == (UNIT != 0);  // (queries may lie in the output's place: a row is stored once)
  float to_o = 1.f;
  if constexpr (UNIT != 0) {
    if (whole) to_o = __builtin_amdgcn_ldexpf(1.f, UNIT);
    else move_unit(UNIT, m, l, to_o);
  }
  if (mine && whole) {
    char* to = a.out + t * a.o_tok + head * a.o_head;
    const float inv = 1.f / l;
#pragma unroll
    for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(to + (d * 16 + g4 * 4) * 4) = o[d] * inv * to_o;
  } else if (mine) {
    const int64_t hq = (int64_t)a.b.n_kv_heads * a.b.group;
    const int64_t pr = ((int64_t)it.split * a.b.total_new + t) * hq + head;
#pragma unroll
    for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(a.part_o + pr * D + d * 16 + g4 * 4) = o[d] * to_o;
    if (g4 == 0) {
      a.part_m[pr] = m;
      a.part_l[pr] = l;
    }
  }
  if constexpr (!Q8 || UNIT != 0) return false;
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(again[0] | again[1] | again[2] | again[3]) != 0;
}

template <int D, bool Q8>
__global__ __launch_bounds__(kAttnF32Threads) void chunk_attn_f32_kernel(ChunkAttnArgs a) {
  using G = F32Shape<D>;
  __shared__ __align__(16) unsigned char k_lds[2][G::TK * G::KP];
  __shared__ __align__(16) float v_lds[2][D * G::VP];
  __shared__ uint32_t again[4];
  if ((int)blockIdx.x >= a.wide.items) {
    report_status<256>(a.b, (int)blockIdx.x - a.wide.items, true);
    return;
  }
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (!f32_rows_pass<D, Q8, 0>(a, (int)blockIdx.x, (int)threadIdx.x & 63, wave, k_lds, v_lds, again)) return;
  if constexpr (Q8) {
    const Again g = again_from((int)blockIdx.x, wave);
    f32_rows_pass<D, Q8, kUnit>(g.a, g.x, lane_id(), g.wave, k_lds, v_lds, again);
  }
}

constexpr int kMergeMany = 16;  // splits of a sequence above which a row has a workgroup of the merge

// out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s over a row's splits, M = max_s m_s.  A row is a (token, head)
// pair; D / 4 lanes take four of its columns each.  Rows of few splits: such a group of lanes per row, four splits at a
// time with a running M.  Rows of more: all the groups of the workgroup take splits of one row, each all of its own at
// once, and are joined through LDS.  Rows of one split are written already.
//
// Bound by the partials' bytes where there are many rows: 512 tokens of 32 heads of 128 in 4 splits (38 MB), 9.8 us, 3.9 TB/s;
// 1500 tokens of 16 heads of 64, 5.8 to 6.8 us (a wave per row with a lane per split: 11.8; workgroups per row from 5 splits
// on: 103 us for the whole call, not 69).  One token of 28 heads in 64 splits (0.9 MB): 4.4 us (four at a time, all groups: 5.8).
template <typename T, int D>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkAttnArgs a) {
  constexpr int G = D / 4, NG = 256 / G;
  __shared__ __align__(16) float part[NG][D];
  const int c = threadIdx.x % G, g = threadIdx.x / G, lane = threadIdx.x & 63;
  int b;
  const ChunkSeq sq = seq_of_token(a.b, blockIdx.x, b);
  if (sq.n == 0) return;
  const int hq = a.b.n_kv_heads * a.b.group, i = (int)blockIdx.x - sq.t0;
  const ChunkGeom& ge = sq.n * a.b.group <= a.few_rows ? a.few : a.wide;
  if (sq.L + sq.n <= ge.split_rows) return;
  const bool many = (int)div_by((uint32_t)(sq.L + sq.n - 1), ge.split) >= kMergeMany;  // (1 + that: the splits)
  const int per = many ? 1 : NG;
  const int64_t step = (int64_t)a.b.total_new * hq;  // rows between a row's splits
  for (int h0 = (int)blockIdx.y * per; h0 < hq; h0 += gridDim.y * per) {
    const int h = many ? h0 : min(h0 + g, hq - 1), hh = h - (int)div_by((uint32_t)h, a.group) * a.b.group;
    const int limit = block_limit(a, ge, sq, row_block(ge, i * a.b.group + hh));
    const int ns = (int)div_by((uint32_t)(limit - 1), ge.split) + 1;  // (at most 64)
    if (ns <= 1) continue;                           // (where `many`: the whole workgroup)
    const int64_t pr = (int64_t)blockIdx.x * hq + h;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (many) {
      constexpr int U = 64 / NG;
      f32x4 o[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g + u * NG < ns) o[u] = *reinterpret_cast<const f32x4*>(a.part_o + ((g + u * NG) * step + pr) * D + c * 4);
      const float ms = lane < ns ? a.part_m[lane * step + pr] : kNegInf, ls = lane < ns ? a.part_l[lane * step + pr] : 0.f;
      const float M = wave_max(ms);
      float wt = ms == kNegInf ? 0.f : exp2f(ms - M);  // of split `lane`
      wt /= wave_sum(wt * ls);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float w = __shfl(wt, g + u * NG, 64);
        if (g + u * NG < ns) {
#pragma unroll
          for (int x = 0; x < 4; ++x) acc[x] = __builtin_fmaf(w, o[u][x], acc[x]);
        }
      }
      __syncthreads();  // (the row before has been read)
      *reinterpret_cast<f32x4*>(&part[g][c * 4]) = acc;
      __syncthreads();
      if (g != 0) continue;
#pragma unroll
      for (int k = 1; k < NG; ++k) acc += *reinterpret_cast<const f32x4*>(&part[k][c * 4]);
    } else {
      float M = kNegInf, l = 0.f;
      for (int s0 = 0; s0 < ns; s0 += 4) {
        f32x4 o[4];
        float m[4], lw[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int64_t r = min(s0 + u, ns - 1) * step + pr;
          o[u] = *reinterpret_cast<const f32x4*>(a.part_o + r * D + c * 4);
          m[u] = a.part_m[r];
          lw[u] = a.part_l[r];
        }
        const float to = fmaxf(fmaxf(fmaxf(M, m[0]), fmaxf(m[1], m[2])), m[3]), ref = to == kNegInf ? 0.f : to;
        const float e = exp2f(M - ref);
        l *= e;
        acc *= e;
        M = to;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (s0 + u < ns) {
            const float w = m[u] == kNegInf ? 0.f : exp2f(m[u] - ref);
            l = __builtin_fmaf(w, lw[u], l);
#pragma unroll
            for (int x = 0; x < 4; ++x) acc[x] = __builtin_fmaf(w, o[u][x], acc[x]);
          }
        }
      }
      acc /= l;
      if (h0 + g >= hq) continue;
    }
    char* to = a.out + (int64_t)blockIdx.x * a.o_tok + (int64_t)h * a.o_head;
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4*>(to + c * 16) = acc;
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x) Elem<T>::store(to, c * 4 + x, acc[x]);
    }
  }
}

template <typename T, int D>
hipError_t go_merge(const ChunkAttnArgs& a, hipStream_t s) {
  // rows of many tokens have several heads to a workgroup
  const int hq = a.b.n_kv_heads * a.b.group, per = max(a.few.nsplit, a.wide.nsplit) > kMergeMany ? 1 : 1024 / D;
  const int y = max(1, min((hq + per - 1) / per, 16384 / a.b.total_new));
  hipLaunchKernelGGL((chunk_merge_kernel<T, D>), dim3(a.b.total_new, y), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn_f32(int head_dim, bool q8, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  const dim3 grid(a.wide.items + (status ? a.b.batch : 0));
  if (q8 && head_dim == 128) hipLaunchKernelGGL((chunk_attn_f32_kernel<128, true>), grid, dim3(kAttnF32Threads), 0, s, a);
  else if (q8) hipLaunchKernelGGL((chunk_attn_f32_kernel<64, true>), grid, dim3(kAttnF32Threads), 0, s, a);
  else if (head_dim == 128) hipLaunchKernelGGL((chunk_attn_f32_kernel<128, false>), grid, dim3(kAttnF32Threads), 0, s, a);
  else hipLaunchKernelGGL((chunk_attn_f32_kernel<64, false>), grid, dim3(kAttnF32Threads), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_chunk_merge(int dtype, int head_dim, const ChunkAttnArgs& a, hipStream_t s) {
  if (dtype == 1) return head_dim == 128 ? go_merge<bf16_t, 128>(a, s) : go_merge<bf16_t, 64>(a, s);
  return head_dim == 128 ? go_merge<float, 128>(a, s) : go_merge<float, 64>(a, s);
}

}  // namespace respec

// Keys and values of new tokens into the pages of an 8-bit cache.
//
// A block of 2^shift rows of one KV head has one power-of-two scale, 2^k with the largest new magnitude at most 448 2^k, no
// smaller than the scale that earlier rows of the block have.  Every new row is read once, in 2 or 4 bytes per
// element, and written in one, so memory bounds it.
//
// A wave takes 16 rows of a block, for K or for V, all of them in registers: a lane has D / 64 segments of 16 elements, which it
// reads in 16-byte pieces and writes as one.  The waves of a larger block meet once, in LDS, for the largest magnitude.
// Earlier rows are read only where their scale grows.
//
// 8057 tokens of 32 heads of 128, bf16, blocks of 32 rows (198 MB): 41 to 43 us, 4.6 to 4.8 TB/s, as a large copy.  96 sequences of one
// token each, 8 heads: 4.5 to 5.4 us, which is a launch and three dependent reads (lengths, page id, scale).  Every wave walks over the
// batch for its block: 1024 sequences 21 us, 4096 175, 16384 2241 (calls).
#include "q8.hpp"

namespace respec {
namespace {

// Block y of the batch's list of blocks that new rows touch, by a whole wave (n = 0: none).
struct BlockItem {
  ChunkSeq seq;
  int b, blk;
};
__device__ __forceinline__ BlockItem find_block(const ChunkBatch& c, int shift, int y) {
  const int lane = (int)(threadIdx.x & 63);
  BlockItem it{ChunkSeq{0, 0, 0, 0}, 0, 0};
  for (int b0 = 0; b0 < c.batch; b0 += 64) {
    ChunkSeq s{0, 0, 0, 0};
    int blocks = 0;
    if (b0 + lane < c.batch) {
      s = chunk_seq(c, b0 + lane);
      if (s.n > 0) blocks = ((s.L + s.n - 1) >> shift) - (s.L >> shift) + 1;
    }
    int incl = blocks;
    if (c.batch > 1) incl = wave_prefix_sum(incl);
    const uint64_t past = __ballot(y < incl);
    if (past) {
      const int l = __builtin_ctzll(past);
      blocks = __builtin_amdgcn_readlane(blocks, l);
      y -= __builtin_amdgcn_readlane(incl, l) - blocks;
      if ((uint32_t)y >= (uint32_t)blocks) return it;  // (offsets that overlap: more blocks than 32 bits count)
      it.b = b0 + l;
      it.seq = ChunkSeq{__builtin_amdgcn_readlane(s.t0, l), __builtin_amdgcn_readlane(s.n, l), __builtin_amdgcn_readlane(s.L, l), 0};
      it.blk = (it.seq.L >> shift) + y;
      return it;
    }
    y -= __builtin_amdgcn_readlane(incl, 63);
  }
  return it;
}

__device__ __forceinline__ uint32_t finite_bits(uint32_t f) {  // magnitude's bits of a finite float, else 0
  f &= 0x7FFFFFFFu;
  return f < 0x7F800000u ? f : 0u;
}
template <int LEVEL>
__device__ __forceinline__ uint32_t max_level(uint32_t v) {
  return max(v, (uint32_t)xchg<LEVEL>((int)v));
}

template <int ES, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void append_q8_kernel(AppendQ8Args a) {
  constexpr int SEGS = D / 64;      // segments of a lane
  constexpr int SPR = D / 16;       // segments of a row
  constexpr int NP = ES;            // 16-byte pieces of a segment (16 elements)
  if ((int)blockIdx.x >= a.wgs) {
    report_status<64 * WAVES>(a.b, (int)blockIdx.x - a.wgs, false);
    return;
  }
  __shared__ uint32_t tops[WAVES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int shift = a.q8.shift, per = 1 << (shift - 4);  // waves of a block
  const uint32_t x = blockIdx.x * (uint32_t)(WAVES / per) + (uint32_t)(wave / per);
  const uint32_t y = div_by(x, a.per_block);
  const int rest = (int)(x - y * a.per_block.d), g = rest >> 1;
  const bool of_v = rest & 1;
  const BlockItem it = find_block(a.b, shift, (int)y);
  const ChunkSeq& s = it.seq;
  const int first = it.blk << shift, row0 = first + (wave % per) * 16;  // of the block, of this wave
  const int end = s.L + s.n;

  u32x4 raw[SEGS][NP];
  bool fresh[SEGS];
  const char* from = (of_v ? a.v_new : a.k_new) + (int64_t)g * (of_v ? a.v_head : a.k_head);
  const int64_t step = of_v ? a.v_tok : a.k_tok;
#pragma unroll
  for (int u = 0; u < SEGS; ++u) {
    const int seg = u * 64 + lane, r = row0 + seg / SPR;
    fresh[u] = r >= s.L && r < end;
    if (fresh[u]) {
      const char* p = from + (int64_t)(s.t0 + (r - s.L)) * step + seg % SPR * (16 * ES);
#pragma unroll
      for (int i = 0; i < NP; ++i) raw[u][i] = ld16(p + i * 16);
    }
  }
  char* codes = nullptr;
  uint8_t* scale = nullptr;
  if (s.n > 0) {
    const uint32_t p = div_by((uint32_t)first, a.b.page);
    const int32_t id = a.b.table[(int64_t)it.b * a.b.table_stride + p];
    if ((uint32_t)id < (uint32_t)a.b.n_pages) {  // (a page out of range is left out and reported)
      codes = (of_v ? a.b.v : a.b.k) + id * a.b.page_stride + (int64_t)g * a.b.head_stride +
              (int64_t)((uint64_t)(row0 - (int)(p * a.b.page.d)) * a.b.row_stride);
      scale = (of_v ? a.q8.v : a.q8.k) + scale_offset(a.b, a.q8, id, (uint32_t)first, g);
    }
  }
  int was = 0;  // exponent byte of the earlier rows
  if (scale && first < s.L) was = *scale;
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < SEGS; ++u)
    if (fresh[u]) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (ES == 2) top = max(top, max(finite_bits(raw[u][i][e] << 16), finite_bits(raw[u][i][e] & 0xFFFF0000u)));
          else top = max(top, finite_bits(raw[u][i][e]));
        }
    }
  top = max_level<5>(max_level<4>(max_level<3>(max_level<2>(max_level<1>(max_level<0>(top))))));
  if (shift > 4) {
    if (lane == 0) tops[wave] = top;
    __syncthreads();
    const int w0 = wave / per * per;
    for (int w = 0; w < per; ++w) top = max(top, tops[w0 + w]);
  }
  if (!codes) return;
  // the least k with top <= 448 2^k: top = m 2^e, 1 <= m < 2, and 448 = 1.75 2^8
  const int k = max(-126, (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u));
  const int byte = max(k + 127, was);
  if ((wave % per) == 0 && lane == 0 && byte != was) *scale = (uint8_t)byte;
  const bool grown = first < s.L && byte > was;  // (uniform)
#pragma unroll
  for (int u = 0; u < SEGS; ++u) {
    const int seg = u * 64 + lane, r = row0 + seg / SPR;
    char* to = codes + (int64_t)((uint64_t)(seg / SPR) * a.b.row_stride) + seg % SPR * 16;
    u32x4 y;
    if (fresh[u]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          uint32_t b;
          if constexpr (ES == 2) {
            const uint32_t w = raw[u][i / 2][(i % 2) * 2 + e / 2];
            b = e & 1 ? w & 0xFFFF0000u : w << 16;
          } else {
            b = raw[u][i][e];
          }
          f[e] = __builtin_amdgcn_ldexpf(__uint_as_float(b), 127 - byte);
        }
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
        y[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], c, true);
      }
      *reinterpret_cast<u32x4*>(to) = y;
    } else if (grown && r < s.L) {
      const u32x4 old = ld16(to);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const q8_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(old[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(old[i], true);
        const int e = was - byte;
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_ldexpf(lo.x, e), __builtin_amdgcn_ldexpf(lo.y, e), 0, false);
        y[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_ldexpf(hi.x, e), __builtin_amdgcn_ldexpf(hi.y, e), c, true);
      }
      *reinterpret_cast<u32x4*>(to) = y;
    }
  }
}

template <int ES, int D>
hipError_t go(const AppendQ8Args& a, hipStream_t s) {
  const dim3 grid((unsigned)a.wgs + (a.b.status ? a.b.batch : 0));
  if (a.q8.shift == 7) hipLaunchKernelGGL((append_q8_kernel<ES, D, 8>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((append_q8_kernel<ES, D, kAppendQ8Waves>), grid, dim3(64 * kAppendQ8Waves), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append_q8(int es, int head_dim, const AppendQ8Args& a, hipStream_t s) {
  if (es == 2) return head_dim == 128 ? go<2, 128>(a, s) : go<2, 64>(a, s);
  return head_dim == 128 ? go<4, 128>(a, s) : go<4, 64>(a, s);
}

}  // namespace respec

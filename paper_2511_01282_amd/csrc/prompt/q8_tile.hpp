// Tiles of an 8-bit paged cache (see q8.hpp), for the bf16 attention kernels (gfx950).
//
// Sixteen rows from a multiple of 16 lie in one page and share a scale (scale blocks are multiples of 16 rows, pages of
// blocks), so a wave's rows come 16 at a time from one address, whole also where the sequence ends inside them (what
// is behind the end is masked).  bf16 holds e4m3 values times a power of two exactly.
#pragma once

#include "chunk_tile.hpp"
#include "q8.hpp"

namespace respec {

__device__ __forceinline__ float q8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Page ids and scales of 16 rows each, a lane for each: rows r0 .. r0 + 15 of the sequence (r0 a multiple of 16, from the
// sequence's end on its last 16 instead).
struct Q8Window {
  int32_t id;
  uint32_t k, v;  // exponent bytes
  __device__ __forceinline__ void fill(const ChunkAttnArgs& a, const Item& it, int r0, int hi_row) {
    const uint32_t r = (uint32_t)max(0, min(r0, (hi_row - 1) & ~15));
    id = a.b.table[(int64_t)it.b * a.b.table_stride + div_by(r, a.b.page)];
    const int64_t at = scale_offset(a, id, r, it.g);
    k = a.q8.k[at];
    v = a.q8.v[at];
  }
};

// 16 rows of K and V on their way through a wave's registers into tiles of bf16 (as chunk_tile.hpp's).
template <int D>
struct Q8Rows {
  static constexpr int PPR = D / 16, N = D / 64;  // 16-byte pieces per row, of a lane
  u32x4 k[N], v[N];
  float k_scale, v_scale;
  __device__ __forceinline__ void fetch(const ChunkAttnArgs& a, int g, const Q8Window& w, int entry, int r0, int lane) {
    const int32_t id = __builtin_amdgcn_readlane(w.id, entry);
    k_scale = q8_scale((uint32_t)__builtin_amdgcn_readlane((int)w.k, entry));
    v_scale = q8_scale((uint32_t)__builtin_amdgcn_readlane((int)w.v, entry));
    const int64_t off = offset_in(a.b, id, (uint32_t)r0) + (int64_t)g * a.b.head_stride;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int p = u * 64 + lane;
      const uint32_t in = (uint32_t)(p / PPR) * a.b.row_stride + (uint32_t)(p % PPR * 16);
      k[u] = ld16(a.b.k + off + in);
      v[u] = ld16(a.b.v + off + in);
    }
  }
  __device__ __forceinline__ void to_lds(unsigned char* k_tile, unsigned char* v_tile, int row0, int lane) const {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int p = u * 64 + lane, r = row0 + p / PPR, c = 2 * (p % PPR);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        *reinterpret_cast<u32x4*>(k_tile + r * D * 2 + ((c + h) ^ k_chunk<D>(r)) * 16) = q8_bf16(u32x2{k[u][2 * h], k[u][2 * h + 1]}, k_scale);
        *reinterpret_cast<u32x4*>(v_tile + r * D * 2 + ((c + h) ^ v_chunk<D>(r)) * 16) = q8_bf16(u32x2{v[u][2 * h], v[u][2 * h + 1]}, v_scale);
      }
    }
  }
};

// Tiles of 32 rows of D codes, their 16-byte chunks permuted inside the row: reads of 16 rows (K), or of two chunks of 8 rows
// (V), touch every bank once.
template <int D>
__device__ __forceinline__ int k8_chunk(int r) {
  return D == 128 ? ((r >> 1) & 7) : ((r >> 2) & 3);
}
template <int D>
__device__ __forceinline__ int v8_chunk(int r) {
  return D == 128 ? (r & 2) + ((r & 8) >> 1) : ((r & 8) >> 2);
}

// K fragments of 32 keys (A operand: lane l holds key l & 31, elements 32 (ks / 2) + 16 (l / 32) + 8 (ks % 2) ..).
template <int D>
__device__ __forceinline__ void read_k8(const unsigned char* tile, int lane, float scale, u32x4 (&kf)[D / 16]) {
  const int r32 = lane & 31, hi = lane >> 5;
#pragma unroll
  for (int kk = 0; kk < D / 32; ++kk) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(tile + r32 * D + (((2 * kk + hi) ^ k8_chunk<D>(r32)) << 4));
    kf[2 * kk] = q8_bf16(u32x2{x.x, x.y}, scale);
    kf[2 * kk + 1] = q8_bf16(u32x2{x.z, x.w}, scale);
  }
}

// V^T fragments of 32 keys as read_v's, by transposing reads: lane j of a 16-lane group addresses columns 8 (j % 2) .. of row
// j / 2 of eight and receives column j of them.
template <int D>
__device__ __forceinline__ void read_v8(const unsigned char* tile, int lane, float s0, float s1, u32x4 (&vf)[D / 32][2]) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
  const int lr = lane & 15, dh = (lane >> 4) & 1, hi = lane >> 5, i = lr >> 1;
  const int r = 4 * hi + i + (i & 4);  // rows 4 hi .. + 3 and 8 + 4 hi .. + 3 (and 16 further: the same permutation)
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) {
      const unsigned char* p = tile + (16 * k2 + r) * D + (((2 * db + dh) ^ v8_chunk<D>(r)) << 4) + (lr & 1) * 8;
      const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)p));
      vf[db][k2] = q8_bf16(x, k2 ? s1 : s0);
    }
}

// add_not_finite() over a tile of codes.
template <int D, int G>
__device__ __forceinline__ void add_not_finite8(Rows<D> (&rows)[G], const unsigned char* v_tile, float s0, float s1, int key0,
                                                const int (&end)[G], int lane) {
#pragma unroll 1
  for (int key = 0; key < 32; ++key)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = 32 * db + 8 * q + 4 * (lane >> 5);
        const uint32_t x = *reinterpret_cast<const uint32_t*>(v_tile + key * D + (((col >> 4) ^ v8_chunk<D>(key)) << 4) + (col & 15));
        const u32x4 y = q8_bf16(u32x2{x, 0u}, key < 16 ? s0 : s1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = bf16_to_f32((uint16_t)(y[e / 2] >> (16 * (e % 2))));
          const bool odd = !(fabsf(v) < __builtin_huge_valf());
#pragma unroll
          for (int g = 0; g < G; ++g) rows[g].o[db][4 * q + e] += odd && key0 + key < end[g] ? v : 0.f;
        }
      }
}

}  // namespace respec

// Tiles of an 8-bit paged cache (see q8.hpp), for the bf16 attention kernels (gfx950).
//
// Sixteen rows from a multiple of 16 lie in one page and share a scale (scale blocks are multiples of 16 rows, pages of
// blocks), so a wave's rows come 16 at a time from one address, whole also where the sequence ends inside them: keys
// behind the end are masked in the scores, and their values, which a reused page may well hold NaNs in, count as zeros.
// bf16 holds e4m3 values times a power of two (all but the very least and largest, see q8.hpp).
#pragma once

#include "chunk_tile.hpp"
#include "q8.hpp"

namespace respec {

__device__ __forceinline__ float q8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
template <int UNIT>
__device__ __forceinline__ float q8_scale(uint32_t byte) { return q8_scale((uint32_t)max((int)byte - UNIT, 0)); }

// Places and scales of 16 rows each, a lane for each: rows r0 .. r0 + 15 of the sequence (r0 a multiple of 16, from the
// sequence's end on its last 16 instead).
struct Q8Window {
  uint32_t lo, hi;  // offset of the rows in a KV head of the cache (64 bits)
  uint32_t scales;  // exponent bytes: K's, and from bit 16 on V's
  __device__ __forceinline__ void fill(const ChunkAttnArgs& a, const Item& it, int r0, int hi_row) {
    const uint32_t r = (uint32_t)max(0, min(r0, (hi_row - 1) & ~15));
    const int32_t id = a.b.table[(int64_t)it.b * a.b.table_stride + div_by(r, a.b.page)];
    const int64_t at = scale_offset(a, id, r, it.g);
    scales = a.q8.k[at] | (uint32_t)a.q8.v[at] << 16;
    const uint64_t off = (uint64_t)offset_in(a.b, id, r);
    lo = (uint32_t)off;
    hi = (uint32_t)(off >> 32);
  }
  __device__ __forceinline__ uint64_t offset(int l) const {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi, l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)lo, l);
  }
};

// 16 rows of K or V on their way through a wave's registers into a tile of bf16 (as chunk_tile.hpp's).
template <int D>
struct Q8Rows {
  static constexpr int PPR = D / 16, N = D / 64;  // 16-byte pieces per row, of a lane
  u32x4 x[N];
  // A lane's places: in memory, from the first row on, and in a tile of bf16 (its first 16 bytes of 32), row 0 on.
  static __device__ __forceinline__ uint32_t from(uint32_t stride, int lane) { return (uint32_t)(lane / PPR) * stride + (uint32_t)(lane % PPR * 16); }
  template <bool K>
  static __device__ __forceinline__ uint32_t to(int lane) {
    const int r = lane / PPR, c = 2 * (lane % PPR);
    return (uint32_t)(r * D * 2 + ((c ^ (K ? k_chunk<D>(r) : v_chunk<D>(r))) << 4));
  }
  // Rows at `rows` (this head's), `stride` bytes apart.
  __device__ __forceinline__ void fetch(const char* rows, uint32_t stride, uint32_t from) {
#pragma unroll
    for (int u = 0; u < N; ++u) x[u] = ld16(rows + u * 8 * (uint64_t)stride + from);
  }
  // Rows from `valid` on become zeros.
  __device__ __forceinline__ void clear_from(int valid, int lane) {
#pragma unroll
    for (int u = 0; u < N; ++u)
      if ((u * 64 + lane) / PPR >= valid) x[u] = u32x4{0u, 0u, 0u, 0u};
  }
  // Into a tile at its row `row0`, 0 or 16: chunk c + 1 is c's neighbour (c is even), and 8 rows further the permutation has
  // its bit of 8 changed (K's of 128 columns) or is the same.
  template <bool K>
  __device__ __forceinline__ void to_lds(unsigned char* tile, int row0, float scale, uint32_t to) const {
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)tile + (uint32_t)(row0 * D * 2) + to;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t here = (at ^ (uint32_t)(16 * h + (K ? 128 * u : 0))) + (uint32_t)(u * 8 * D * 2);
        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)here = q8_bf16(u32x2{x[u][2 * h], x[u][2 * h + 1]}, scale);
      }
  }
};

// Tiles of 32 rows of D codes for products of 16 query rows, v_mfma_f32_16x16x32_bf16.  S^T = K Q^T of 16 keys leaves, in lane l,
// the scores of query row l % 16 with keys 4 (l / 16) .. + 3; those of both halves of a tile are the B operand of O^T += V^T P^T
// as they stand, if V's A operand takes its keys in the same order.
//
// The rows' 16-byte chunks are permuted inside the row (by the DMA's source addresses): the 16 rows that a quarter of a K read
// takes, and the 16 that half of a transposing V read does, touch every bank once.
template <int D>
__device__ __forceinline__ int k8_chunk(int r) {
  return D == 128 ? ((r >> 1) & 7) : ((r >> 2) & 3);
}
template <int D>
__device__ __forceinline__ int v8_chunk(int r) {
  return D == 128 ? ((r >> 1) & 3) + ((r & 16) >> 2) : ((r >> 2) & 1) + ((r & 16) >> 3);
}

__device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) { return mma_k64(bf16_t{}, a, b, c); }

// K fragments of 16 keys (A operand): lane l holds key l % 16, for step 2 j + e the elements 16 (4 j + l / 16) + 8 e .. + 7.
template <int D>
__device__ __forceinline__ void read_k8(const unsigned char* tile, int lane, int half, float scale, u32x4 (&kf)[D / 32]) {
  const int r = 16 * half + (lane & 15), g = lane >> 4;
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(tile + r * D + (((4 * j + g) ^ k8_chunk<D>(r)) << 4));
    kf[2 * j] = q8_bf16(u32x2{x.x, x.y}, scale);
    kf[2 * j + 1] = q8_bf16(u32x2{x.z, x.w}, scale);
  }
}

// V^T fragments of 32 keys (A operand): lane l holds column 16 cb + l % 16 of keys 4 (l / 16) .. + 3 and 16 further, by transposing
// reads: lane j of a 16-lane group addresses columns 8 (j % 2) .. of row j / 2 of eight and receives column j of them.
// Keys from `valid` on count as zeros.
template <int D>
__device__ __forceinline__ void read_v8(const unsigned char* tile, int lane, float s0, float s1, int valid, u32x4 (&vf)[D / 16]) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
  const int j = lane & 15, i = j >> 1, r = 4 * (lane >> 4) + (i & 3) + 4 * (i & 4);
  const unsigned char* row = tile + r * D + (j & 1) * 8;
  u32x2 x[D / 16];
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb)
    x[cb] = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(row + ((cb ^ v8_chunk<D>(r)) << 4))));
  if (valid < 32) {  // (uniform)
    u32x2 mask;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int keys = valid - 16 * h - 4 * (lane >> 4);  // of these four
      mask[h] = keys >= 4 ? ~0u : keys <= 0 ? 0u : (1u << (8 * keys)) - 1;
    }
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) x[cb] &= mask;
  }
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb) {
    const u32x4 lo = q8_bf16(x[cb], s0), hi = q8_bf16(x[cb], s1);
    vf[cb] = u32x4{lo.x, lo.y, hi.z, hi.w};
  }
}

// 16 query rows of a wave (lane l: row l % 16; its four lanes hold a quarter of the keys and columns each).
template <int D>
struct Rows16 {
  f32x4 o[D / 16];  // columns 16 cb + 4 (l / 16) .. + 3
  float m, l;       // as Rows'
  float limit;

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) o[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = kNoRef;
    l = 0.f;
    limit = kSumLimit16;
  }
  static constexpr float kSumLimit16 = 2048.f;  // 8 weights of at most 2^8
};

// weights() and settle() of a tile's 8 scores per lane.
template <bool FAR = false>
__device__ __forceinline__ float weights16(const f32x4 (&s)[2], float scale_log2, float m, u32x4& p) {
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float p0 = __builtin_amdgcn_exp2f(less_ref<FAR>(s[w / 2][2 * (w % 2)], scale_log2, m));
    const float p1 = __builtin_amdgcn_exp2f(less_ref<FAR>(s[w / 2][2 * (w % 2) + 1], scale_log2, m));
    const bf16x2 h = __builtin_convertvector(f32x2{p0, p1}, bf16x2);
    sum = __builtin_amdgcn_fdot2_f32_bf16(h, ones, sum, false);
    p[w] = __builtin_bit_cast(uint32_t, h);
  }
  return sum;
}
template <int D>
__device__ __forceinline__ void settle16(Rows16<D>& r, const f32x4 (&s)[2], float scale_log2, u32x4& p, float sum) {
  if (__any(sum > r.limit)) {
    float x = max_of(s[0][0], s[1][0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) x = max_of(x, max_of(s[0][i], s[1][i]));
    x = max_of(x, xchg<4>(x));
    const float top = max_of(x, xchg<5>(x)) * scale_log2;
    const float to = top > r.m + kRefMargin ? top : r.m;
    const float alpha = __builtin_amdgcn_exp2f(r.m - to);
    r.m = to;
    r.limit = fabsf(to) > kFarRef && to != kNoRef ? -1.f : Rows16<D>::kSumLimit16;
    r.l *= alpha;
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) r.o[cb] *= alpha;
    sum = weights16<true>(s, scale_log2, to, p);
  }
  r.l += sum;
}

// Values that are not finite, in tiles that some row does not see whole: see take_out_not_finite() and add_not_finite().
template <int D>
__device__ __forceinline__ bool take_out_not_finite16(u32x4 (&vf)[D / 16]) {
  u16x2 top = {0, 0};
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb)
#pragma unroll
    for (int w = 0; w < 4; ++w) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[cb][w] & 0x7FFF7FFFu));
  if (!__any(top[0] >= 0x7F80 || top[1] >= 0x7F80)) return false;
#pragma unroll
  for (int cb = 0; cb < D / 16; ++cb)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t x = vf[cb][w];
      vf[cb][w] = ((x & 0x7F80u) == 0x7F80u ? 0u : x & 0xFFFFu) | ((x & 0x7F800000u) == 0x7F800000u ? 0u : x & 0xFFFF0000u);
    }
  return true;
}
template <int D, int G>
__device__ __forceinline__ void add_not_finite16(Rows16<D> (&rows)[G], const unsigned char* v_tile, float s0, float s1, int key0,
                                                 const int (&end)[G], int lane) {
#pragma unroll 1
  for (int key = 0; key < 32; ++key)
#pragma unroll
    for (int cb = 0; cb < D / 16; ++cb) {
      const uint32_t x = *reinterpret_cast<const uint32_t*>(v_tile + key * D + ((cb ^ v8_chunk<D>(key)) << 4) + 4 * (lane >> 4));
      const u32x4 y = q8_bf16(u32x2{x, 0u}, key < 16 ? s0 : s1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v = bf16_to_f32((uint16_t)(y[e / 2] >> (16 * (e % 2))));
        const bool odd = !(fabsf(v) < __builtin_huge_valf());
#pragma unroll
        for (int g = 0; g < G; ++g) rows[g].o[cb][e] += odd && key0 + key < end[g] ? v : 0.f;
      }
    }
}

}  // namespace respec

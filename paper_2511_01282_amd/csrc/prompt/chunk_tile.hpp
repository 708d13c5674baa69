// Tiles of a paged KV cache in LDS and their fragments, for the bf16 attention kernels (gfx950).
//
// Matrix cores: v_mfma_f32_32x32x16_bf16.  S^T = K Q^T leaves, in lane l, 16 scores of ONE query row
// (row l & 31): element i is key 8 (i / 4) + 4 (l / 32) + i % 4 of 32.  Rounded to bf16 in pairs they
// are the B operand of O^T += V^T P^T as they stand, if V's A operand takes its keys in the same order.
//
// K and V rows lie in LDS as in memory, D elements each, their 16-byte chunks permuted inside the
// row (by the DMA's source addresses) so that fragment reads touch every bank once.
#pragma once

#include "chunk.hpp"

namespace respec {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// Softmax reference of a row that has seen nothing: no finite score is below it, and exp2 of an ordinary score less this
// is inf, which a row's first tile always corrects (see settle).
constexpr float kNoRef = -3.402823466e38f;
// A row's reference maximum is raised only where a weight exceeds 2^8 or so (log2 units), so that the
// accumulators are seldom rescaled; the weights' sum in a tile shows it without looking for the maximum.
constexpr float kRefMargin = 8.f;
constexpr float kSumLimit = 4096.f;  // 16 weights of at most 2^8
constexpr float kFarRef = 33554432.f;  // 2^25, see settle()

template <int D>
__device__ __forceinline__ int k_chunk(int r) {  // permutation of a K row's chunks (an xor)
  return D == 128 ? (r & 15) : ((r >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int v_chunk(int r) {  // ... of a V row's: a half-wave of a transposing read takes 64
  return D == 128 ? ((r & 3) << 2) : ((r & 2) << 1);  // bytes of each of 4 rows
}

__device__ __forceinline__ f32x16 mma32(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// max(a, b) without the canonicalisation of fmaxf's operands (none is a signalling NaN).
__device__ __forceinline__ float max_of(float a, float b) { return __builtin_amdgcn_fmed3f(a, b, __builtin_huge_valf()); }

// N DMA requests of 1 KB: request q moves 16 bytes per lane from base + off[q] + 1024 q to LDS at
// dst + 1024 q (the instruction's offset counts on both sides; dst and base uniform).
template <int N>
__device__ __forceinline__ void dma_rows(uint32_t dst, uint64_t base, const uint32_t (&off)[N]) {
  uint32_t saved;
  dst = __builtin_amdgcn_readfirstlane(dst);
  base = uniform_u64(base);
  static_assert(N == 1 || N == 2 || N == 4, "requests");
  if constexpr (N == 1) {
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %3\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "s"(dst), "v"(off[0]), "s"(base)
        : "memory");
  } else if constexpr (N == 2) {
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %4\n\t"
        "global_load_lds_dwordx4 %3, %4 offset:1024\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "s"(dst), "v"(off[0]), "v"(off[1]), "s"(base)
        : "memory");
  } else {
    asm volatile(
        "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
        "global_load_lds_dwordx4 %2, %6\n\t"
        "global_load_lds_dwordx4 %3, %6 offset:1024\n\t"
        "global_load_lds_dwordx4 %4, %6 offset:2048\n\t"
        "global_load_lds_dwordx4 %5, %6 offset:3*1024\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "s"(dst), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base)
        : "memory");
  }
}
// One request from an address of each lane's own.
__device__ __forceinline__ void dma_lanes(uint32_t dst, uint64_t addr) {
  uint32_t saved;
  dst = __builtin_amdgcn_readfirstlane(dst);
  asm volatile(
      "s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\t"
      "global_load_lds_dwordx4 %2, off\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(saved)
      : "s"(dst), "v"(addr)
      : "memory");
}

// What a wave brings of every tile: R rows (NR requests) of K and of V, rows r0 .. r0 + R - 1 of the sequence
// into LDS at k_dst and v_dst.  The page ids of the rows lie in LDS.  (R and the first row's place in its tile
// are multiples of 8; the chunks' permutation repeats every 16 rows.)
template <int D, int R>
struct RowFeed {
  static constexpr int CPR = D / 8, RPI = 64 / CPR, NR = R / RPI;  // chunks per row, rows per request, requests
  const char* k;   // this head of page 0
  const char* v;
  uint32_t k_off[NR], v_off[NR];  // within R rows of one page
  int first;       // the first row's place in its tile

  __device__ __forceinline__ void init(const ChunkBatch& c, int g, int first_, int lane) {
    first = first_;
    k = c.k + (int64_t)g * c.head_stride;
    v = c.v + (int64_t)g * c.head_stride;
#pragma unroll
    for (int q = 0; q < NR; ++q) {
      const int r = q * RPI + lane / CPR, pos = lane % CPR;
      const uint32_t row = (uint32_t)r * c.row_stride + 1024u * (NR - 1 - q);
      k_off[q] = row + (uint32_t)((pos ^ k_chunk<D>(first + r)) * 16);
      v_off[q] = row + (uint32_t)((pos ^ v_chunk<D>(first + r)) * 16);
    }
  }
  // Offset from k and v of R rows in page `id` (uniform), the first at row `at` of it, for dma_rows with k_off and v_off.
  __device__ __forceinline__ int64_t page_offset(const ChunkBatch& c, int id, uint32_t at) const {
    const int64_t page = (uint32_t)id < (uint32_t)c.n_pages ? id : 0;
    return page * c.page_stride + (int64_t)((uint64_t)at * c.row_stride) - 1024 * (NR - 1);
  }
  // Such rows.
  __device__ __forceinline__ void from_page(const ChunkBatch& c, uint32_t k_dst, uint32_t v_dst, int id, uint32_t at) const {
    const int64_t off = page_offset(c, id, at);
    dma_rows<NR>(k_dst, (uint64_t)(k + off), k_off);
    dma_rows<NR>(v_dst, (uint64_t)(v + off), v_off);
  }
  // Rows r0 .. in any pages (ids: LDS, entry 0 is page p0 of the sequence); rows from hi on repeat row hi - 1.
  __device__ __forceinline__ void from_rows(const ChunkBatch& c, uint32_t k_dst, uint32_t v_dst, const int32_t* ids, uint32_t p0,
                                            int r0, int hi, int lane) const {
#pragma unroll
    for (int q = 0; q < NR; ++q) {
      const int r = q * RPI + lane / CPR, pos = lane % CPR;
      const uint32_t row = (uint32_t)min(r0 + r, hi - 1), p = div_by(row, c.page);
      const int32_t id = ids[p - p0];
      const int64_t page = (uint32_t)id < (uint32_t)c.n_pages ? id : 0;
      const int64_t off = page * c.page_stride + (int64_t)((uint64_t)(row - p * c.page.d) * c.row_stride);
      dma_lanes(k_dst + 1024 * q, (uint64_t)(k + off + (pos ^ k_chunk<D>(first + r)) * 16));
      dma_lanes(v_dst + 1024 * q, (uint64_t)(v + off + (pos ^ v_chunk<D>(first + r)) * 16));
    }
  }
};

// K fragments of 32 keys (A operand: lane l holds key l & 31).
template <int D>
__device__ __forceinline__ u32x4 read_k1(const unsigned char* tile, int lane, int ks) {
  const int r32 = lane & 31, hi = lane >> 5;
  return *reinterpret_cast<const u32x4*>(tile + r32 * D * 2 + (((2 * ks + hi) ^ k_chunk<D>(r32)) << 4));
}
template <int D>
__device__ __forceinline__ void read_k(const unsigned char* tile, int lane, u32x4 (&kf)[D / 16]) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) kf[ks] = read_k1<D>(tile, lane, ks);
}

// V^T fragments of 32 keys (A operand: lane l holds column 32 db + (l & 31), keys 16 k2 + {0..3, 8..11} + 4 (l / 32)),
// by transposing reads: lane j of a 16-lane group addresses row + j / 4, columns 4 (j % 4) .. and receives column j
// of the four rows.
template <int D>
__device__ __forceinline__ u32x4 read_v1(const unsigned char* tile, int lane, int db, int k2) {
  typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
  const int lr = lane & 15, dh = (lane >> 4) & 1, hi = lane >> 5;
  const int r = 4 * hi + lr / 4;  // (rows + 8 and + 16 share the permutation)
  const int col = 32 * db + 16 * dh + 4 * (lr % 4);
  const unsigned char* p = tile + r * D * 2 + ((col >> 3) ^ v_chunk<D>(r)) * 16 + (col & 7) * 2 + 16 * k2 * D * 2;
  const u32x2 h0 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p));
  const u32x2 h1 = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 8 * D * 2)));
  return u32x4{h0.x, h0.y, h1.x, h1.y};
}
template <int D>
__device__ __forceinline__ void read_v(const unsigned char* tile, int lane, u32x4 (&vf)[D / 32][2]) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2) vf[db][k2] = read_v1<D>(tile, lane, db, k2);
}

// 32 query rows of a wave (lane l: row l & 31; both halves of the wave hold half of its keys and columns).
template <int D>
struct Rows {
  f32x16 o[D / 32];  // column 32 db + 8 (i / 4) + 4 (l / 32) + i % 4
  float m, l;        // reference maximum (log2 units), sum of this half's weights
  float limit;       // sum of a tile's weights above which settle() looks at them

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o[db] = f32x16{};
    m = kNoRef;
    l = 0.f;
    limit = kSumLimit;
  }
};

// A score's exponent against reference m; FAR: with the product rounded first.
template <bool FAR>
__device__ __forceinline__ float less_ref(float s, float scale_log2, float m) {
#pragma clang fp contract(off)
  return FAR ? s * scale_log2 - m : __builtin_fmaf(s, scale_log2, -m);
}

// Weights of 32 keys against reference m, as bf16 pairs, and their sum.  The sum is of the rounded weights, so
// the division by it undoes what rounding does to all of them alike.  Each rounding, to 8 bits, is half a step
// of the output's own rounding at most, and they are many and of either sign: 0.0020 to 0.0022 of the result's norm off
// from 64 bits, where the output's rounding alone is 0.00166.  A second product with the weights' low parts, as in the tree
// attention of a verification step (whose sums meet decision margins before they are rounded), leaves that alone, but takes
// 736 us for 540 (8192-token prompt, 32 heads of 128), 193 for 143 (512 tokens over 16384 rows), 108 for 105 (32 decoding
// tokens, D = 128), 77 for 70 (D = 64).
template <bool FAR = false>
__device__ __forceinline__ float weights(const f32x16& s, float scale_log2, float m, u32x4 (&p)[2]) {
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
  float sum = 0.f;
#pragma unroll
  for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float p0 = __builtin_amdgcn_exp2f(less_ref<FAR>(s[8 * k2 + 2 * w], scale_log2, m));
      const float p1 = __builtin_amdgcn_exp2f(less_ref<FAR>(s[8 * k2 + 2 * w + 1], scale_log2, m));
      const bf16x2 h = __builtin_convertvector(f32x2{p0, p1}, bf16x2);
      sum = __builtin_amdgcn_fdot2_f32_bf16(h, ones, sum, false);
      p[k2][w] = __builtin_bit_cast(uint32_t, h);
    }
  return sum;
}

// After weights(): where some row's sum shows a weight above the margin, its reference becomes the tile's
// maximum, what it has accumulated is rescaled and the tile's weights are taken again.  The reference is a score's
// rounded product with the scale, off from the exact one by up to half a unit of its last place: where that is more than a
// few (2^31 and up it is 128: a weight of inf or 0 that should be 1), every tile's weights are taken again, against rounded
// products (kFarRef; as a limit of the row's own it costs nothing, a test of the reference in every tile 3-5% of mixed batches).
template <int D>
__device__ __forceinline__ void settle(Rows<D>& r, const f32x16& s, float scale_log2, u32x4 (&p)[2], float sum) {
  if (__any(sum > r.limit)) {
    float x = max_of(s[0], s[1]);
#pragma unroll
    for (int i = 2; i < 16; ++i) x = max_of(x, s[i]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    const float top = max_of(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale_log2;
    const float to = top > r.m + kRefMargin ? top : r.m;
    const float alpha = __builtin_amdgcn_exp2f(r.m - to);
    r.m = to;
    r.limit = fabsf(to) > kFarRef && to != kNoRef ? -1.f : kSumLimit;
    r.l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) r.o[db] *= alpha;
    sum = weights<true>(s, scale_log2, to, p);
  }
  r.l += sum;
}

// Scores of keys from position `end` on (s[0] is at key0 + 4 (lane / 32)) are masked.
__device__ __forceinline__ void mask_scores(f32x16& s, int key0, int end, int lane) {
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = key0 + 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3) < end ? s[i] : kNegInf;
}

// A masked weight is zero, and zero times a NaN or an infinity is not.  In tiles that some row does not
// see whole, values that are not finite are taken out of the fragments (true is returned), and
// add_not_finite() brings them to the rows that see them: whatever the weight, they make a NaN or an
// infinity of the sum.
template <int D>
__device__ __forceinline__ bool take_out_not_finite(u32x4 (&vf)[D / 32][2]) {
  u16x2 top = {0, 0};
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int w = 0; w < 4; ++w)
        top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, vf[db][k2][w] & 0x7FFF7FFFu));
  if (!__any(top[0] >= 0x7F80 || top[1] >= 0x7F80)) return false;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t x = vf[db][k2][w];
        vf[db][k2][w] = ((x & 0x7F80u) == 0x7F80u ? 0u : x & 0xFFFFu) | ((x & 0x7F800000u) == 0x7F800000u ? 0u : x & 0xFFFF0000u);
      }
  return true;
}
template <int D, int G>
__device__ __forceinline__ void add_not_finite(Rows<D> (&rows)[G], const unsigned char* v_tile, int key0, const int (&end)[G],
                                               int lane) {
#pragma unroll 1
  for (int key = 0; key < 32; ++key)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = 32 * db + 8 * q + 4 * (lane >> 5);
        const u32x2 x = *reinterpret_cast<const u32x2*>(v_tile + key * D * 2 + (((col >> 3) ^ v_chunk<D>(key)) << 4) + (col & 7) * 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float v = bf16_to_f32((uint16_t)(x[e / 2] >> (16 * (e % 2))));
          const bool odd = !(fabsf(v) < __builtin_huge_valf());
#pragma unroll
          for (int g = 0; g < G; ++g) rows[g].o[db][4 * q + e] += odd && key0 + key < end[g] ? v : 0.f;
        }
      }
}

// Unnormalised partial (a split's) or normalised output of a lane's row.
template <int D>
__device__ __forceinline__ void store_rows(Rows<D>& r, const ChunkAttnArgs& a, bool whole, int split, int64_t t, int64_t head,
                                           bool live, int lane) {
  const int hi = lane >> 5;
  const float l = r.l + xchg<5>(r.l);
  if (!live) return;
  if (whole) {
    char* to = a.out + t * a.o_tok + head * a.o_head;
    const float inv = 1.f / l;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        u32x2 x;
#pragma unroll
        for (int w = 0; w < 2; ++w)
          x[w] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{r.o[db][4 * q + 2 * w] * inv, r.o[db][4 * q + 2 * w + 1] * inv}, bf16x2));
        *reinterpret_cast<u32x2*>(to + (32 * db + 8 * q + 4 * hi) * 2) = x;
      }
  } else {
    const int64_t pr = ((int64_t)split * a.b.total_new + t) * ((int64_t)a.b.n_kv_heads * a.b.group) + head;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(a.part_o + pr * D + 32 * db + 8 * q + 4 * hi) =
            f32x4{r.o[db][4 * q], r.o[db][4 * q + 1], r.o[db][4 * q + 2], r.o[db][4 * q + 3]};
    if (hi == 0) {
      a.part_m[pr] = r.m;
      a.part_l[pr] = l;
    }
  }
}

}  // namespace respec

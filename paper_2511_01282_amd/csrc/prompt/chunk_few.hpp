// Causal attention of a few query rows over a paged cache, bf16: decoding steps and short chunks.
//
// Up to 32 or 64 query rows (tokens times the heads of a group) of a sequence and KV head: the cache is
// read once and memory bounds it.  A workgroup takes a split of the cache rows; its four waves own all the query rows
// and every fourth tile of 32 cache rows each, with a ring of their own in LDS that they fill by DMA, so
// nothing but a wave's own requests is ever waited for.  (With one group of 32 rows it is all of them, in every tile: the
// queries are first used inside the loop, the compiler waits for their loads at its head, and the DMA, of which it does not
// know, is waited for with them.)  At the end the waves' (m, l, O) are joined through LDS.
// Measured: 32 sequences of one token, 32 heads on 8 of 128, 300 to 16000 rows (536 MB), 101 us, 5.3 TB/s; one
// sequence over 32768 rows, 28 heads on 4 (67 MB), 16 us, 4.2 TB/s.
#pragma once

#include "chunk_pages.hpp"
#include "chunk_tile.hpp"

namespace respec {

constexpr int kFewTile = 32;

template <int D>
struct FewShape {
  static constexpr int S = D == 128 ? 2 : 4;       // ring slots of a wave
  static constexpr int kHalf = kFewTile * D * 2;      // bytes of a K or V tile
  static constexpr int kSlot = 2 * kHalf;
  static constexpr int kWave = S * kSlot;
  static constexpr int kPageIds = 1024;            // page ids of a wave's window
  static constexpr int kIds = 4 * kWave;
  static constexpr int kMl = kIds + 4 * kPageIds * 4;
  static constexpr int kLds = kMl + 4 * 64 * 8;
  static_assert(D * 64 * 2 <= kWave, "the waves hand their O over through their rings");
  static_assert(kLds <= 163840, "LDS of a CU");
};

// Item x, by four waves (256 threads); GR groups of 32 query rows.  LEAN, for waves of at most 256 registers: what depends
// on the lane alone is worked out in every tile (`at`); held along, as the compiler would have it, it spills.
template <int D, int GR, bool LEAN>
__device__ __forceinline__ void few_rows_item(const ChunkAttnArgs& a, int x, unsigned char* smem) {
  using G = FewShape<D>;
  using Feed = RowFeed<D, kFewTile / 2>;
  constexpr int KS = D / 16, DB = D / 32, NR = Feed::NR, S = G::S;
  const ChunkGeom& ge = a.few;
  const Item it = find_item(a.b, ge, 1, a.few_rows, x);
  const ChunkSeq& sq = it.seq;
  if (sq.n == 0) return;
  const int rows = sq.n * a.b.group;
  const int limit = block_limit(a, ge, sq, 0);
  const int lo = it.split * ge.split_rows;
  if (lo >= limit) return;
  const bool whole = limit <= ge.split_rows;
  const int hi_row = whole ? limit : min(limit, lo + ge.split_rows);
  const int nt = (hi_row - lo + kFewTile - 1) / kFewTile;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, hi = lane >> 5;
  const uint32_t lds0 =
      (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)smem + (uint32_t)(wave * G::kWave);
  const unsigned char* ring = smem + wave * G::kWave;
  const int my_nt = nt > wave ? (nt - wave + 3) / 4 : 0;

  int64_t tok[GR], head[GR];
  int end[GR];
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const int row = min(g * 32 + r32, rows - 1), i = (int)div_by((uint32_t)row, a.group);
    tok[g] = sq.t0 + i;
    head[g] = (int64_t)it.g * a.b.group + (row - i * a.b.group);
    end[g] = min(sq.L + i + 1, hi_row);
  }
  const int unmasked = min(sq.L + 1, hi_row);  // rows that every query row sees

  Feed feed;
  feed.init(a.b, it.g, 0, lane);
  PageIds<G::kPageIds> ids{reinterpret_cast<int32_t*>(smem + G::kIds) + wave * G::kPageIds, a.b.table + (int64_t)it.b * a.b.table_stride, 0u, 0u,
              div_by((uint32_t)(hi_row - 1), a.b.page) + 1u};
  const bool in_page = a.b.page.d % 16 == 0;  // 16 rows from a multiple of 16 lie in one page
  int produced = 0;
  auto produce = [&]() {
    int at = lane;
    if constexpr (LEAN) asm("" : "+v"(at));
    const uint32_t dst = lds0 + (uint32_t)((produced % S) * G::kSlot);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int t0 = lo + (produced * 4 + wave) * kFewTile + h * 16;
      const uint32_t pa = div_by((uint32_t)min(t0, hi_row - 1), a.b.page), to = dst + (uint32_t)(h * 16 * D * 2);
      ids.need(pa, div_by((uint32_t)min(t0 + 15, hi_row - 1), a.b.page), lane);
      if (in_page && t0 + 16 <= hi_row)
        feed.from_page(a.b, to, to + G::kHalf, ids.uniform(pa), (uint32_t)t0 - pa * a.b.page.d);
      else
        feed.from_rows(a.b, to, to + G::kHalf, ids.ids, ids.p0, t0, hi_row, at);
    }
    ++produced;
  };
  for (int t = 0; t < min(my_nt, S); ++t) produce();

  u32x4 qf[GR][KS];
  Rows<D> r[GR];
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const char* q = a.q + tok[g] * a.q_tok + head[g] * a.q_head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[g][ks] = ld16(q + (2 * ks + hi) * 16);
    r[g].init();
  }
  if constexpr (GR > 1) {  // (the queries in accumulation registers, which the products read as they are)
#pragma unroll
    for (int g = 0; g < GR; ++g)
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) asm("" : "+a"(qf[g][ks]));
  }
#pragma unroll 1
  for (int j = 0; j < my_nt; ++j) {
    switch (produced - 1 - j) {  // tiles requested after this one, 4 NR requests each
      case 0: asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); break;
      case 1: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * NR) : "memory"); break;
      case 2: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(8 * NR) : "memory"); break;
      default: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(12 * NR) : "memory"); break;
    }
    const unsigned char* t = ring + (j % S) * G::kSlot;
    const int key0 = lo + (j * 4 + wave) * kFewTile;
    u32x4 kf[KS], vf[DB][2], p[GR][2];
    int at = lane;
    if constexpr (LEAN) asm("" : "+v"(at));
    read_k<D>(t, at, kf);
    read_v<D>(t + G::kHalf, at, vf);
    f32x16 s[GR];
#pragma unroll
    for (int g = 0; g < GR; ++g) {
      s[g] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[g] = mma32(kf[ks], qf[g][ks], s[g]);
    }
    if (key0 + kFewTile <= unmasked) {
#pragma unroll
      for (int g = 0; g < GR; ++g) settle(r[g], s[g], a.scale_log2, p[g], weights(s[g], a.scale_log2, r[g].m, p[g]));
    } else {
#pragma unroll
      for (int g = 0; g < GR; ++g) {
        mask_scores(s[g], key0, end[g], at);
        settle(r[g], s[g], a.scale_log2, p[g], weights(s[g], a.scale_log2, r[g].m, p[g]));
      }
      if (take_out_not_finite<D>(vf)) add_not_finite<D, GR>(r, t + G::kHalf, key0, end, at);
    }
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < GR; ++g) r[g].o[db] = mma32(vf[db][k2], p[g][k2], r[g].o[db]);
    // this wave's reads of the slot are done before it is filled again
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (produced < my_nt) produce();
  }

  // ---- O = sum_w 2^(m_w - M) O_w, l likewise: every wave writes its own, and joins a quarter of the columns ----
  float2* ml = reinterpret_cast<float2*>(smem + G::kMl);
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    if (g > 0) __syncthreads();
    f32x4* to = reinterpret_cast<f32x4*>(smem + wave * G::kWave) + lane;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        to[(db * 4 + q) * 64] = f32x4{r[g].o[db][4 * q], r[g].o[db][4 * q + 1], r[g].o[db][4 * q + 2], r[g].o[db][4 * q + 3]};
    ml[wave * 64 + lane] = make_float2(r[g].m, r[g].l);
    __syncthreads();
    float M = kNoRef, w[4], l = 0.f;
#pragma unroll
    for (int w_ = 0; w_ < 4; ++w_) M = fmaxf(M, ml[w_ * 64 + lane].x);
#pragma unroll
    for (int w_ = 0; w_ < 4; ++w_) {
      w[w_] = __builtin_amdgcn_exp2f(ml[w_ * 64 + lane].x - M);
      l += w[w_] * ml[w_ * 64 + lane].y;
    }
    l += xchg<5>(l);
    const bool mine = g * 32 + r32 < rows;
    const int64_t pr = ((int64_t)it.split * a.b.total_new + tok[g]) * ((int64_t)a.b.n_kv_heads * a.b.group) + head[g];
    const float inv = 1.f / l;
#pragma unroll
    for (int c = 0; c < DB; ++c) {  // (4 DB blocks of 8 columns, DB per wave)
      const int blk = wave * DB + c;
      f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w_ = 0; w_ < 4; ++w_) v += (reinterpret_cast<const f32x4*>(smem + w_ * G::kWave) + lane)[blk * 64] * w[w_];
      const int col = 32 * (blk / 4) + 8 * (blk % 4) + 4 * hi;
      if (!mine) continue;
      if (whole) {
        u32x2 y;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          y[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * e] * inv, v[2 * e + 1] * inv}, bf16x2));
        *reinterpret_cast<u32x2*>(a.out + tok[g] * a.o_tok + head[g] * a.o_head + col * 2) = y;
      } else {
        *reinterpret_cast<f32x4*>(a.part_o + pr * D + col) = v;
      }
    }
    if (!whole && mine && wave == 0 && hi == 0) {
      a.part_m[pr] = M;
      a.part_l[pr] = l;
    }
  }
}

}  // namespace respec

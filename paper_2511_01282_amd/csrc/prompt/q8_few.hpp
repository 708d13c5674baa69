// Causal attention of a few query rows over an 8-bit paged cache: decoding steps and short chunks.
//
// As chunk_few.hpp's: four waves own all the query rows and every fourth tile of 32 cache rows each, with rings of their own
// in LDS, filled by DMA as the codes lie in memory.  The codes become bf16, exactly, on the way from LDS into the products'
// operands.
#pragma once

#include "chunk_few.hpp"
#include "q8_tile.hpp"

namespace respec {

template <int D>
struct Q8FewShape {
  static constexpr int S = D == 128 ? 4 : 8;  // ring slots of a wave
  static constexpr int kHalf = kFewTile * D;  // bytes of a K or V tile
  static constexpr int kSlot = 2 * kHalf;
  static constexpr int kWave = S * kSlot;
  static constexpr int kMl = 4 * kWave;
  static constexpr int kLds = kMl + 4 * 64 * 8;
  static_assert(kLds <= 163840 - 1024, "LDS of a CU, less report_status()'s");
};

// Waits until at most n tiles of R requests each are under way (n from 0 to 7).
template <int R>
__device__ __forceinline__ void wait_tiles(int n) {
  switch (n) {
    case 0: asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); break;
    case 1: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(R) : "memory"); break;
    case 2: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * R) : "memory"); break;
    case 3: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * R) : "memory"); break;
    case 4: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * R) : "memory"); break;
    case 5: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(5 * R) : "memory"); break;
    case 6: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(6 * R) : "memory"); break;
    default: asm volatile("s_waitcnt vmcnt(%0)" ::"n"(7 * R) : "memory"); break;
  }
}

// Item x, by four waves (256 threads); GR groups of 32 query rows.
template <int D, int GR, bool LEAN>
__device__ __forceinline__ void q8_few_rows_item(const ChunkAttnArgs& a, int x, unsigned char* smem) {
  using G = Q8FewShape<D>;
  constexpr int KS = D / 16, DB = D / 32, S = G::S;
  constexpr int NR = D / 64, RPI = 1024 / D, CPR = D / 16;  // requests of 16 rows, rows of a request, chunks of a row
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
  u32x4 qf[GR][KS];
  Rows<D> r[GR];
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const int row = min(g * 32 + r32, rows - 1), i = (int)div_by((uint32_t)row, a.group);
    tok[g] = sq.t0 + i;
    head[g] = (int64_t)it.g * a.b.group + (row - i * a.b.group);
    end[g] = min(sq.L + i + 1, hi_row);
    const char* q = a.q + tok[g] * a.q_tok + head[g] * a.q_head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[g][ks] = ld16(q + (4 * (ks / 2) + 2 * hi + ks % 2) * 16);  // (as read_k8 orders them)
    r[g].init();
  }
  const int unmasked = min(sq.L + 1, hi_row);  // rows that every query row sees

  // ---- tiles: pages and scales of 64 of the wave's at a time, a lane for each; DMA of their rows, 16 at a time ----
  const char* kb = a.b.k + (int64_t)it.g * a.b.head_stride;
  const char* vb = a.b.v + (int64_t)it.g * a.b.head_stride;
  uint32_t k_off[NR], v_off[NR];
#pragma unroll
  for (int q = 0; q < NR; ++q) {
    const int rr = q * RPI + lane / CPR, pos = lane % CPR;
    const uint32_t row = (uint32_t)rr * a.b.row_stride + 1024u * (NR - 1 - q);
    k_off[q] = row + (uint32_t)((pos ^ k8_chunk<D>(rr)) * 16);
    v_off[q] = row + (uint32_t)((pos ^ v8_chunk<D>(rr)) * 16);
  }
  int32_t ids[2];
  uint32_t scales[2] = {0u, 0u};  // of 64 tiles each, by turns: bytes K, K, V, V of a tile's two halves
  auto fill = [&](int base) {
    uint32_t bytes = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      Q8Window w;
      w.fill(a, it, lo + ((base + lane) * 4 + wave) * kFewTile + h * 16, hi_row);
      ids[h] = w.id;
      bytes |= (w.k | w.v << 16) << (8 * h);
    }
    if (base & 64) scales[1] = bytes;
    else scales[0] = bytes;
  };
  int produced = 0;
  auto produce = [&]() {
    if (produced > 0 && (produced & 63) == 0) fill(produced);
    const uint32_t dst = lds0 + (uint32_t)((produced % S) * G::kSlot);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t t0 = (uint32_t)min(lo + (produced * 4 + wave) * kFewTile + h * 16, (hi_row - 1) & ~15);
      const int64_t off = offset_in(a.b, __builtin_amdgcn_readlane(ids[h], produced & 63), t0) - 1024 * (NR - 1);
      const uint32_t to = dst + (uint32_t)(h * 16 * D);
      dma_rows<NR>(to, (uint64_t)(kb + off), k_off);
      dma_rows<NR>(to + G::kHalf, (uint64_t)(vb + off), v_off);
    }
    ++produced;
  };
  if (my_nt > 0) fill(0);
  // (the queries and scales have arrived before the first request: the compiler, which does not know of the DMA, waits for
  // them here, and not in the loop, where it would wait for the tiles, too)
#pragma unroll
  for (int g = 0; g < GR; ++g)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if constexpr (GR > 1) asm volatile("" : "+a"(qf[g][ks]));
      else asm volatile("" : "+v"(qf[g][ks]));
    }
  asm volatile("" : "+v"(scales[0]));
  for (int t = 0; t < min(my_nt, S); ++t) produce();

#pragma unroll 1
  for (int j = 0; j < my_nt; ++j) {
    wait_tiles<4 * NR>(produced - 1 - j);
    const unsigned char* t = ring + (j % S) * G::kSlot;
    const int key0 = lo + (j * 4 + wave) * kFewTile;
    const uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)(j & 64 ? scales[1] : scales[0]), j & 63);
    const float v0 = q8_scale((word >> 16) & 0xFF), v1 = q8_scale(word >> 24);
    u32x4 kf[KS], vf[DB][2], p[GR][2];
    int at = lane;
    if constexpr (LEAN) asm("" : "+v"(at));
    read_k8<D>(t, at, q8_scale((at & 16 ? word >> 8 : word) & 0xFF), kf);
    read_v8<D>(t + G::kHalf, at, v0, v1, vf);
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
      if (take_out_not_finite<D>(vf)) add_not_finite8<D, GR>(r, t + G::kHalf, v0, v1, key0, end, at);
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
  join_waves<D, GR, G::kWave>(a, r, smem, reinterpret_cast<float2*>(smem + G::kMl), whole, it.split, tok, head, rows, wave, lane);
}

}  // namespace respec

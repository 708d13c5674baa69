// Causal attention of a few query rows over an 8-bit paged cache: decoding steps and short chunks.
//
// As chunk_few.hpp's: four waves own all the query rows and every fourth tile of 32 cache rows each, with rings of their own
// in LDS, filled by DMA as the codes lie in memory.  The codes become bf16 (see q8.hpp) on the way from LDS into the products'
// operands.  The cache's bytes bound it, if the matrix and vector work on them hides behind their arrival:
//
// * Groups of 16 query rows: a conversion costs the same for any number of rows, products and softmax less the fewer
//   rows there are (32 tokens over 300-16000 rows, 32 heads on 8 of 128: groups of 32 136 us, of 16 74 then).
// * Two workgroups to a CU with two slots of 32 rows per wave: three with slots of half a tile 86 us, one with four slots 83,
//   two 73.  Slots given back between K's and V's products: 81.  Heads of 64 columns with four slots: 64 tokens over 200-3000 rows
//   23.8 us, with two, and so up to four workgroups to a CU, 22.0.
// * Pages and scales of 64 tiles are looked up at once, a lane each; keys behind the sequence's end are cleared
//   before they are converted, so that what a reused page holds there never takes the slow way of values that are not finite
//   (40 us for such a tile).  With both, 60 us.
// * Sequences' lines of tiles dealt evenly over the workgroups: 62 us.  The longest splits first: 61, and 64 tokens over 200-3000 rows 38
//   instead of 33.
//
// The 32 tokens: 268 MB in 52 to 58 us (4.6 to 5.1 TB/s; batches of equal lengths 5.2 to 5.4), and 5 for the merge.  One token
// over 32767 rows, 28 heads on 4: 33.6 MB in 9.8 to 12.3 us.  Two groups: 24 sequences of 4 to 8 tokens over 2000-16000 rows, 32 heads on 8
// of 128, 339 MB in 86 us; four groups, 9 to 16 tokens, 341 MB in 145: one workgroup to a CU.
#pragma once

#include "q8_tile.hpp"

namespace respec {

constexpr int kQ8Tile = 32;

template <int D>
struct Q8FewShape {
  static constexpr int S = 2;                 // ring slots of a wave
  static constexpr int kHalf = kQ8Tile * D;   // bytes of a K or V tile
  static constexpr int kSlot = 2 * kHalf;
  static constexpr int kWave = S * kSlot;
  static constexpr int kMl = 4 * kWave;
  static constexpr int kAgain = kMl + 4 * 64 * 8;  // 64 bits of each wave
  static constexpr int kLds = kAgain + 4 * 8;
  static_assert(D * 64 <= kWave, "the waves hand their O over through their rings");
  static_assert(kLds <= 163840 / 2 - 1024, "two workgroups to a CU");
};

// Waits until at most n tiles of R requests each are under way, n < 2.
template <int R>
__device__ __forceinline__ void wait_tiles(int n) {
  if (n == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(R) : "memory");
  else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// One pass over item x, by four waves (256 threads); GR groups of 16 query rows.  V is taken in units of 2^UNIT (see kUnit); in units of
// more than 1, the rows that the pass before found large, and did not store, are stored alone.  Returns whether this one found any.
template <int D, int GR, int UNIT>
__device__ __forceinline__ bool q8_few_rows_pass(const ChunkAttnArgs& a, int x, int lane, int wave, unsigned char* smem) {
  using G = Q8FewShape<D>;
  constexpr int KS = D / 32, CB = D / 16, S = G::S;
  constexpr int NR = D / 64, RPI = 1024 / D, CPR = D / 16;  // requests of 16 rows, rows of a request, chunks of a row
  static_assert(S == 2, "wait_tiles()");
  const ChunkGeom& ge = a.few;
  const Item it = find_item(a.b, ge, 1, a.few_rows, x, lane);
  const ChunkSeq& sq = it.seq;
  if (sq.n == 0) return false;
  const int rows = sq.n * a.b.group;
  const int limit = block_limit(a, ge, sq, 0);
  const int lo = it.split * ge.split_rows;
  if (lo >= limit) return false;
  const bool whole = limit <= ge.split_rows;
  const int hi_row = whole ? limit : min(limit, lo + ge.split_rows);
  const int nt = (hi_row - lo + kQ8Tile - 1) / kQ8Tile;

  const int r16 = lane & 15, g4 = lane >> 4;
  const uint32_t lds0 =
      (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)smem + (uint32_t)(wave * G::kWave);
  const unsigned char* ring = smem + wave * G::kWave;
  const int my_nt = nt > wave ? (nt - wave + 3) / 4 : 0;

  // (a row's token, its head: worked out again for the output, not kept in registers)
  struct Place {
    int i;
    int64_t tok, head;
  };
  auto place = [&](int g, int of) __attribute__((always_inline)) {
    const int row = min(g * 16 + of, rows - 1), i = (int)div_by((uint32_t)row, a.group);
    return Place{i, (int64_t)sq.t0 + i, (int64_t)it.g * a.b.group + (row - i * a.b.group)};
  };
  int end[GR];
  u32x4 qf[GR][KS];
  Rows16<D> r[GR];
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const Place at = place(g, r16);
    end[g] = min(sq.L + at.i + 1, hi_row);
    const char* q = a.q + at.tok * a.q_tok + at.head * a.q_head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[g][ks] = ld16(q + (2 * (4 * (ks / 2) + g4) + ks % 2) * 16);  // (as read_k8 orders them)
    r[g].init();
  }
  const int unmasked = min(sq.L + 1, hi_row);  // rows that every query row sees

  // ---- tiles: pages and scales of 64 of the wave's at a time, a lane for each; DMA of their rows, 16 at a time ----
  const char* kb = a.b.k + (int64_t)it.g * a.b.head_stride - 1024 * (NR - 1);
  const char* vb = a.b.v + (int64_t)it.g * a.b.head_stride - 1024 * (NR - 1);
  uint32_t k_off[NR], v_off[2][NR];
#pragma unroll
  for (int q = 0; q < NR; ++q) {
    const int rr = q * RPI + lane / CPR, pos = lane % CPR;
    const uint32_t row = (uint32_t)rr * a.b.row_stride + 1024u * (NR - 1 - q);
    k_off[q] = row + (uint32_t)((pos ^ k8_chunk<D>(rr)) * 16);
#pragma unroll
    for (int h = 0; h < 2; ++h) v_off[h][q] = row + (uint32_t)((pos ^ v8_chunk<D>(16 * h + rr)) * 16);
  }
  Q8Window window[2];             // of a tile's halves
  uint32_t scales[2] = {0u, 0u};  // of 64 tiles each, by turns: bytes K, K, V, V of a tile's two halves
  auto fill = [&](int base) {
#pragma unroll
    for (int h = 0; h < 2; ++h) window[h].fill(a, it, lo + ((base + lane) * 4 + wave) * kQ8Tile + h * 16, hi_row);
    const uint32_t bytes = window[0].scales | window[1].scales << 8;
    if (base & 64) scales[1] = bytes;
    else scales[0] = bytes;
  };
  int produced = 0;
  auto produce = [&]() {
    if (produced > 0 && (produced & 63) == 0) fill(produced);
    const uint32_t dst = lds0 + (uint32_t)((produced % S) * G::kSlot);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint64_t off = window[h].offset(produced & 63);
      const uint32_t to = dst + (uint32_t)(h * 16 * D);
      dma_rows<NR>(to, (uint64_t)(kb + off), k_off);
      dma_rows<NR>(to + G::kHalf, (uint64_t)(vb + off), v_off[h]);
    }
    ++produced;
  };
  if (my_nt > 0) fill(0);
  // (the queries and scales have arrived before the first request: the compiler, which does not know of the DMA, waits for
  // them here, and not in the loop, where it would wait for the tiles, too)
#pragma unroll
  for (int g = 0; g < GR; ++g)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[g][ks]));
  asm volatile("" : "+v"(scales[0]));
  for (int t = 0; t < min(my_nt, S); ++t) produce();

#pragma unroll 1
  for (int j = 0; j < my_nt; ++j) {
    wait_tiles<4 * NR>(produced - 1 - j);
    const unsigned char* t = ring + (j % S) * G::kSlot;
    const int key0 = lo + (j * 4 + wave) * kQ8Tile;
    const uint32_t word = (uint32_t)__builtin_amdgcn_readlane((int)(j & 64 ? scales[1] : scales[0]), j & 63);
    const float v0 = q8_scale<UNIT>((word >> 16) & 0xFF), v1 = q8_scale<UNIT>(word >> 24);
    u32x4 vf[CB], p[GR];
    f32x4 s[GR][2];
#pragma unroll
    for (int g = 0; g < GR; ++g) s[g][0] = s[g][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (neighbouring products are of different sums, the halves' of one group or the groups' of one half: one that waits for the
    // product before it costs more)
    constexpr int HH = GR == 1 ? 2 : 1;
#pragma unroll
    for (int h0 = 0; h0 < 2; h0 += HH) {
      u32x4 kf[HH][KS];
#pragma unroll
      for (int h = 0; h < HH; ++h) read_k8<D>(t, lane, h0 + h, q8_scale((word >> (8 * (h0 + h))) & 0xFF), kf[h]);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int g = 0; g < GR; ++g)
#pragma unroll
          for (int h = 0; h < HH; ++h) s[g][h0 + h] = mma16(kf[h][ks], qf[g][ks], s[g][h0 + h]);
    }
    read_v8<D>(t + G::kHalf, lane, v0, v1, hi_row - key0, vf);
    if (key0 + kQ8Tile <= unmasked) {
#pragma unroll
      for (int g = 0; g < GR; ++g) settle16(r[g], s[g], a.scale_log2, p[g], weights16(s[g], a.scale_log2, r[g].m, p[g]));
    } else {
#pragma unroll
      for (int g = 0; g < GR; ++g) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[g][h][i] = key0 + 16 * h + 4 * g4 + i < end[g] ? s[g][h][i] : kNegInf;
        settle16(r[g], s[g], a.scale_log2, p[g], weights16(s[g], a.scale_log2, r[g].m, p[g]));
      }
      if (take_out_not_finite16<D>(vf)) add_not_finite16<D, GR>(r, t + G::kHalf, v0, v1, key0, end, lane);
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int g = 0; g < GR; ++g) r[g].o[cb] = mma16(vf[cb], p[g], r[g].o[cb]);
    // this wave's reads of the slot are done before it is filled again
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (produced < my_nt) produce();
  }

  // ---- O = sum_w 2^(m_w - M) O_w, l likewise: every wave writes its own, and joins a quarter of the columns ----
  float2* ml = reinterpret_cast<float2*>(smem + G::kMl);
  f32x4 v[GR][CB / 4];
  float M[GR], l[GR];
  uint64_t large = 0;  // rows of large sums in this wave's columns, a bit each
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    if (g > 0) __syncthreads();
    f32x4* to = reinterpret_cast<f32x4*>(smem + wave * G::kWave) + lane;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) to[cb * 64] = r[g].o[cb];
    ml[wave * 64 + lane] = make_float2(r[g].m, r[g].l);
    __syncthreads();
    float w[4];
    M[g] = kNoRef;
    l[g] = 0.f;
#pragma unroll
    for (int w_ = 0; w_ < 4; ++w_) M[g] = fmaxf(M[g], ml[w_ * 64 + lane].x);
#pragma unroll
    for (int w_ = 0; w_ < 4; ++w_) {
      w[w_] = __builtin_amdgcn_exp2f(ml[w_ * 64 + lane].x - M[g]);
      l[g] += w[w_] * ml[w_ * 64 + lane].y;
    }
    l[g] += xchg<4>(l[g]);
    l[g] += xchg<5>(l[g]);
    float size = 0.f;
#pragma unroll
    for (int c = 0; c < CB / 4; ++c) {
      v[g][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w_ = 0; w_ < 4; ++w_)
        v[g][c] += (reinterpret_cast<const f32x4*>(smem + w_ * G::kWave) + lane)[(wave * (CB / 4) + c) * 64] * w[w_];
      add_sizes(size, v[g][c]);
    }
    if constexpr (UNIT == 0) {
      uint64_t of = __ballot(!(size < kLarge));
      of |= of >> 32;
      large |= ((of | of >> 16) & 0xFFFF) << (16 * g);
    }
  }
  // each wave knows of its columns: all of them together
  uint64_t* again = reinterpret_cast<uint64_t*>(smem + G::kAgain);
  if constexpr (UNIT == 0) {
    if (lane == 0) again[wave] = large;
    __syncthreads();
  }
  large = uniform_u64(again[0] | again[1] | again[2] | again[3]);
  int of = r16;
  asm volatile("" : "+v"(of));
#pragma unroll
  for (int g = 0; g < GR; ++g) {
    const Place at = place(g, of);
    // (queries may lie in the output's place: a row is stored once)
    if (g * 16 + r16 >= rows || (large >> (g * 16 + r16) & 1) != (UNIT != 0)) continue;
    const int64_t pr = ((int64_t)it.split * a.b.total_new + at.tok) * ((int64_t)a.b.n_kv_heads * a.b.group) + at.head;
    const float inv = 1.f / l[g];
    float to_o = 1.f;
    if constexpr (UNIT != 0) {
      if (whole) to_o = __builtin_amdgcn_ldexpf(1.f, UNIT);
      else move_unit(UNIT, M[g], l[g], to_o);
    }
#pragma unroll
    for (int c = 0; c < CB / 4; ++c) {
      const int col = 16 * (wave * (CB / 4) + c) + 4 * g4;
      const f32x4 x = v[g][c];
      if (whole) {
        u32x2 y;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          y[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x[2 * e] * inv * to_o, x[2 * e + 1] * inv * to_o}, bf16x2));
        *reinterpret_cast<u32x2*>(a.out + at.tok * a.o_tok + at.head * a.o_head + col * 2) = y;
      } else {
        *reinterpret_cast<f32x4*>(a.part_o + pr * D + col) = x * to_o;
      }
    }
    if (!whole && wave == 0 && g4 == 0) {
      a.part_m[pr] = M[g];
      a.part_l[pr] = l[g];
    }
  }
  return UNIT == 0 && large != 0;
}

// Item x, by four waves (256 threads), `wave` this one; GR groups of 16 query rows.
template <int D, int GR>
__device__ __forceinline__ void q8_few_rows_item(const ChunkAttnArgs& a, int x, int wave, unsigned char* smem) {
  if (!q8_few_rows_pass<D, GR, 0>(a, x, (int)threadIdx.x & 63, wave, smem)) return;
  const Again g = again_from(x, wave);
  q8_few_rows_pass<D, GR, kUnit>(g.a, g.x, lane_id(), g.wave, smem);
}

}  // namespace respec

// Causal attention of long chunks over a paged cache, bf16: 256 query rows per workgroup.
//
// Eight waves, two per SIMD, own 32 query rows each and walk over the same cache rows, tile by tile of 32.
// Tiles go round an LDS ring by DMA (or, of an 8-bit cache, through registers), four of them per pass and barrier.
//
// Over a bf16 cache, 8192 tokens, 32 heads of 128 (0.55 TFLOP): 511 to 556 us with the card's temperature, 0.99 to 1.08
// PFLOP/s, where a large bf16 matrix product reaches 1.22.  The matrix cores are busy half of the cycles, at 1.96 GHz; matrix
// and vector instructions of a SIMD's two waves hardly overlap (512 and some 480 cycles of the 1010 that a wave's tile takes),
// and the waves wait 30% of their time.  (Forms that leave one kind of work out, the weights' exponentials or the tiles' reads, took
// 9 to 14% less each; none of them bounds it alone.)  Four waves of 64 rows, with the tiles' fragments read half as often, took
// a tenth more clocks and the same time (537 to 545 us, the clock at 2.2 GHz), and chunks 3-5% longer; two tiles per pass and
// three passes requested ahead at D = 128, 558 against 546 us.
// 512 tokens over 16384 rows, 32 heads on 8: 134 to 150 us, and 10 us for the merge of the splits.
#pragma once

#include <type_traits>

#include "chunk_pages.hpp"
#include "chunk_tile.hpp"
#include "q8_tile.hpp"

namespace respec {

constexpr int kWideTile = 32;  // cache rows of a tile
constexpr int kWideWaves = kAttnWideThreads / 64;

template <int D, bool Q8>
struct WideShape {
  static constexpr int kPass = 4;              // tiles between two barriers
  static constexpr int kAhead = D == 128 || Q8 ? 1 : 3;  // passes requested ahead
  static constexpr int S = kPass * (kAhead + 1) + 1;   // ring slots: a pass and the tile after it, and those under way
  static constexpr int kRows = kPass * kWideTile / kWideWaves;  // cache rows of a pass that a wave brings
  static constexpr int kHalf = kWideTile * D * 2;      // bytes of a K or V tile
  static constexpr int kSlot = 2 * kHalf;
  static constexpr int kPageIds = 384;             // page ids of a wave's window
  static constexpr int kIds = S * kSlot;
  static constexpr int kLds = kIds + (Q8 ? kWideWaves * 4 : kWideWaves * kPageIds * 4);  // (Q8: a word of each wave)
  static_assert(kLds <= 163840 - 1024, "LDS of a CU, less report_status()'s");
};

// Q8: the cache holds e4m3 values with a scale per block.  A wave brings its rows of a pass, 16 that share a page and a
// scale, through registers, and they become bf16 (see q8.hpp) on the way into LDS.  So each value is converted
// once for all 256 rows, and what follows is the same.  At 64 columns both are on their way during a whole pass (K written in its
// middle: 1% more).  At 128 K is on its way during the first half of a pass and V during the
// second, for want of registers: both during all of it spilled 76, and 512 tokens over 16384 rows, 32 heads on 8 of 128, took 561 us.
// Like this 144 to 158 with the card's temperature, the merge's 10 among them; 8192 tokens, 32 heads, 514 to 562 us, as over the bf16 cache.
// V's writes meet banks twice, 17% of the LDS cycles.  Waves at a higher priority in their products: 160 instead of 155 us
// (512 tokens).  Values left as they are in LDS after the first passes, which is wrong, 138 of 152: what the conversion costs.
//
// V is taken in units of 2^UNIT (see kUnit in q8.hpp); in units of more than 1, the rows that the pass before found large, and did not
// store, are stored alone.  Returns whether this one found any (Q8).
template <int D, bool Q8, int UNIT>
__device__ __forceinline__ bool wide_rows_pass(const ChunkAttnArgs& a, int x, int lane, int wave, unsigned char* smem) {
  using G = WideShape<D, Q8>;
  using Feed = RowFeed<D, G::kRows>;
  constexpr int KS = D / 16, DB = D / 32, S = G::S, kPass = G::kPass, kRows = G::kRows, NR = Feed::NR;
  const ChunkGeom& ge = a.wide;
  const Item it = find_item(a.b, ge, a.few_rows + 1, INT32_MAX, x, lane);
  const ChunkSeq& sq = it.seq;
  if (sq.n == 0) return false;
  const int rows = sq.n * a.b.group, row0 = it.rb * ge.rows_per_wg;
  const int limit = block_limit(a, ge, sq, it.rb);
  const int lo = it.split * ge.split_rows;
  if (lo >= limit) return false;
  const bool whole = limit <= ge.split_rows;  // the block's only split
  const int hi_row = whole ? limit : min(limit, lo + ge.split_rows);
  const int np = (hi_row - lo + kWideTile * kPass - 1) / (kWideTile * kPass);  // passes

  const int r32 = lane & 31, hi = lane >> 5;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)smem;

  // ---- this wave's rows ----
  const int wrow = row0 + wave * 32;
  const int row = min(wrow + r32, rows - 1), tok_i = (int)div_by((uint32_t)row, a.group);
  const int64_t tok = sq.t0 + tok_i, head = (int64_t)it.g * a.b.group + (row - tok_i * a.b.group);
  const int end[1] = {min(sq.L + tok_i + 1, hi_row)};  // cache rows that this lane's row sees end here, within the split
  u32x4 qf[KS];
  {
    const char* q = a.q + tok * a.q_tok + head * a.q_head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = ld16(q + (2 * ks + hi) * 16);
  }
  // (uniform) tiles that some row of the wave sees, and those that every row sees whole; none for a wave without rows
  const int my_end = min(sq.L + (int)div_by((uint32_t)min(wrow + 31, rows - 1), a.group) + 1, hi_row);
  const int my_first = min(sq.L + (int)div_by((uint32_t)min(wrow, rows - 1), a.group) + 1, hi_row);
  const int my_tiles = wrow < rows && my_end > lo ? (my_end - lo + kWideTile - 1) / kWideTile : 0;
  const int unmasked = my_tiles > 0 ? max(my_first - lo, 0) / kWideTile : 0;

  // ---- DMA: unit u is tiles kPass u + 1 .. kPass u + kPass (unit -1: tile 0), kRows rows of each by every wave ----
  Feed feed;
  if constexpr (!Q8) feed.init(a.b, it.g, wave * kRows % kWideTile, lane);
  PageIds<G::kPageIds> ids{reinterpret_cast<int32_t*>(smem + G::kIds) + wave * G::kPageIds,
                           a.b.table + (int64_t)it.b * a.b.table_stride, 0u, 0u, div_by((uint32_t)(hi_row - 1), a.b.page) + 1u};
  const bool in_page = a.b.page.d % kRows == 0;  // a wave's rows of a unit lie in one page
  const int w_tile = wave * kRows / kWideTile, w_row = wave * kRows % kWideTile;  // ... within the unit, and the tile
  // units that this wave requests something of end here (it asks for rows of the last tile, no further ones)
  const int n_units = ((hi_row - lo + kWideTile - 1) / kWideTile - 1 - w_tile + kPass - 1) / kPass;
  int unit = -1;
  // Offset of the ring slot that this wave's rows of the next unit go into, and of the one that they went into last.  (Slots are
  // counted on, not divided for, and a unit's place is looked up with its page: scalar instructions stand in a wave's line with the
  // others.  12 chunks of 1-700 tokens over 33-9000 rows, 8-bit cache, 64 columns: 61 and, so, 58 us; 2 prompts of 3000 tokens 116.5
  // and 110, bf16 105 and 102.7.)
  int into_next = (S + 1 - kPass + w_tile) % S * G::kSlot, into = 0;
  // (Q8: a wave's window of 64 units, a lane for each; the unit that is on its way)
  static_assert(!Q8 || kRows == 16, "16 rows share a page and a scale");
  constexpr bool kBoth = D == 64;  // K and V are on their way together, during a whole pass
  Q8Window window;
  Q8Rows<D> q8[kBoth ? 2 : 1];
  auto &k8 = q8[0], &v8 = q8[kBoth];
  int coming = -1, entry = 0;  // its first tile (none: -1), its lane of the window
  uint64_t q8_off = 0;
  const uint32_t q8_from = Q8Rows<D>::from(a.b.row_stride, lane), q8_k = Q8Rows<D>::template to<true>(lane), q8_v = Q8Rows<D>::template to<false>(lane);
  auto q8_begin = [&](int u) __attribute__((always_inline)) {  // K of unit u is requested (kBoth: and V)
    const int t = kPass * u + 1 + w_tile;
    coming = -1;
    if (u >= n_units) return;
    entry = (u + 1) & 63;
    if (entry == 0) window.fill(a, it, lo + (kPass * (u + lane) + 1 + w_tile) * kWideTile + w_row, hi_row);
    if (t < 0) return;
    coming = t;
    q8_off = window.offset(entry) + (uint64_t)((int64_t)it.g * a.b.head_stride);
    k8.fetch(a.b.k + q8_off, a.b.row_stride, q8_from);
    if constexpr (kBoth) v8.fetch(a.b.v + q8_off, a.b.row_stride, q8_from);
  };
  auto q8_scales = [&]() __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readlane((int)window.scales, entry); };
  auto q8_middle = [&]() __attribute__((always_inline)) {  // (not kBoth) K is in LDS, V is requested
    if (kBoth || coming < 0) return;
    k8.template to_lds<true>(smem + into, w_row, q8_scale(q8_scales() & 0xFF), q8_k);
    v8.fetch(a.b.v + q8_off, a.b.row_stride, q8_from);
  };
  auto q8_end = [&]() __attribute__((always_inline)) {  // all of it is in LDS
    if (coming < 0) return;
    if constexpr (kBoth) k8.template to_lds<true>(smem + into, w_row, q8_scale(q8_scales() & 0xFF), q8_k);
    const int valid = hi_row - (lo + coming * kWideTile + w_row);  // rows that some token sees
    if (valid < kRows) v8.clear_from(valid, lane);
    v8.template to_lds<false>(smem + into + G::kHalf, w_row, q8_scale<UNIT>(q8_scales() >> 16), q8_v);
  };
  auto request = [&]() __attribute__((always_inline)) {
    const int u = unit++, t = kPass * u + 1 + w_tile, t0 = lo + t * kWideTile + w_row;
    into = into_next;
    into_next += kPass * G::kSlot - (into_next >= (S - kPass) * G::kSlot ? S * G::kSlot : 0);
    if constexpr (Q8) {
      q8_begin(u);
      return;
    }
    if (t < 0 || u >= n_units) return;
    const uint32_t dst = lds0 + (uint32_t)(into + w_row * D * 2);
    const uint32_t pa = div_by((uint32_t)min(t0, hi_row - 1), a.b.page);
    ids.need(pa, div_by((uint32_t)min(t0 + kRows - 1, hi_row - 1), a.b.page), lane);
    if (in_page && t0 + kRows <= hi_row)
      feed.from_page(a.b, dst, dst + G::kHalf, ids.uniform(pa), (uint32_t)t0 - pa * a.b.page.d);
    else
      feed.from_rows(a.b, dst, dst + G::kHalf, ids.ids, ids.p0, t0, hi_row, lane);
  };
  // Unit u has landed for every wave: of this one's requests only those of later units are under way, and its reads of the
  // slots that are filled next have arrived (their products stand before this, but nothing else keeps them there).
  auto landed = [&](int u) __attribute__((always_inline)) {
    if constexpr (Q8) {
      q8_end();
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      return;
    }
    const int newer = min(n_units, u + G::kAhead) - 1 - u;
    if (newer >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * NR) : "memory");
    else if (newer == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NR) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  static_assert(G::kAhead <= 3, "landed() tells two newer units apart");
  // The queries have arrived here: first used inside the loops, they would be waited for at each loop's head, and with them the
  // unit just requested, of which the compiler does not know (8192 tokens, bf16 cache: 543 us; like this 533).
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[ks]));
#pragma unroll 1
  for (int u = -1; u < G::kAhead; ++u) {
    request();
    if constexpr (Q8) {
      q8_middle();
      if (u < 0) q8_end();
    }
  }

  Rows<D> r[1];
  r[0].init();
  f32x16 s[2];
  u32x4 p[2], kf[KS], vf[DB][2];
  int slot = 0;  // offset of the slot of the tile at hand
  landed(0);
  if (my_tiles > 0) {
    read_k<D>(smem, lane, kf);
    s[0] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[0] = mma32(kf[ks], qf[ks], s[0]);
    mask_scores(s[0], lo, end[0], lane);
  }
  auto take_in = [&]() __attribute__((always_inline)) {  // O += V^T P
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int db = 0; db < DB; ++db) r[0].o[db] = mma32(vf[db][k2], p[k2], r[0].o[db]);
  };
  // Tile t, whose scores are s[t % 2]: the next tile's scores, this one's weights, O += V^T P.  Where no row is masked, O is that
  // of the tile before: its products, and the next tile's scores', then stand between two of settle()'s branches with nothing
  // that they wait for (16384 rows, 512 tokens, 32 heads on 8 of 64: 100.5 and, like this, 97.2 us; bf16 94.5 and 92.5; of 128
  // 152 and 152, bf16 148.5 and 147).  Orders of products and vector instructions that were asked for one by one took up
  // to 4% more at 64 columns and up to 1% less at 128.
  auto tile = [&](auto masked_c, auto u_c, int t) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked_c)::value;
    constexpr int U = decltype(u_c)::value;
    const unsigned char* v_tile = smem + slot + G::kHalf;
    slot = slot == (S - 1) * G::kSlot ? 0 : slot + G::kSlot;
    const int key0 = lo + t * kWideTile;
    if constexpr (!MASKED) take_in();
    read_k<D>(smem + slot, lane, kf);
    s[1 - U] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[1 - U] = mma32(kf[ks], qf[ks], s[1 - U]);
    read_v<D>(v_tile, lane, vf);
    bool odd = false;
    if constexpr (MASKED) odd = take_out_not_finite<D>(vf);
    const float sum = weights(s[U], a.scale_log2, r[0].m, p);
    settle(r[0], s[U], a.scale_log2, p, sum);
    if constexpr (MASKED) {
      take_in();
      if (odd) add_not_finite<D, 1>(r, v_tile, key0, end, lane);
      mask_scores(s[1 - U], key0 + kWideTile, end[0], lane);
    }
  };
  using I0 = std::integral_constant<int, 0>;
  using I1 = std::integral_constant<int, 1>;
  auto pass = [&](auto masked_c, int j) __attribute__((always_inline)) {
    const int t = kPass * j;
#pragma unroll
    for (int u = 0; u < kPass; u += 2) {
      tile(masked_c, I0{}, t + u);
      tile(masked_c, I1{}, t + u + 1);
      if (Q8 && u == 0) q8_middle();
    }
  };
  // (every wave passes np barriers; a tile takes the next one's scores, too)
  int j = 0;
  p[0] = p[1] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
  for (int db = 0; db < DB; ++db) vf[db][0] = vf[db][1] = p[0];
#pragma unroll 1
  for (; kPass * j + kPass + 1 <= unmasked; ++j) {
    if (j > 0) landed(j);
    request();
    pass(std::integral_constant<bool, false>{}, j);
  }
  if (j > 0) take_in();
#pragma unroll 1
  for (; j < np; ++j) {
    if (j > 0) landed(j);
    request();
#pragma unroll 1
    for (int u = 0; u < kPass; u += 2) {
      const int t = kPass * j + u;
      using Yes = std::integral_constant<bool, true>;
      if (t < my_tiles) tile(Yes{}, I0{}, t);
      if (t + 1 < my_tiles) tile(Yes{}, I1{}, t + 1);
      if (Q8 && u == 0) q8_middle();
    }
  }
  // the requests past the last pass land before the workgroup's LDS is released
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if constexpr (!Q8) {
    store_rows<D>(r[0], a, whole, it.split, tok, head, wrow + r32 < rows, lane);
    return false;
  } else {
    uint32_t* again = reinterpret_cast<uint32_t*>(smem + G::kIds);  // the waves' rows, a bit each
    const bool row_here = wrow + r32 < rows;
    if constexpr (UNIT == 0) {
      float size = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) add_sizes(size, r[0].o[db]);
      const uint64_t large = __ballot(row_here && !(size < kLarge));
      if (lane == 0) again[wave] = (uint32_t)large | (uint32_t)(large >> 32);
      wave_lds_sync();
    }
    // (queries may lie in the output's place: a row is stored once)
    store_rows<D>(r[0], a, whole, it.split, tok, head, row_here && (again[wave] >> r32 & 1) == (UNIT != 0), lane, UNIT);
    if constexpr (UNIT != 0) return false;
    __syncthreads();
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < kWideWaves; ++w) any |= again[w];
    return __builtin_amdgcn_readfirstlane(any) != 0;
  }
}

template <int D, bool Q8>
__device__ __forceinline__ void wide_rows_item(const ChunkAttnArgs& a, int x, unsigned char* smem) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (!wide_rows_pass<D, Q8, 0>(a, x, (int)threadIdx.x & 63, wave, smem)) return;
  if constexpr (Q8) {
    const Again g = again_from(x, wave);
    wide_rows_pass<D, Q8, kUnit>(g.a, g.x, lane_id(), g.wave, smem);
  }
}

}  // namespace respec

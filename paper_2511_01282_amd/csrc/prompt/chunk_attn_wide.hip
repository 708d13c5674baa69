// Causal attention of long chunks over a paged cache, bf16: 256 query rows per workgroup.
//
// Eight waves, two per SIMD, own 32 query rows each and walk over the same cache rows, tile by tile of 32.
// Tiles go round an LDS ring by DMA, four of them per pass and barrier.
//
// 8192 tokens, 32 heads of 128 (0.55 TFLOP): 511 to 556 us with the card's temperature, 0.99 to 1.08 PFLOP/s, where a large
// bf16 matrix product reaches 1.22.  The matrix cores are busy half of the cycles, at 1.96 GHz; matrix and vector
// instructions of a SIMD's two waves hardly overlap (512 and some 480 cycles of the 1010 that a wave's tile takes), and the
// waves wait 30% of their time.  Part of that is the queries': they are first used inside the loops, so the compiler counts
// their loads as under way at each loop's head and waits for them there.  It does not know of the DMA, and these waits
// (vmcnt(7) .. vmcnt(0) before the first score products of a pass, and of every masked tile) are for the unit just
// requested as well: it lands beside that tile, not beside the whole pass.
// With those waits in place: four waves of 64 rows, with the tiles' fragments read half as often, took a tenth more clocks and
// the same time (537 to 545 us, the clock at 2.2 GHz), and chunks 3-5% longer; two tiles per pass and three passes requested
// ahead at D = 128, 558 against 546 us.
// 512 tokens over 16384 rows, 32 heads on 8: 134 to 150 us and 10 us for the merge of the splits.
#include <type_traits>

#include "chunk_few.hpp"

namespace respec {
namespace {

constexpr int kTile = 32;  // cache rows of a tile
constexpr int kWaves = kAttnWideThreads / 64;

template <int D>
struct WideShape {
  static constexpr int kPass = 4;              // tiles between two barriers
  static constexpr int kAhead = D == 128 ? 1 : 3;  // passes requested ahead
  static constexpr int S = kPass * (kAhead + 1) + 1;   // ring slots: a pass and the tile after it, and those under way
  static constexpr int kRows = kPass * kTile / kWaves;  // cache rows of a pass that a wave brings
  static constexpr int kHalf = kTile * D * 2;      // bytes of a K or V tile
  static constexpr int kSlot = 2 * kHalf;
  static constexpr int kPageIds = 384;             // page ids of a wave's window
  static constexpr int kIds = S * kSlot;
  static constexpr int kLds = kIds + kWaves * kPageIds * 4;
  static_assert(kLds <= 163840 - 1024, "LDS of a CU, less report_status()'s");
};

template <int D>
__device__ __forceinline__ void wide_rows_item(const ChunkAttnArgs& a, int x, unsigned char* smem) {
  using G = WideShape<D>;
  using Feed = RowFeed<D, G::kRows>;
  constexpr int KS = D / 16, DB = D / 32, S = G::S, kPass = G::kPass, kRows = G::kRows, NR = Feed::NR;
  const ChunkGeom& ge = a.wide;
  const Item it = find_item(a.b, ge, a.few_rows + 1, INT32_MAX, x);
  const ChunkSeq& sq = it.seq;
  if (sq.n == 0) return;
  const int rows = sq.n * a.b.group, row0 = it.rb * ge.rows_per_wg;
  const int limit = block_limit(a, ge, sq, it.rb);
  const int lo = it.split * ge.split_rows;
  if (lo >= limit) return;
  const bool whole = limit <= ge.split_rows;  // the block's only split
  const int hi_row = whole ? limit : min(limit, lo + ge.split_rows);
  const int np = (hi_row - lo + kTile * kPass - 1) / (kTile * kPass);  // passes

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  const int my_tiles = wrow < rows && my_end > lo ? (my_end - lo + kTile - 1) / kTile : 0;
  const int unmasked = my_tiles > 0 ? max(my_first - lo, 0) / kTile : 0;

  // ---- DMA: unit u is tiles kPass u + 1 .. kPass u + kPass (unit -1: tile 0), kRows rows of each by every wave ----
  Feed feed;
  feed.init(a.b, it.g, wave * kRows % kTile, lane);
  PageIds<G::kPageIds> ids{reinterpret_cast<int32_t*>(smem + G::kIds) + wave * G::kPageIds,
                           a.b.table + (int64_t)it.b * a.b.table_stride, 0u, 0u, div_by((uint32_t)(hi_row - 1), a.b.page) + 1u};
  const bool in_page = a.b.page.d % kRows == 0;  // a wave's rows of a unit lie in one page
  const int w_tile = wave * kRows / kTile, w_row = wave * kRows % kTile;  // ... within the unit, and the tile
  // units that this wave requests something of end here (it asks for rows of the last tile, no further ones)
  const int n_units = ((hi_row - lo + kTile - 1) / kTile - 1 - w_tile + kPass - 1) / kPass;
  int unit = -1;
  auto request = [&]() __attribute__((always_inline)) {
    const int u = unit++, t = kPass * u + 1 + w_tile, t0 = lo + t * kTile + w_row;
    if (t < 0 || u >= n_units) return;
    const uint32_t dst = lds0 + (uint32_t)((t % S) * G::kSlot + w_row * D * 2);
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
    const int newer = min(n_units, u + G::kAhead) - 1 - u;
    if (newer >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * NR) : "memory");
    else if (newer == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NR) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  static_assert(G::kAhead <= 3, "landed() tells two newer units apart");
#pragma unroll 1
  for (int u = -1; u < G::kAhead; ++u) request();

  Rows<D> r[1];
  r[0].init();
  f32x16 s[2];
  u32x4 p[2], kf[KS], vf[DB][2];
  auto slot = [&](int t) __attribute__((always_inline)) { return smem + (t % S) * G::kSlot; };
  landed(0);
  if (my_tiles > 0) {
    read_k<D>(slot(0), lane, kf);
    s[0] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[0] = mma32(kf[ks], qf[ks], s[0]);
    mask_scores(s[0], lo, end[0], lane);
  }
  // Tile t, whose scores are s[t % 2]: the next tile's scores, this one's weights, O += V^T P.
  auto tile = [&](auto masked_c, auto u_c, int t) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked_c)::value;
    constexpr int U = decltype(u_c)::value;
    const unsigned char* v_tile = slot(t) + G::kHalf;
    const int key0 = lo + t * kTile;
    read_k<D>(slot(t + 1), lane, kf);
    s[1 - U] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) s[1 - U] = mma32(kf[ks], qf[ks], s[1 - U]);
    read_v<D>(v_tile, lane, vf);
    bool odd = false;
    if constexpr (MASKED) odd = take_out_not_finite<D>(vf);
    const float sum = weights(s[U], a.scale_log2, r[0].m, p);
    settle(r[0], s[U], a.scale_log2, p, sum);
#pragma unroll
    for (int k2 = 0; k2 < 2; ++k2)
#pragma unroll
      for (int db = 0; db < DB; ++db) r[0].o[db] = mma32(vf[db][k2], p[k2], r[0].o[db]);
    if constexpr (MASKED) {
      if (odd) add_not_finite<D, 1>(r, v_tile, key0, end, lane);
      mask_scores(s[1 - U], key0 + kTile, end[0], lane);
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
    }
  };
  // (every wave passes np barriers; a tile takes the next one's scores, too)
  int j = 0;
#pragma unroll 1
  for (; kPass * j + kPass + 1 <= unmasked; ++j) {
    if (j > 0) landed(j);
    request();
    pass(std::integral_constant<bool, false>{}, j);
  }
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
    }
  }
  // the requests past the last pass land before the workgroup's LDS is released
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  store_rows<D>(r[0], a, whole, it.split, tok, head, wrow + r32 < rows, lane);
}

// MIXED: sequences of few query rows are there, too, and have workgroups of their own, of which four waves work (a
// launch for each kind, one after the other: 13 sequences of 1-90 tokens over 146-217 rows, 28 heads on 4, 32.2 us,
// like this 22.1; 9 of 1-307 over 352-564, 32 on 8, 47.3 and 38.8).
template <int D, bool MIXED>
__global__ __launch_bounds__(64 * kWaves, 1) void chunk_attn_wide_kernel(ChunkAttnArgs a) {
  extern __shared__ __align__(1024) unsigned char smem[];
  int x = (int)blockIdx.x;
  if (x < a.wide.items) {
    wide_rows_item<D>(a, x, smem);
    return;
  }
  x -= a.wide.items;
  if constexpr (MIXED) {
    if (x < a.few.items) {
      if (threadIdx.x < 256) few_rows_item<D, 1, D == 128>(a, x, smem);
      return;
    }
    x -= a.few.items;
  }
  report_status<64 * kWaves>(a.b, x, true);
}

template <int D, bool MIXED>
hipError_t go(bool launch, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  constexpr int kLds = MIXED && FewShape<D>::kLds > WideShape<D>::kLds ? FewShape<D>::kLds : WideShape<D>::kLds;
  if (!launch)
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&chunk_attn_wide_kernel<D, MIXED>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  const int items = a.wide.items + (MIXED ? a.few.items : 0) + (status ? a.b.batch : 0);
  hipLaunchKernelGGL((chunk_attn_wide_kernel<D, MIXED>), dim3(items), dim3(64 * kWaves), kLds, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn_wide(int head_dim, const ChunkAttnArgs& a, bool mixed, bool status, hipStream_t s) {
  if (mixed) return head_dim == 128 ? go<128, true>(true, a, status, s) : go<64, true>(true, a, status, s);
  return head_dim == 128 ? go<128, false>(true, a, status, s) : go<64, false>(true, a, status, s);
}
hipError_t set_chunk_attn_wide_lds_limit(int head_dim) {
  const ChunkAttnArgs none{};
  const hipError_t e = head_dim == 128 ? go<128, false>(false, none, false, nullptr) : go<64, false>(false, none, false, nullptr);
  if (e != hipSuccess) return e;
  return head_dim == 128 ? go<128, true>(false, none, false, nullptr) : go<64, true>(false, none, false, nullptr);
}

}  // namespace respec

// Causal attention of long chunks over a paged cache, bf16: 256 query rows per workgroup.
//
// Four waves own 64 rows each, as two groups of 32, so that a K or V fragment read from LDS serves
// two matrix products: with 32 rows per wave the fragments of four waves' worth of rows would take the LDS's whole
// bandwidth (128 bytes per clock) at the matrix cores' rate.  One wave per SIMD, then, with up to 512
// registers, and it has to keep the matrix core busy by itself: while one group's products run, the
// other group's softmax does.  Per 32 keys:
//   phase A:  S_0 = K Q_0^T (next keys), O_0 += V^T P_0 (these)   beside   P_1 of S_1 (these)
//   phase B:  S_1 = K Q_1^T (next keys), O_1 += V^T P_1 (these)   beside   P_0 of S_0 (next)
// 16 products of 32 clocks per phase against 16 exponentials of 16 clocks and 32 other instructions of
// 4.  The fragments of the next 32 keys are read from LDS in the same phases.
//
// Tiles of 64 cache rows go round an LDS ring by DMA, each wave bringing 16 of the rows.
#include <type_traits>

#include "chunk_pages.hpp"
#include "chunk_tile.hpp"

namespace respec {
namespace {

constexpr int kTile = 64;

template <int D>
struct WideShape {
  static constexpr int S = 4;                      // ring slots
  static constexpr int kHalf = kTile * D * 2;      // bytes of a K or V tile
  static constexpr int kSlot = 2 * kHalf;
  static constexpr int kIds = S * kSlot;
  static constexpr int kLds = kIds + 4 * kPageIds * 4;
  static_assert(kLds <= 163840, "LDS of a CU");
};

template <int D>
__global__ __launch_bounds__(256, 1) void chunk_attn_wide_kernel(ChunkAttnArgs a, int items) {
  using G = WideShape<D>;
  using Feed = RowFeed<D, 16>;
  constexpr int KS = D / 16, DB = D / 32, NR = Feed::NR, S = G::S;
  extern __shared__ __align__(1024) unsigned char smem[];
  if ((int)blockIdx.x >= items) {
    report_status<256>(a.b, (int)blockIdx.x - items, true);
    return;
  }
  const ChunkGeom& ge = a.wide;
  const Item it = item_of(a.b, ge, blockIdx.x);
  const ChunkSeq sq = chunk_seq(a.b, it.b);
  const int rows = sq.n * a.b.group, row0 = it.rb * ge.rows_per_wg;
  if (row0 >= rows || rows <= a.few_rows) return;
  const int limit = block_limit(a, ge, sq, it.rb);
  const int lo = it.split * ge.split_rows;
  if (lo >= limit) return;
  const bool whole = limit <= ge.split_rows;  // the block's only split
  const int hi_row = ge.nsplit == 1 ? limit : min(limit, lo + ge.split_rows);
  const int nt = (hi_row - lo + kTile - 1) / kTile;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, hi = lane >> 5;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)smem;

  // ---- this wave's rows ----
  const int wrow = row0 + wave * 64;
  const bool live = wrow < rows;
  int64_t tok[2], head[2];
  int end[2];  // cache rows that this lane's row of each group sees, within the split
  u32x4 qf[2][KS];
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const int row = min(wrow + g * 32 + r32, rows - 1), i = (int)div_by((uint32_t)row, a.group);
    tok[g] = sq.t0 + i;
    head[g] = (int64_t)it.g * a.b.group + (row - i * a.b.group);
    end[g] = min(sq.L + i + 1, hi_row);
    const char* q = a.q + tok[g] * a.q_tok + head[g] * a.q_head;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[g][ks] = ld16(q + (2 * ks + hi) * 16);
  }
  // (the queries in accumulation registers, which the products read as they are)
#pragma unroll
  for (int g = 0; g < 2; ++g)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) asm("" : "+a"(qf[g][ks]));
  // (uniform) tiles that some row of the wave sees, and those from which on some row does not see all
  const int last = min(wrow + 63, rows - 1);
  const int my_end = min(sq.L + (int)div_by((uint32_t)last, a.group) + 1, hi_row);
  const int my_first = min(sq.L + (int)div_by((uint32_t)min(wrow, rows - 1), a.group) + 1, hi_row);
  const int my_nt = live && my_end > lo ? (my_end - lo + kTile - 1) / kTile : 0;
  const int unmasked = max(my_first - lo, 0) / kTile;  // tiles that every row sees whole

  // ---- DMA ----
  Feed feed;
  feed.init(a.b, it.g, lane);
  PageIds ids{reinterpret_cast<int32_t*>(smem + G::kIds) + wave * kPageIds, a.b.table + (int64_t)it.b * a.b.table_stride, 0u, 0u,
              div_by((uint32_t)(hi_row - 1), a.b.page) + 1u};
  const bool in_page = a.b.page.d % 16 == 0;  // a wave's 16 rows of a tile lie in one page
  int produced = 0;
  // The next tile's requests: `fast`, and from where to where, if the wave's rows lie whole in one page; requested
  // as a tile's products go on.  Other tiles are requested at once.
  bool fast = false;
  uint64_t next_k = 0, next_v = 0;
  uint32_t next_dst = 0;
  int next_id = 0;  // page of the wave's first row of the next tile, read ahead where the window holds it
  auto prepare = [&]() __attribute__((always_inline)) {
    const int t0 = lo + produced * kTile + wave * 16;
    next_dst = lds0 + (uint32_t)((produced % S) * G::kSlot + wave * 16 * D * 2);
    ++produced;
    const uint32_t pa = div_by((uint32_t)min(t0, hi_row - 1), a.b.page);
    fast = in_page && t0 + 16 <= hi_row && pa < ids.p1;
    if (fast) {
      const int64_t off = feed.page_offset(a.b, __builtin_amdgcn_readfirstlane(next_id), (uint32_t)t0 - pa * a.b.page.d);
      next_k = (uint64_t)(feed.k + off);
      next_v = (uint64_t)(feed.v + off);
    } else {
      ids.need(pa, div_by((uint32_t)min(t0 + 15, hi_row - 1), a.b.page), lane);
      feed.from_rows(a.b, next_dst, next_dst + G::kHalf, ids.ids, ids.p0, t0, hi_row, lane);
    }
    const uint32_t pn = div_by((uint32_t)min(t0 + kTile, hi_row - 1), a.b.page);
    if (pn < ids.p1) next_id = ids.ids[pn - ids.p0];
  };
  auto request = [&](bool v) __attribute__((always_inline)) {
    if (fast) dma_rows<NR>(v ? next_dst + G::kHalf : next_dst, v ? next_v : next_k, v ? feed.v_off : feed.k_off);
  };
  // Tiles up to t have landed for every wave (t < produced).
  auto landed = [&](int t) __attribute__((always_inline)) {
    const int newer = produced - 1 - t;
    if (newer >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(4 * NR) : "memory");
    else if (newer == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NR) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // (what a wave has read of the slots it is done with it has used in products, so nothing of them is under way)
    asm volatile("s_barrier" ::: "memory");
  };
  for (int t = 0; t < min(nt, S - 1); ++t) {
    prepare();
    request(false);
    request(true);
  }

  // ---- rows' state; the first tile's scores ----
  Rows<D> r[2];
  r[0].init();
  r[1].init();
  f32x16 s[2];
  u32x4 p[2][2], kf[KS], vf[DB][2];
  landed(0);
  if (my_nt > 0) {
    read_k<D>(smem, lane, kf);
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      s[g] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[g] = mma32(kf[ks], qf[g][ks], s[g]);
      mask_scores(s[g], lo, end[g], lane);
    }
    read_k<D>(smem + 32 * D * 2, lane, kf);
    settle(r[0], s[0], a.scale_log2, p[0], weights(s[0], a.scale_log2, r[0].m, p[0]));
  }

  // A phase: the scores `to` of 32 keys (kf) and O += V^T P of a group, beside the other group's weights `w` of scores
  // `from`.  Each product is followed by its share of the vector instructions, in this order: the scheduler
  // would put them together.
  auto phase = [&](auto masked_c, f32x16& to, const u32x4(&q)[KS], Rows<D>& rows_, const u32x4(&pv)[2], const f32x16& from, float m,
                   u32x4(&w)[2], auto load) __attribute__((always_inline)) {
    constexpr int N = KS + 2 * DB;  // products
    float x[16], sum = 0.f;
    const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
    auto slice = [&](int n) __attribute__((always_inline)) {  // step n of 18: score n's exponent and exponential, pair n - 2
      if (n < 16) x[n] = __builtin_fmaf(from[n], a.scale_log2, -m);
      if (n >= 1 && n < 17) x[n - 1] = __builtin_amdgcn_exp2f(x[n - 1]);
      if (n >= 3 && n % 2 == 1) {
        const bf16x2 h = __builtin_convertvector(f32x2{x[n - 3], x[n - 2]}, bf16x2);
        const int pair = (n - 3) / 2;
        sum = __builtin_amdgcn_fdot2_f32_bf16(h, ones, sum, false);
        w[pair / 4][pair % 4] = __builtin_bit_cast(uint32_t, h);
      }
    };
    int done = 0;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (n < KS) {
        to = mma32(kf[n], q[n], n == 0 ? f32x16{} : to);
      } else {
        const int k2 = (n - KS) / DB, db = (n - KS) % DB;
        rows_.o[db] = mma32(vf[db][k2], pv[k2], rows_.o[db]);
      }
      load(n);
#pragma unroll
      for (; done < min(18, ((n + 1) * 18 + N - 3) / (N - 2)); ++done) slice(done);
      if constexpr (!decltype(masked_c)::value) __builtin_amdgcn_sched_barrier(0);
    }
    return sum;
  };
  // 32 keys from key0: V rows at v_cur; kf holds the next 32 keys' K fragments, k_next are those after them.
  auto substep = [&](auto masked_c, auto u_c, const unsigned char* v_cur, const unsigned char* k_next, int key0) __attribute__((always_inline)) {
    constexpr bool MASKED = decltype(masked_c)::value;
    constexpr int U = decltype(u_c)::value;
    // phase A
    bool odd = false;
    if constexpr (MASKED) {
      read_v<D>(v_cur, lane, vf);
      odd = take_out_not_finite<D>(vf);
    }
    const float sum1 = phase(masked_c, s[0], qf[0], r[0], p[0], s[1], r[1].m, p[1], [&](int n) __attribute__((always_inline)) {
      if (!MASKED && n < 2 * DB) vf[n % DB][n / DB] = read_v1<D>(v_cur, lane, n % DB, n / DB);
      if (U == 0 && (n == 1 || n == KS)) request(n > 1);
    });
    settle(r[1], s[1], a.scale_log2, p[1], sum1);
    // phase B
    if constexpr (MASKED) mask_scores(s[0], key0 + 32, end[0], lane);
    const float sum0 = phase(masked_c, s[1], qf[1], r[1], p[1], s[0], r[0].m, p[0], [&](int n) __attribute__((always_inline)) {
      if (n >= KS) kf[n - KS] = read_k1<D>(k_next, lane, n - KS);
    });
    if constexpr (MASKED) {
      mask_scores(s[1], key0 + 32, end[1], lane);
      if (odd) add_not_finite<D, 2>(r, v_cur, key0, end, lane);
    }
    settle(r[0], s[0], a.scale_log2, p[0], sum0);
  };
  auto tile = [&](auto masked_c, int j) __attribute__((always_inline)) {
    const unsigned char* t_cur = smem + (j % S) * G::kSlot;
    const unsigned char* t_next = smem + ((j + 1) % S) * G::kSlot;
    substep(masked_c, std::integral_constant<int, 0>{}, t_cur + G::kHalf, t_next, lo + j * kTile);
    substep(masked_c, std::integral_constant<int, 1>{}, t_cur + G::kHalf + 32 * D * 2, t_next + 32 * D * 2, lo + j * kTile + 32);
  };
  // Tile j + 1 has landed, and every wave is done with tile j - 1, whose slot is filled again.
  auto begin = [&](int j) __attribute__((always_inline)) {
    landed(min(j + 1, nt - 1));
    fast = false;
    if (produced < nt) prepare();
  };
  // (a tile takes the next one's scores, too; every wave passes nt barriers)
  int j = 0;
#pragma unroll 1
  for (; j + 2 <= unmasked && j < my_nt; ++j) {
    begin(j);
    tile(std::integral_constant<bool, false>{}, j);
  }
#pragma unroll 1
  for (; j < my_nt; ++j) {
    begin(j);
    tile(std::integral_constant<bool, true>{}, j);
  }
#pragma unroll 1
  for (; j < nt; ++j) {
    begin(j);
    request(false);
    request(true);
  }
#pragma unroll
  for (int g = 0; g < 2; ++g)
    store_rows<D>(r[g], a, whole, it.split, tok[g], head[g], wrow + g * 32 + r32 < rows, lane);
}

template <int D>
hipError_t go(bool launch, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  if (!launch)
    return hipFuncSetAttribute(reinterpret_cast<const void*>(&chunk_attn_wide_kernel<D>),
                               hipFuncAttributeMaxDynamicSharedMemorySize, WideShape<D>::kLds);
  const int items = (int)item_count(a.b, a.wide);
  hipLaunchKernelGGL(chunk_attn_wide_kernel<D>, dim3(items + (status ? a.b.batch : 0)), dim3(256), WideShape<D>::kLds, s, a, items);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attn_wide(int head_dim, const ChunkAttnArgs& a, bool status, hipStream_t s) {
  return head_dim == 128 ? go<128>(true, a, status, s) : go<64>(true, a, status, s);
}
hipError_t set_chunk_attn_wide_lds_limit(int head_dim) {
  const ChunkAttnArgs none{};
  return head_dim == 128 ? go<128>(false, none, false, nullptr) : go<64>(false, none, false, nullptr);
}

}  // namespace respec

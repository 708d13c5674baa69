// Host side of the prompt side's C ABI: plans, argument validation, launches.
// See include/respec_prompt.h and, for the 8-bit cache, include/respec_cache.h for the contract.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <atomic>
#include <new>

#include "../../../include/respec_cache.h"
#include "../../../include/respec_prompt.h"
#include "../attn_route.hpp"
#include "../overlap.hpp"
#include "prompt.hpp"

using namespace respec;

struct respec_chunk_plan {
  respec_chunk_shape s;
  int es;            // bytes per element
  size_t part_rows;  // rows of partials that the workspace holds
  size_t total;
};

struct respec_score_plan {
  respec_score_shape s;
  int ko;            // width of the key lists: 8 or 16
  size_t total;
};

namespace {

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
bool aligned(const void* p, size_t n) { return ((uintptr_t)p % n) == 0; }
bool known(int32_t dtype) { return dtype == RESPEC_F32 || dtype == RESPEC_BF16; }
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

constexpr int kMaxSplits = 64;           // a lane of the merge per split
constexpr size_t kMaxPartial = 1u << 25;  // columns of partials: 134 MB
constexpr int kMaxStride = 1 << 24;
constexpr int kMaxRows = 1 << 30;         // cache rows of a sequence: positions a tile further fit 32 bits

// Whether a launch of so many workgroups can be made: a dispatch counts its threads in 32 bits.
bool launchable(long long workgroups, int threads) { return workgroups * threads < 1ll << 32; }

// Checks of a stride in elements: non-negative and whole 16-byte pieces.
bool stride_ok(int64_t s, int es) { return s >= 0 && s < (1ll << 50) && s * es % 16 == 0; }

// `ces`: bytes per element of the cache.
respec_status check_batch(const respec_chunk_plan* plan, const respec_chunk_batch& b, int ces) {
  const respec_chunk_shape& s = plan->s;
  if (b.batch < 0 || b.total_new < 0 || b.max_new_in_batch < 0 || b.max_kv_len_in_batch < 0) return RESPEC_ERR_SHAPE;
  if (b.batch > s.max_batch || b.total_new > s.max_new || b.max_kv_len_in_batch > s.max_kv_len) return RESPEC_ERR_CAPACITY;
  if (b.max_new_in_batch > b.total_new) return RESPEC_ERR_SHAPE;
  if (b.batch == 0) return RESPEC_OK;
  const respec_paged_cache& c = b.cache;
  if (!b.new_off || !b.kv_len || !c.k || !c.v || !c.page_table) return RESPEC_ERR_NULL;
  if (c.n_pages < 1 || c.page_size < 1 || c.table_width < 1) return RESPEC_ERR_SHAPE;
  if (b.batch > 1 && c.table_stride < c.table_width) return RESPEC_ERR_SHAPE;
  if (!stride_ok(c.page_stride, ces) || !stride_ok(c.head_stride, ces) || !stride_ok(c.row_stride, ces) ||
      c.row_stride > kMaxStride)
    return RESPEC_ERR_SHAPE;
  if (!aligned(c.k, 16) || !aligned(c.v, 16)) return RESPEC_ERR_SHAPE;
  return RESPEC_OK;
}

// Whether the statuses lie apart from what the kernels read: a sequence's is written while other workgroups still look up lengths
// and pages.
bool status_apart(const respec_chunk_batch& b) {
  const respec_paged_cache& c = b.cache;
  const int64_t ints = 4ll * b.batch;
  return !overlap(b.seq_status, ints, b.new_off, 1, 0, ints + 4) && !overlap(b.seq_status, ints, b.kv_len, 1, 0, ints) &&
         !overlap(b.seq_status, ints, c.page_table, b.batch, b.batch > 1 ? (__int128)4 * c.table_stride : 0, 4ll * c.table_width);
}

ChunkBatch device_batch(const respec_chunk_plan* plan, const respec_chunk_batch& b, int ces) {
  const respec_paged_cache& c = b.cache;
  ChunkBatch d;
  d.new_off = b.new_off;
  d.kv_len = b.kv_len;
  d.table = c.page_table;
  d.status = b.seq_status;
  d.k = static_cast<char*>(c.k);
  d.v = static_cast<char*>(c.v);
  d.page_stride = c.page_stride * ces;
  d.head_stride = c.head_stride * ces;
  d.table_stride = c.table_stride;
  d.row_stride = (uint32_t)(c.row_stride * ces);
  d.page = fast_div((uint32_t)c.page_size);
  d.batch = b.batch;
  d.total_new = b.total_new;
  d.max_new = b.max_new_in_batch;
  d.max_kv = b.max_kv_len_in_batch;
  d.n_pages = c.n_pages;
  d.table_width = c.table_width;
  d.n_kv_heads = plan->s.n_kv_heads;
  d.group = plan->s.n_q_heads / plan->s.n_kv_heads;
  d.kv_heads = fast_div((uint32_t)d.n_kv_heads);
  return d;
}

// Whether attention's output rows share bytes with nothing that another workgroup reads or writes: they may be the queries' own.
bool output_apart(const respec_chunk_plan* plan, const respec_chunk_attn_args& x) {
  const int es = plan->es, heads = plan->s.n_q_heads;
  const int64_t row = (int64_t)plan->s.head_dim * es, t = x.b.total_new;
  const RowSet q = row_set(x.q, t, x.q_token_stride * es, heads, x.q_head_stride * es, row);
  const RowSet out = row_set(x.out, t, x.out_token_stride * es, heads, x.out_head_stride * es, row);
  return !overlap_within(t, x.out_token_stride * es, heads, x.out_head_stride * es, row) && (same_rows(q, out) || !overlap(q, out));
}

// An 8-bit cache's batch as one over pages of one-byte elements; its scales' checks.
respec_chunk_batch codes_batch(const respec_q8_batch& b) {
  const respec_q8_cache& c = b.cache;
  return respec_chunk_batch{b.batch, b.total_new, b.max_new_in_batch, b.max_kv_len_in_batch, b.new_off, b.kv_len,
                            respec_paged_cache{c.k, c.v, c.n_pages, c.page_size, c.page_stride, c.head_stride, c.row_stride,
                                               c.page_table, c.table_width, c.table_stride},
                            b.seq_status};
}
respec_status check_scales(const respec_q8_cache& c) {
  if (!c.k_scale || !c.v_scale) return RESPEC_ERR_NULL;
  if (c.scale_block != 16 && c.scale_block != 32 && c.scale_block != 64 && c.scale_block != 128) return RESPEC_ERR_SHAPE;
  if (c.page_size % c.scale_block != 0) return RESPEC_ERR_SHAPE;
  for (int64_t s : {c.scale_page_stride, c.scale_head_stride})
    if (s < 0 || s >= 1ll << 50) return RESPEC_ERR_SHAPE;
  return RESPEC_OK;
}
Q8Scales device_scales(const respec_q8_cache& c) {
  return Q8Scales{c.k_scale, c.v_scale, c.scale_page_stride, c.scale_head_stride, __builtin_ctz((unsigned)c.scale_block)};
}

// How long an attention kernel takes over one cache row of a block, with all the workgroups of a CU that the pace was
// taken with, to start a workgroup, and to launch the merge (us); and how much of the work that longest sequences would be a batch
// is taken to be.
struct Pace {
  double row, start, merge = 4, share = 0.5;
};

// Splits of the sequences: the number n (of a coarser choice upwards; at most `held`, each of `least` cache rows or
// more, in multiples of `unit`) with the least estimated time  rounds * (rows / n * row + start) + merge,
// rounds = items * n / (CUs * per_cu); fewer than per_cu workgroups on a CU are so much faster.  One sequence's lengths
// are known, and its workgroups run in whole rounds; of a batch the host knows the longest alone, so half the work that
// longest sequences would be is assumed, and half a round of tail (80 drawn batches of chunks, geometric mean: a third
// 30.5 us, 0.4 29.5, 0.5 29.4, 0.8 29.2; of decoding tokens 21.8, 21.2, 21.8, 21.9).  Float32, 60 drawn sequences: with a lone
// workgroup's true pace 13.1 us, with four workgroups' for any 13.9, where calls of a few rows were split in vain.
ChunkGeom geometry(const ChunkBatch& b, int rows_per_wg, long long blocks, long long limit, int unit, int least,
                   int per_cu, Pace pace, int row_bytes, long long held) {
  ChunkGeom g{rows_per_wg, 1, INT_MAX, 0, fast_div(INT_MAX)};
  const long long items = blocks * b.n_kv_heads;
  double best = 0;
  long long most = std::min({ceil_div(limit, least), (long long)kMaxSplits, held, items > 0 ? (long long)INT_MAX / items : 1});
  for (long long n = 1, rows_before = 0; n <= std::max(most, 1ll); n += 1 + n / 6) {
    const long long rows = ceil_div(ceil_div(limit, n), unit) * unit;
    if (rows == rows_before) continue;
    rows_before = rows;
    const double wgs = (double)items * ceil_div(limit, std::max(rows, 1ll)) / (kCUs * per_cu);
    const double rounds = b.batch == 1 ? ceil(wgs) : std::max(1.0, wgs * pace.share) + 0.5;
    const double joined = 1e-6 * n * b.total_new * b.n_kv_heads * b.group * row_bytes * 2 / 4.5;
    const double merge = n == 1 ? 0 : pace.merge + joined * (b.batch == 1 ? 1 : pace.share);
    const double crowd = std::min(1.0, ceil(wgs * per_cu) / per_cu);  // workgroups of a CU, of the per_cu that set the pace
    const double t = rounds * (rows * pace.row * crowd + pace.start) + merge;
    if (n == 1 || t < best) {
      best = t;
      g.split_rows = n == 1 || rows >= limit ? INT_MAX : (int)rows;
    }
  }
  g.split = fast_div((uint32_t)g.split_rows);
  g.nsplit = g.split_rows == INT_MAX ? 1 : (int)ceil_div(limit, g.split_rows);
  g.items = (int)std::min(items * g.nsplit, (long long)INT_MAX);
  return g;
}

// Checks of the new rows of an append's arguments (either kind of cache).
template <typename Args>
respec_status check_new_rows(const respec_chunk_plan* plan, const Args& x) {
  if (!x.k_new || !x.v_new) return RESPEC_ERR_NULL;
  if (!aligned(x.k_new, 16) || !aligned(x.v_new, 16)) return RESPEC_ERR_SHAPE;
  for (int64_t s : {x.k_token_stride, x.k_head_stride, x.v_token_stride, x.v_head_stride})
    if (!stride_ok(s, plan->es)) return RESPEC_ERR_SHAPE;
  return RESPEC_OK;
}

// Raise the LDS limits of the attention kernels on the current device, once (a call into the runtime that also
// loads the kernels: the first step pays it).
bool raise_lds_limits(int head_dim, bool q8) {
  constexpr int kMaxDevices = 64;
  static std::atomic<uint64_t> done[4];  // [head size, cache], a bit per device
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return false;
  std::atomic<uint64_t>& d = done[(head_dim == 128) + 2 * q8];
  const uint64_t bit = dev < kMaxDevices ? 1ull << dev : 0;  // (past the last: every call raises them)
  if (d.load(std::memory_order_acquire) & bit) return true;
  if (q8) {
    if (set_q8_attn_lds_limits(head_dim) != hipSuccess) return false;
  } else if (set_chunk_attn_few_lds_limit(head_dim) != hipSuccess || set_chunk_attn_wide_lds_limit(head_dim) != hipSuccess) {
    return false;
  }
  d.fetch_or(bit, std::memory_order_release);
  return true;
}

// Attention over a cache of the plan's type or, with its scales, of 8-bit values.
respec_status attend(const respec_chunk_plan* plan, const respec_chunk_attn_args& x, const respec_q8_cache* q8, void* workspace,
                     void* stream) {
  if (!workspace || !aligned(workspace, 256)) return RESPEC_ERR_WORKSPACE;
  const int ces = q8 ? 1 : plan->es;
  const respec_status st = check_batch(plan, x.b, ces);
  if (st != RESPEC_OK) return st;
  if (q8 && x.b.batch > 0) {
    const respec_status scales = check_scales(*q8);
    if (scales != RESPEC_OK) return scales;
  }
  if (!(x.scale >= 0.f) || isinf(x.scale)) return RESPEC_ERR_PARAM;
  if (x.b.batch == 0) return RESPEC_OK;
  if (x.b.total_new > 0) {
    if (!x.q || !x.out) return RESPEC_ERR_NULL;
    if (!aligned(x.q, 16) || !aligned(x.out, 16)) return RESPEC_ERR_SHAPE;
    for (int64_t s : {x.q_token_stride, x.q_head_stride, x.out_token_stride, x.out_head_stride})
      if (!stride_ok(s, plan->es)) return RESPEC_ERR_SHAPE;
  }
  if (x.b.max_new_in_batch == 0 && !x.b.seq_status) return RESPEC_OK;  // (no sequence has tokens)
  const respec_chunk_shape& s = plan->s;
  ChunkAttnArgs a;
  a.b = device_batch(plan, x.b, ces);
  a.q8 = q8 ? device_scales(*q8) : Q8Scales{nullptr, nullptr, 0, 0, 0};
  a.q = static_cast<const char*>(x.q);
  a.out = static_cast<char*>(x.out);
  a.q_tok = x.q_token_stride * plan->es;
  a.q_head = x.q_head_stride * plan->es;
  a.o_tok = x.out_token_stride * plan->es;
  a.o_head = x.out_head_stride * plan->es;
  a.group = fast_div((uint32_t)a.b.group);
  char* ws = static_cast<char*>(workspace);
  const size_t o_bytes = align256(plan->part_rows * s.head_dim * 4), m_bytes = align256(plan->part_rows * 4);
  a.part_o = reinterpret_cast<float*>(ws);
  a.part_m = reinterpret_cast<float*>(ws + o_bytes);
  a.part_l = reinterpret_cast<float*>(ws + o_bytes + m_bytes);
  a.scale_log2 = (float)(1.4426950408889634 * (x.scale > 0.f ? (double)x.scale : 1.0 / sqrt((double)s.head_dim)));
  if (isinf(a.scale_log2)) return RESPEC_ERR_PARAM;
  const long long limit = (long long)a.b.max_kv + a.b.max_new;  // rows that the last token of the longest sequence sees
  const long long all_rows = (long long)a.b.total_new * a.b.group, rows = (long long)a.b.max_new * a.b.group;  // per KV head
  const long long seqs = std::min(a.b.batch, a.b.total_new);    // sequences that can have tokens
  const long long held = x.b.total_new > 0 ? (long long)(plan->part_rows / ((size_t)x.b.total_new * s.n_q_heads)) : 1;
  // row blocks of all sequences: each sequence's last one may be short
  auto blocks = [&](int per_wg) { return std::min(ceil_div(all_rows, per_wg) + (seqs > 1 ? seqs - 1 : 0), seqs * ceil_div(rows, per_wg)); };
  const int rb = (s.head_dim + 2) * 4;
  hipStream_t stm = static_cast<hipStream_t>(stream);
  const bool status = a.b.status != nullptr;
  const long long reports = status ? a.b.batch : 0;  // workgroups that report a sequence's status
  auto apart = [&] { return status_apart(x.b) && (x.b.total_new == 0 || output_apart(plan, x)); };
  hipError_t e;
  if (s.dtype == RESPEC_F32) {
    a.few_rows = 0;
    a.few = ChunkGeom{1, 1, INT_MAX, 0, fast_div(INT_MAX)};
    a.wide = geometry(a.b, 64, blocks(64), limit, 32, 32, 2, s.head_dim == 128 ? Pace{0.16, 5} : Pace{0.1, 5}, rb, held);
    if (!launchable(a.wide.items + reports, kAttnF32Threads) || !apart()) return RESPEC_ERR_SHAPE;
    e = launch_chunk_attn_f32(s.head_dim, q8 != nullptr, a, status, stm);
  } else {
    // Calls of at most 64 query rows per KV head have the few-row kernel, of one or two groups of 32 (over an 8-bit cache: of one,
    // two or four of 16); others have 256-row blocks, and sequences of up to 32 rows among them the few-row kernel's way in the same launch.
    const bool wide = rows > 64, mixed = wide && a.b.batch > 1;
    a.few_rows = !wide ? (q8 && rows <= 16 ? 16 : rows <= 32 ? 32 : 64) : mixed ? 32 : 0;
    // Few rows over an 8-bit cache: up to 32 rows, two workgroups to a CU, 33-64 rows one.  (25 batches of decoding tokens and short
    // chunks, over the best of eleven splits each: 1.02 times its time, with the other cache's paces 1.08; 13 more with heads of
    // 64: 1.04.)  Long chunks have the other cache's paces (44 calls, over the best of thirteen splits each: 1.04; paces fitted to
    // these calls 1.03).
    if (q8 && !wide)
      a.few = a.few_rows <= 32 ? geometry(a.b, a.few_rows, seqs, limit, 128, 512, 2, Pace{0.005, 4, 6, 0.4}, rb, held)
                               : geometry(a.b, a.few_rows, seqs, limit, 128, 256, 1, Pace{0.0142, 5, 6, 0.4}, rb, held);
    else
      a.few = !wide || mixed ? geometry(a.b, a.few_rows, seqs, limit, 128, 128, 1,
                                        s.head_dim == 128 ? Pace{0.02, 6} : Pace{0.01, 6}, rb, held)
                             : ChunkGeom{1, 1, INT_MAX, 0, fast_div(INT_MAX)};
    a.wide = wide ? geometry(a.b, 256, blocks(256), limit, 128, 256, 1, s.head_dim == 128 ? Pace{0.032, 6} : Pace{0.018, 6}, rb, held)
                  : ChunkGeom{1, 1, INT_MAX, 0, fast_div(INT_MAX)};
    if (!launchable((long long)a.few.items + a.wide.items + reports, wide ? kAttnWideThreads : kAttnFewThreads) || !apart())
      return RESPEC_ERR_SHAPE;
    if (!raise_lds_limits(s.head_dim, q8 != nullptr)) return RESPEC_ERR_HIP;
    if (q8)
      e = wide ? launch_q8_attn_wide(s.head_dim, a, mixed, status, stm) : launch_q8_attn_few(s.head_dim, a, status, stm);
    else
      e = wide ? launch_chunk_attn_wide(s.head_dim, a, mixed, status, stm) : launch_chunk_attn_few(s.head_dim, a, status, stm);
  }
  if (e != hipSuccess) return RESPEC_ERR_HIP;
  if (x.b.total_new > 0 && (a.few.nsplit > 1 || a.wide.nsplit > 1) &&
      launch_chunk_merge(s.dtype, s.head_dim, a, stm) != hipSuccess)
    return RESPEC_ERR_HIP;
  return RESPEC_OK;
}

}  // namespace

extern "C" {

respec_status respec_chunk_create(const respec_chunk_shape* shape, respec_chunk_plan** out) {
  if (!shape || !out) return RESPEC_ERR_NULL;
  *out = nullptr;
  const respec_chunk_shape& s = *shape;
  if (!known(s.dtype)) return RESPEC_ERR_DTYPE;
  if (s.head_dim != 64 && s.head_dim != 128) return RESPEC_ERR_SHAPE;
  if (s.n_q_heads < 1 || s.n_q_heads > RESPEC_CHUNK_MAX_HEADS || s.n_kv_heads < 1 || s.n_q_heads % s.n_kv_heads != 0)
    return RESPEC_ERR_SHAPE;
  if (s.max_batch < 1 || s.max_batch > RESPEC_CHUNK_MAX_BATCH || s.max_new < 1 || s.max_kv_len < 0) return RESPEC_ERR_SHAPE;
  if ((long long)s.max_new * s.n_q_heads > INT_MAX || (long long)s.max_new + s.max_kv_len > kMaxRows) return RESPEC_ERR_SHAPE;
  respec_chunk_plan* p = new (std::nothrow) respec_chunk_plan();
  if (!p) return RESPEC_ERR_CAPACITY;
  p->s = s;
  p->es = s.dtype == RESPEC_BF16 ? 2 : 4;
  p->part_rows = std::min((size_t)s.max_new * s.n_q_heads * kMaxSplits, kMaxPartial / s.head_dim);
  p->total = align256(p->part_rows * s.head_dim * 4) + 2 * align256(p->part_rows * 4);
  *out = p;
  return RESPEC_OK;
}

void respec_chunk_destroy(respec_chunk_plan* plan) { delete plan; }

size_t respec_chunk_workspace_bytes(const respec_chunk_plan* plan) { return plan ? plan->total : 0; }

respec_status respec_chunk_append(const respec_chunk_plan* plan, const respec_chunk_append_args* args, void* stream) {
  if (!plan || !args) return RESPEC_ERR_NULL;
  const respec_chunk_append_args& x = *args;
  const respec_status st = check_batch(plan, x.b, plan->es);
  if (st != RESPEC_OK) return st;
  if (x.b.batch == 0) return RESPEC_OK;
  if (x.b.total_new > 0) {
    const respec_status rows = check_new_rows(plan, x);
    if (rows != RESPEC_OK) return rows;
  } else if (!x.b.seq_status) {
    return RESPEC_OK;
  }
  AppendArgs a;
  a.b = device_batch(plan, x.b, plan->es);
  a.k_new = static_cast<const char*>(x.k_new);
  a.v_new = static_cast<const char*>(x.v_new);
  a.k_tok = x.k_token_stride * plan->es;
  a.k_head = x.k_head_stride * plan->es;
  a.v_tok = x.v_token_stride * plan->es;
  a.v_head = x.v_head_stride * plan->es;
  const int pieces = 2 * plan->s.n_kv_heads * plan->s.head_dim * plan->es / 16;  // of a token
  a.per_tok = fast_div((uint32_t)pieces);
  a.tok_per_wg = std::max(1, std::min(2048 / pieces, kAppendMaxTok));
  if (!launchable(ceil_div(x.b.total_new, a.tok_per_wg) + (x.b.seq_status ? x.b.batch : 0), kAppendThreads) || !status_apart(x.b))
    return RESPEC_ERR_SHAPE;
  return launch_chunk_append(plan->es, plan->s.head_dim, a, static_cast<hipStream_t>(stream)) == hipSuccess
             ? RESPEC_OK
             : RESPEC_ERR_HIP;
}

respec_status respec_chunk_attn(const respec_chunk_plan* plan, const respec_chunk_attn_args* args, void* workspace,
                                void* stream) {
  if (!plan || !args) return RESPEC_ERR_NULL;
  return attend(plan, *args, nullptr, workspace, stream);
}

respec_status respec_chunk_attn_q8(const respec_chunk_plan* plan, const respec_q8_attn_args* args, void* workspace,
                                   void* stream) {
  if (!plan || !args) return RESPEC_ERR_NULL;
  const respec_q8_attn_args& x = *args;
  return attend(plan,
                respec_chunk_attn_args{codes_batch(x.b), x.q, x.q_token_stride, x.q_head_stride, x.out, x.out_token_stride,
                                       x.out_head_stride, x.scale},
                &x.b.cache, workspace, stream);
}

respec_status respec_chunk_append_q8(const respec_chunk_plan* plan, const respec_q8_append_args* args, void* stream) {
  if (!plan || !args) return RESPEC_ERR_NULL;
  const respec_q8_append_args& x = *args;
  const respec_chunk_batch b = codes_batch(x.b);
  const respec_status st = check_batch(plan, b, 1);
  if (st != RESPEC_OK) return st;
  if (b.batch == 0) return RESPEC_OK;
  const respec_status scales = check_scales(x.b.cache);
  if (scales != RESPEC_OK) return scales;
  if (b.total_new > 0) {
    const respec_status rows = check_new_rows(plan, x);
    if (rows != RESPEC_OK) return rows;
  }
  AppendQ8Args a;
  a.b = device_batch(plan, b, 1);
  a.q8 = device_scales(x.b.cache);
  a.k_new = static_cast<const char*>(x.k_new);
  a.v_new = static_cast<const char*>(x.v_new);
  a.k_tok = x.k_token_stride * plan->es;
  a.k_head = x.k_head_stride * plan->es;
  a.v_tok = x.v_token_stride * plan->es;
  a.v_head = x.v_head_stride * plan->es;
  a.per_block = fast_div((uint32_t)(2 * plan->s.n_kv_heads));
  // blocks that the new rows can touch: a sequence's n tokens at most (n + block - 2) / block + 1 and n
  const long long block = x.b.cache.scale_block, total = b.total_new, seqs = std::min((long long)b.batch, total);
  const long long each = std::min((long long)b.max_new_in_batch, (b.max_new_in_batch + block - 2) / block + 1);
  const long long blocks = std::min({total, total / block + 2 * seqs, seqs * each});
  const int waves = block == 128 ? 8 : kAppendQ8Waves, per_wg = waves / (int)(block / 16);
  const long long wgs = ceil_div(blocks * 2 * plan->s.n_kv_heads, per_wg), reports = b.seq_status ? b.batch : 0;
  if (wgs + reports == 0) return RESPEC_OK;
  if (!launchable(wgs + reports, 64 * waves) || !status_apart(b)) return RESPEC_ERR_SHAPE;
  a.wgs = (int)wgs;
  return launch_append_q8(plan->es, plan->s.head_dim, a, static_cast<hipStream_t>(stream)) == hipSuccess ? RESPEC_OK : RESPEC_ERR_HIP;
}

respec_status respec_score_create(const respec_score_shape* shape, respec_score_plan** out) {
  if (!shape || !out) return RESPEC_ERR_NULL;
  *out = nullptr;
  const respec_score_shape& s = *shape;
  if (!known(s.dtype)) return RESPEC_ERR_DTYPE;
  if (s.topk_out < 1 || s.topk_out > RESPEC_MAX_TOPK_OUT || s.vocab < s.topk_out || s.vocab >= 1 << 30 || s.max_rows < 1)
    return RESPEC_ERR_SHAPE;
  if (!launchable(s.max_rows, kScoreThreads)) return RESPEC_ERR_SHAPE;  // (more parts than rows: kScoreParts in all)
  respec_score_plan* p = new (std::nothrow) respec_score_plan();
  if (!p) return RESPEC_ERR_CAPACITY;
  p->s = s;
  p->ko = s.topk_out <= 8 ? 8 : 16;
  // rows in parts: at most kScoreParts workgroups in all (one row: kScoreMaxKeys / ko)
  const long long records = std::min({(long long)s.max_rows * (kScoreMaxKeys / p->ko), (long long)kScoreParts});
  p->total = align256((size_t)records * (kScoreWords + 2 * p->ko) * 4);
  *out = p;
  return RESPEC_OK;
}

void respec_score_destroy(respec_score_plan* plan) { delete plan; }

size_t respec_score_workspace_bytes(const respec_score_plan* plan) { return plan ? plan->total : 0; }

respec_status respec_score(const respec_score_plan* plan, const respec_score_args* args, void* workspace,
                           void* stream) {
  if (!plan || !args) return RESPEC_ERR_NULL;
  if (!workspace || !aligned(workspace, 256)) return RESPEC_ERR_WORKSPACE;
  const respec_score_shape& s = plan->s;
  const respec_score_args& x = *args;
  if (x.rows < 0) return RESPEC_ERR_SHAPE;
  if (x.rows > s.max_rows) return RESPEC_ERR_CAPACITY;
  if (x.rows == 0) return RESPEC_OK;
  if (!x.logits) return RESPEC_ERR_NULL;
  const int es = s.dtype == RESPEC_BF16 ? 2 : 4;
  if (!aligned(x.logits, es) || (x.rows > 1 && (x.row_stride < s.vocab || x.row_stride >= 1ll << 50))) return RESPEC_ERR_SHAPE;
  ScoreArgs a;
  a.z = x.logits;
  a.row_stride = x.row_stride;
  a.token = x.token;
  a.part = static_cast<float*>(workspace);
  a.tok_logprob = x.tok_logprob;
  a.tok_rank = x.tok_rank;
  a.lse = x.lse;
  a.entropy = x.entropy;
  a.topk_id = x.topk_id;
  a.topk_logprob = x.topk_logprob;
  a.rows = x.rows;
  a.vocab = s.vocab;
  a.topk_out = s.topk_out;
  a.parts = std::max(1, std::min({kScoreParts / x.rows, kScoreMaxKeys / plan->ko, s.vocab / 2048}));
  return launch_score(s.dtype, plan->ko, a, static_cast<hipStream_t>(stream)) == hipSuccess ? RESPEC_OK : RESPEC_ERR_HIP;
}

}  // extern "C"

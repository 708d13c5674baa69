// Host side of the prompt side's C ABI: plans, argument validation, launches.
// See include/respec_prompt.h for the contract.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <atomic>
#include <new>

#include "../../../include/respec_prompt.h"
#include "../attn_route.hpp"
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

respec_status check_batch(const respec_chunk_plan* plan, const respec_chunk_batch& b) {
  const respec_chunk_shape& s = plan->s;
  if (b.batch < 0 || b.total_new < 0 || b.max_new_in_batch < 0 || b.max_kv_len_in_batch < 0) return RESPEC_ERR_SHAPE;
  if (b.batch > s.max_batch || b.total_new > s.max_new || b.max_kv_len_in_batch > s.max_kv_len) return RESPEC_ERR_CAPACITY;
  if (b.max_new_in_batch > b.total_new) return RESPEC_ERR_SHAPE;
  if (b.batch == 0) return RESPEC_OK;
  const respec_paged_cache& c = b.cache;
  if (!b.new_off || !b.kv_len || !c.k || !c.v || !c.page_table) return RESPEC_ERR_NULL;
  if (c.n_pages < 1 || c.page_size < 1 || c.table_width < 1) return RESPEC_ERR_SHAPE;
  if (b.batch > 1 && c.table_stride < c.table_width) return RESPEC_ERR_SHAPE;
  if (!stride_ok(c.page_stride, plan->es) || !stride_ok(c.head_stride, plan->es) || !stride_ok(c.row_stride, plan->es) ||
      c.row_stride > kMaxStride)
    return RESPEC_ERR_SHAPE;
  if (!aligned(c.k, 16) || !aligned(c.v, 16)) return RESPEC_ERR_SHAPE;
  return RESPEC_OK;
}

ChunkBatch device_batch(const respec_chunk_plan* plan, const respec_chunk_batch& b) {
  const respec_paged_cache& c = b.cache;
  ChunkBatch d;
  d.new_off = b.new_off;
  d.kv_len = b.kv_len;
  d.table = c.page_table;
  d.status = b.seq_status;
  d.k = static_cast<char*>(c.k);
  d.v = static_cast<char*>(c.v);
  d.page_stride = c.page_stride * plan->es;
  d.head_stride = c.head_stride * plan->es;
  d.table_stride = c.table_stride;
  d.row_stride = (uint32_t)(c.row_stride * plan->es);
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

// How long an attention kernel takes over one cache row of a block, with all the workgroups of a CU that the pace was
// taken with, and to start a workgroup (us).
struct Pace {
  double row, start;
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
  constexpr double kShare = 0.5;
  ChunkGeom g{rows_per_wg, 1, INT_MAX, 0, fast_div(INT_MAX)};
  const long long items = blocks * b.n_kv_heads;
  double best = 0;
  long long most = std::min({ceil_div(limit, least), (long long)kMaxSplits, held, items > 0 ? (long long)INT_MAX / items : 1});
  for (long long n = 1, rows_before = 0; n <= std::max(most, 1ll); n += 1 + n / 6) {
    const long long rows = ceil_div(ceil_div(limit, n), unit) * unit;
    if (rows == rows_before) continue;
    rows_before = rows;
    const double wgs = (double)items * ceil_div(limit, std::max(rows, 1ll)) / (kCUs * per_cu);
    const double rounds = b.batch == 1 ? ceil(wgs) : std::max(1.0, wgs * kShare) + 0.5;
    const double joined = 1e-6 * n * b.total_new * b.n_kv_heads * b.group * row_bytes * 2 / 4.5;
    const double merge = n == 1 ? 0 : 4 + joined * (b.batch == 1 ? 1 : kShare);
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

// Raise the LDS limits of the attention kernels on the current device, once (a call into the runtime that also
// loads the kernels: the first step pays it).
bool raise_lds_limits(int head_dim) {
  constexpr int kMaxDevices = 64;
  static std::atomic<uint64_t> done[2];  // [head size], a bit per device
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return false;
  std::atomic<uint64_t>& d = done[head_dim == 128];
  const uint64_t bit = dev < kMaxDevices ? 1ull << dev : 0;  // (past the last: every call raises them)
  if (d.load(std::memory_order_acquire) & bit) return true;
  if (set_chunk_attn_few_lds_limit(head_dim) != hipSuccess || set_chunk_attn_wide_lds_limit(head_dim) != hipSuccess) return false;
  d.fetch_or(bit, std::memory_order_release);
  return true;
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
  const respec_status st = check_batch(plan, x.b);
  if (st != RESPEC_OK) return st;
  if (x.b.batch == 0) return RESPEC_OK;
  if (x.b.total_new > 0) {
    if (!x.k_new || !x.v_new) return RESPEC_ERR_NULL;
    if (!aligned(x.k_new, 16) || !aligned(x.v_new, 16)) return RESPEC_ERR_SHAPE;
    for (int64_t s : {x.k_token_stride, x.k_head_stride, x.v_token_stride, x.v_head_stride})
      if (!stride_ok(s, plan->es)) return RESPEC_ERR_SHAPE;
  } else if (!x.b.seq_status) {
    return RESPEC_OK;
  }
  AppendArgs a;
  a.b = device_batch(plan, x.b);
  a.k_new = static_cast<const char*>(x.k_new);
  a.v_new = static_cast<const char*>(x.v_new);
  a.k_tok = x.k_token_stride * plan->es;
  a.k_head = x.k_head_stride * plan->es;
  a.v_tok = x.v_token_stride * plan->es;
  a.v_head = x.v_head_stride * plan->es;
  const int pieces = 2 * plan->s.n_kv_heads * plan->s.head_dim * plan->es / 16;  // of a token
  a.per_tok = fast_div((uint32_t)pieces);
  a.tok_per_wg = std::max(1, std::min(2048 / pieces, kAppendMaxTok));
  if (!launchable(ceil_div(x.b.total_new, a.tok_per_wg) + (x.b.seq_status ? x.b.batch : 0), kAppendThreads)) return RESPEC_ERR_SHAPE;
  return launch_chunk_append(plan->es, plan->s.head_dim, a, static_cast<hipStream_t>(stream)) == hipSuccess
             ? RESPEC_OK
             : RESPEC_ERR_HIP;
}

respec_status respec_chunk_attn(const respec_chunk_plan* plan, const respec_chunk_attn_args* args, void* workspace,
                                void* stream) {
  if (!plan || !args) return RESPEC_ERR_NULL;
  if (!workspace || !aligned(workspace, 256)) return RESPEC_ERR_WORKSPACE;
  const respec_chunk_attn_args& x = *args;
  const respec_status st = check_batch(plan, x.b);
  if (st != RESPEC_OK) return st;
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
  a.b = device_batch(plan, x.b);
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
  hipError_t e;
  if (s.dtype == RESPEC_F32) {
    a.few_rows = 0;
    a.few = ChunkGeom{1, 1, INT_MAX, 0, fast_div(INT_MAX)};
    a.wide = geometry(a.b, 64, blocks(64), limit, 32, 32, 2, s.head_dim == 128 ? Pace{0.16, 5} : Pace{0.1, 5}, rb, held);
    if (!launchable(a.wide.items + reports, kAttnF32Threads)) return RESPEC_ERR_SHAPE;
    e = launch_chunk_attn_f32(s.head_dim, a, status, stm);
  } else {
    // Calls of at most 64 query rows per KV head have the few-row kernel, of one or two groups of 32; others have
    // 256-row blocks, and sequences of up to 32 rows among them the few-row kernel's way in the same launch.
    const bool wide = rows > 64, mixed = wide && a.b.batch > 1;
    a.few_rows = !wide ? (rows <= 32 ? 32 : 64) : mixed ? 32 : 0;
    a.few = !wide || mixed ? geometry(a.b, a.few_rows, seqs, limit, 128, 128, 1,
                                      s.head_dim == 128 ? Pace{0.02, 6} : Pace{0.01, 6}, rb, held)
                           : ChunkGeom{1, 1, INT_MAX, 0, fast_div(INT_MAX)};
    a.wide = wide ? geometry(a.b, 256, blocks(256), limit, 128, 256, 1, s.head_dim == 128 ? Pace{0.032, 6} : Pace{0.018, 6}, rb, held)
                  : ChunkGeom{1, 1, INT_MAX, 0, fast_div(INT_MAX)};
    if (!launchable((long long)a.few.items + a.wide.items + reports, wide ? kAttnWideThreads : kAttnFewThreads)) return RESPEC_ERR_SHAPE;
    if (!raise_lds_limits(s.head_dim)) return RESPEC_ERR_HIP;
    e = wide ? launch_chunk_attn_wide(s.head_dim, a, mixed, status, stm) : launch_chunk_attn_few(s.head_dim, a, status, stm);
  }
  if (e != hipSuccess) return RESPEC_ERR_HIP;
  if (x.b.total_new > 0 && (a.few.nsplit > 1 || a.wide.nsplit > 1) &&
      launch_chunk_merge(s.dtype, s.head_dim, a, stm) != hipSuccess)
    return RESPEC_ERR_HIP;
  return RESPEC_OK;
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

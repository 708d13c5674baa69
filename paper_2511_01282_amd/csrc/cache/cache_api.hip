// Host side of rotary positions, kept rows and copied pages: argument validation and launches.
// See include/respec_cache.h for the contract.
#include <limits.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "../../../include/respec_cache.h"
#include "../overlap.hpp"
#include "cache.hpp"

using namespace respec;

struct respec_rotary_plan {
  respec_rotary_shape s;
  int es;
  uint64_t turns[kRotaryMaxPairs];
};

namespace {

bool aligned(const void* p, size_t n) { return ((uintptr_t)p % n) == 0; }
bool known(int32_t dtype) { return dtype == RESPEC_F32 || dtype == RESPEC_BF16; }
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }
constexpr long long kMaxStride = 1ll << 50;  // bytes or elements
bool stride_ok(int64_t s, int es) { return s >= 0 && s < kMaxStride && s * es % 16 == 0; }
// A dispatch counts its threads in 32 bits (and its workgroups of the second and third dimension in 16).
bool launchable(long long workgroups, int threads) { return workgroups >= 0 && workgroups < (1ll << 32) / threads; }

// Whether rotary outputs share bytes with nothing that another thread reads or writes: an output may be its input.
bool outputs_apart(const respec_rotary_plan* plan, const respec_rotary_args& x) {
  const int es = plan->es;
  const int64_t t = x.tokens, row = (int64_t)plan->s.head_dim * es;
  const int hq = plan->s.n_q_heads, hkv = plan->s.n_kv_heads;
  auto rows = [&](const void* p, int64_t token, int h, int64_t head) { return row_set(p, t, token * es, h, head * es, row); };
  const RowSet in[2] = {rows(x.q, x.q_token_stride, hq, x.q_head_stride), rows(x.k, x.k_token_stride, hkv, x.k_head_stride)};
  const RowSet out[2] = {rows(x.q_out, x.q_out_token_stride, hq, x.q_out_head_stride), rows(x.k_out, x.k_out_token_stride, hkv, x.k_out_head_stride)};
  for (int i = 0; i < 2; ++i) {
    if (!out[i].at) continue;
    if (i == 0 ? overlap_within(t, x.q_out_token_stride * es, hq, x.q_out_head_stride * es, row)
               : overlap_within(t, x.k_out_token_stride * es, hkv, x.k_out_head_stride * es, row))
      return false;
    for (int j = 0; j < 2; ++j)
      if (in[j].at && !(i == j && same_rows(out[i], in[j])) && overlap(out[i], in[j])) return false;
  }
  return !(out[0].at && out[1].at && overlap(out[0], out[1]));
}

constexpr double kTurn = 6.283185307179586;  // 2 pi, rounded down
// 2^64 times the fraction of a turn that w radians are, to 2^-63 of w and half a unit: under 2^-62, so that 2^31 positions further the
// angle is within 2^-31 of a turn.
uint64_t turns_of(double w) {
  const long double turns = fmodl((long double)w / (2 * 3.141592653589793238462643383279502884L), 1.0L);
  const long double scaled = roundl(ldexpl(turns, 64));
  return scaled >= ldexpl(1.0L, 64) ? 0 : (uint64_t)scaled;
}

}  // namespace

extern "C" {

respec_status respec_rotary_create(const respec_rotary_shape* shape, const double* frequency, respec_rotary_plan** out) {
  if (!shape || !frequency || !out) return RESPEC_ERR_NULL;
  *out = nullptr;
  const respec_rotary_shape& s = *shape;
  if (!known(s.dtype)) return RESPEC_ERR_DTYPE;
  if (s.head_dim != 64 && s.head_dim != 128) return RESPEC_ERR_SHAPE;
  if (s.n_q_heads < 1 || s.n_q_heads > RESPEC_CHUNK_MAX_HEADS || s.n_kv_heads < 1 || s.n_kv_heads > RESPEC_CHUNK_MAX_HEADS)
    return RESPEC_ERR_SHAPE;
  if (s.rotary_dim < 16 || s.rotary_dim > s.head_dim || s.rotary_dim % 16 != 0) return RESPEC_ERR_SHAPE;
  if (s.max_tokens < 1 || s.max_tokens > RESPEC_ROTARY_MAX_TOKENS) return RESPEC_ERR_SHAPE;
  if (s.layout != RESPEC_ROTARY_HALF && s.layout != RESPEC_ROTARY_INTERLEAVED) return RESPEC_ERR_PARAM;
  if (!(s.amplitude >= 0.f) || isinf(s.amplitude)) return RESPEC_ERR_PARAM;
  for (int i = 0; i < s.rotary_dim / 2; ++i)
    if (!(frequency[i] >= 0.0) || frequency[i] > kTurn) return RESPEC_ERR_PARAM;
  respec_rotary_plan* p = new (std::nothrow) respec_rotary_plan();
  if (!p) return RESPEC_ERR_CAPACITY;
  p->s = s;
  p->es = s.dtype == RESPEC_BF16 ? 2 : 4;
  for (int i = 0; i < s.rotary_dim / 2; ++i) p->turns[i] = turns_of(frequency[i]);
  *out = p;
  return RESPEC_OK;
}

void respec_rotary_destroy(respec_rotary_plan* plan) { delete plan; }

respec_status respec_rotary(const respec_rotary_plan* plan, const respec_rotary_args* args, void* stream) {
  if (!plan || !args) return RESPEC_ERR_NULL;
  const respec_rotary_shape& s = plan->s;
  const respec_rotary_args& x = *args;
  const int es = plan->es;
  if (x.tokens < 0) return RESPEC_ERR_SHAPE;
  if (x.tokens > s.max_tokens) return RESPEC_ERR_CAPACITY;
  if (!x.positions) {
    if (x.batch < 0 || x.batch > RESPEC_CHUNK_MAX_BATCH) return RESPEC_ERR_SHAPE;
    if (x.batch > 0 && (!x.new_off || !x.kv_len)) return RESPEC_ERR_NULL;
  } else if (x.seq_status) {
    return RESPEC_ERR_PARAM;
  }
  if (x.tokens > 0) {
    if (!x.q != !x.q_out || !x.k != !x.k_out) return RESPEC_ERR_NULL;
    for (const void* p : {x.q, (const void*)x.q_out, x.k, (const void*)x.k_out})
      if (p && !aligned(p, 16)) return RESPEC_ERR_SHAPE;
    if (x.q)
      for (int64_t v : {x.q_token_stride, x.q_head_stride, x.q_out_token_stride, x.q_out_head_stride})
        if (!stride_ok(v, es)) return RESPEC_ERR_SHAPE;
    if (x.k)
      for (int64_t v : {x.k_token_stride, x.k_head_stride, x.k_out_token_stride, x.k_out_head_stride})
        if (!stride_ok(v, es)) return RESPEC_ERR_SHAPE;
  }
  const int reports = !x.positions && x.seq_status ? (int)ceil_div(x.batch, kRotaryThreads) : 0;
  const bool rows = x.tokens > 0 && (x.q || x.k) && (x.positions || x.batch > 0);
  if (!rows && reports == 0) return RESPEC_OK;
  RotaryArgs a;
  memset(&a, 0, sizeof a);
  a.positions = x.positions;
  // (a sequence as chunk_seq() checks it: tokens of the call, positions below 2^30)
  a.b.new_off = x.new_off;
  a.b.kv_len = x.kv_len;
  a.b.status = x.seq_status;
  a.b.batch = x.batch;
  a.b.total_new = a.b.max_new = x.tokens;
  a.b.max_kv = 1 << 30;
  a.b.table_width = 1 << 30;
  a.b.page = fast_div(1);
  auto side = [&](const void* from, int64_t ft, int64_t fh, void* to, int64_t tt, int64_t th) {
    return RotaryRows{static_cast<const char*>(from), static_cast<char*>(to), ft * es, fh * es, tt * es, th * es};
  };
  a.q = side(x.q, x.q_token_stride, x.q_head_stride, x.q_out, x.q_out_token_stride, x.q_out_head_stride);
  a.k = side(x.k, x.k_token_stride, x.k_head_stride, x.k_out, x.k_out_token_stride, x.k_out_head_stride);
  a.q_heads = x.q ? s.n_q_heads : 0;
  a.heads = std::max(1, a.q_heads + (x.k ? s.n_kv_heads : 0));
  a.tokens = rows ? x.tokens : 0;
  a.amplitude = s.amplitude > 0.f ? s.amplitude : 1.f;
  memcpy(a.turns, plan->turns, sizeof a.turns);
  const int units = s.head_dim * es / 32;
  a.turned = s.rotary_dim * es / 32;
  // Four heads to a thread where that still leaves each CU a workgroup: the angles are half of a thread's work otherwise.  (32 + 8 heads
  // of 128, bf16, one and four heads: 512 tokens 9.2 and 9.2 us, 2048 12.3 and 11.4, 4096 18.9 and 16.9, 8192 38.1 and 38.8; 28 + 4: 512
  // 8.5 and 9.2, 4096 16.1 and 14.4.)
  const long long items = (long long)a.tokens * a.heads * units;
  const int r = items >= 4ll * kRotaryThreads * 256 ? 4 : 1;
  a.stride = fast_div((uint32_t)ceil_div(a.heads, r));
  const int slots = (int)a.stride.d * units;
  a.tok_per_wg = std::max(1, kRotaryThreads / slots);
  a.status_wgs = reports;
  const long long wgs = reports + ceil_div(a.tokens, a.tok_per_wg), per_token = a.tok_per_wg > 1 ? 1 : ceil_div(slots, kRotaryThreads);
  if (!launchable(wgs * per_token, kRotaryThreads)) return RESPEC_ERR_SHAPE;
  if (rows && !outputs_apart(plan, x)) return RESPEC_ERR_SHAPE;
  // (a status is written while workgroups of tokens still read offsets and lengths)
  if (reports > 0 && (overlap(x.seq_status, 4ll * x.batch, x.new_off, 1, 0, 4ll * x.batch + 4) ||
                      overlap(x.seq_status, 4ll * x.batch, x.kv_len, 1, 0, 4ll * x.batch)))
    return RESPEC_ERR_SHAPE;
  return launch_rotary(es, s.head_dim, s.layout == RESPEC_ROTARY_HALF, r, (int)wgs, (int)per_token, a, static_cast<hipStream_t>(stream)) ==
                 hipSuccess
             ? RESPEC_OK
             : RESPEC_ERR_HIP;
}

respec_status respec_cache_keep(const respec_cache_keep_args* args, void* stream) {
  if (!args) return RESPEC_ERR_NULL;
  const respec_cache_keep_args& x = *args;
  const respec_paged_cache& c = x.cache;
  if (!known(x.dtype)) return RESPEC_ERR_DTYPE;
  const int es = x.dtype == RESPEC_BF16 ? 2 : 4;
  if (x.batch < 0 || x.batch > RESPEC_CHUNK_MAX_BATCH || x.n_layers < 1 || x.n_layers > 65535) return RESPEC_ERR_SHAPE;
  if (x.n_kv_heads < 1 || x.n_kv_heads > RESPEC_CHUNK_MAX_HEADS || (x.head_dim != 64 && x.head_dim != 128)) return RESPEC_ERR_SHAPE;
  if (x.path_width < 1 || x.path_width > kKeepMaxPath) return RESPEC_ERR_SHAPE;
  if (x.batch == 0) return RESPEC_OK;
  if (!c.k || !c.v || !c.page_table || !x.kv_len || !x.path || !x.acc_len) return RESPEC_ERR_NULL;
  if (c.n_pages < 1 || c.page_size < 1 || c.table_width < 1) return RESPEC_ERR_SHAPE;
  if (x.batch > 1 && (c.table_stride < c.table_width || x.path_stride < x.path_width)) return RESPEC_ERR_SHAPE;
  for (int64_t s : {c.page_stride, c.head_stride, c.row_stride, x.layer_stride})
    if (!stride_ok(s, es)) return RESPEC_ERR_SHAPE;
  if (c.row_stride > 1 << 24 || !aligned(c.k, 16) || !aligned(c.v, 16)) return RESPEC_ERR_SHAPE;
  KeepArgs a;
  memset(&a, 0, sizeof a);
  a.b.kv_len = x.kv_len;
  a.b.table = c.page_table;
  a.b.status = x.seq_status;
  a.b.k = static_cast<char*>(c.k);
  a.b.v = static_cast<char*>(c.v);
  a.b.page_stride = c.page_stride * es;
  a.b.head_stride = c.head_stride * es;
  a.b.row_stride = (uint32_t)(c.row_stride * es);
  a.b.table_stride = c.table_stride;
  a.b.page = fast_div((uint32_t)c.page_size);
  a.b.batch = x.batch;
  a.b.n_pages = c.n_pages;
  a.b.table_width = c.table_width;
  a.layer_stride = x.layer_stride * es;
  a.path = x.path;
  a.path_stride = x.path_stride;
  a.path_width = x.path_width;
  a.acc_len = x.acc_len;
  a.kv_len_out = x.kv_len_out;
  a.pieces = x.n_kv_heads * x.head_dim * es / 16;
  if (!launchable(ceil_div(2 * a.pieces, kKeepThreads) * x.n_layers * x.batch, kKeepThreads)) return RESPEC_ERR_SHAPE;
  const int64_t row = (int64_t)x.head_dim * es;
  if (overlap_within(x.n_layers, a.layer_stride, row) || overlap_within(c.n_pages, c.page_stride * es, row) ||
      overlap_within(x.n_kv_heads, c.head_stride * es, row) || overlap_within(c.page_size, c.row_stride * es, row))
    return RESPEC_ERR_SHAPE;  // (rows in one place would be moved more than once)
  // A sequence's length and status are written by its first workgroup, while those of other layers may not have started.
  const int64_t ints = 4ll * x.batch;
  const __int128 path_step = x.batch > 1 ? (__int128)4 * x.path_stride : 0, table_step = x.batch > 1 ? (__int128)4 * c.table_stride : 0;
  for (const int32_t* to : {x.kv_len_out, x.seq_status})
    if (overlap(to, ints, x.kv_len, 1, 0, ints) || overlap(to, ints, x.acc_len, 1, 0, ints) ||
        overlap(to, ints, x.path, x.batch, path_step, 4ll * x.path_width) ||
        overlap(to, ints, c.page_table, x.batch, table_step, 4ll * c.table_width))
      return RESPEC_ERR_SHAPE;
  if (overlap(x.kv_len_out, ints, x.seq_status, 1, 0, ints)) return RESPEC_ERR_SHAPE;
  return launch_keep(x.head_dim * es, x.n_layers, a, static_cast<hipStream_t>(stream)) == hipSuccess ? RESPEC_OK : RESPEC_ERR_HIP;
}

respec_status respec_cache_copy(const respec_cache_copy_args* args, void* stream) {
  if (!args) return RESPEC_ERR_NULL;
  const respec_cache_copy_args& x = *args;
  if (x.pairs < 0 || x.pairs > RESPEC_CACHE_MAX_PAIRS || x.n_pages < 1 || x.n_planes < 1 || x.n_planes > RESPEC_CACHE_MAX_PLANES)
    return RESPEC_ERR_SHAPE;
  if (!x.planes) return RESPEC_ERR_NULL;
  CopyArgs a;
  memset(&a, 0, sizeof a);
  a.src = x.src;
  a.dst = x.dst;
  a.status = x.status;
  a.n_pages = x.n_pages;
  a.n_planes = x.n_planes;
  long long wgs = 0;
  int layers = 1;
  for (int i = 0; i < x.n_planes; ++i) {
    const respec_page_plane& p = x.planes[i];
    if (!p.base) return RESPEC_ERR_NULL;
    if (p.n_layers < 1 || p.n_layers > 65535 || p.heads < 1 || p.heads > 65535 || p.rows < 1 || p.row_bytes < 1) return RESPEC_ERR_SHAPE;
    for (int64_t s : {p.page_stride, p.layer_stride, p.head_stride, p.row_stride})
      if (s < 0 || s >= kMaxStride) return RESPEC_ERR_SHAPE;
    if (p.row_bytes > INT_MAX || (long long)p.heads * p.rows > INT_MAX || p.row_bytes > INT_MAX / ((long long)p.heads * p.rows)) return RESPEC_ERR_SHAPE;
    // runs that lie side by side are one
    long long heads = p.heads, rows = p.rows, run = p.row_bytes;
    if (rows == 1 || p.row_stride == run) {
      run *= rows;
      rows = 1;
      if (heads == 1 || p.head_stride == run) {
        run *= heads;
        heads = 1;
      }
    }
    // the widest piece that every address is a multiple of
    uint64_t bits = (uint64_t)(uintptr_t)p.base | (uint64_t)run | (uint64_t)p.page_stride | 16;
    if (p.n_layers > 1) bits |= (uint64_t)p.layer_stride;
    if (heads > 1) bits |= (uint64_t)p.head_stride;
    if (rows > 1) bits |= (uint64_t)p.row_stride;
    CopyPlane& d = a.plane[i];
    d.piece = (int)(bits & (~bits + 1));
    d.base = static_cast<char*>(p.base);
    d.page_stride = p.page_stride;
    d.layer_stride = p.layer_stride;
    d.head_stride = p.head_stride;
    d.row_stride = p.row_stride;
    d.n_layers = p.n_layers;
    d.first_wg = (int)wgs;
    const uint32_t per_row = (uint32_t)(run / d.piece);
    d.per_row = fast_div(per_row);
    d.per_head = fast_div((uint32_t)(per_row * rows));
    d.pieces = (uint32_t)(per_row * rows * heads);
    wgs += ceil_div(d.pieces, kCopyThreads * kCopyPieces);
    layers = std::max(layers, (int)p.n_layers);
  }
  if (x.pairs == 0) return RESPEC_OK;
  if (!x.src || !x.dst) return RESPEC_ERR_NULL;
  if (wgs > INT_MAX || !launchable(wgs, kCopyThreads) || !launchable(wgs * layers, kCopyThreads) ||
      !launchable(wgs * layers * x.pairs, kCopyThreads))
    return RESPEC_ERR_SHAPE;
  // (a pair's status is written while its other workgroups still read the ids)
  for (const int32_t* ids : {x.src, x.dst})
    if (overlap(x.status, 4ll * x.pairs, ids, 1, 0, 4ll * x.pairs)) return RESPEC_ERR_SHAPE;
  return launch_copy((int)wgs, layers, x.pairs, a, static_cast<hipStream_t>(stream)) == hipSuccess ? RESPEC_OK : RESPEC_ERR_HIP;
}

}  // extern "C"

// Internal launch interface of the prompt side's kernels (not part of the C ABI).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace respec {

// n / d for 32-bit n and a divisor fixed on the host: with l = ceil(log2 d) and
// m = floor(2^32 (2^l - d) / d) + 1, n / d = (t + (n - t) / 2^min(l,1)) / 2^max(l-1,0), t = floor(m n / 2^32)
// (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994).
struct FastDiv {
  uint32_t d, m, s1, s2;
};
inline FastDiv fast_div(uint32_t d) {  // d >= 1
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  FastDiv f;
  f.d = d;
  f.m = (uint32_t)((((1ull << l) - d) << 32) / d + 1);
  f.s1 = l < 1 ? l : 1;
  f.s2 = l < 1 ? 0 : l - 1;
  return f;
}
__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv& f) {
  const uint32_t t = __umulhi(f.m, n);
  return (t + ((n - t) >> f.s1)) >> f.s2;
}

// A chunk batch as the kernels see it; strides in bytes.
struct ChunkBatch {
  const int32_t* new_off;  // [B+1]
  const int32_t* kv_len;   // [B]
  const int32_t* table;
  int32_t* status;         // [B] or null
  char* k;
  char* v;
  int64_t page_stride, head_stride, table_stride;  // (table_stride: entries)
  uint32_t row_stride;
  FastDiv page;            // rows per page
  int32_t batch, total_new, max_new, max_kv, n_pages, table_width;
  int32_t n_kv_heads, group;
  FastDiv kv_heads;        // by n_kv_heads
};

struct AppendArgs {
  ChunkBatch b;
  const char* k_new;
  const char* v_new;
  int64_t k_tok, k_head, v_tok, v_head;  // bytes
  FastDiv per_tok;                        // 16-byte pieces of a token's K and V rows
  int32_t tok_per_wg;
};

// How an attention kernel cuts its sequences: a workgroup per (row block, split, KV head, sequence).
struct ChunkGeom {
  int32_t rows_per_wg;  // query rows, (token, head-in-group) pairs, of a block: a power of two
  int32_t nsplit;       // splits of the longest sequence; 1: no partials
  int32_t split_rows;   // cache rows of a split
  int32_t items;        // grid: (row block, split, sequence, KV head), see find_item
  FastDiv split;        // by split_rows
};

struct ChunkAttnArgs {
  ChunkBatch b;
  const char* q;
  char* out;
  int64_t q_tok, q_head, o_tok, o_head;  // bytes
  FastDiv group;
  float* part_o;      // [nsplit][total_new * Hq][D] unnormalised
  float* part_m;      // [nsplit][total_new * Hq] (log2 units)
  float* part_l;
  float scale_log2;   // scale * log2(e)
  // sequences of up to few_rows query rows per KV head are the first geometry's, the others the second's
  int32_t few_rows;
  ChunkGeom few, wide;
};

struct ScoreArgs {
  const void* z;
  int64_t row_stride;  // elements
  const int32_t* token;
  float* part;         // [rows][parts][kScoreWords + 2 KO]
  float* tok_logprob; int32_t* tok_rank; float* lse; float* entropy; int32_t* topk_id; float* topk_logprob;
  int32_t rows, vocab, topk_out, parts;
};
// threads of the kernels' workgroups
constexpr int kAppendThreads = 256, kScoreThreads = 256, kAttnF32Threads = 256, kAttnFewThreads = 256, kAttnWideThreads = 512;
constexpr int kAppendMaxTok = 16;  // tokens of an append workgroup
constexpr int kScoreWords = 4;  // m, S, T, rank count
constexpr int kScoreMaxKeys = 256;
constexpr int kScoreParts = 512;  // workgroups that a few rows are cut into (65 rows of 152064 float32
                                  // logits: 384 20.4 us, 512 18.9, 1024 19.7)

hipError_t launch_chunk_append(int es, int head_dim, const AppendArgs& a, hipStream_t s);
// float32; `status`: whether this launch reports the sequences' status
hipError_t launch_chunk_attn_f32(int head_dim, const ChunkAttnArgs& a, bool status, hipStream_t s);
// bf16: sequences of at most / more than few_rows query rows per KV head; mixed: of both kinds
hipError_t launch_chunk_attn_few(int head_dim, const ChunkAttnArgs& a, bool status, hipStream_t s);
hipError_t launch_chunk_attn_wide(int head_dim, const ChunkAttnArgs& a, bool mixed, bool status, hipStream_t s);
hipError_t set_chunk_attn_few_lds_limit(int head_dim);
hipError_t set_chunk_attn_wide_lds_limit(int head_dim);
hipError_t launch_chunk_merge(int dtype, int head_dim, const ChunkAttnArgs& a, hipStream_t s);
hipError_t launch_score(int dtype, int ko, const ScoreArgs& a, hipStream_t s);

}  // namespace respec

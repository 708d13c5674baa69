/* respec_prompt.h -- C ABI of the prompt side of a decoding process on MI355X (gfx950).
 *
 * What comes before the first verification step of respec_verify.h, and between
 * steps when a conversation goes on: the keys and values of new tokens go into
 * a cache, the new tokens attend to it, and their logits give the entropies
 * that the drafting session's trigger reads (respec_draft_session_append).
 *
 *   respec_chunk_append   K/V rows of new tokens into a paged cache
 *   respec_chunk_attn     causal attention of the new tokens over that cache: single
 *                         decoding tokens, pieces of a prompt, whole prompts, mixed
 *   respec_score          log probability and rank of given tokens, entropy and top
 *                         alternatives, one row of logits each
 *
 * The cache.  Row r (0-based position) of sequence b lies in page
 * page_table[b][r / page_size], at row r % page_size of it; element d of KV head
 * h at  page * page_stride + h * head_stride + (r % page_size) * row_stride + d.
 * A page may serve several sequences (a shared prefix).  The cache of a
 * verification step, [B][Hkv][L_cap][D], is the case page_size = L_cap with one
 * page per sequence.
 *
 * The new tokens.  Sequence b owns the packed tokens new_off[b] .. new_off[b+1]-1
 * (possibly none); its token i stands at position kv_len[b] + i: kv_len counts
 * the rows in front of the chunk, as in a verification step.
 *
 * Conventions (as in respec_verify.h)
 *  - Every tensor pointer is caller-owned DEVICE memory.  Nothing is allocated,
 *    freed or synchronised; a call only enqueues kernels on the caller's stream
 *    (a hipStream_t passed as void*, NULL = the null stream) and can be captured
 *    in a hipGraph.  The stream's device must be the current one.
 *  - Plans hold host metadata only, are immutable and may be shared by threads.
 *    Calls that may overlap need workspaces of their own; calls in order on one
 *    stream, captured or not, can share one.  A workspace needs no initialisation.
 *  - Host-side checks return a status and launch nothing; RESPEC_ERR_SHAPE, too,
 *    for a call whose kernel would have 2^32 threads or more (for example appends
 *    of 2^28 tokens of one narrow KV head, or 65535 sequences of 256 KV heads of
 *    one token with a status).  Errors in device data
 *    are reported per sequence in seq_status[b] (when it is not NULL): the kernels
 *    never trap and never touch memory outside the buffers described here.
 *    What a sequence with a non-zero status leaves in its own output rows is
 *    unspecified, and so are those of sequences behind offsets that decrease, and of
 *    tokens that these share with a sequence before; other rows are not affected.
 *  - Rows of outputs behind the last sequence's tokens, and before the first's,
 *    keep what they held: total_new may exceed new_off[B] (a captured call that
 *    is replayed with fewer tokens).
 *  - No exceptions cross this ABI and nothing is printed. */
#ifndef RESPEC_PROMPT_H
#define RESPEC_PROMPT_H

#include <stddef.h>
#include <stdint.h>

#include "respec_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------- chunks of new tokens */

/* Limits of this implementation. */
enum { RESPEC_CHUNK_MAX_BATCH = 65535, RESPEC_CHUNK_MAX_HEADS = 256 };

/* Shapes and capacities, fixed when the plan is created. */
typedef struct {
  int32_t n_q_heads;   /* Hq, at most RESPEC_CHUNK_MAX_HEADS                                 */
  int32_t n_kv_heads;  /* Hkv, divides Hq                                                     */
  int32_t head_dim;    /* D: 64 or 128                                                        */
  int32_t dtype;       /* respec_dtype of q, k_new, v_new, the cache and out                  */
  int32_t max_batch;   /* capacity in sequences, at most RESPEC_CHUNK_MAX_BATCH               */
  int32_t max_new;     /* capacity in new tokens of all sequences of a call; max_new * Hq
                          < 2^31                                                              */
  int32_t max_kv_len;  /* capacity in rows in front of a chunk, max_kv_len + max_new <= 2^30  */
} respec_chunk_shape;

/* A paged cache.  k and v are laid out alike; strides are in elements, each a
 * multiple of 16 bytes, non-negative; k and v are 16-byte aligned. */
typedef struct {
  void* k;
  void* v;
  int32_t n_pages;             /* pages that k and v hold                                     */
  int32_t page_size;           /* rows per page, >= 1                                         */
  int64_t page_stride;
  int64_t head_stride;
  int64_t row_stride;          /* at most 2^24                                                */
  const int32_t* page_table;   /* [B] rows of table_width entries, table_stride apart.  Only the
                                  entries of a sequence's live rows are read as pages; any of
                                  them outside [0, n_pages) gives RESPEC_ERR_PAGE             */
  int32_t table_width;
  int64_t table_stride;        /* >= table_width (any value for one sequence)                 */
} respec_paged_cache;

typedef struct {
  int32_t batch;               /* B, 0 <= B <= max_batch                                      */
  int32_t total_new;           /* rows of the packed tensors, 0 <= total_new <= max_new        */
  int32_t max_new_in_batch;    /* >= every new_off[b+1] - new_off[b], <= total_new             */
  int32_t max_kv_len_in_batch; /* >= every kv_len[b], <= max_kv_len                            */
  const int32_t* new_off;      /* [B+1] int32, non-decreasing                                  */
  const int32_t* kv_len;       /* [B] int32                                                    */
  respec_paged_cache cache;
  int32_t* seq_status;         /* [B] or NULL: RESPEC_OK, RESPEC_ERR_SHAPE (new_off: decreasing,
                                  outside [0, total_new], or more than max_new_in_batch tokens),
                                  RESPEC_ERR_CAPACITY (kv_len outside [0, max_kv_len_in_batch], or
                                  more rows than table_width pages hold), RESPEC_ERR_PAGE.  Shares no
                                  byte with new_off, kv_len and the page table's rows (the call:
                                  RESPEC_ERR_SHAPE), which other workgroups may still read      */
} respec_chunk_batch;

/* Strides of the packed tensors are in elements and multiples of 16 bytes;
 * pointers are 16-byte aligned; the last dimension is contiguous. */
typedef struct {
  respec_chunk_batch b;
  const void* k_new;           /* [total_new][Hkv][D]                                          */
  const void* v_new;
  int64_t k_token_stride, k_head_stride;
  int64_t v_token_stride, v_head_stride;
} respec_chunk_append_args;

typedef struct {
  respec_chunk_batch b;
  const void* q;               /* [total_new][Hq][D]                                           */
  int64_t q_token_stride, q_head_stride;
  void* out;                   /* [total_new][Hq][D], may be q itself with q's strides; else shares no
                                  byte with q's rows, nor one of its rows with another
                                  (RESPEC_ERR_SHAPE)                                            */
  int64_t out_token_stride, out_head_stride;
  float scale;                 /* of the scores, finite and > 0; 0 = 1 / sqrt(D)                */
} respec_chunk_attn_args;

typedef struct respec_chunk_plan respec_chunk_plan;

/* Create a plan (host).  Validates the shape; *out receives the plan. */
respec_status respec_chunk_create(const respec_chunk_shape* shape, respec_chunk_plan** out);

/* Destroy a plan (host).  NULL is ignored. */
void respec_chunk_destroy(respec_chunk_plan* plan);

/* Bytes of device workspace that respec_chunk_attn needs (host); 0 for a NULL plan. */
size_t respec_chunk_workspace_bytes(const respec_chunk_plan* plan);

/* Write row kv_len[b] + i of sequence b from k_new / v_new of its token i, for
 * every new token.  Needs no workspace.  Rows that two sequences write to the
 * same place (a shared page) end as either's. */
respec_status respec_chunk_append(const respec_chunk_plan* plan, const respec_chunk_append_args* args, void* stream);

/* out[t][h] = sum over rows r = 0 .. kv_len[b] + i of  p_r V[r][h / (Hq / Hkv)],
 * p = softmax over those rows of  scale * q[t][h] . K[r][h / (Hq / Hkv)],
 * for token t = new_off[b] + i.  The rows of the new tokens themselves are read
 * from the cache (respec_chunk_append, earlier on the stream).  Rows that a
 * token does not see have no part in its output, whatever they hold.
 * Scores and sums are float32.  bf16 rounds p to bf16 before its product with V
 * (0.0019 to 0.0022 of the output's norm in all, where rounding the output alone
 * is 0.0017); float32 rounds nothing further.  Sums are divided in the end, and of values above 2^119 / rows
 * (float32: 2^128 / rows) they may be infinities.
 * workspace: respec_chunk_workspace_bytes(plan) bytes, 256-byte aligned. */
respec_status respec_chunk_attn(const respec_chunk_plan* plan, const respec_chunk_attn_args* args, void* workspace,
                                void* stream);

/* ------------------------------------------------------------- scores of given tokens */

typedef struct {
  int32_t vocab;     /* V >= topk_out, < 2^30                                                  */
  int32_t dtype;     /* respec_dtype of the logits                                             */
  int32_t max_rows;  /* capacity in rows, 1 .. 2^24 - 1                                        */
  int32_t topk_out;  /* width of the top-k output, 1..RESPEC_MAX_TOPK_OUT                      */
} respec_score_shape;

/* One row of logits z [V] each.  p = softmax(z); natural logarithms.
 * A row whose logits are all -inf has lse -inf, log probabilities -inf and entropy 0.
 * A row that holds a NaN or +inf gets NaN in its float outputs and -1 in the
 * others.  Every output may be NULL. */
typedef struct {
  int32_t rows;          /* R, 0 <= R <= max_rows                                              */
  const void* logits;    /* [R][V] dtype, aligned to its elements                              */
  int64_t row_stride;    /* elements between rows, >= V                                        */
  const int32_t* token;  /* [R] int32 token to score; -1: none (log probability 0, rank -1); any
                            other id outside [0, V): log probability NaN, rank -1.  NULL: none in
                            every row                                                          */
  float* tok_logprob;    /* [R] log p(token)                                                    */
  int32_t* tok_rank;     /* [R] #{u : z[u] > z[token]} + #{u < token : z[u] == z[token]}        */
  float* lse;            /* [R] log sum_v exp z                                                 */
  float* entropy;        /* [R] -sum_v p log p, nats                                            */
  int32_t* topk_id;      /* [R][topk_out] ids by (z desc, id asc)                               */
  float* topk_logprob;   /* [R][topk_out] log p of those ids                                    */
} respec_score_args;

typedef struct respec_score_plan respec_score_plan;

/* As their respec_chunk_* namesakes. */
respec_status respec_score_create(const respec_score_shape* shape, respec_score_plan** out);
void respec_score_destroy(respec_score_plan* plan);
size_t respec_score_workspace_bytes(const respec_score_plan* plan);

/* Score `rows` rows.  workspace as above. */
respec_status respec_score(const respec_score_plan* plan, const respec_score_args* args, void* workspace,
                           void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RESPEC_PROMPT_H */

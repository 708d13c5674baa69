/* respec_cache.h -- C ABI of what a cache goes through around the steps on MI355X (gfx950).
 *
 * Beside respec_prompt.h's append and attention over a cache of the model's type:
 *
 *   respec_rotary            rotary positions of queries and keys, of new tokens and of
 *                            the nodes of a draft tree (a verification step takes a node's
 *                            query from its hidden state as it is: for it, of the keys)
 *   respec_chunk_append_q8   K/V rows of new tokens into a paged cache of 8-bit values
 *   respec_chunk_attn_q8     causal attention of new tokens over that cache
 *   respec_cache_keep        the accepted path of every verified draft tree moves to the
 *                            front of its nodes' rows, in all layers
 *   respec_cache_copy        pages are copied: a fork's partly filled page, beams' pages
 *
 * Conventions are respec_prompt.h's: caller-owned device memory, calls that only
 * enqueue kernels on the caller's stream and can be captured, host checks that return
 * a status and launch nothing (RESPEC_ERR_SHAPE, too, for a launch of 2^32 threads or more),
 * errors in device data reported per sequence or pair (when the caller gives an
 * array for them, which shares no byte with what the call reads: RESPEC_ERR_SHAPE)
 * with no access outside the buffers described here. */
#ifndef RESPEC_CACHE_H
#define RESPEC_CACHE_H

#include <stddef.h>
#include <stdint.h>

#include "respec_prompt.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------- rotary positions */

/* Which columns make a pair: i and i + rotary_dim / 2, or 2 i and 2 i + 1. */
typedef enum { RESPEC_ROTARY_HALF = 0, RESPEC_ROTARY_INTERLEAVED = 1 } respec_rotary_layout;

enum { RESPEC_ROTARY_MAX_TOKENS = 1 << 24 };

typedef struct {
  int32_t n_q_heads;   /* heads of q, 1 .. RESPEC_CHUNK_MAX_HEADS                               */
  int32_t n_kv_heads;  /* heads of k, 1 .. RESPEC_CHUNK_MAX_HEADS                               */
  int32_t head_dim;    /* D: 64 or 128                                                        */
  int32_t rotary_dim;  /* columns 0 .. rotary_dim - 1 are turned: a multiple of 16, 16 .. D     */
  int32_t layout;      /* respec_rotary_layout                                                */
  int32_t dtype;       /* respec_dtype of the tensors                                         */
  int32_t max_tokens;  /* capacity in tokens, 1 .. RESPEC_ROTARY_MAX_TOKENS                     */
  float amplitude;     /* of cosines and sines, finite and > 0; 0 = 1                          */
} respec_rotary_shape;

/* Row t of q and k (one head's D columns) at position p: with w_i = frequency[i],
 *   y_a = amplitude (x_a cos(p w_i) - x_b sin(p w_i)),  y_b = amplitude (x_b cos(p w_i) + x_a sin(p w_i))
 * for pair i = (a, b); columns from rotary_dim on are copied.  Angles are within 2^-31 of
 * a turn at every position; cosines, sines and products are float32, the result is rounded once.
 * Positions are given one per token, or as a chunk batch's: token i of sequence b
 * stands at kv_len[b] + i.  A token at a negative position, one of no sequence and those of a
 * sequence with a non-zero status keep what their output rows held.
 * An output shares no byte with an input, the other output or itself (RESPEC_ERR_SHAPE), but may be
 * its input with the same strides; tensors may lie between each other's rows. */
typedef struct {
  int32_t tokens;              /* rows of the tensors, 0 <= tokens <= max_tokens                */
  const int32_t* positions;    /* [tokens] int32, or NULL: new_off and kv_len                   */
  int32_t batch;               /* (of new_off and kv_len; 0 .. RESPEC_CHUNK_MAX_BATCH)           */
  const int32_t* new_off;      /* [batch + 1] int32, non-decreasing                             */
  const int32_t* kv_len;       /* [batch] int32                                                 */
  const void* q;               /* [tokens][Hq][D], or NULL (with q_out): no queries              */
  int64_t q_token_stride, q_head_stride;
  void* q_out;                 /* as q                                                          */
  int64_t q_out_token_stride, q_out_head_stride;
  const void* k;               /* [tokens][Hkv][D], or NULL (with k_out)                         */
  int64_t k_token_stride, k_head_stride;
  void* k_out;
  int64_t k_out_token_stride, k_out_head_stride;
  int32_t* seq_status;         /* [batch] or NULL (and NULL with positions): RESPEC_OK or RESPEC_ERR_SHAPE
                                  (new_off: decreasing or outside [0, tokens]), RESPEC_ERR_CAPACITY (kv_len
                                  negative, or positions from 2^30 on)                           */
} respec_rotary_args;

typedef struct respec_rotary_plan respec_rotary_plan;

/* frequency: HOST array of rotary_dim / 2 doubles, radians per position, 0 .. 2 pi (copied). */
respec_status respec_rotary_create(const respec_rotary_shape* shape, const double* frequency, respec_rotary_plan** out);
void respec_rotary_destroy(respec_rotary_plan* plan);
respec_status respec_rotary(const respec_rotary_plan* plan, const respec_rotary_args* args, void* stream);

/* ------------------------------------------------------------- a cache of 8-bit values */

/* The values are e4m3 (4 exponent, 3 mantissa bits, no infinities, largest 448); the
 * rows of a block (rows r with the same r / scale_block, of one page and KV head) share
 * a power-of-two scale, held as its exponent byte e: the scale is 2^(e - 127), 0 <= e <= 254.
 * Row r's element is its e4m3 value times the scale of its block.  (Of a float's kind, e4m3
 * has the same relative precision over its range, so a scale's own mantissa would buy
 * next to nothing, and a power of two makes every later change of scale exact but for
 * values that leave the range at its bottom.)
 * The byte of block j of KV head h of a page is at
 *   page * scale_page_stride + h * scale_head_stride + j.
 * Strides of k and v are in elements (bytes), multiples of 16, non-negative. */
typedef struct {
  void* k;
  void* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int32_t n_pages;
  int32_t page_size;           /* rows per page, a multiple of scale_block                       */
  int32_t scale_block;         /* rows that share a scale: 16, 32, 64 or 128                     */
  int64_t page_stride;
  int64_t head_stride;
  int64_t row_stride;          /* at most 2^24                                                   */
  int64_t scale_page_stride;   /* (any non-negative; of k_scale and v_scale alike)                */
  int64_t scale_head_stride;
  const int32_t* page_table;   /* as respec_paged_cache's                                        */
  int32_t table_width;
  int64_t table_stride;
} respec_q8_cache;

typedef struct {
  int32_t batch;               /* as respec_chunk_batch's                                        */
  int32_t total_new;
  int32_t max_new_in_batch;
  int32_t max_kv_len_in_batch;
  const int32_t* new_off;
  const int32_t* kv_len;
  respec_q8_cache cache;
  int32_t* seq_status;
} respec_q8_batch;

typedef struct {
  respec_q8_batch b;
  const void* k_new;           /* [total_new][Hkv][D] of the plan's dtype                        */
  const void* v_new;
  int64_t k_token_stride, k_head_stride;
  int64_t v_token_stride, v_head_stride;
} respec_q8_append_args;

typedef struct {
  respec_q8_batch b;
  const void* q;               /* as respec_chunk_attn_args'                                     */
  int64_t q_token_stride, q_head_stride;
  void* out;
  int64_t out_token_stride, out_head_stride;
  float scale;
} respec_q8_attn_args;

/* respec_chunk_append into an 8-bit cache, of the same plan.  In every block that new rows touch,
 * with a the largest finite magnitude of its new rows and k the least integer from -126 on with
 * a <= 448 2^k:  the scale is 2^k or, where rows of the sequence stand in the block already
 * (from its first row to kv_len - 1), the larger of that and the scale that they have; these
 * rows' values are rounded again if their scale grows.  A new value x becomes x 2^-k
 * rounded to nearest even; a NaN or an infinity becomes a NaN.  (A number within 2^-5 of 2^128 of
 * its size may round to 2^128, which attention takes for an infinity in a key.)  Rows of the block behind the new
 * ones keep their bytes.
 * A block belongs to one sequence while it is written: what the rows of a block hold that two
 * sequences of the call write is unspecified (share whole blocks, copy a partly filled page
 * first). */
respec_status respec_chunk_append_q8(const respec_chunk_plan* plan, const respec_q8_append_args* args, void* stream);

/* respec_chunk_attn over an 8-bit cache, of the same plan and workspace.  The cache's values go into the products as they
 * are: what is rounded is what respec_chunk_attn rounds.  (bf16 plans take them in bf16, whose least step is 2^-133: values under
 * blocks of exponent bytes 0 to 2 are rounded to it.  A key of 2^128 or more in size counts as an infinity.)  The mean of values of
 * any size is as accurate as another, also where their sum is no float32: such rows are computed twice, as those
 * with a NaN are. */
respec_status respec_chunk_attn_q8(const respec_chunk_plan* plan, const respec_q8_attn_args* args, void* workspace,
                                   void* stream);

/* ------------------------------------------------------------- rows kept, pages copied */

/* After a verification step: row kv_len[b] + path[b][i] of every layer's cache moves to row
 * kv_len[b] + i, for i = 0 .. acc_len[b] (path and acc_len as respec_verify_step leaves them: node
 * ids, ascending, the root's 0 first), and kv_len_out[b] = kv_len[b] + acc_len[b] + 1.
 * acc_len[b] = -1 (a step that failed for the sequence): nothing moves, kv_len_out[b] = kv_len[b].
 * A sequence with a non-zero status: nothing moves, kv_len_out[b] = kv_len[b].
 * A page with rows that move, or that rows move to, belongs to one sequence (copy a shared, partly filled page first), and rows
 * of layers, pages and heads to one place each (RESPEC_ERR_SHAPE for a stride of less than a row).
 * kv_len_out and seq_status share no byte with kv_len, acc_len, the paths, the page table's rows or each other
 * (RESPEC_ERR_SHAPE): they are written while other workgroups may still read. */
typedef struct {
  int32_t batch;               /* 0 .. RESPEC_CHUNK_MAX_BATCH                                    */
  int32_t n_layers;            /* 1 .. 65535                                                     */
  int32_t n_kv_heads;          /* 1 .. RESPEC_CHUNK_MAX_HEADS                                    */
  int32_t head_dim;            /* D: 64 or 128                                                   */
  int32_t dtype;               /* respec_dtype of the cache                                      */
  respec_paged_cache cache;    /* of layer 0                                                     */
  int64_t layer_stride;        /* elements from a layer to the next, a multiple of 16 bytes,
                                  non-negative                                                   */
  const int32_t* kv_len;       /* [B] int32                                                      */
  const int32_t* path;         /* [B] rows of path_width entries, path_stride apart               */
  int32_t path_width;          /* 1 .. RESPEC_MAX_DEPTH + 1                                       */
  int64_t path_stride;         /* >= path_width (any value for one sequence)                     */
  const int32_t* acc_len;      /* [B] int32                                                      */
  int32_t* kv_len_out;         /* [B] or NULL                                                    */
  int32_t* seq_status;         /* [B] or NULL: RESPEC_OK, RESPEC_ERR_TREE (acc_len below -1 or not below
                                  path_width; path not ascending from a node id >= 0),
                                  RESPEC_ERR_CAPACITY (kv_len negative, or more rows than the table's
                                  pages hold), RESPEC_ERR_PAGE                                    */
} respec_cache_keep_args;

respec_status respec_cache_keep(const respec_cache_keep_args* args, void* stream);

enum { RESPEC_CACHE_MAX_PLANES = 8, RESPEC_CACHE_MAX_PAIRS = 65535 };

/* One array of pages: every layer's page p is `heads` times `rows` runs of row_bytes bytes.  All
 * strides in bytes, non-negative. */
typedef struct {
  void* base;
  int64_t page_stride;
  int32_t n_layers;            /* 1 .. 65535                                                     */
  int64_t layer_stride;
  int32_t heads;               /* 1 .. 65535                                                     */
  int64_t head_stride;
  int32_t rows;                /* >= 1                                                           */
  int64_t row_stride;
  int64_t row_bytes;           /* >= 1; heads * rows * row_bytes < 2^31                           */
} respec_page_plane;

/* Page dst[i] of every plane and layer becomes a copy of its page src[i], i < pairs.  A pair
 * with src[i] = -1 is left out.  No page may be the destination of two pairs, or of one and the
 * source of another: what such a page's copy holds is unspecified. */
typedef struct {
  int32_t pairs;               /* 0 .. RESPEC_CACHE_MAX_PAIRS                                     */
  const int32_t* src;          /* [pairs] int32                                                  */
  const int32_t* dst;          /* [pairs] int32                                                  */
  int32_t n_pages;             /* pages of every plane, >= 1                                      */
  int32_t n_planes;            /* 1 .. RESPEC_CACHE_MAX_PLANES                                     */
  const respec_page_plane* planes;   /* HOST array                                               */
  int32_t* status;             /* [pairs] or NULL: RESPEC_OK, or RESPEC_ERR_PAGE (an id outside
                                  [0, n_pages); nothing is copied)                               */
} respec_cache_copy_args;

respec_status respec_cache_copy(const respec_cache_copy_args* args, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* RESPEC_CACHE_H */

// Device helpers shared by the kernels that work on chunks of new tokens.
#pragma once

#include "../common.hpp"
#include "prompt.hpp"

namespace respec {

constexpr int kStShape = 2, kStCapacity = 6, kStPage = 11;

// Sequence b of a chunk batch; a sequence with unusable lengths has no tokens.
struct ChunkSeq {
  int t0, n, L, status;
};
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkBatch& c, int b) {
  const int t0 = c.new_off[b], t1 = c.new_off[b + 1], L = c.kv_len[b];
  ChunkSeq s{t0, 0, L, 0};
  // (as 64-bit: no difference or sum of the device's words wraps)
  const long long n = (long long)t1 - t0;
  if (t0 < 0 || n < 0 || t1 > c.total_new || n > c.max_new)
    s.status = kStShape;
  else if (L < 0 || L > c.max_kv || (long long)L + n > (long long)c.table_width * c.page.d)
    s.status = kStCapacity;
  else
    s.n = (int)n;
  return s;
}

// Byte offset, within a KV head of the cache, of row r of a sequence, in the page of id `id`.  An id out of
// range (reported by report_status) reads page 0 instead.
__device__ __forceinline__ int64_t offset_in(const ChunkBatch& c, int32_t id, uint32_t r) {
  const int64_t page = (uint32_t)id < (uint32_t)c.n_pages ? id : 0;
  return page * c.page_stride + (int64_t)((uint64_t)(r - div_by(r, c.page) * c.page.d) * c.row_stride);
}

// The sequence that owns packed token t (n = 0: none), by a whole wave: a lane per sequence.
__device__ __forceinline__ ChunkSeq seq_of_token(const ChunkBatch& c, int t, int& b) {
  for (int b0 = 0; b0 < c.batch; b0 += 64) {
    const int k = b0 + (int)(threadIdx.x & 63);
    ChunkSeq s{0, 0, 0, 0};
    if (k < c.batch) s = chunk_seq(c, k);
    const uint64_t own = __ballot(t >= s.t0 && t - s.t0 < s.n);
    if (own) {
      const int l = __builtin_ctzll(own);
      b = b0 + l;
      return ChunkSeq{__builtin_amdgcn_readlane(s.t0, l), __builtin_amdgcn_readlane(s.n, l),
                      __builtin_amdgcn_readlane(s.L, l), 0};
    }
  }
  b = 0;
  return ChunkSeq{0, 0, 0, 0};
}

// Status of sequence b, by one workgroup of NT threads: its lengths, then the page ids of
// rows [lo, L + n), lo = 0 or L.
template <int NT>
__device__ __forceinline__ void report_status(const ChunkBatch& c, int b, bool from_zero) {
  const ChunkSeq s = chunk_seq(c, b);
  __shared__ int bad;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  if (s.n > 0) {
    const int32_t* table = c.table + (int64_t)b * c.table_stride;
    const uint32_t p0 = from_zero ? 0u : div_by((uint32_t)s.L, c.page), p1 = div_by((uint32_t)(s.L + s.n - 1), c.page);
    bool any = false;
    for (uint32_t p = p0 + threadIdx.x; p <= p1; p += NT) any |= (uint32_t)table[p] >= (uint32_t)c.n_pages;
    if (any) bad = 1;
  }
  __syncthreads();
  if (threadIdx.x == 0) c.status[b] = s.status ? s.status : (bad ? kStPage : 0);
}

__device__ __forceinline__ int wave_prefix_sum(int v) {  // inclusive
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);  // from 1, 2, 4 and 8 lanes below in rows of 16,
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // lanes 15 and 47 to the rows after theirs,
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // and lane 31 to the upper half
  return v;
}

__device__ __forceinline__ int row_block(const ChunkGeom& ge, int row) { return row >> __builtin_ctz(ge.rows_per_wg); }

// A workgroup's item.  Item x is of KV head x % Hkv (a head's workgroups meet on one XCD where the heads are a
// multiple of 8, and read its tiles at about the same time) and entry x / Hkv of the list of (sequence, split, row
// block), a block's rows descending: the longest first.  A sequence of `rows` query rows from `least` to `most`
// has its row blocks times its splits of entries; the grid holds as many as any lengths within the call's bounds
// need, and those past the list's end find nothing (n = 0).  The list is walked 64 sequences at a time, and so is it for a
// token's sequence: hundreds of sequences cost nothing that shows, but thousands do (one token each over 16 rows, 8 heads on 2 of
// 64, append and attention: 256 sequences 12 and 12 us, 1024 19 and 52, 4096 70 and 478, 16384 284 and 6480).
struct Item {
  int split, g, rb, b;
  ChunkSeq seq;
};
__device__ __forceinline__ Item find_item(const ChunkBatch& c, const ChunkGeom& ge, int least, int most, int x, int lane) {
  int y = (int)div_by((uint32_t)x, c.kv_heads);
  Item it{0, x - y * c.n_kv_heads, 0, 0, ChunkSeq{0, 0, 0, 0}};
  for (int b0 = 0; b0 < c.batch; b0 += 64) {
    ChunkSeq s{0, 0, 0, 0};
    int blocks = 0, splits = 1;
    if (b0 + lane < c.batch) {
      s = chunk_seq(c, b0 + lane);
      const int rows = s.n * c.group;
      if (rows >= least && rows <= most) {
        blocks = row_block(ge, rows - 1) + 1;
        splits = (int)div_by((uint32_t)(s.L + s.n - 1), ge.split) + 1;
      }
    }
    // (a lane's entries: its blocks times its splits, as many as the grid holds for it; 64 lanes' fit 32 bits)
    int incl = blocks * splits;
    if (c.batch > 1) incl = wave_prefix_sum(incl);
    const uint64_t past = __ballot(y < incl);
    if (past) {
      const int l = __builtin_ctzll(past);
      blocks = __builtin_amdgcn_readlane(blocks, l);
      y -= __builtin_amdgcn_readlane(incl, l) - blocks * __builtin_amdgcn_readlane(splits, l);
      it.b = b0 + l;
      it.split = __popcll(__ballot((uint32_t)(lane + 1) * (uint32_t)blocks <= (uint32_t)y));  // y / blocks, at most 63
      it.rb = blocks - 1 - (y - it.split * blocks);
      if ((uint32_t)it.rb >= (uint32_t)blocks) return it;  // (offsets that overlap: more entries than 32 bits count)
      it.seq = ChunkSeq{__builtin_amdgcn_readlane(s.t0, l), __builtin_amdgcn_readlane(s.n, l),
                        __builtin_amdgcn_readlane(s.L, l), 0};
      return it;
    }
    y -= __builtin_amdgcn_readlane(incl, 63);
  }
  return it;
}

// Cache rows that the rows of block rb see (at least one).
__device__ __forceinline__ int block_limit(const ChunkAttnArgs& a, const ChunkGeom& ge, const ChunkSeq& s, int rb) {
  const int last = min((rb + 1) * ge.rows_per_wg, s.n * a.b.group) - 1;
  return s.L + (int)div_by((uint32_t)last, a.group) + 1;
}

}  // namespace respec

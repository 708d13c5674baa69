// Internal launch interface of the kernels of include/respec_cache.h that need no chunk plan (not part of the C ABI).
#pragma once

#include "../prompt/chunk.hpp"

namespace respec {

constexpr int kRotaryThreads = 256, kKeepThreads = 256, kCopyThreads = 256;
constexpr int kRotaryMaxPairs = 64;
constexpr int kKeepMaxPath = 65;
constexpr int kCopyMaxPlanes = 8;
constexpr int kCopyPieces = 4;  // pieces of a copying thread

// One of q and k; strides in bytes.
struct RotaryRows {
  const char* x;
  char* y;
  int64_t x_tok, x_head, y_tok, y_head;
};

struct RotaryArgs {
  ChunkBatch b;              // (without positions: offsets and lengths alone)
  const int32_t* positions;  // or null
  RotaryRows q, k;
  int32_t q_heads, heads;    // of q (0: none), of q and k
  FastDiv stride;            // a thread takes heads j, j + stride, j + 2 stride, ..
  int32_t tokens, tok_per_wg, turned, status_wgs;  // turned: units of a head that are turned (the others are copied)
  float amplitude;
  uint64_t turns[kRotaryMaxPairs];  // 2^64 times turns per position
};

struct KeepArgs {
  ChunkBatch b;                // kv_len, table and cache
  int64_t layer_stride;
  const int32_t* path;
  const int32_t* acc_len;
  int32_t* kv_len_out;
  int64_t path_stride;
  int32_t path_width, pieces;  // pieces: 16-byte pieces of a row of all KV heads
};

struct CopyPlane {
  char* base;
  int64_t page_stride, layer_stride, head_stride, row_stride;
  int32_t n_layers, first_wg;  // first_wg: of a layer's and pair's workgroups
  uint32_t pieces;             // of a page in a layer
  FastDiv per_row, per_head;   // pieces of a run, and of a head's runs
  int32_t piece;               // bytes of a piece: 16, 8, 4, 2 or 1
};
struct CopyArgs {
  const int32_t* src;
  const int32_t* dst;
  int32_t* status;
  int32_t n_pages, n_planes;
  CopyPlane plane[kCopyMaxPlanes];
};

hipError_t launch_rotary(int es, int head_dim, bool half, int heads_per_thread, int wgs, int wgs_of_token, const RotaryArgs& a,
                         hipStream_t s);
hipError_t launch_keep(int head_bytes, int layers, const KeepArgs& a, hipStream_t s);
hipError_t launch_copy(int wgs, int layers, int pairs, const CopyArgs& a, hipStream_t s);

}  // namespace respec

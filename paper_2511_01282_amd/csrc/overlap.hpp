// Host checks of what a call writes against what its workgroups read.
#pragma once

#include <stdint.h>

namespace respec {

// Whether `size` bytes at `a` share one with `n` rows of `row` bytes, `stride` bytes apart (not negative), from `b` on.
inline bool overlap(const void* a, int64_t size, const void* b, int64_t n, __int128 stride, int64_t row) {
  if (!a || !b || size <= 0 || n <= 0 || row <= 0) return false;
  const __int128 lo = (__int128)(uintptr_t)a - (uintptr_t)b, hi = lo + size;  // from the first row on
  if (hi <= 0 || lo >= (n - 1) * stride + row) return false;
  const __int128 i = stride == 0 || lo < row ? 0 : (lo - row) / stride + 1;   // the first row that ends behind `lo`
  return i < n && i * stride < hi;
}

}  // namespace respec

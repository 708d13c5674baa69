// Host checks of what a call writes against what its workgroups read.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace respec {

// Whether `size` bytes at `a` share one with `n` rows of `row` bytes, `stride` bytes apart (not negative), from `b` on.
inline bool overlap(const void* a, int64_t size, const void* b, int64_t n, __int128 stride, int64_t row) {
  if (!a || !b || size <= 0 || n <= 0 || row <= 0) return false;
  const __int128 lo = (__int128)(uintptr_t)a - (uintptr_t)b, hi = lo + size;  // from the first row on
  if (hi <= 0 || lo >= (n - 1) * stride + row) return false;
  const __int128 i = stride == 0 || lo < row ? 0 : (lo - row) / stride + 1;   // the first row that ends behind `lo`
  return i < n && i * stride < hi;
}

// `n` rows, `step` bytes apart.
struct Comb {
  int64_t n, step;
};
constexpr int64_t kMost = 1ll << 60;  // (more bytes than there are addresses)
// Rows of a two-dimensional tensor, the dimension of the larger step first; dimensions of one place (or of step 0) have n = 1.
struct RowSet {
  uintptr_t at;
  Comb outer, inner;
  int64_t row, inner_size, size;  // bytes of a row, of an outer place's rows from the first to the last, of all
};
inline RowSet row_set(const void* at, int64_t n0, int64_t step0, int64_t n1, int64_t step1, int64_t row) {
  auto comb = [](int64_t n, int64_t step) { return n > 1 && step != 0 ? Comb{n, step} : Comb{1, 0}; };
  const Comb a = comb(n0, step0), b = comb(n1, step1);
  RowSet s{(uintptr_t)at, a.step >= b.step ? a : b, a.step >= b.step ? b : a, row, 0, 0};
  const __int128 inner = (__int128)(s.inner.n - 1) * s.inner.step + row, all = (__int128)(s.outer.n - 1) * s.outer.step + inner;
  s.inner_size = inner < kMost ? (int64_t)inner : kMost;
  s.size = all < kMost ? (int64_t)all : kMost;
  return s;
}
inline bool same_rows(const RowSet& a, const RowSet& b) {
  auto same = [](const Comb& x, const Comb& y) { return x.n == y.n && x.step == y.step; };
  return a.at == b.at && same(a.outer, b.outer) && same(a.inner, b.inner);
}

inline int64_t floor_div(int64_t x, int64_t d) { return x / d - (x % d < 0); }

// Whether a place of `a` from 0 on and one of `b` from `to` on have rows of `row` bytes that share one.
inline bool overlap(Comb a, Comb b, int64_t to, int64_t row) {
  if (a.n > b.n) {
    const Comb c = a;
    a = b, b = c, to = -to;
  }
  if (a.step == b.step && a.step > 0) {  // distances are multiples of the step: the two next to `to`, or the last that there is
    for (int64_t e : {floor_div(to, a.step), floor_div(to, a.step) + 1}) {
      e = e <= -b.n ? 1 - b.n : e >= a.n ? a.n - 1 : e;
      if (e * a.step < to + row && to < e * a.step + row) return true;
    }
    return false;
  }
  for (int64_t i = 0; i < a.n; ++i) {
    const int64_t x = i * a.step - to;  // from b's first row on
    const int64_t j = b.step == 0 || x < row ? 0 : (x - row) / b.step + 1;
    if (j < b.n && j * b.step < x + row && x < j * b.step + row) return true;
  }
  return false;
}
// Whether two tensors' rows (of the same size) share a byte; a few steps where their outer steps are the same, as slices of one
// tensor have them.
inline bool overlap(const RowSet& a, const RowSet& b) {
  if (a.at >= b.at + b.size || b.at >= a.at + a.size || a.size == kMost || b.size == kMost) return false;
  const int64_t to = (int64_t)(b.at - a.at);
  if (a.outer.n == 1 || b.outer.n == 1 || a.outer.step == b.outer.step) {
    const int64_t step = a.outer.n > 1 ? a.outer.step : b.outer.step;
    if (step == 0) return overlap(a.inner, b.inner, to, a.row);
    // a's place i and b's j, d = i - j: their spans meet
    int64_t d = floor_div(to - a.inner_size, step) + 1, last = -floor_div(-(to + b.inner_size), step) - 1;
    if (d <= -b.outer.n) d = 1 - b.outer.n;
    if (last >= a.outer.n) last = a.outer.n - 1;
    for (; d <= last; ++d)
      if (overlap(a.inner, b.inner, to - d * step, a.row)) return true;
    return false;
  }
  if (a.outer.n > b.outer.n) return overlap(b, a);
  for (int64_t i = 0; i < a.outer.n; ++i) {
    const int64_t x = i * a.outer.step - to;  // of a's place, from b's first row on
    int64_t j = floor_div(x - b.inner_size, b.outer.step) + 1;
    if (j < 0) j = 0;
    for (; j < b.outer.n && j * b.outer.step < x + a.inner_size; ++j)
      if (overlap(a.inner, b.inner, j * b.outer.step - x, a.row)) return true;
  }
  return false;
}
// Whether two places of a tensor are sure to share a byte: neighbours in one dimension.
inline bool overlap_within(int64_t n, int64_t step, int64_t row) { return n > 1 && step < row; }
// Whether two places of a two-dimensional tensor share a byte.
inline bool overlap_within(int64_t n0, int64_t step0, int64_t n1, int64_t step1, int64_t row) {
  if (overlap_within(n0, step0, row) || overlap_within(n1, step1, row)) return true;
  const RowSet s = row_set(nullptr, n0, step0, n1, step1, row);
  if (s.outer.n == 1 || s.inner.n == 1 || s.outer.step >= s.inner_size || s.size == kMost) return false;
  // places i and j further in the one dimension and the other: the two i next to j's distance
  const Comb a = s.outer.n < s.inner.n ? s.outer : s.inner, b = s.outer.n < s.inner.n ? s.inner : s.outer;
  for (int64_t j = 1; j < a.n; ++j) {
    const int64_t x = j * a.step, i = x / b.step;
    if ((i > 0 && i < b.n && x - i * b.step < row) || (i + 1 < b.n && (i + 1) * b.step - x < row)) return true;
  }
  return false;
}

}  // namespace respec

// Which addresses the rows and heads of a tensor cover, and whether two tensors have some in common.  Host code only.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace fsx {

// Runs of dim bytes, at + r row + h head for rows 0 .. rows - 1 and heads 0 .. heads - 1; strides of 0 and more.
struct Extent {
  int64_t at, rows, row, heads, head, dim;
  int64_t end() const { return at + (rows - 1) * row + (heads - 1) * head + dim; }
};
inline Extent block(const void* p, int64_t bytes) { return {(int64_t)(uintptr_t)p, 1, 0, 1, 0, bytes}; }

// Whether no two runs of x overlap: whichever stride is the larger, blocks of the smaller one's runs lie apart.
inline bool apart(const Extent& x) {
  const bool head_major = x.head > x.row;
  const int64_t lo = head_major ? x.row : x.head, hi = head_major ? x.head : x.row;
  const int64_t n_lo = head_major ? x.rows : x.heads, n_hi = head_major ? x.heads : x.rows;
  return !((n_lo > 1 && lo < x.dim) || (n_hi > 1 && hi < (n_lo - 1) * lo + x.dim));
}

// Whether a run of x, whose runs are apart, has a byte of from .. to - 1.
inline bool meets(const Extent& x, int64_t from, int64_t to) {
  const bool head_major = x.head > x.row;
  const int64_t lo = head_major ? x.row : x.head, hi = head_major ? x.head : x.row;
  const int64_t n_lo = head_major ? x.rows : x.heads, n_hi = head_major ? x.heads : x.rows;
  // the first run that ends behind `from`: the first that begins behind `before`
  const int64_t before = from - x.dim - x.at;
  int64_t first = 0;
  if (before >= 0) {
    const int64_t o = n_hi > 1 ? std::min(before / hi, n_hi - 1) : 0, i = n_lo > 1 ? (before - o * hi) / lo + 1 : 1;
    if (i < n_lo) first = o * hi + i * lo;
    else if (o + 1 < n_hi) first = (o + 1) * hi;
    else return false;
  }
  return x.at + first < to;
}

// Whether a (of any strides) and b (whose runs are apart) have a byte in common.
inline bool meet(Extent a, Extent b) {
  if (a.end() <= b.at || b.end() <= a.at) return false;  // as nearly always
  if (a.head == 0) a.heads = 1;
  if (a.row == 0) a.rows = 1;
  if (a.heads > 1 && a.head == a.dim) a.dim *= a.heads, a.heads = 1;
  if (a.heads == 1 && a.rows > 1 && a.row == a.dim) a.dim *= a.rows, a.rows = 1;
  // Rows of the same length: row r of a lies to row s of b as its row 0 to row s - r, so one row against all differences.
  if (a.rows > 1 && a.row == b.row && b.row >= (b.heads - 1) * b.head + b.dim) {
    b.at -= (a.rows - 1) * b.row;
    b.rows += a.rows - 1;
    a.rows = 1;
  }
  for (int64_t r = 0; r < a.rows; ++r)
    for (int64_t h = 0; h < a.heads; ++h) {
      const int64_t from = a.at + r * a.row + h * a.head;
      if (meets(b, from, from + a.dim)) return true;
    }
  return false;
}

}  // namespace fsx

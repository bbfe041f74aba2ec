// reader_checks.h -- what the C entries of the reader's operators check their
// arguments with (reader.cpp, tokens.cpp).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <string>
#include <utility>

#include "mafat_internal.h"

namespace mafat {
namespace {

constexpr int64_t kMax31 = int64_t{1} << 31;

inline int fail(int status, const std::string& msg) {
  set_error(msg);
  return status;
}

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

inline size_t elt_size(int dtype) { return dtype == MAFAT_F32 ? 4 : dtype == MAFAT_BF16 ? 2 : 1; }

// Rows of `width` bytes every `pitch` bytes.
struct Span {
  const void* p;
  int64_t rows;
  int64_t width, pitch;
};

// Whether n rows of a stride have an extent that byte arithmetic can hold.
inline bool fits(int64_t n, int64_t stride) { return n < 1 || stride < (int64_t{1} << 58) / n; }

// Whether two tensors share a byte.  Tensors of one pitch may lie side by side
// in the rows of one buffer; others count as overlapping if their extents do.
inline bool overlap(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.p), b0 = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t a1 = a0 + static_cast<uintptr_t>((a.rows - 1) * a.pitch + a.width);
  const uintptr_t b1 = b0 + static_cast<uintptr_t>((b.rows - 1) * b.pitch + b.width);
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.pitch != b.pitch) return true;
  const int64_t d = static_cast<int64_t>(b0 >= a0 ? (b0 - a0) % a.pitch : (a.pitch - (a0 - b0) % a.pitch) % a.pitch);
  return d < a.width || d + b.width > a.pitch;
}

inline int launched(hipError_t e, const char* what) {
  return e == hipSuccess ? MAFAT_OK : fail(MAFAT_EHIP, std::string(what) + " launch failed: " + hipGetErrorString(e));
}

// Heads and rows as one extent (strides in any order).
inline Span extent(const void* p, int64_t esz, int64_t d, std::initializer_list<std::pair<int64_t, int64_t>> axes) {
  int64_t n = d;
  for (const auto& a : axes)
    if (a.first > 0) n += (a.first - 1) * a.second;
  return {p, 1, n * esz, n * esz};
}

// Rows of heads: rows of one pitch, which may lie side by side with others in
// the rows of one buffer, where heads lie within a row; else one extent.
inline Span rows_of_heads(const void* p, int64_t esz, int64_t d, int64_t rows, int64_t row, int64_t heads, int64_t head) {
  const int64_t width = (heads - 1) * head + d;
  if (rows <= 1 || row >= width) return {p, rows, width * esz, (rows <= 1 ? width : row) * esz};
  return extent(p, esz, d, {{rows, row}, {heads, head}});
}

// `d` values of each of `heads` heads in `rows` rows, strides in elements.
struct Heads {
  const void* p;
  int64_t esz, d, rows, row, heads, head;
  Span span() const { return rows_of_heads(p, esz, d, rows, row, heads, head); }
};

// Whether two such tensors share a byte.  Those of one pair of strides may lie
// between each other in any order (queries, keys and values head by head, say):
// then heads j - i = m and rows apart by n are D + m head + n row bytes apart, D the
// tensors' distance.  Others count as `overlap` says.
inline bool heads_overlap(const Heads& a, const Heads& b) {
  if (!overlap(a.span(), b.span())) return false;
  if (a.esz != b.esz || (a.rows > 1 && b.rows > 1 && a.row != b.row) || (a.heads > 1 && b.heads > 1 && a.head != b.head)) return true;
  const int64_t row = (a.rows > 1 ? a.row : b.row) * a.esz, head = (a.heads > 1 ? a.head : b.head) * a.esz;
  const int64_t wa = a.d * a.esz, wb = b.d * b.esz;
  const int64_t apart = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
  for (int64_t m = 1 - a.heads; m < b.heads; ++m) {
    const int64_t x = apart + m * head;
    // rows n with -wb < x + n row < wa, the first of them by a quotient towards minus infinity
    const int64_t from = -wb - x;
    int64_t n = (from >= 0 ? from / row : -((row - 1 - from) / row)) + 1;
    if (n < 1 - a.rows) n = 1 - a.rows;
    if (n < b.rows && x + n * row < wa) return true;
  }
  return false;
}

// Whether one such tensor, which is written, has a byte twice.
inline bool heads_collide(const Heads& a) {
  const int64_t in_row = (a.heads - 1) * a.head + a.d, in_head = (a.rows - 1) * a.row + a.d;
  if (!a.p || a.rows <= 1 || a.heads <= 1 || a.row >= in_row || a.head >= in_head) return false;
  for (int64_t m = 1; m < a.heads; ++m) {  // m heads up and n rows down
    const int64_t x = m * a.head, n = x / a.row;
    if ((n < a.rows && x - n * a.row < a.d) || (n + 1 < a.rows && (n + 1) * a.row - x < a.d)) return true;
  }
  return false;
}

}  // namespace
}  // namespace mafat

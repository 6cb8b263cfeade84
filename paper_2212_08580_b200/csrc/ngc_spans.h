// Checks of the memory that an entry point's arguments name: alignment, and which of them share bytes.
#pragma once
#include <cstddef>
#include <cstdint>
#include <initializer_list>

namespace ngc {

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Bytes of an argument (none: a null pointer).
struct Span {
  uintptr_t first, last;
  Span(const void *p, size_t bytes) : first(reinterpret_cast<uintptr_t>(p)), last(p ? first + bytes : first) {}
};
inline Span matrix_span(const void *p, long long rows, int n_classes, long long ld, size_t e) {
  return Span(p, rows > 0 ? (size_t)((rows - 1) * ld + n_classes) * e : 0);
}
inline bool apart(const Span &a, const Span &b) { return a.last <= b.first || b.last <= a.first || a.first == a.last || b.first == b.last; }
inline bool apart(const Span &a, std::initializer_list<Span> others) {
  for (const Span &b : others)
    if (!apart(a, b)) return false;
  return true;
}
// The same of matrices, which may also be column blocks of one buffer: rows of `row` bytes, `stride` bytes apart (0: not evenly).
struct MatrixSpan {
  Span span;
  uintptr_t row, stride;
  MatrixSpan(const void *p, long long rows, int columns, long long ld, size_t e)
      : span(matrix_span(p, rows, columns, ld, e)), row((uintptr_t)columns * e), stride((uintptr_t)ld * e) {}
  MatrixSpan(const Span &all, uintptr_t row_bytes, uintptr_t stride_bytes) : span(all), row(row_bytes), stride(stride_bytes) {}
};
inline bool apart(const MatrixSpan &a, const MatrixSpan &b) {
  if (apart(a.span, b.span)) return true;
  if (a.stride != b.stride || a.stride == 0) return false;
  const uintptr_t on = b.span.first >= a.span.first ? (b.span.first - a.span.first) % a.stride
                                                    : (a.stride - (a.span.first - b.span.first) % a.stride) % a.stride;
  return on >= a.row && on + b.row <= a.stride;
}
// An output that may take an input's place, number for number: whoever writes a row's (or a pair's) has read it by then.
inline bool apart_or_same(const Span &a, std::initializer_list<Span> others) {
  for (const Span &b : others)
    if (!apart(a, b) && a.first != b.first) return false;
  return true;
}

}  // namespace ngc

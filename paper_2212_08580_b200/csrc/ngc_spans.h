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
// An output that may take an input's place, number for number: whoever writes a row's (or a pair's) has read it by then.
inline bool apart_or_same(const Span &a, std::initializer_list<Span> others) {
  for (const Span &b : others)
    if (!apart(a, b) && a.first != b.first) return false;
  return true;
}

}  // namespace ngc

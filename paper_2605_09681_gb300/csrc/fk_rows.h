// Whether tensors of rows meet in memory (host).
#pragma once

#include <cstdint>

namespace fk {

// rows of `width` bytes, `stride` bytes apart
struct Rows {
  uintptr_t p;
  int64_t stride, width;
};

// All that rows extend over, as one.
inline Rows whole(const Rows& a, int64_t tokens) {
  const int64_t n = (tokens - 1) * a.stride + a.width;
  return Rows{a.p, n, n};
}

// Whether rows of one meet rows of the other.  With one stride, slices of the same wide rows are told apart; else whole
// extents are compared.
inline bool meet(const Rows& a, const Rows& b, int64_t tokens) {
  const Rows x = whole(a, tokens), y = whole(b, tokens);
  if (x.p + (uintptr_t)x.width <= y.p || y.p + (uintptr_t)y.width <= x.p) return false;
  if (a.stride != b.stride || tokens == 1) return true;
  const int64_t d = (int64_t)(a.p < b.p ? b.p - a.p : a.p - b.p) % a.stride;
  const int64_t low = a.p < b.p ? a.width : b.width, high = a.p < b.p ? b.width : a.width;
  return d < low || a.stride - d < high;
}

}  // namespace fk

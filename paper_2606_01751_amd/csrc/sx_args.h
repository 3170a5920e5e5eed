// Checks of pointer arguments shared by the host translation units.
#pragma once

#include <algorithm>
#include <cstdint>

namespace sx {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

inline bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && na > 0 && nb > 0 && x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

// n rows of `width` bytes, `ld` bytes apart.
struct Rows {
  const void* p;
  int64_t n, width, ld;
};
inline Rows whole(const void* p, int64_t bytes) { return {p, 1, bytes, bytes}; }

// Whether some row of x and some row of y have a byte in common.
inline bool rows_overlap(Rows x, Rows y) {
  typedef __int128 wide;
  if (!x.p || !y.p || x.n <= 0 || y.n <= 0 || x.width <= 0 || y.width <= 0) return false;
  for (Rows* r : {&x, &y})
    if (r->n > 1 && r->ld == r->width && r->n <= INT64_MAX / r->ld) *r = whole(r->p, r->n * r->ld);   // contiguous: one row
  const wide d = (wide)(uintptr_t)y.p - (wide)(uintptr_t)x.p;   // from x's first row to y's
  if (d >= (wide)(x.n - 1) * x.ld + x.width || -d >= (wide)(y.n - 1) * y.ld + y.width) return false;
  if (x.n == 1) x.ld = y.ld;
  if (y.n == 1) y.ld = x.ld;
  if (x.ld == y.ld) {
    // row j of y begins at d + k ld of row i of x, k = j - i: the first k whose row ends behind x's begin decides
    const wide t = -d - y.width;
    const wide below = t >= 0 ? t / x.ld : -((-t + x.ld - 1) / x.ld);   // floor(t / ld)
    const wide k = std::max<wide>(below + 1, -(wide)(x.n - 1));
    return k < y.n && d + k * x.ld < x.width;
  }
  if (x.n > y.n) std::swap(x, y);
  for (int64_t i = 0; i < x.n; ++i)
    if (rows_overlap({(const char*)x.p + i * x.ld, 1, x.width, x.width}, y)) return true;
  return false;
}

}  // namespace sx

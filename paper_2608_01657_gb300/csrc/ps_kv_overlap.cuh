// Whether arrays of a call lie on one another (host code).
#pragma once

#include <cstddef>
#include <cstdint>

namespace pskv {

// 'tokens' x 'heads' runs of 'dim' 16-bit elements, run (t, h) at p + 2 (t s0 + h
// s1) bytes; strides are not negative.
struct HeadRuns {
  const void* p;
  int64_t s0, s1;
  int64_t heads;
};

// Some a <= x <= b with |x s + c| < dim?
inline bool near_zero(int64_t s, int64_t a, int64_t b, int64_t c, int64_t dim) {
  int64_t x = s ? -c / s : 0;  // the nearest two are this one and a neighbour
  for (int64_t y = x - 1; y <= x + 1; ++y) {
    const int64_t z = y < a ? a : (y > b ? b : y), d = z * s + c;
    if (d > -dim && d < dim) return true;
  }
  return false;
}

// Does a run of x have an element in common with one of y (or, where x is y itself,
// with another one of x)?  'self': x and y are one array.
inline bool heads_overlap(HeadRuns x, HeadRuns y, int64_t tokens, int64_t dim, bool self = false) {
  const int64_t T = tokens;
  const int64_t off = ((intptr_t)x.p - (intptr_t)y.p) / 2;
  // an axis of one place is never stepped over
  if (T == 1) x.s0 = y.s0 = 0;
  if (x.heads == 1) x.s1 = y.s1;
  if (y.heads == 1) y.s1 = x.s1;
  const int64_t ex = (T - 1) * x.s0 + (x.heads - 1) * x.s1 + dim, ey = (T - 1) * y.s0 + (y.heads - 1) * y.s1 + dim;
  if (off >= ey || off + ex <= 0) return false;
  if (self) {  // the differences of two runs: dt s0 + dh s1, one of each sign's pair
    if (x.s1 >= dim && x.s0 >= (x.heads - 1) * x.s1 + dim) return false;
    for (int64_t dh = 0; dh < x.heads; ++dh) {
      if (dh > 0 && near_zero(x.s0, -(T - 1), T - 1, dh * x.s1, dim)) return true;
      if (dh == 0 && T > 1 && x.s0 < dim) return true;
    }
    return false;
  }
  const int64_t wx = (x.heads - 1) * x.s1 + dim, wy = (y.heads - 1) * y.s1 + dim;  // elements from a token's first to its last
  if (x.s0 == y.s0 && x.s0 > 0) {  // side by side within a token's step?
    const int64_t r = (off % x.s0 + x.s0) % x.s0;
    if (r >= wy && r + wx <= x.s0) return false;
  }
  if (x.s0 == y.s0 && x.s1 == y.s1) {
    for (int64_t dh = -(y.heads - 1); dh < x.heads; ++dh)
      if (near_zero(x.s0, -(T - 1), T - 1, off + dh * x.s1, dim)) return true;
    return false;
  }
  // Different strides, and not side by side: each run of x is looked up among y's,
  // in the one or two tokens that it can meet where y's tokens follow one another.
  for (int64_t t = 0; t < T; ++t)
    for (int64_t h = 0; h < x.heads; ++h) {
      const int64_t at = off + t * x.s0 + h * x.s1;
      if (T == 1 || y.s0 >= wy) {
        const int64_t u = y.s0 ? at / y.s0 : 0;
        for (int64_t v = u - 1; v <= u + 1; ++v)
          if (v >= 0 && v < T && near_zero(y.s1, -(y.heads - 1), 0, at - v * y.s0, dim)) return true;
      } else {
        for (int64_t g = 0; g < y.heads; ++g)
          if (near_zero(y.s0, -(T - 1), 0, at - g * y.s1, dim)) return true;
      }
    }
  return false;
}

// Arrays of a call, for finding outputs that lie on inputs or on one another.
struct Span {
  const void* p;
  int64_t bytes;
  bool out;
};
template <size_t N>
inline bool outputs_apart(const Span (&s)[N]) {
  for (size_t i = 0; i < N; ++i)
    for (size_t j = 0; j < N; ++j) {
      if (i == j || !s[i].out || !s[i].p || !s[j].p || s[i].bytes <= 0 || s[j].bytes <= 0) continue;
      const int64_t d = (intptr_t)s[i].p - (intptr_t)s[j].p;
      if (d < s[j].bytes && -d < s[i].bytes) return false;
    }
  return true;
}

}  // namespace pskv

// Whether two strided pieces of memory have a byte in common.  Host code.
#pragma once

#include <cstdint>

namespace costa {

// `lines` lines of `line` bytes each, `pitch` bytes (at least `line`) apart.
struct Span {
  uintptr_t at;
  int64_t line, pitch, lines;
};

// The smallest j >= 0 with lo <= a j mod m <= hi (0 <= lo <= hi < m), or -1: where no
// multiple of a lies in [lo, hi], the multiples of m that may be taken off one are, modulo
// a, a problem of the same kind with a in m's place (as in Euclid's algorithm).
inline int64_t first_in(int64_t a, int64_t m, int64_t lo, int64_t hi) {
  if (lo == 0) return 0;
  a %= m;
  if (a == 0) return -1;
  const int64_t c = (lo + a - 1) / a;
  if ((__int128)c * a <= hi) return c;
  const int64_t y = first_in(m % a, a, a - hi % a, a - lo % a);
  if (y < 0) return -1;
  return (int64_t)(((__int128)m * y + lo + a - 1) / a);
}

inline bool spans_meet(Span a, Span b) {
  for (Span* s : {&a, &b}) {
    if (s->line <= 0 || s->lines <= 0) return false;
    if (s->lines == 1 || s->pitch == s->line) *s = Span{s->at, s->line * s->lines, s->line * s->lines, 1};
  }
  auto extent = [](const Span& s) { return (s.lines - 1) * s.pitch + s.line; };
  const __int128 x0 = (__int128)b.at - (__int128)a.at;  // b's first line from a's
  if (x0 >= extent(a) || -x0 >= extent(b)) return false;
  if (a.lines == 1 && b.lines == 1) return true;
  const int64_t p = b.pitch, q = a.pitch;
  // the first line of b that begins at x or later
  auto line_from = [&](__int128 x) { return x <= x0 ? (__int128)0 : (x - x0 + p - 1) / p; };
  auto any_in = [&](__int128 lo, __int128 hi) { return line_from(lo) < b.lines && x0 + line_from(lo) * p < hi; };
  const __int128 last = (__int128)(a.lines - 1) * q;  // where a's last line begins
  // lines of b that begin before a's first line and reach into it, or within its last one
  if (any_in(1 - (__int128)b.line, 0) || any_in(last, last + a.line)) return true;
  // those that begin in between meet the line before them or the next one: their places
  // modulo q are below a.line or above q - b.line
  const __int128 from = line_from(0);
  const __int128 to = line_from(last) < b.lines ? line_from(last) : (__int128)b.lines;
  if (from >= to) return false;
  if (a.line > q - b.line) return true;
  const int64_t s = (int64_t)((x0 + from * p + b.line - 1) % q), top = a.line + b.line - 2;
  if (s <= top) return true;
  const int64_t j = first_in(p, q, q - s, q - s + top);
  return j >= 0 && from + j < to;
}

}  // namespace costa

// Whether two operands of a call share a byte: workgroups run in any order, so that an output may share memory with an input only where
// every element is written by the lane that has read it.  Exact for every pair of layouts -- slices of one packed matrix lie between
// each other without meeting -- and a few comparisons where the operands lie apart, as they mostly do.
#pragma once
#include <stddef.h>
#include <stdint.h>

typedef __int128 wide_t;                             // (strides are the caller's: no product of them may wrap)

// inner runs of `width` bytes every inner_step, in turn every outer_step (bytes), all within [lo, hi).  at = null: not there.
struct Extent {
  const void* at = nullptr;
  int64_t outer = 1, inner = 1;
  wide_t outer_step = 0, inner_step = 0, width = 0, lo = 0, hi = 0;
  Extent() {}
  Extent(const void* p, int64_t n_outer, wide_t s_outer, int64_t n_inner, wide_t s_inner, wide_t w)
      : at(p), outer(n_outer), inner(n_inner), outer_step(n_outer > 1 ? s_outer : 0), inner_step(n_inner > 1 ? s_inner : 0), width(w) {
    if (!p) return;                                  // (an empty range: it meets nothing)
    lo = hi = (wide_t)(uintptr_t)p;
    hi += w;
    const wide_t o = (outer - 1) * outer_step, i = (inner - 1) * inner_step;
    (o < 0 ? lo : hi) += o;
    (i < 0 ? lo : hi) += i;
  }
};
static inline Extent extent_rows(const void* at, int64_t rows, int64_t ld, int64_t cols, int64_t size) {
  return Extent(at, rows, (wide_t)ld * size, 1, 0, (wide_t)cols * size);
}
static inline Extent extent_heads(const void* at, int64_t tokens, int64_t token, int64_t heads, int64_t head, int64_t d, int64_t size) {
  return Extent(at, tokens, (wide_t)token * size, heads, (wide_t)head * size, (wide_t)d * size);
}
static inline Extent extent_bytes(const void* at, wide_t bytes) { return Extent(at, 1, 0, 1, 0, bytes); }

static inline wide_t wide_max(wide_t a, wide_t b) { return a > b ? a : b; }
static inline wide_t floor_div(wide_t a, wide_t b) { return a / b - (a % b != 0 && a < 0); }      // b > 0

// n intervals of `width` bytes, the first at `at`, `step` apart (at least 0).
struct Run {
  wide_t at;
  int64_t n;
  wide_t step, width;
  Run(wide_t a, int64_t count, wide_t s, wide_t w) : at(a), n(s ? count : 1), step(n > 1 ? s : 0), width(w) {
    if (step < 0) { at += (n - 1) * step; step = -step; }
  }
  wide_t end() const { return at + (n - 1) * step + width; }
};
// Calls f(k) for every k = j - i for which interval j of b can meet interval i of a, both of the same step (or one of them alone);
// f is given the distance from a's interval to b's.  True as soon as f is.
template <typename F>
static inline bool each_meeting(const Run& a, const Run& b, F f) {
  if (a.end() <= b.at || b.end() <= a.at) return false;
  const wide_t step = a.n > 1 ? a.step : b.step;
  if (!step) return f(b.at - a.at);
  for (wide_t k = wide_max(floor_div(a.at - b.at - b.width, step) + 1, -(a.n - 1)); k <= b.n - 1 && b.at - a.at + k * step < a.width; ++k)
    if (f(b.at - a.at + k * step)) return true;
  return false;
}
// The same for any two steps: the shorter run's intervals one by one.
template <typename F>
static inline bool meets(const Run& a, const Run& b, F f) {
  if (a.end() <= b.at || b.end() <= a.at) return false;
  if (a.n == 1 || b.n == 1 || a.step == b.step) return each_meeting(a, b, f);
  const Run& few = a.n <= b.n ? a : b;
  for (int64_t i = 0; i < few.n; ++i) {
    const Run one(few.at + i * few.step, 1, 0, few.width);
    if (a.n <= b.n ? each_meeting(one, b, f) : each_meeting(a, one, f)) return true;
  }
  return false;
}
// The longer step outside.
static inline Extent extent_sorted(Extent e) {
  const wide_t o = e.outer_step < 0 ? -e.outer_step : e.outer_step, i = e.inner_step < 0 ? -e.inner_step : e.inner_step;
  return o >= i ? e : Extent(e.at, e.inner, e.inner_step, e.outer, e.outer_step, e.width);
}
static inline bool extents_in_turn_meet(const Extent& x, const Extent& y) {
  const Extent a = extent_sorted(x), b = extent_sorted(y);
  const Run ia(0, a.inner, a.inner_step, a.width), ib(0, b.inner, b.inner_step, b.width);      // (from the first byte of an outer step)
  const Run oa((wide_t)(uintptr_t)a.at + ia.at, a.outer, a.outer_step, ia.end() - ia.at);
  const Run ob((wide_t)(uintptr_t)b.at + ib.at, b.outer, b.outer_step, ib.end() - ib.at);
  return meets(oa, ob, [&](wide_t apart) {
    const Run from_a(0, ia.n, ia.step, ia.width), from_b(apart, ib.n, ib.step, ib.width);
    return meets(from_a, from_b, [](wide_t) { return true; });
  });
}
static inline bool extents_meet(const Extent& a, const Extent& b) { return a.lo < b.hi && b.lo < a.hi && extents_in_turn_meet(a, b); }
// Element for element the same memory.
static inline bool extents_same(const Extent& a, const Extent& b) {
  return a.at == b.at && a.width == b.width && a.outer == b.outer && a.inner == b.inner && a.outer_step == b.outer_step && a.inner_step == b.inner_step;
}
static inline bool meets_but_in_place(const Extent& out, const Extent& in) { return extents_meet(out, in) && !extents_same(out, in); }
// No byte of it belongs to two runs.
static inline bool extent_distinct(const Extent& x) {
  const Extent e = extent_sorted(x);
  const wide_t o = e.outer_step < 0 ? -e.outer_step : e.outer_step, i = e.inner_step < 0 ? -e.inner_step : e.inner_step;
  return (e.inner == 1 || i >= e.width) && (e.outer == 1 || o >= (e.inner - 1) * i + e.width);
}

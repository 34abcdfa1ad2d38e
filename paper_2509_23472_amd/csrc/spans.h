// Whether the memory of many tensors is written twice, or written and read, by one call (host).
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <new>

struct Span {                                        // bytes that a call writes, or reads
  uintptr_t lo, hi;
  bool operator<(const Span& o) const { return lo < o.lo; }
};
// Whether what the step writes (parameters, copies, states) shares memory with itself or with what it reads.  Sorted intervals: a parameter that
// is in the list twice is found among a thousand tensors too.  -1: no host memory for them.
static inline int adamw_meets(void* const* p, const void* const* g, void* const* copy, const int64_t* n, int64_t count, int p_size, int g_size,
                       const Span (&state)[3], const Span (&scalars)[3]) {
  Span* const out = new (std::nothrow) Span[(size_t)(2 * count + 3)];
  if (!out) return -1;
  size_t k = 0;
  for (const Span& s : state)
    if (s.hi > s.lo) out[k++] = s;
  for (int64_t i = 0; i < count; ++i)
    if (n[i] > 0) out[k++] = {(uintptr_t)p[i], (uintptr_t)p[i] + (uintptr_t)n[i] * p_size};
  for (int64_t i = 0; copy && i < count; ++i)
    if (n[i] > 0 && copy[i]) out[k++] = {(uintptr_t)copy[i], (uintptr_t)copy[i] + (uintptr_t)n[i] * 2};
  if (!std::is_sorted(out, out + k)) std::sort(out, out + k);
  int meets = 0;
  for (size_t i = 1; i < k; ++i) meets |= out[i].lo < out[i - 1].hi;
  // The written intervals are apart here: the last one that begins before s ends is the one to look at.  Lists mostly ascend: it is the one of
  // the tensor before, or one of the next few.
  const Span *at = out, *const end = out + k;
  auto met = [&](Span s) {
    for (int i = 0; i < 3 && at != end && at->lo < s.hi; ++i) ++at;
    if ((at != end && at->lo < s.hi) || (at != out && (at - 1)->lo >= s.hi)) at = std::lower_bound(out, out + k, Span{s.hi, s.hi});
    return s.hi > s.lo && at != out && (at - 1)->hi > s.lo;
  };
  for (int64_t i = 0; i < count && !meets; ++i)
    if (n[i] > 0) meets = met({(uintptr_t)g[i], (uintptr_t)g[i] + (uintptr_t)n[i] * g_size});
  for (const Span& s : scalars) meets |= !meets && met(s);
  delete[] out;
  return meets;
}

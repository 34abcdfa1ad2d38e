// Log probabilities of given tokens under logits (tokens x vocabulary), with the entropy and the largest alternatives, and their gradient.
//
//   c = 1 / (T ln 2),  M = max x,  u_j = (x_j - M) c,  S = sum 2^u_j,  W = sum u_j 2^u_j
//   log p_j = (x_j - M) / T - ln 2 log2 S,   H = ln 2 (log2 S - W / S)      (no cancellation: log2 S >= 0, W <= 0)
//   dx_j = (1 / T) [ g (delta_jt - p_j) - h p_j (log p_j + H) ]
//
// Exponents are binary logarithms, so that an element costs a difference, a product and the exponential: a CU has 30 vector operations for each bf16
// that it reads and writes at the rate of a copy, and an exponential is four of them.  c is rounded once for all elements (a relative error of at most
// 2^-24 of the temperature), u twice.  The maximum is one of x itself: a row of the type's lowest value, which x c may not hold, is as good as equal.
// S and W are kept beside a running maximum in one pass: a new maximum M' takes S to S 2^((M - M') c), W to (W + (M - M') c S) 2^((M - M') c).
// In W u is cut off at -300, where 2^u is 0: an infinite u times 0 never occurs; NaN stays in S.
// The running maximum starts at the lowest finite number, so that a row of nothing but -inf ends with S = 0.
//
// The k largest: a workgroup first finds the largest element of each of 64 groups of its columns (k up to 32) or of 256; the k-th largest of those bounds the k-th
// largest element from below, and few elements lie above it (in random order -G ln(1 - k / G) of them for G groups: 24 for k = 20, 74 for 64).  A second pass over the row, which is in L2, collects these in LDS, where they
// are ranked by counting.  Elements are ordered by one 64-bit number, the value's order above the index's complement: no two are equal, so ties
// go to the lowest index and the order of the atomic counter does not show.  Where too many lie above the bound (a row in descending
// order), they are found one by one.
//
// Bound by memory: the logits are read once, the gradient written once.  8192 x 32000: forward 98 us (5.3 TB/s; a copy 5.1), backward 211, both in one
// call 200 (5.2); float32 4096 x 32000 the same.  1001 x 50257 float32 forward 39, backward 86 (4.7) each in a row; one after the other 55 and 69: the
// gradient's last lines leave the caches during the next forward pass.
#pragma once
#include "common.h"

#include <algorithm>
#include <cfloat>

#define LP_THREADS 256
#define LP_CANDIDATES 1024
#define LP_SPLITS 64

struct LpArgs {
  const void* x;
  int64_t ld, m, n;
  int64_t row0;          // of a launch
  const void* targets;   // int32 or int64, or null
  int target_64;
  float inv_t, c;        // 1 / T, 1 / (T ln 2)
  float *logp, *stats;   // m; 3 x m: M, log2 S, H
  int top;
  float* top_logp;       // m x top
  int32_t* top_ids;
  int64_t chunk;         // columns per workgroup
  int splits;
  float* part;           // m x splits x 4: M, S, W
  uint64_t* part_top;    // m x splits x top
  const float *d_logp, *d_entropy;
  void* grad;
  int64_t ldg;
};

struct LpSum {
  float m, s, w;
};
__device__ inline LpSum lp_none() { return {-FLT_MAX, 0.0f, 0.0f}; }
#define LP_LN2 0.693147181f
__device__ inline float lp_cut(float u) { return fmaxf(u, -300.0f); }
__device__ inline LpSum lp_moved(const LpSum& a, float m, float c) {
  const float d = lp_cut((a.m - m) * c), f = __builtin_amdgcn_exp2f(d);
  return {m, a.s * f, (a.w + d * a.s) * f};
}
__device__ inline LpSum lp_wave_merge(LpSum a, float c) {
  float m = a.m;
#pragma unroll
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  a = lp_moved(a, m, c);
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    a.s += __shfl_xor(a.s, d);
    a.w += __shfl_xor(a.w, d);
  }
  return a;
}
// Log probability of an element of logit x (what is below nothing, a row without a distribution, gives -inf).  By 1 / T, not by c, which takes the lowest
// values of a type, finite masks, past float32's range: their log p is finite as they are.
__device__ inline float lp_log(const LpArgs& g, float x, const LpSum& a, float log_s) {
  return a.s == 0.0f ? -__builtin_inff() : fmaf(-LP_LN2, log_s, (x - a.m) * g.inv_t);
}
__device__ inline float lp_log_sum(float s) { return s == 0.0f ? 0.0f : log2f(s); }
__device__ inline float lp_entropy(const LpSum& a, float log_s) { return a.s == 0.0f ? 0.0f : (log_s - a.w / a.s) * LP_LN2; }
__device__ inline int64_t lp_target(const LpArgs& g, int64_t row) {
  return g.target_64 ? ((const int64_t*)g.targets)[row] : (int64_t)((const int32_t*)g.targets)[row];
}
// What a row ends with, by one thread.
template <typename T>
__device__ inline void lp_finish(const LpArgs& g, int64_t row, const LpSum& a, float log_s) {
  const bool none = a.s == 0.0f;
  g.stats[row] = none ? -__builtin_inff() : a.m;
  g.stats[g.m + row] = log_s;
  g.stats[2 * g.m + row] = lp_entropy(a, log_s);
  if (!g.logp) return;
  const int64_t t = lp_target(g, row);
  g.logp[row] = t < 0 ? 0.0f : (t >= g.n ? __builtin_nanf("") : lp_log(g, (float)((const T*)g.x)[row * g.ld + t], a, log_s));
}

// Order of elements: larger values first, then lower indices; what is no number counts as -inf, and both zeros as one.
__device__ inline uint64_t lp_key(float x, int col) {
  const unsigned b = x != x ? 0xff800000u : __float_as_uint(x + 0.0f);
  return (uint64_t)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | ~(uint32_t)col;
}
__device__ inline float lp_value(uint64_t key) {
  const unsigned b = (unsigned)(key >> 32);
  return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ inline int32_t lp_index(uint64_t key) { return (int32_t)~(uint32_t)key; }

template <typename T>
struct LpPiece {
  static constexpr int E = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef vec any __attribute__((aligned(sizeof(T))));
};
// Elements of a run before the first whole piece.
template <typename T>
__device__ inline int64_t lp_head(const T* at, int64_t n) {
  const int64_t head = (int64_t)((16 - ((uintptr_t)at & 15)) & 15) / (int64_t)sizeof(T);
  return head < n ? head : n;
}
// Where the elements [c0, c1) of a row lie for a thread: whole pieces, then for thread i < 2 E one of the few around them (lone, -1: none).
// (Columns are 32 bits: a row has 2^30 at most.)
struct LpRun {
  int first, pieces, lone;
};
template <typename T>
__device__ inline LpRun lp_run(const T* row, int c0, int c1) {
  constexpr int E = LpPiece<T>::E;
  const int head = (int)lp_head(row + c0, c1 - c0), first = c0 + head, pieces = (c1 - first) / E, tail = c1 - first - pieces * E;
  const int i = threadIdx.x;
  return {first, pieces, i < head ? c0 + i : (i >= E && i < E + tail ? first + pieces * E + i - E : -1)};
}
// Calls f(values, column, how many) for all elements [c0, c1) of a row, U pieces in flight.
template <typename T, int U, int THREADS, typename F>
__device__ inline void lp_each(const T* row, int c0, int c1, F f) {
  constexpr int E = LpPiece<T>::E;
  const LpRun r = lp_run(row, c0, c1);
  const T* const first = row + r.first;
  float x[E];
  for (int v = threadIdx.x; v < r.pieces; v += THREADS * U) {
    typename LpPiece<T>::vec raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (v + u * THREADS < r.pieces) raw[u] = *(const typename LpPiece<T>::vec*)(first + (unsigned)(v + u * THREADS) * E);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (v + u * THREADS >= r.pieces) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = (float)raw[u][e];
      f(x, r.first + (v + u * THREADS) * E, E);
    }
  }
  if (r.lone < 0) return;
  x[0] = (float)row[r.lone];
#pragma unroll
  for (int e = 1; e < E; ++e) x[e] = -__builtin_inff();
  f(x, r.lone, 1);
}
// Fills the elements [c0, c1) of a row.
template <typename T>
__device__ inline void lp_fill(T* row, int c0, int c1, T value) {
  constexpr int E = LpPiece<T>::E;
  const LpRun r = lp_run(row, c0, c1);
  typename LpPiece<T>::vec all;
#pragma unroll
  for (int e = 0; e < E; ++e) all[e] = value;
  for (int v = threadIdx.x; v < r.pieces; v += LP_THREADS) *(typename LpPiece<T>::vec*)(row + r.first + (unsigned)v * E) = all;
  if (r.lone >= 0) row[r.lone] = value;
}

// Ranks the `count` candidates in LDS (all different, count at most LP_CANDIDATES): rank r < k goes to out(r, key).
template <int THREADS, typename F>
__device__ inline void lp_rank(const uint64_t* cand, int count, int k, F out) {
  for (int i = threadIdx.x; i < count; i += THREADS) {
    const uint64_t mine = cand[i];
    int above = 0;
#pragma unroll 16
    for (int j = 0; j < count; ++j) above += cand[j] > mine;
    if (above < k) out(above, mine);
  }
}

// One pass for the sums, a second for the candidates.  (Kept in registers between the two, the columns of small workgroups gain nothing: 256 x 32000 with 20
// alternatives 14.1 us both ways, 512 x 32000 24 kept and 19 read again.)
template <typename T, int THREADS, bool TOP>
__global__ __launch_bounds__(THREADS) void logprob_kernel(LpArgs g) {
  constexpr int E = LpPiece<T>::E, WAVES = THREADS / 64;
  __shared__ LpSum sums[WAVES];
  __shared__ uint64_t best_of[TOP ? THREADS : 1], cand[TOP ? LP_CANDIDATES : 1], bound;
  __shared__ int found;
  const int tid = threadIdx.x, split = blockIdx.y;
  const int n = (int)g.n, chunk = (int)g.chunk, c0 = split * chunk, c1 = n - c0 < chunk ? n : c0 + chunk;
  const int64_t row = g.row0 + blockIdx.x;
  const T* const x = (const T*)g.x + row * g.ld;
  auto each = [&](auto f) { lp_each<T, 4, THREADS>(x, c0, c1, f); };
  LpSum a = lp_none();
  float best = -__builtin_inff();
  int best_col = -1;
  each([&](const float (&v)[E], int col, int count) {
    float top = v[0];
#pragma unroll
    for (int e = 1; e < E; ++e) top = fmaxf(top, v[e]);
    if (top > a.m) a = lp_moved(a, top, g.c);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (e >= count) break;
      const float u = (v[e] - a.m) * g.c, p = __builtin_amdgcn_exp2f(u);
      a.s += p;
      a.w = fmaf(lp_cut(u), p, a.w);
    }
    if (TOP && (best_col < 0 || top > best)) {
      best = top > best ? top : best;
      int at = 0;
#pragma unroll
      for (int e = E - 1; e >= 0; --e)
        if (v[e] == best) at = e;
      best_col = col + (best == -__builtin_inff() ? 0 : at);
    }
  });
  a = lp_wave_merge(a, g.c);
  if ((tid & 63) == 0) sums[tid >> 6] = a;
  if (TOP) best_of[tid] = best_col < 0 ? 0 : lp_key(best, best_col);
  if (TOP && tid == 0) { bound = 0; found = 0; }
  __syncthreads();
  a = (tid & 63) < WAVES ? sums[tid & 63] : lp_none();
  a = lp_wave_merge(a, g.c);
  const float log_s = lp_log_sum(a.s);
  if (tid == 0) {
    if (g.splits == 1) lp_finish<T>(g, row, a, log_s);
    else *(f32x4*)(g.part + (row * g.splits + split) * 4) = (f32x4){a.m, a.s, a.w, 0.0f};
  }
  if constexpr (TOP) {
    // The bound, found by one wave, or four: of the maxima of 256 groups of threads, or of 64 where that will do.
    const int groups = g.top <= 32 ? 64 : 256;
    uint64_t mine = best_of[tid];
    int above = 0;
    if (tid < groups) {
      for (int i = tid + groups; i < THREADS; i += groups) mine = best_of[i] > mine ? best_of[i] : mine;
      cand[tid] = mine;
    }
    if (groups > 64) __syncthreads();
    else sb_wave_sync();
    if (tid < groups) {
#pragma unroll 16
      for (int i = 0; i < groups; ++i) above += cand[i] > mine;
      if (above == g.top - 1 && mine) bound = mine;        // (all different but for groups without elements)
    }
    __syncthreads();
    const uint64_t least = bound;
    const float least_value = least ? lp_value(least) : -__builtin_inff();
    each([&](const float (&v)[E], int col, int count) {
      float top = v[0];
#pragma unroll
      for (int e = 1; e < E; ++e) top = fmaxf(top, v[e]);
      if (top < least_value) return;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (e >= count) break;
        if (v[e] < least_value) continue;          // (passed by most waves as a whole)
        const uint64_t key = lp_key(v[e], col + e);
        if (key >= least) {
          const int at = atomicAdd(&found, 1);
          if (at < LP_CANDIDATES) cand[at] = key;
        }
      }
    });
    __syncthreads();
    const int count = found;
    auto put = [&](int r, uint64_t key) {
      if (g.splits > 1) {
        g.part_top[(row * g.splits + split) * g.top + r] = key;
      } else {
        g.top_ids[row * g.top + r] = lp_index(key);
        g.top_logp[row * g.top + r] = lp_log(g, lp_value(key), a, log_s);
      }
    };
    if (count <= LP_CANDIDATES) {
      lp_rank<THREADS>(cand, count, g.top, put);
      if (g.splits > 1)
        for (int r = count + tid; r < g.top; r += THREADS) put(r, 0);
    } else {                                       // one by one, each below the one before
      uint64_t last = ~0ull;
      for (int r = 0; r < g.top; ++r) {
        uint64_t next = 0;
        lp_each<T, 1, THREADS>(x, c0, c1, [&](const float (&v)[E], int col, int cnt) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (e >= cnt) break;
            const uint64_t key = lp_key(v[e], col + e);
            if (key < last && key > next) next = key;
          }
        });
#pragma unroll
        for (int d = 32; d; d >>= 1) {
          const uint64_t other = __shfl_xor((unsigned long long)next, d);
          next = other > next ? other : next;
        }
        __syncthreads();
        if ((tid & 63) == 0) best_of[tid >> 6] = next;
        __syncthreads();
        last = best_of[0];
        for (int w = 1; w < WAVES; ++w) last = best_of[w] > last ? best_of[w] : last;
        if (tid == 0) put(r, last);
      }
    }
  }
  __syncthreads();
}

// Joins the parts of split rows: their sums in a fixed tree, and the ranks of the candidates among those that are not below a bound of the k-th
// largest: the largest of the lists' last entries, or the smallest of their (k / splits)-th ones.
template <typename T>
__global__ __launch_bounds__(LP_THREADS) void logprob_join_kernel(LpArgs g) {
  extern __shared__ uint64_t cand[];                 // splits x top
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63, total = g.splits * g.top;
  const int64_t row = g.row0 + blockIdx.x;
  const uint64_t* const lists = g.part_top + row * total;
  LpSum a = lp_none();
  uint64_t last = 0, early = ~0ull;
  if (lane < g.splits) {
    const f32x4 p = *(const f32x4*)(g.part + (row * g.splits + lane) * 4);
    if (g.top) {
      last = lists[lane * g.top + g.top - 1];
      early = lists[lane * g.top + (g.top - 1) / g.splits];
    }
    a = {p[0], p[1], p[2]};
  }
  a = lp_wave_merge(a, g.c);
  const float log_s = lp_log_sum(a.s);
  if (tid == 0) lp_finish<T>(g, row, a, log_s);
  if (g.top) {
#pragma unroll
    for (int d = 32; d; d >>= 1) {
      const uint64_t l = __shfl_xor((unsigned long long)last, d), e = __shfl_xor((unsigned long long)early, d);
      last = l > last ? l : last;
      early = e < early ? e : early;
    }
    const uint64_t least = last > early ? last : early;
    if (tid == 0) found = 0;
    __syncthreads();
    for (int i = tid; i < total; i += LP_THREADS) {
      const uint64_t key = lists[i];
      if (key && key >= least) cand[atomicAdd(&found, 1)] = key;
    }
    __syncthreads();
    lp_rank<LP_THREADS>(cand, found, g.top, [&](int r, uint64_t key) {
      g.top_ids[row * g.top + r] = lp_index(key);
      g.top_logp[row * g.top + r] = lp_log(g, lp_value(key), a, log_s);
    });
    __syncthreads();
  }
}

// What the gradient of a row needs.
struct LpRow {
  float m, inv_s;        // M, 1 / S
  float by, by_u;        // dx_j = 2^u_j (by + by_u u_j) but at the target, which has g more
  float g;
  int64_t target;
  bool zero, bad;
};
__device__ inline LpRow lp_row(const LpArgs& g, int64_t row, float m, float s, float log_s, float entropy) {
  LpRow r;
  r.target = g.targets ? lp_target(g, row) : -1;
  r.bad = r.target >= g.n;
  r.g = r.target >= 0 && g.d_logp ? g.d_logp[row] * g.inv_t : 0.0f;
  const float d = g.d_entropy ? g.d_entropy[row] * g.inv_t : 0.0f, inv_s = 1.0f / s;
  r.zero = !r.bad && ((r.g == 0.0f && d == 0.0f) || s == 0.0f);
  r.m = m;
  r.by_u = -d * LP_LN2 * inv_s;
  r.by = -(r.g + d * fmaf(-LP_LN2, log_s, entropy)) * inv_s;
  return r;
}
template <bool ENTROPY>
__device__ inline float lp_slope(const LpRow& r, float u, float p) { return ENTROPY ? p * fmaf(r.by_u, lp_cut(u), r.by) : p * r.by; }

// Gradient from the statistics: a chunk of a row per workgroup.
template <typename T, bool ENTROPY>
__global__ __launch_bounds__(LP_THREADS) void logprob_backward_kernel(LpArgs g) {
  constexpr int E = LpPiece<T>::E;
  const int n = (int)g.n, chunk = (int)g.chunk, c0 = (int)blockIdx.y * chunk, c1 = n - c0 < chunk ? n : c0 + chunk;
  const int64_t row = g.row0 + blockIdx.x;
  const float m = g.stats[row], log_s = g.stats[g.m + row];
  const LpRow r = lp_row(g, row, m, m == -__builtin_inff() ? 0.0f : exp2f(log_s), log_s, g.stats[2 * g.m + row]);
  const T* const x = (const T*)g.x + row * g.ld;
  T* const y = (T*)g.grad + row * g.ldg;
  if (r.zero || r.bad) {
    const T fill = (T)(r.bad ? __builtin_nanf("") : 0.0f);
    lp_fill(y, c0, c1, fill);
    return;
  }
  lp_each<T, 4, LP_THREADS>(x, c0, c1, [&](const float (&v)[E], int col, int count) {
    typename LpPiece<T>::vec out;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      if (e >= count) break;
      const float u = (v[e] - r.m) * g.c;
      out[e] = (T)lp_slope<ENTROPY>(r, u, __builtin_amdgcn_exp2f(u));
    }
    if (r.target >= col && r.target < col + count) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (col + e == r.target) {
          const float u = (v[e] - r.m) * g.c;
          out[e] = (T)(r.g + lp_slope<ENTROPY>(r, u, __builtin_amdgcn_exp2f(u)));
        }
    }
    if (count == E) *(typename LpPiece<T>::any*)(y + col) = out;
    else y[col] = out[0];
  });
}

// Both in one call: a row stays in the registers of a workgroup between the sums and the gradient.  V pieces per thread.  The exponentials are formed
// again for the gradient: kept, they take twice the row's registers, and no second workgroup of the CU could work while one waits for memory.
// REST: what lies behind V pieces per thread (65536 float32, 131072 bf16) is summed beside a running maximum and read again for the gradient.
// (1024 threads with eight pieces have 64 registers each for two workgroups to a CU and keep two more words in scratch memory: 8192 x 50257 bf16 takes 324 us, at the
// copy's rate 320.)
template <typename T, int THREADS, int V, bool ENTROPY, bool REST = false>
__global__ __launch_bounds__(THREADS, V < 8 || THREADS * V == 8192 ? 8 : (V == 8 ? 7 : 4)) void logprob_grad_kernel(LpArgs g) {
  constexpr int E = LpPiece<T>::E, WAVES = THREADS / 64;
  __shared__ float tops[WAVES];
  __shared__ float sums[2][WAVES];
  const int tid = threadIdx.x;
  const int64_t row = g.row0 + blockIdx.x;
  const T* const x = (const T*)g.x + row * g.ld;
  const int n = (int)g.n, head = (int)lp_head(x, g.n), pieces = (n - head) / E, tail = n - head - pieces * E;
  const T* const body = x + head;
  typename LpPiece<T>::vec raw[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int at = tid + u * THREADS;
    if (at < pieces) raw[u] = *(const typename LpPiece<T>::vec*)(body + (unsigned)at * E);
  }
  const int lone = tid < head ? tid : (tid >= E && tid < E + tail ? head + pieces * E + tid - E : -1);
  const float alone = lone >= 0 ? (float)x[lone] : -__builtin_inff();
  // f(values, piece) for the pieces that are not held
  auto rest = [&](auto f) {
    for (int at = tid + V * THREADS; at < pieces; at += 2 * THREADS) {
      typename LpPiece<T>::vec two[2];
      two[0] = *(const typename LpPiece<T>::vec*)(body + (unsigned)at * E);
      if (at + THREADS < pieces) two[1] = *(const typename LpPiece<T>::vec*)(body + (unsigned)(at + THREADS) * E);
      f(two[0], at);
      if (at + THREADS < pieces) f(two[1], at + THREADS);
    }
  };
  LpSum more = lp_none();
  if constexpr (REST)
    rest([&](const typename LpPiece<T>::vec& v, int) {
      float t = (float)v[0];
#pragma unroll
      for (int e = 1; e < E; ++e) t = fmaxf(t, (float)v[e]);
      if (t > more.m) more = lp_moved(more, t, g.c);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float u = ((float)v[e] - more.m) * g.c, p = __builtin_amdgcn_exp2f(u);
        more.s += p;
        more.w = fmaf(lp_cut(u), p, more.w);
      }
    });
  float top = REST ? fmaxf(alone, more.m) : alone;
#pragma unroll
  for (int u = 0; u < V; ++u)
    if (tid + u * THREADS < pieces) {
#pragma unroll
      for (int e = 0; e < E; ++e) top = fmaxf(top, (float)raw[u][e]);
    }
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
  top = tops[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) top = fmaxf(top, tops[w]);
  LpSum a = {fmaxf(top, -FLT_MAX), 0.0f, 0.0f};
  if constexpr (REST) a = lp_moved(more, a.m, g.c);
  auto add = [&](float v) {
    const float u = (v - a.m) * g.c, p = __builtin_amdgcn_exp2f(u);
    a.s += p;
    a.w = fmaf(lp_cut(u), p, a.w);
  };
  if (lone >= 0) add(alone);
#pragma unroll
  for (int u = 0; u < V; ++u)
    if (tid + u * THREADS < pieces) {
#pragma unroll
      for (int e = 0; e < E; ++e) add((float)raw[u][e]);
    }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    a.s += __shfl_xor(a.s, d);
    a.w += __shfl_xor(a.w, d);
  }
  if ((tid & 63) == 0) { sums[0][tid >> 6] = a.s; sums[1][tid >> 6] = a.w; }
  __syncthreads();
  a.s = sums[0][0];
  a.w = sums[1][0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) { a.s += sums[0][w]; a.w += sums[1][w]; }
  const float log_s = lp_log_sum(a.s);
  const LpRow r = lp_row(g, row, a.m, a.s, log_s, lp_entropy(a, log_s));
  if (tid == 0) lp_finish<T>(g, row, a, log_s);
  const float asked = r.g != 0.0f && !r.bad && r.target >= 0 ? (float)x[r.target] : 0.0f;
  __syncthreads();                                 // (the target's logit is read before the gradient may take its place)
  T* const y = (T*)g.grad + row * g.ldg;
  if (r.zero || r.bad) {
    const T fill = (T)(r.bad ? __builtin_nanf("") : 0.0f);
    if (lone >= 0) y[lone] = fill;
#pragma unroll
    for (int u = 0; u < V; ++u)
      if (tid + u * THREADS < pieces) {
        typename LpPiece<T>::vec out;
#pragma unroll
        for (int e = 0; e < E; ++e) out[e] = fill;
        *(typename LpPiece<T>::any*)(y + head + (unsigned)(tid + u * THREADS) * E) = out;
      }
    if constexpr (REST) {
      typename LpPiece<T>::vec out;
#pragma unroll
      for (int e = 0; e < E; ++e) out[e] = fill;
      for (int at = tid + V * THREADS; at < pieces; at += THREADS) *(typename LpPiece<T>::any*)(y + head + (unsigned)at * E) = out;
    }
    return;
  }
  const int hit = r.g != 0.0f && r.target >= 0 ? (int)r.target : -1;
  auto slope = [&](float v) {
    const float u = (v - r.m) * g.c;
    return lp_slope<ENTROPY>(r, u, __builtin_amdgcn_exp2f(u));
  };
  if (lone >= 0) y[lone] = (T)(slope(alone) + (lone == hit ? r.g : 0.0f));
  auto put = [&](const typename LpPiece<T>::vec& v, int at) {
    const int col = head + at * E;
    typename LpPiece<T>::vec out;
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = (T)slope((float)v[e]);
    if (hit >= col && hit < col + E) {
      const T own = (T)(r.g + slope(asked));
#pragma unroll
      for (int e = 0; e < E; ++e) out[e] = col + e == hit ? own : out[e];
    }
    *(typename LpPiece<T>::any*)(y + head + (unsigned)at * E) = out;
  };
#pragma unroll
  for (int u = 0; u < V; ++u)
    if (tid + u * THREADS < pieces) put(raw[u], tid + u * THREADS);
  if constexpr (REST) rest(put);
}

// Workgroups of 1024 threads where they are enough for the card and 256 threads are not.  us with 1024 and with 256 threads, 32000 columns in bf16: 256 rows 9.0 and
// 10.5 (20 alternatives: 15.2 and 18.6; 21 split between workgroups of 256 and joined), 512 rows 11.9 and 12.6 (18.8 and 21.7), 768 rows 16.0 and 15.1 (27.1 and 24.6), 1024 rows
// 19.0 and 17.8 (31.2 and 28.5).  Longer rows gain from 1024 threads for longer: 50257 columns in float32 768 rows 31.1 and 32.3 (51.9 and 53.8), 1024 rows 39.5
// and 40.5 (64.1 and 68.6).  One border for all of them costs 14 % at worst (2048 rows of 50257 in
// float32 with alternatives 135, 119).  Fewer rows are split between workgroups of 256, as many as make 1024 of
// them, of 512 pieces at least: a row of 128000 with 5 alternatives 7 us and 4 for the join.  (The gradient in the same call takes a third launch then: one row
// of 32000 8.6 us, 64 rows 10.5, 127 rows 14.1; 128 rows, a workgroup each, 9.9.)
static bool lp_wide(int64_t m, int64_t n, bool bf16) { return m >= 128 && m < 1024 && n >= (bf16 ? 8192 : 4096); }
static int lp_splits(int64_t m, int64_t n, bool bf16) {
  const int64_t want = m >= 128 ? 1 : 1024 / m;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, n / (bf16 ? 4096 : 2048)), LP_SPLITS));
}
static int64_t lp_chunk(int64_t n, int splits) { return (int64_t)align_up((size_t)ceil_div64(n, splits), 64); }
static size_t lp_part_bytes(int64_t m, int64_t n, int top, bool bf16) {
  const int s = lp_splits(m, n, bf16);
  return s > 1 ? (size_t)m * s * (16 + 8 * (size_t)top) : 0;
}
// A workgroup per row holds what it can of it in registers; few rows are split between workgroups, in two passes, and so are rows of which less than half
// could be held.
static bool lp_held(int64_t m, int64_t n, bool bf16) { return lp_splits(m, n, bf16) == 1 && n / (bf16 ? 8 : 4) <= 32 * 1024; }

#define LP_ROWS (1 << 20)                            // of a launch: fewer than 2^32 threads
template <typename T>
static int launch_logprobs(hipStream_t s, LpArgs g) {
  g.splits = lp_splits(g.m, g.n, sizeof(T) == 2);
  g.chunk = lp_chunk(g.n, g.splits);
  g.splits = (int)ceil_div64(g.n, g.chunk);
#define LP_FORWARD(THREADS)                                                                                                   \
  do {                                                                                                                         \
    if (g.top) LORACT_LAUNCH("token_logprobs", s, (logprob_kernel<T, THREADS, true>), grid, dim3(THREADS), 0, g);               \
    else LORACT_LAUNCH("token_logprobs", s, (logprob_kernel<T, THREADS, false>), grid, dim3(THREADS), 0, g);                   \
  } while (0)
  for (g.row0 = 0; g.row0 < g.m; g.row0 += LP_ROWS) {
    const dim3 grid((unsigned)std::min<int64_t>(g.m - g.row0, LP_ROWS), (unsigned)g.splits);
    if (lp_wide(g.m, g.n, sizeof(T) == 2)) LP_FORWARD(1024);
    else LP_FORWARD(LP_THREADS);
    if (g.splits > 1) LORACT_LAUNCH("token_logprobs_join", s, logprob_join_kernel<T>, dim3(grid.x), dim3(LP_THREADS), (unsigned)(g.splits * g.top * 8), g);
  }
#undef LP_FORWARD
  return LORACT_OK;
}
template <typename T>
static int launch_logprobs_backward(hipStream_t s, LpArgs g) {
  g.chunk = std::max<int64_t>(LP_THREADS * 4 * LpPiece<T>::E, lp_chunk(g.n, 64));
  for (g.row0 = 0; g.row0 < g.m; g.row0 += 1 << 17) {
    const dim3 grid((unsigned)std::min<int64_t>(g.m - g.row0, 1 << 17), (unsigned)ceil_div64(g.n, g.chunk));
    if (g.d_entropy) LORACT_LAUNCH("token_logprobs_backward", s, (logprob_backward_kernel<T, true>), grid, dim3(LP_THREADS), 0, g);
    else LORACT_LAUNCH("token_logprobs_backward", s, (logprob_backward_kernel<T, false>), grid, dim3(LP_THREADS), 0, g);
  }
  return LORACT_OK;
}
template <typename T>
static int launch_logprobs_grad(hipStream_t s, LpArgs g) {
  if (!lp_held(g.m, g.n, sizeof(T) == 2)) {
    LORACT_TRY(launch_logprobs<T>(s, g));
    return launch_logprobs_backward<T>(s, g);
  }
  const int64_t pieces = g.n / LpPiece<T>::E;
#define LP_GRAD(THREADS, V, REST)                                                                                                        \
  do {                                                                                                                                    \
    if (g.d_entropy) LORACT_LAUNCH("token_logprobs_grad", s, (logprob_grad_kernel<T, THREADS, V, true, REST>), grid, dim3(THREADS), 0, g);  \
    else LORACT_LAUNCH("token_logprobs_grad", s, (logprob_grad_kernel<T, THREADS, V, false, REST>), grid, dim3(THREADS), 0, g);           \
  } while (0)
  for (g.row0 = 0; g.row0 < g.m; g.row0 += LP_ROWS) {
    const dim3 grid((unsigned)std::min<int64_t>(g.m - g.row0, LP_ROWS));
    // (512 threads with eight pieces: 8192 x 32000 bf16 203 us, with 1024 and four 239, 16384 x 16400 201 and 253: fewer waves wait for the same row; 4096 x 16000
    // float32 106 and 103)
    if (pieces <= 256 * 2) LP_GRAD(256, 2, false);
    else if (pieces <= 256 * 8) LP_GRAD(256, 8, false);
    else if (pieces <= 512 * 8) LP_GRAD(512, 8, false);
    else if (pieces <= 1024 * 8) LP_GRAD(1024, 8, false);
    else if (pieces <= 1024 * 16) LP_GRAD(1024, 16, false);
    else LP_GRAD(1024, 16, true);
  }
#undef LP_GRAD
  return LORACT_OK;
}

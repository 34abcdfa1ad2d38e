// Dropout from a counter: whether element (i, j) of an m x n matrix is kept depends on (seed, i, j) alone, so the
// mask is made again wherever it is needed and never stored.
//
//   word(i, g) = splitmix64 output number i ceil(n / 4) + g + 1 of the seed,   field(i, j) = bits 16 (j % 4) .. + 15 of word(i, j / 4)
//   y_ij = x_ij 65536 / (65536 - thr)  where field(i, j) >= thr = round(65536 p),   0 elsewhere
//
// Four elements share a 64-bit output: two 64-bit products per four elements, a third of the vector rate that a CU has
// left while it streams bf16 at the rate of a copy.  A group of four never crosses a row, so any four aligned columns of
// any row can be masked by themselves (the epilogues of the products do).  A dropped element is 0 whatever it held: it is
// selected, not multiplied.
//
// Bound by memory: 8192 x 4096 bf16 with a residual 38.5 us, 5.2 TB/s, the rate of a copy.
#pragma once
#include "common.h"

#include <algorithm>

struct DropArgs {
  uint64_t seed;
  int64_t groups;        // ceil(n / 4)
  uint32_t thr;          // 0: everything is kept
  float scale;
};

static inline DropArgs drop_args(double p, uint64_t seed, int64_t n) {
  DropArgs d;
  const double t = p * 65536.0 + 0.5;
  d.thr = t >= 65535.0 ? 65535u : (uint32_t)t;
  d.scale = (float)(65536.0 / (65536.0 - (double)d.thr));
  d.seed = seed;
  d.groups = ceil_div64(n, 4);
  return d;
}

__device__ inline uint64_t drop_word(const DropArgs& d, int64_t row, int64_t group) {
  return splitmix64_mix(d.seed + (uint64_t)(row * d.groups + group + 1) * SPLITMIX_GOLDEN);
}
__device__ inline float drop_one(const DropArgs& d, uint64_t word, int i, float v) {
  return ((uint32_t)(word >> (16 * i)) & 0xffffu) >= d.thr ? v * d.scale : 0.0f;
}

struct DropoutArgs {
  const void* X;
  int64_t ldx;
  const void* R;         // optional residual
  int64_t ldr;
  void* Y;
  int64_t ldy;
  int64_t m, n;
  int64_t step_rows, step_pieces;   // the grid's stride in rows and pieces of a row
  DropArgs d;
};

// One piece of E columns per thread and trip (E = 16 bytes' worth; E = 4, element by element, where rows do not allow
// that), U of them in flight.  The place (row, piece) advances by the grid's stride, so there is one division per thread.
template <typename T, int E, bool VEC, int U>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs g) {
  typedef T piece __attribute__((ext_vector_type(E)));
  const int64_t per_row = (g.n + E - 1) / E;
  const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int64_t row = first / per_row, at = first - row * per_row;
  while (row < g.m) {
    T x[U][E], r[U][E];
    int64_t rows[U], cols[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      rows[u] = row;
      cols[u] = at * E;
      at += g.step_pieces;
      row += g.step_rows;
      if (at >= per_row) { at -= per_row; ++row; }
      if (rows[u] >= g.m) continue;
      const T* xp = (const T*)g.X + rows[u] * g.ldx + cols[u];
      const T* rp = (const T*)g.R + rows[u] * g.ldr + cols[u];
      if (VEC) {
        *(piece*)x[u] = *(const piece*)xp;
        if (g.R) *(piece*)r[u] = *(const piece*)rp;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const bool in = cols[u] + e < g.n;
          x[u][e] = in ? xp[e] : (T)0.0f;
          r[u][e] = in && g.R ? rp[e] : (T)0.0f;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (rows[u] >= g.m) break;
      T y[E];
#pragma unroll
      for (int q = 0; q < E / 4; ++q) {
        const uint64_t word = drop_word(g.d, rows[u], cols[u] / 4 + q);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float v = drop_one(g.d, word, e, (float)x[u][4 * q + e]);
          if (g.R) v += (float)r[u][4 * q + e];
          y[4 * q + e] = (T)v;
        }
      }
      T* yp = (T*)g.Y + rows[u] * g.ldy + cols[u];
      if (VEC) {
        *(piece*)yp = *(const piece*)y;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (cols[u] + e < g.n) yp[e] = y[e];
      }
    }
  }
}

template <typename T>
static int launch_dropout(hipStream_t s, DropoutArgs g, bool vec) {
  constexpr int E = 16 / sizeof(T), U = 2;
  const int64_t per_row = ceil_div64(g.n, vec ? E : 4);
  const int64_t blocks = std::min<int64_t>(ceil_div64(g.m * per_row, 256 * U), 2048);
  g.step_rows = blocks * 256 / per_row;
  g.step_pieces = blocks * 256 % per_row;
  if (vec) LORACT_LAUNCH("dropout", s, (dropout_kernel<T, E, true, U>), dim3((unsigned)blocks), dim3(256), 0, g);
  else LORACT_LAUNCH("dropout", s, (dropout_kernel<T, 4, false, U>), dim3((unsigned)blocks), dim3(256), 0, g);
  return LORACT_OK;
}

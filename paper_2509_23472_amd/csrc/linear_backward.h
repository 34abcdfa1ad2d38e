// Backward of loract_linear's epilogue in one pass over dY and Z:
//   dP_ij = act'(Z_ij) D(dY)_ij,   db_j = sum_i dP_ij,   dB = s T^T dP   (r x n)
// with the mask of D made again from the counter.
//
// The element-wise result never leaves the registers for the sums: a lane holds E consecutive columns of one row, four rows per
// wave instruction, which is the operand layout of v_mfma_f32_16x16x4_f32 when its column index is read as "every E-th
// column": the e-th product of a lane takes its e-th element, row l / 16, column E (l % 16) + e, and T's rows as the other
// operand.  The sums are therefore exact float32 products of the unrounded dP, and neither LDS nor a second reading of dP is
// needed.  Waves of a workgroup take turns over its rows and are joined in LDS, workgroups over the rows of a
// column strip through partial sums, both in a fixed order.
//
// Bound by memory: 8192 x 11008 bf16 with SiLU and 16 columns of T 119 us and 5 for the join (4.6 TB/s; a copy 5.1).  With GELU, dropout
// and more columns by vector and float32 matrix instructions, one after the other in a wave: 32 columns 191 us, 64 302 (238 without the two).
#pragma once
#include "linear_epilogue.h"

struct LinBackArgs {
  const void* dY;
  int64_t lddy;
  const void* Z;         // null: no activation
  int64_t ldz;
  const void* T;         // m x r contiguous, or null
  int64_t r;
  void* dP;
  int64_t lddp;
  int64_t m, n;
  int act;
  int64_t chunk;         // rows per workgroup
  float* part;           // [chunk][1 + 16 RB][columns of all strips]; null: no sums
  int64_t n_pad;
  DropArgs d;
};

#define LB_WAVES 4

// Columns per lane: 16 bytes' worth; 8 for bf16 with more than 32 columns of T, whose accumulators would leave room for one wave
// per SIMD.
constexpr int lb_columns(int size, int rb) { return size == 2 && rb <= 2 ? 8 : 4; }

// VEC: rows allow pieces of lb_columns elements.  RB: blocks of 16 columns of T (0: the bias gradient alone, or nothing).  The
// i-th row of the products' block b stands for column RB i + b of T, so that a lane's RB values of T lie together.
template <typename T, bool VEC, int RB>
__global__ __launch_bounds__(64 * LB_WAVES) void linear_backward_kernel(LinBackArgs g) {
  constexpr int E = lb_columns(sizeof(T), RB), U = E == 4 && sizeof(T) == 2 ? 4 : 2;
  typedef T piece __attribute__((ext_vector_type(E)));
  typedef T t_piece __attribute__((ext_vector_type(RB ? RB : 1)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = lane & 15, k = lane >> 4;
  const int64_t strip = (int64_t)blockIdx.z * gridDim.x + blockIdx.x;
  if (strip * (16 * E) >= g.n) return;               // (the last of several blockIdx.z may not be full)
  const int64_t col = strip * (16 * E) + c * E;
  const int64_t r_beg = (int64_t)blockIdx.y * g.chunk;
  const int64_t r_end = r_beg + g.chunk < g.m ? r_beg + g.chunk : g.m;
  const bool on = col < g.n;
  const bool t_vec = g.r == 16 * RB && RB != 3 && (uintptr_t)g.T % (RB * sizeof(T) + (RB == 0)) == 0;
  float sum[E];
  f32x4 acc[RB ? RB : 1][E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    sum[e] = 0.0f;
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b][e] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  }
  for (int64_t r0 = r_beg + wave * (4 * U); r0 < r_end; r0 += LB_WAVES * 4 * U) {
    T y[U][E], z[U][E];
    float tv[U][RB ? RB : 1], p[U][E];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = r0 + 4 * u + k;
      const bool live = on && row < r_end;
#pragma unroll
      for (int e = 0; e < E; ++e) { y[u][e] = (T)0.0f; z[u][e] = (T)0.0f; }
      if (live) {
        const T* yp = (const T*)g.dY + row * g.lddy + col;
        const T* zp = (const T*)g.Z + row * g.ldz + col;
        if (VEC) {
          *(piece*)y[u] = *(const piece*)yp;
          if (g.Z) *(piece*)z[u] = *(const piece*)zp;
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (col + e < g.n) {
              y[u][e] = yp[e];
              if (g.Z) z[u][e] = zp[e];
            }
        }
      }
      if (RB) {
        const T* tp = (const T*)g.T + row * g.r + RB * c;
#pragma unroll
        for (int b = 0; b < RB; ++b) tv[u][b] = 0.0f;
        if (row < r_end) {
          if (t_vec) {
            const t_piece t = *(const t_piece*)tp;
#pragma unroll
            for (int b = 0; b < RB; ++b) tv[u][b] = (float)t[b];
          } else {
#pragma unroll
            for (int b = 0; b < RB; ++b)
              if (RB * c + b < g.r) tv[u][b] = (float)tp[b];
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < E; ++e) p[u][e] = (float)y[u][e];
    if (g.d.thr) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
          const uint64_t word = drop_word(g.d, r0 + 4 * u + k, col / 4 + q);
#pragma unroll
          for (int e = 0; e < 4; ++e) p[u][4 * q + e] = drop_one(g.d, word, e, p[u][4 * q + e]);
        }
    }
    // (one choice for all of them)
    auto slopes = [&](int act) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e) p[u][e] = lin_act_back<sizeof(T) == 4>(act, (float)z[u][e], p[u][e]);
    };
    if (g.act == LORACT_ACT_RELU) slopes(LORACT_ACT_RELU);
    else if (g.act == LORACT_ACT_GELU) slopes(LORACT_ACT_GELU);
    else if (g.act == LORACT_ACT_SILU) slopes(LORACT_ACT_SILU);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t row = r0 + 4 * u + k;
      T o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (row >= r_end) p[u][e] = 0.0f;            // (the slope of a zero need not be finite times zero)
        o[e] = (T)p[u][e];
        sum[e] += p[u][e];
      }
      if (on && row < r_end) {
        T* dp = (T*)g.dP + row * g.lddp + col;
        if (VEC) {
          *(piece*)dp = *(const piece*)o;
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (col + e < g.n) dp[e] = o[e];
        }
      }
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[b][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(tv[u][b], p[u][e], acc[b][e], 0, 0, 0);
    }
  }
  if (!g.part) return;
  // db: the four row groups of the wave; then the waves of the workgroup, one after the other
  __shared__ float red[1 + 16 * RB][16 * E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    sum[e] += __shfl_xor(sum[e], 16);
    sum[e] += __shfl_xor(sum[e], 32);
  }
  for (int w = 0; w < LB_WAVES; ++w) {
    if (wave == w) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (k == 0) red[0][c * E + e] = (w ? red[0][c * E + e] : 0.0f) + sum[e];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            float* at = &red[1 + RB * (4 * k + q) + b][c * E + e];
            *at = (w ? *at : 0.0f) + acc[b][e][q];
          }
      }
    }
    __syncthreads();
  }
  float* out = g.part + (int64_t)blockIdx.y * (1 + 16 * RB) * g.n_pad + strip * (16 * E);
  for (int i = threadIdx.x; i < (1 + 16 * RB) * 16 * E; i += 64 * LB_WAVES)
    out[(int64_t)(i / (16 * E)) * g.n_pad + i % (16 * E)] = red[i / (16 * E)][i % (16 * E)];
}

// db and dB from the workgroups' partial sums, added in their order.
__global__ __launch_bounds__(256) void linear_backward_join_kernel(const float* part, int chunks, int rows, int64_t n_pad, int64_t n,
                                                                   int64_t r, float scale, float* db, float* dB) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  const int row = blockIdx.y;                      // 0: db, 1 + j: row j of dB
  const float* src = part + row * n_pad + i;
  const int64_t step = rows * n_pad;
  float s = 0.0f;
  for (int z = 0; z < chunks; z += 16) {
    float v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = src[(z + u < chunks ? z + u : chunks - 1) * step];
#pragma unroll
    for (int u = 0; u < 16; ++u)
      if (z + u < chunks) s += v[u];
  }
  if (row == 0) { if (db) db[i] = s; }
  else if (row <= r) dB[(int64_t)(row - 1) * n + i] = s * scale;
}

struct LinBackPlan {
  int64_t strips, chunk, chunks, n_pad;
  int rb;
  size_t bytes;
};
// Rows are cut so that there are four workgroups per CU, 64 rows each at least.
static LinBackPlan linear_backward_plan(int64_t m, int64_t n, int64_t r, bool bf16) {
  LinBackPlan p;
  p.rb = (int)ceil_div64(r, 16);
  const int width = 16 * lb_columns(bf16 ? 2 : 4, p.rb);
  p.strips = ceil_div64(n, width);
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>(std::max<int64_t>(1, 1024 / p.strips), ceil_div64(m, 64)));
  p.chunk = ceil_div64(ceil_div64(m, want), 64) * 64;
  p.chunks = ceil_div64(m, p.chunk);
  p.n_pad = p.strips * width;
  p.bytes = (size_t)p.chunks * (1 + 16 * p.rb) * p.n_pad * 4;
  return p;
}

template <typename T>
static int launch_linear_backward(hipStream_t s, LinBackArgs g, const LinBackPlan& p, bool vec, float scale, float* db, float* dB) {
  g.chunk = p.chunk;
  g.n_pad = p.n_pad;
  const int64_t x = std::min<int64_t>(p.strips, 1 << 23);               // (fewer than 2^32 threads in a direction)
  const dim3 grid((unsigned)x, (unsigned)p.chunks, (unsigned)ceil_div64(p.strips, x));
#define LB_LAUNCH(V, RB) LORACT_LAUNCH("linear_backward", s, (linear_backward_kernel<T, V, RB>), grid, dim3(64 * LB_WAVES), 0, g)
#define LB_RB(RB) { if (vec) LB_LAUNCH(true, RB); else LB_LAUNCH(false, RB); break; }
  switch (p.rb) {
    case 0: LB_RB(0)
    case 1: LB_RB(1)
    case 2: LB_RB(2)
    case 3: LB_RB(3)
    default: LB_RB(4)
  }
#undef LB_RB
#undef LB_LAUNCH
  if (!g.part) return LORACT_OK;
  LORACT_LAUNCH("linear_backward_join", s, linear_backward_join_kernel,
                dim3((unsigned)ceil_div64(g.n, 256), (unsigned)(1 + g.r)), dim3(256), 0, (const float*)g.part, (int)p.chunks,
                1 + 16 * p.rb, p.n_pad, g.n, g.r, scale, db, dB);
  return LORACT_OK;
}

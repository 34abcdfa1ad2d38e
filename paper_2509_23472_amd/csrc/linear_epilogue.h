// What follows the product in loract_linear, on values that are still in registers:
//   P = acc + bias (kept as Z where the caller asks),  Y = R + D(act(P)).
// Everything is float32 until the one rounding to the type of Y (and of Z).
#pragma once
#include "dropout.h"

// The activations and their slopes: exp and the reciprocal by the hardware's instructions (both within one unit), and Phi from
//   erfc(x) = t q(t) exp(-x^2),  t = 1 / (1 + 0.4 x),  x >= 0,
// q a polynomial of least relative error (1.4e-7, 4e-7 evaluated in float32).  What is stored as bf16 needs no more: the argument of exp is rounded
// once, which costs |x| 2^-23 of the result at most, up to 2^-17 where exp itself is 2^-126.  EXACT (what is stored as float32, and the
// slopes of float32 operands): that rounding is made good, SiLU divides, and Phi near 0 comes from a polynomial in z, which leaves what
// erff, expf and a division would: largest relative errors in units of 2^-24 (with those) SiLU 3.6 (3.0), GELU above -1 4.3 (4.5), from there to -6,
// where 1 + erf cancels, 21 (all).
// Those functions have five times the instructions, which an epilogue has nothing to hide behind: 8192 x 4096 -> 11008 bf16 with SiLU 747 us with
// them and 685 so (642 without an activation), the backward of 8192 x 11008 SiLU 169 and 123, GELU 215 and 131, of 12608 x 768
// float32 GELU 38 and 33 (32.4 without the polynomial in z), SiLU's division 32.6 (the reciprocal: 32.0).  8192 x 4096 -> 4096 of bf16 to
// float32: GELU 248 us (238 as for bf16), SiLU 239 (236); where little else is done, 3200 x 64 -> 1664 float32 GELU 33.7 (31.7).
// exp of any x, or (BELOW) of x <= 0, of which less than -104 gives 0 as -104 does: no choice between finite and infinite is needed then.
template <bool EXACT, bool BELOW>
__device__ inline float lin_exp(float x) {
  if (EXACT && BELOW) x = fmaxf(x, -104.0f);
  constexpr float L = 1.44269504088896341f, L_REST = 1.92596299112661746e-8f;      // log2(e) and what its rounding leaves
  const float t = x * L;
  const float e = __builtin_amdgcn_exp2f(t);
  if (!EXACT) return e;
  const float rest = fmaf(x, L_REST, fmaf(x, L, -t));                              // (not a number where t overflows)
  return BELOW || (t > -150.0f && t < 128.0f) ? fmaf(e, 0.693147180559945309f * rest, e) : e;  // (from 128 on e is infinite: nothing to make good)
}
// 1 / (1 + exp(-z)) and z times it.  EXACT: by a division, since the reciprocal's instruction makes zero of what is below 2^-126 (z < -87.3),
// of which z times as much need not be.
template <bool EXACT>
__device__ inline float lin_sigmoid(float z, float times) {
  const float below = 1.0f + lin_exp<EXACT, false>(-z);
  return EXACT ? times / below : times * __builtin_amdgcn_rcpf(below);
}
// Phi(z); *density: exp(-z^2 / 2)
template <bool EXACT>
__device__ inline float lin_phi(float z, float* density) {
  const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(z), 0.4f * 0.70710678118654752f, 1.0f));
  float q = 0.05026593804359436f;
  q = fmaf(q, t, -0.182917058467865f);
  q = fmaf(q, t, 0.16911154985427856f);
  q = fmaf(q, t, -0.005630594678223133f);
  q = fmaf(q, t, 0.1414429396390915f);
  q = fmaf(q, t, 0.16853874921798706f);
  q = fmaf(q, t, 0.20784316956996918f);
  q = fmaf(q, t, 0.22566956281661987f);
  q = fmaf(q, t, 0.22567586600780487f);
  const float u = z * z;
  *density = lin_exp<EXACT, true>(-0.5f * u);
  const float half = 0.5f * q * t * *density;
  const float tail = z < 0.0f ? half : 1.0f - half;
  if (!EXACT) return tail;
  // within sqrt(2) of 0, where the tail's error would be most of the result's: Phi = 1/2 + z r(z^2), r within 2e-8 / z
  float r = 4.3545057337723847e-07f;
  r = fmaf(r, u, -8.859667104843538e-06f);
  r = fmaf(r, u, 0.00011466867726994678f);
  r = fmaf(r, u, -0.0011868048459291458f);
  r = fmaf(r, u, 0.009973385371267796f);
  r = fmaf(r, u, -0.06649035960435867f);
  r = fmaf(r, u, 0.3989422917366028f);
  return u < 2.0f ? fmaf(z, r, 0.5f) : tail;
}
// (one choice for all of them: the values' chains of operations then run side by side)
template <bool EXACT, int N>
__device__ inline void lin_act(int act, float (&v)[N]) {
  if (act == LORACT_ACT_RELU) {
#pragma unroll
    for (int u = 0; u < N; ++u) v[u] = v[u] < 0.0f ? 0.0f : v[u];                  // (a NaN stays one)
  } else if (act == LORACT_ACT_GELU) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      float density;
      v[u] *= lin_phi<EXACT>(v[u], &density);
    }
  } else if (act == LORACT_ACT_SILU) {
#pragma unroll
    for (int u = 0; u < N; ++u) v[u] = lin_sigmoid<EXACT>(v[u], v[u]);
  }
}
// act'(z) g.  Where max(z, 0) is flat the gradient is 0 whatever g holds: selected, as a dropped element is.
template <bool EXACT>
__device__ inline float lin_act_back(int act, float z, float g) {
  switch (act) {
    case LORACT_ACT_RELU: return z > 0.0f ? g : 0.0f;
    case LORACT_ACT_GELU: {
      float density;
      const float phi = lin_phi<EXACT>(z, &density);
      return g * (phi + z * (density * 0.39894228040143268f));
    }
    case LORACT_ACT_SILU: {
      const float s = lin_sigmoid<EXACT>(z, 1.0f);
      return g * (s * (1.0f + z * (1.0f - s)));
    }
    default: return g;
  }
}

struct LinEpilogue {
  const float* bias;     // n, or null
  const void* R;         // m x n of the inputs' type, or null
  int64_t ldr;
  void* Y;
  int64_t ldy;
  void* Z;               // m x n of the inputs' type, or null
  int64_t ldz;
  int64_t m, n;
  int act;
  int y_f32;             // Y is float32 (the inputs may be bf16)
  int vec;               // R, Y and Z take four (bf16 large tiles: eight) elements at a time
  DropArgs d;
};

template <typename T>
struct LinQuad {
  typedef T type __attribute__((ext_vector_type(4)));
};

// Four columns col .. col + 3 (col a multiple of 4) of one row: the residual, to be loaded ahead, and the rest.
template <typename T>
__device__ inline f32x4 lin_load4(const LinEpilogue& e, int64_t row, int64_t col) {
  f32x4 r = {0.0f, 0.0f, 0.0f, 0.0f};
  if (!e.R || row >= e.m || col >= e.n) return r;
  typedef typename LinQuad<T>::type quad;
  const T* rp = (const T*)e.R + row * e.ldr + col;
  if (e.vec) {
    const quad q = *(const quad*)rp;
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = (float)q[u];
  } else {
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (col + u < e.n) r[u] = (float)rp[u];
  }
  return r;
}
template <typename T>
__device__ inline void lin_store4(const LinEpilogue& e, int64_t row, int64_t col, f32x4 v, f32x4 r) {
  if (row >= e.m || col >= e.n) return;
  typedef typename LinQuad<T>::type quad;
  float b[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  T* zp = (T*)e.Z + row * e.ldz + col;
#pragma unroll
  for (int u = 0; u < 4; ++u)
    if (e.bias && col + u < e.n) b[u] = e.bias[col + u];
  quad zq;
  f32x4 y;
  float a[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    a[u] = v[u] + b[u];
    zq[u] = (T)a[u];
  }
  if (sizeof(T) == 4 || e.y_f32) lin_act<true>(e.act, a);
  else lin_act<false>(e.act, a);
  const uint64_t word = e.d.thr ? drop_word(e.d, row, col / 4) : 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (e.d.thr) a[u] = drop_one(e.d, word, u, a[u]);
    y[u] = e.R ? a[u] + r[u] : a[u];
  }
  if (e.vec) {
    if (e.Z) *(quad*)zp = zq;
    if (e.y_f32) {
      *(f32x4*)((float*)e.Y + row * e.ldy + col) = y;
    } else {
      quad yq;
#pragma unroll
      for (int u = 0; u < 4; ++u) yq[u] = (T)y[u];
      *(quad*)((T*)e.Y + row * e.ldy + col) = yq;
    }
    return;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    if (col + u >= e.n) break;
    if (e.Z) zp[u] = zq[u];
    if (e.y_f32) ((float*)e.Y)[row * e.ldy + col + u] = y[u];
    else ((T*)e.Y)[row * e.ldy + col + u] = (T)y[u];
  }
}

// Sum of the K splits' partial tiles (in their order), then the epilogue.  part: [split][m][n_pad], n_pad = n up to a multiple of 4.
template <typename T>
__global__ __launch_bounds__(256) void linear_join_kernel(const float* part, int splits, int64_t n_pad, LinEpilogue e) {
  const int64_t quads = n_pad / 4, total = e.m * quads;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / quads, col = (i - row * quads) * 4;
    const float* src = part + row * n_pad + col;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    const f32x4 r = lin_load4<T>(e, row, col);
    for (int z = 0; z < splits; z += 4) {
      f32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *(const f32x4*)(src + (int64_t)(z + u < splits ? z + u : splits - 1) * e.m * n_pad);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (z + u < splits) s += v[u];
    }
    lin_store4<T>(e, row, col, s, r);
  }
}

// What follows the product in loract_linear, on values that are still in registers:
//   P = acc + bias (kept as Z where the caller asks),  Y = R + D(act(P)).
// Everything is float32 until the one rounding to the type of Y (and of Z).
#pragma once
#include "dropout.h"

// The activations and their slopes.  FAST (bf16 inputs): exp and the reciprocal by the hardware's instructions, and Phi from
//   erfc(x) = q(t) exp(-x^2),  t = 1 / (1 + 0.4 x),  x >= 0,
// q a polynomial fitted here to the least relative error (1.4e-7, 4e-7 evaluated in float32): relative errors below 2^-20
// wherever the result matters to 8 bits, at a fifth of the instructions of erff, expf and a division -- an epilogue of a large tile is
// vector instructions that nothing hides (8192 x 11008 with SiLU, 4096 in: 986 -> 706 us).  Float32 inputs take the device library's functions.
__device__ inline float lin_exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ inline float lin_sigmoid_fast(float z) { return __builtin_amdgcn_rcpf(1.0f + lin_exp_fast(-z)); }
// Phi(z); *density: exp(-z^2 / 2)
__device__ inline float lin_phi_fast(float z, float* density) {
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
  *density = lin_exp_fast(-0.5f * z * z);
  const float half = 0.5f * q * t * *density;
  return z < 0.0f ? half : 1.0f - half;
}
template <bool FAST>
__device__ inline float lin_act(int act, float z) {
  switch (act) {
    case LORACT_ACT_RELU: return z < 0.0f ? 0.0f : z;                       // (a NaN stays one)
    case LORACT_ACT_GELU: {
      float density;
      return FAST ? z * lin_phi_fast(z, &density) : 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    }
    case LORACT_ACT_SILU: return FAST ? z * lin_sigmoid_fast(z) : z / (1.0f + expf(-z));
    default: return z;
  }
}
template <bool FAST>
__device__ inline float lin_act_slope(int act, float z) {
  switch (act) {
    case LORACT_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case LORACT_ACT_GELU: {
      if (FAST) {
        float density;
        const float phi = lin_phi_fast(z, &density);
        return phi + z * (density * 0.39894228040143268f);
      }
      return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * (expf(-0.5f * z * z) * 0.39894228040143268f);
    }
    case LORACT_ACT_SILU: {
      const float s = FAST ? lin_sigmoid_fast(z) : 1.0f / (1.0f + expf(-z));
      return s * (1.0f + z * (1.0f - s));
    }
    default: return 1.0f;
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

// Four columns col .. col + 3 (col a multiple of 4) of one row.
template <typename T>
__device__ inline void lin_store4(const LinEpilogue& e, int64_t row, int64_t col, f32x4 v) {
  if (row >= e.m || col >= e.n) return;
  typedef typename LinQuad<T>::type quad;
  float b[4] = {0.0f, 0.0f, 0.0f, 0.0f}, r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  const T* rp = (const T*)e.R + row * e.ldr + col;
  T* zp = (T*)e.Z + row * e.ldz + col;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const bool in = col + u < e.n;
    if (e.bias && in) b[u] = e.bias[col + u];
    if (e.R && !e.vec && in) r[u] = (float)rp[u];
  }
  if (e.R && e.vec) {
    const quad q = *(const quad*)rp;
#pragma unroll
    for (int u = 0; u < 4; ++u) r[u] = (float)q[u];
  }
  quad zq;
  f32x4 y;
  const uint64_t word = e.d.thr ? drop_word(e.d, row, col / 4) : 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const float z = v[u] + b[u];
    zq[u] = (T)z;
    float a = lin_act<sizeof(T) == 2>(e.act, z);
    if (e.d.thr) a = drop_one(e.d, word, u, a);
    y[u] = e.R ? a + r[u] : a;
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
    for (int z = 0; z < splits; z += 4) {
      f32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = *(const f32x4*)(src + (int64_t)(z + u < splits ? z + u : splits - 1) * e.m * n_pad);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (z + u < splits) s += v[u];
    }
    lin_store4<T>(e, row, col, s);
  }
}

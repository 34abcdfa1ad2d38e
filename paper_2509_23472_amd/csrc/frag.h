// Operands of the 16 x 16 matrix instructions as a lane holds them: E consecutive k (16 bytes) of row lane % 16, from k = E (lane / 16) on.
#pragma once
#include "common.h"

template <typename T>
struct Ln {
  static constexpr int E = 16 / sizeof(T), STEP = 4 * E;     // k per lane and per step
  typedef T frag __attribute__((ext_vector_type(E)));
  typedef frag frag_any __attribute__((aligned(sizeof(T))));
};
__device__ inline f32x4 ln_mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 ln_mfma(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

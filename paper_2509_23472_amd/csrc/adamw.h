// One step of AdamW over many tensors at once, states in float32 or in 8 bits.
//
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2,  p' = (1 - lr wd) p - rate (m' / (sqrt(v') inv + eps)),
//   rate = lr / (1 - b1^t),  inv = 1 / sqrt(1 - b2^t)
//
// Every operation is rounded by itself, in this order (no fused multiply-adds): the codes of the 8-bit states are then a function
// of the definition alone, whoever computes them.  Only the quotient, which no state depends on, takes the hardware's reciprocal (an ulp).
//
// States in 8 bits.  Of 256 elements m and r = sqrt(v) are held as e4m3 numbers times a power of two each.  A power of two costs no digit of a
// floating-point code, only range (17 binades below the largest element), and scaling by it is exact.  The root, not v, because its range is
// half of v's.  Roundings are random, from a counter: with b2 = 0.999 a step moves v by a thousandth of it at most, which a nearest rounding
// to three digits would undo for ever; the root stays above zero where it is (a zero root below a moment that is not zero would make a step of m / eps).
// bf16 parameters are rounded at random for the same reason.
//
// Bound by memory: p read and written, g read, the states read and written.  4 x 4096 x 4096: all in float32 315 us (6.0 TB/s; more is read than written, a copy
// has 5.1), bf16 with 8-bit states 140 (4.8; 168 before the conversions took the rounding and a reciprocal the division: 85 vector operations per element are as
// much as the reads allow).  448 adapters of 40 M elements, float32 with copies: 256 us in five launches, of which each starts and ends by itself.
// Rate and step from device memory (captured steps): every thread forms the factors in 64 bits before its own work.  With float32 states that is hidden (347 us for 346,
// the adapters 238 for 237); with 8-bit states, whose vector work is what bounds them, it shows: bf16 with float32 gradients 180 us for 157, the adapters 121 for 107 to 118.
#pragma once
#include "common.h"

#include <cmath>

#define ADAMW_CHUNK 2048                             // elements per workgroup: eight per thread, 32 threads to a block of 256

// The tensors of a launch, a kernel argument (4 KB at most with the rest): 98 of them, 122 without copies.
template <bool COPY>
struct AdamwTable {
  static constexpr int MOST = COPY ? 98 : 122;
  void* p[MOST];
  const void* g[MOST];
  bf16_t* copy[COPY ? MOST : 1];
  int64_t n[MOST];                                   // elements
  uint32_t first[MOST];                              // the tensor's place in the state, in blocks of 256
  uint32_t chunk[MOST + 1];                          // first workgroup of each tensor, and their number
};
struct AdamwArgs {
  int count;
  void *m, *v;
  uint8_t* exps;
  const float *lr_dev, *grad_scale_dev;
  const int64_t* step_dev;
  double lr, log2_beta1, log2_beta2, weight_decay;   // (where lr or step are read on the device)
  float beta1, one_beta1, beta2, one_beta2, eps, decay, rate, inv;
  uint64_t seed;
  int64_t step;
};
static_assert(sizeof(AdamwTable<true>) + sizeof(AdamwArgs) <= 4096 && sizeof(AdamwTable<false>) + sizeof(AdamwArgs) <= 4096, "the arguments of a launch");

// rate, inv and decay of a step (host and device).
__host__ __device__ inline void adamw_rates(AdamwArgs& a, double lr, double pow1, double pow2) {
  a.rate = (float)(lr / (1.0 - pow1));
  a.inv = (float)(1.0 / sqrt(1.0 - pow2));
  a.decay = (float)(1.0 - lr * a.weight_decay);
}

template <typename T>
struct Adamw8 {
  typedef T vec __attribute__((ext_vector_type(8)));
  typedef vec any __attribute__((aligned(sizeof(T))));      // parameters and gradients begin at any element
};
template <typename T>
__device__ inline void adamw_load(const T* at, int64_t left, float (&x)[8]) {
  if (left >= 8) {
    const typename Adamw8<T>::vec v = *(const typename Adamw8<T>::any*)at;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < left ? (float)at[e] : 0.0f;
  }
}
template <typename T>
__device__ inline void adamw_store(T* at, int64_t left, const T (&x)[8]) {
  if (left >= 8) {
    typename Adamw8<T>::vec v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e];
    *(typename Adamw8<T>::any*)at = v;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) at[e] = x[e];
  }
}

typedef unsigned adamw_codes __attribute__((ext_vector_type(2)));
// Eight e4m3 numbers (bytes).
__device__ inline void adamw_decode(adamw_codes c, float unit, float (&x)[8]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(c[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c[h], true);
    x[4 * h] = lo[0] * unit;
    x[4 * h + 1] = lo[1] * unit;
    x[4 * h + 2] = hi[0] * unit;
    x[4 * h + 3] = hi[1] * unit;
  }
}
// The byte of a block's exponent from the 32 lanes that hold its elements.
__device__ inline unsigned adamw_exponent(const float (&x)[8]) {
  unsigned top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const unsigned b = __float_as_uint(x[e]) & 0x7fffffffu;
    top = max(top, b < 0x7f800000u ? b : 0u);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d));
  return max((top + 0x2aaaabu) >> 23, 8u) - 7u;
}
// Rounds x 2^(127 - byte) to e4m3 at random and puts it into byte B of `into`: the conversion adds the upper 20 bits of its seed to the 20 bits that
// it cuts off (fewer where codes are 2^-9 apart).
template <int B>
__device__ inline unsigned adamw_code(float x, float scale, unsigned bits, bool above_zero, unsigned into) {
  float y = x * scale;
  if (above_zero) y = x > 0.0f ? fmaxf(y, 0x1p-9f) : y;                // (below 2^-9 it would be 0 or that)
  return (unsigned)__builtin_amdgcn_cvt_sr_fp8_f32(y, (int)(bits << 22 | 1u << 21), (int)into, B);
}
// bf16 from float32 at random; infinities stay, and so does what is no number.
__device__ inline bf16_t adamw_bf16(float x, unsigned bits) {
  if (x != x) return (bf16_t)x;
  return __builtin_bit_cast(bf16_t, (unsigned short)((__float_as_uint(x) + bits * 16u + 8u) >> 16));
}

template <typename P, typename G, bool NARROW, bool COPY>
__global__ __launch_bounds__(256) void adamw_kernel(AdamwTable<COPY> t, AdamwArgs a) {
#pragma clang fp contract(off)
  int lo = 0, hi = a.count;                          // the tensor whose workgroups this one is among
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (t.chunk[mid] <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const int64_t at = (int64_t)(blockIdx.x - t.chunk[lo]) * ADAMW_CHUNK + threadIdx.x * 8;
  const int64_t e0 = (int64_t)t.first[lo] * LORACT_ADAMW_BLOCK + at, left = t.n[lo] - at;
  if ((at & ~(int64_t)255) >= t.n[lo]) return;       // (a whole block of 256: the lanes of the others stay together)
  if (a.lr_dev || a.step_dev) {
    const double lr = a.lr_dev ? (double)*a.lr_dev : a.lr;
    if (a.step_dev) a.step = *a.step_dev;
    adamw_rates(a, lr, exp2((double)a.step * a.log2_beta1), exp2((double)a.step * a.log2_beta2));
  }
  P* const pp = (P*)t.p[lo] + at;
  float p[8], g[8], m[8], v[8], r[8];
  adamw_load<P>(pp, left, p);
  adamw_load<G>((const G*)t.g[lo] + at, left, g);
  if constexpr (NARROW) {
    const uint8_t* const exps = a.exps + (e0 >> 8) * 2;
    const adamw_codes cm = *(const adamw_codes*)((const uint8_t*)a.m + e0), cv = *(const adamw_codes*)((const uint8_t*)a.v + e0);
    adamw_decode(cm, __uint_as_float((unsigned)exps[0] << 23), m);
    adamw_decode(cv, __uint_as_float((unsigned)exps[1] << 23), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * v[e];
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 x = *(const f32x4*)((const float*)a.m + e0 + 4 * h), y = *(const f32x4*)((const float*)a.v + e0 + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) { m[4 * h + e] = x[e]; v[4 * h + e] = y[e]; }
    }
  }
  if (a.grad_scale_dev) {
    const float scale = *a.grad_scale_dev;
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = g[e] * scale;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    m[e] = m[e] * a.beta1 + g[e] * a.one_beta1;
    v[e] = v[e] * a.beta2 + (g[e] * g[e]) * a.one_beta2;
    r[e] = sqrtf(v[e]);
    p[e] = p[e] * a.decay - m[e] * __builtin_amdgcn_rcpf(r[e] * a.inv + a.eps) * a.rate;
  }
  unsigned bits[8];
  if (NARROW || sizeof(P) == 2) {
    uint64_t at_word = splitmix64_mix(a.seed + (uint64_t)a.step * SPLITMIX_GOLDEN) + (uint64_t)(e0 >> 1) * SPLITMIX_GOLDEN;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint64_t word = splitmix64_mix(at_word += SPLITMIX_GOLDEN);
      bits[2 * w] = (unsigned)word;
      bits[2 * w + 1] = (unsigned)(word >> 32);
    }
  }
  if constexpr (NARROW) {
    const unsigned bm = adamw_exponent(m), br = adamw_exponent(r);
    const float sm = __uint_as_float((254u - bm) << 23), sr = __uint_as_float((254u - br) << 23);
    adamw_codes cm = {0, 0}, cr = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const unsigned* const b = bits + 4 * h;
      cm[h] = adamw_code<0>(m[4 * h], sm, b[0], false, cm[h]);
      cm[h] = adamw_code<1>(m[4 * h + 1], sm, b[1], false, cm[h]);
      cm[h] = adamw_code<2>(m[4 * h + 2], sm, b[2], false, cm[h]);
      cm[h] = adamw_code<3>(m[4 * h + 3], sm, b[3], false, cm[h]);
      cr[h] = adamw_code<0>(r[4 * h], sr, b[0] >> 10, true, cr[h]);
      cr[h] = adamw_code<1>(r[4 * h + 1], sr, b[1] >> 10, true, cr[h]);
      cr[h] = adamw_code<2>(r[4 * h + 2], sr, b[2] >> 10, true, cr[h]);
      cr[h] = adamw_code<3>(r[4 * h + 3], sr, b[3] >> 10, true, cr[h]);
    }
    *(adamw_codes*)((uint8_t*)a.m + e0) = cm;
    *(adamw_codes*)((uint8_t*)a.v + e0) = cr;
    if ((threadIdx.x & 31) == 0) *(uint16_t*)(a.exps + (e0 >> 8) * 2) = (uint16_t)(bm | br << 8);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      *(f32x4*)((float*)a.m + e0 + 4 * h) = (f32x4){m[4 * h], m[4 * h + 1], m[4 * h + 2], m[4 * h + 3]};
      *(f32x4*)((float*)a.v + e0 + 4 * h) = (f32x4){v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
    }
  }
  P out[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (sizeof(P) == 2) out[e] = adamw_bf16(p[e], bits[e] >> 20);
    else out[e] = p[e];
  }
  adamw_store<P>(pp, left, out);
  if (COPY && t.copy[lo]) {
    bf16_t c[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) c[e] = (bf16_t)p[e];
    adamw_store<bf16_t>(t.copy[lo] + at, left, c);
  }
}

// Launches as many tables as the tensors need.
template <typename P, typename G, bool COPY>
static int launch_adamw(hipStream_t s, AdamwArgs& a, bool narrow, void* const* p, const void* const* g, void* const* copy, const int64_t* n, int64_t count) {
  AdamwTable<COPY> t;
  a.count = 0;
  t.chunk[0] = 0;
  int64_t first = 0;
  for (int64_t i = 0; i <= count; ++i) {
    const int64_t chunks = i < count ? ceil_div64(n[i], ADAMW_CHUNK) : 0;
    // (fewer than 2^32 threads to a launch)
    if (a.count && (i == count || a.count == t.MOST || t.chunk[a.count] + chunks >= (1 << 24))) {
      const dim3 grid(t.chunk[a.count]), block(256);
      if (narrow) LORACT_LAUNCH("adamw", s, (adamw_kernel<P, G, true, COPY>), grid, block, 0, t, a);
      else LORACT_LAUNCH("adamw", s, (adamw_kernel<P, G, false, COPY>), grid, block, 0, t, a);
      a.count = 0;
    }
    if (!chunks) continue;
    t.p[a.count] = p[i];
    t.g[a.count] = g[i];
    if (COPY) t.copy[a.count] = (bf16_t*)copy[i];
    t.n[a.count] = n[i];
    t.first[a.count] = (uint32_t)(first / LORACT_ADAMW_BLOCK);
    t.chunk[a.count + 1] = t.chunk[a.count] + (uint32_t)chunks;
    ++a.count;
    first += (int64_t)align_up((size_t)n[i], LORACT_ADAMW_BLOCK);
  }
  return LORACT_OK;
}

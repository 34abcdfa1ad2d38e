// P = X W^T + s T B for bf16 maps with few tokens (a step of serving) or few outputs (T = X A): one large operand is read
// once, and everything else is small.
//
// Bound by reading the large operand.  It goes from memory straight into the registers that v_mfma_f32_16x16x32_bf16 takes: a lane
// holds eight consecutive k of one row.  The eight waves of a workgroup share its rows and split K, so that 16 rows are
// enough to keep a CU's share of the memory system busy; their sums are added in LDS in a fixed order, then comes the epilogue.
// One token through 4096 -> 11008 22 us (4.1 TB/s; a copy 5.1), 8192 x 4096 -> 16 17 us (3.9), 65536 x 4096 -> 16 105 us (5.1): what a
// short pass loses is its start.  A second trip's loads ahead of the products gave fewer waves and 31 us instead of 24.
// Accumulators start with the low-rank term (waves 0 and 1, 32 of its rank each), scaled in float32.
#pragma once
#include "linear_large.h"

#define LN_WAVES 8

// Rows along K may start at any multiple of 4 bytes.
// Eight consecutive k of a row along K, zero past the end of K (k_len >= 8).
__device__ inline bf16x8 ln_load(const bf16_t* row, int64_t k, int64_t k_len) {
  return __builtin_bit_cast(bf16x8, gb_shift(gb_load(row, k < k_len ? k : k_len, k_len), k < k_len ? k : k_len, k_len));
}
// Fragment of T (row `row`) or of B (column `col`), 32 of the rank from r0 on.
__device__ inline bf16x8 ln_rank_x(const LinearArgs& g, int64_t row, int r0) {
  bf16x8 v = {};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (r0 + e < g.r) v[e] = ((const bf16_t*)g.T)[row * g.r + r0 + e];
  return v;
}
__device__ inline bf16x8 ln_rank_w(const LinearArgs& g, int64_t col, int r0) {
  bf16x8 v = {};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (r0 + e < g.r) v[e] = ((const bf16_t*)g.B)[(r0 + e) * g.n + col];
  return v;
}

// Adds the waves' sums (part[wave][quads], four consecutive columns each) and finishes them; row and first column by place(quad).
template <typename Place>
__device__ inline void ln_finish(const LinearArgs& g, const f32x4* part, int quads, Place place) {
  for (int i = threadIdx.x; i < quads; i += 64 * LN_WAVES) {
    int64_t row, col;
    place(i, &row, &col);
    f32x4 s = part[i];
#pragma unroll
    for (int w = 1; w < LN_WAVES; ++w) s += part[w * quads + i];
    if (gridDim.y == 1) lin_store4<bf16_t>(g.e, row, col, s, lin_load4<bf16_t>(g.e, row, col));
    else if (row < g.m && col < g.n_pad) *(f32x4*)(g.part + ((int64_t)blockIdx.y * g.m + row) * g.n_pad + col) = s;
  }
}

// OF_W: the rows that are streamed are those of W (n_out x n_in), X is small (16 SMALL rows at most); else they are those of X, and W has
// 16 SMALL columns at most, stored either way (W_KC).  BLOCKS: 16 streamed rows per wave each.
template <bool OF_W, bool W_KC, int BLOCKS, int SMALL>
__global__ __launch_bounds__(64 * LN_WAVES) void linear_thin_kernel(LinearArgs g) {
  constexpr int U = SMALL == 1 ? 4 : 2;                  // steps of 32 of K in flight
  constexpr bool TURN = !OF_W && !W_KC;                  // the small operand passes through LDS to be transposed
  constexpr int QUADS = BLOCKS * SMALL * 64;
  constexpr int TURN_BYTES = TURN ? LN_WAVES * U * SMALL * 1024 : 0, PART_BYTES = LN_WAVES * QUADS * 16;
  __shared__ __attribute__((aligned(16))) unsigned char smem[TURN_BYTES > PART_BYTES ? TURN_BYTES : PART_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t first = (int64_t)blockIdx.x * (16 * BLOCKS);
  const int64_t rows = OF_W ? g.n : g.m, others = OF_W ? g.m : g.n;
  const bf16_t *stream[BLOCKS], *small[SMALL];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int64_t row = first + 16 * b + c < rows ? first + 16 * b + c : rows - 1;      // rows past the end are never stored
    stream[b] = OF_W ? (const bf16_t*)g.W + row * g.ldw : (const bf16_t*)g.X + row * g.ldx;
  }
#pragma unroll
  for (int b = 0; b < SMALL; ++b) {
    const int64_t row = 16 * b + c < others ? 16 * b + c : others - 1;
    if (TURN) small[b] = (const bf16_t*)g.W + (16 * b + 8 * (lane & 1) < g.n ? 16 * b + 8 * (lane & 1) : 0);   // (n is a multiple of 8)
    else small[b] = OF_W ? (const bf16_t*)g.X + row * g.ldx : (const bf16_t*)g.W + row * g.ldw;
  }
  f32x4 acc[BLOCKS][SMALL];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int s = 0; s < SMALL; ++s) acc[b][s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  // the weights' fragment comes first: a lane holds four consecutive columns of one row of Y
  auto mfma = [&](bf16x8 st, bf16x8 sm, f32x4 a) {
    return OF_W ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(st, sm, a, 0, 0, 0) : __builtin_amdgcn_mfma_f32_16x16x32_bf16(sm, st, a, 0, 0, 0);
  };
  if (g.T && blockIdx.y == 0 && 32 * wave < g.r) {
    const int r0 = 32 * wave + 8 * q;
    bf16x8 sm[SMALL];
#pragma unroll
    for (int s = 0; s < SMALL; ++s) {
      const int64_t row = 16 * s + c < others ? 16 * s + c : others - 1;
      sm[s] = OF_W ? ln_rank_x(g, row, r0) : ln_rank_w(g, row, r0);
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const int64_t row = first + 16 * b + c < rows ? first + 16 * b + c : rows - 1;
      const bf16x8 st = OF_W ? ln_rank_w(g, row, r0) : ln_rank_x(g, row, r0);
#pragma unroll
      for (int s = 0; s < SMALL; ++s) acc[b][s] = mfma(st, sm[s], acc[b][s]) * g.lora_scale;
    }
  }
  const int64_t k_beg0 = (int64_t)blockIdx.y * g.k_per_split, k_end0 = k_beg0 + g.k_per_split < g.k ? k_beg0 + g.k_per_split : g.k;
  const int64_t per = ((k_end0 - k_beg0 + 32 * LN_WAVES - 1) / (32 * LN_WAVES)) * 32;
  const int64_t k_beg = k_beg0 + wave * per, k_end = k_beg + per < k_end0 ? k_beg + per : k_end0;
  unsigned char* const turn = smem + wave * (U * SMALL * 1024);
  for (int64_t k0 = k_beg; k0 < k_end; k0 += 32 * U) {
    bf16x8 st[U][BLOCKS], sm[U][SMALL];
    if (k0 + 32 * U <= k_end) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + 32 * u;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) st[u][b] = *(const bf16x8_any*)(stream[b] + k + 8 * q);
#pragma unroll
        for (int s = 0; s < SMALL; ++s)
          sm[u][s] = TURN ? *(const bf16x8*)(small[s] + (k + (lane >> 1)) * g.ldw) : *(const bf16x8_any*)(small[s] + k + 8 * q);
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + 32 * u;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) st[u][b] = ln_load(stream[b], k + 8 * q, k_end);
#pragma unroll
        for (int s = 0; s < SMALL; ++s) {
          if (TURN) {
            const int64_t kr = k + (lane >> 1);
            sm[u][s] = *(const bf16x8*)(small[s] + (kr < k_end ? kr : k_end - 1) * g.ldw);
            if (kr >= k_end) sm[u][s] = (bf16x8){};
          } else {
            sm[u][s] = ln_load(small[s], k + 8 * q, k_end);
          }
        }
      }
    }
    if (TURN) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SMALL; ++s) *(bf16x8*)(turn + (u * SMALL + s) * 1024 + lane * 16) = sm[u][s];
      sb_wave_sync();
      const int s16 = lane & 15, off = (8 * q + (s16 >> 2)) * 32 + (s16 & 3) * 8;
      typedef __attribute__((address_space(3))) gb_s16x4* lds_ptr;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SMALL; ++s) {
          const unsigned char* at = turn + (u * SMALL + s) * 1024 + off;
          const gb_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
          const gb_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * 32));
          sm[u][s] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
      sb_wave_sync();
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
        for (int s = 0; s < SMALL; ++s) acc[b][s] = mfma(st[u][b], sm[u][s], acc[b][s]);
  }
  if (TURN) __syncthreads();
  f32x4* const part = (f32x4*)smem;
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int s = 0; s < SMALL; ++s) part[wave * QUADS + (b * SMALL + s) * 64 + lane] = acc[b][s];
  __syncthreads();
  ln_finish(g, part, QUADS, [&](int i, int64_t* row, int64_t* col) {
    const int b = i / (64 * SMALL), s = i / 64 % SMALL, l = i & 63;      // register u of lane l: column 4 (l / 16) + u, row l % 16
    *row = (OF_W ? 16 * s : first + 16 * b) + (l & 15);
    *col = (OF_W ? first + 16 * b : 16 * s) + 4 * (l >> 4);
  });
}

// Few tokens with W stored n_in x n_out.  A lane reads an 8 x 8 block of W (eight k, eight columns, 16 lanes cover 256 bytes of a row)
// and pairs its rows with byte permutations: the j-th product takes column 8 (l % 16) + j from every lane.
template <int SMALL>
__global__ __launch_bounds__(64 * LN_WAVES) void linear_thin_t_kernel(LinearArgs g) {
  constexpr int QUADS = SMALL * 8 * 64;
  __shared__ __attribute__((aligned(16))) unsigned char smem[LN_WAVES / 2 * QUADS * 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t first = (int64_t)blockIdx.x * 128, col0 = first + 8 * c < g.n ? first + 8 * c : g.n - 8;   // (n is a multiple of 8)
  const bf16_t* small[SMALL];
#pragma unroll
  for (int s = 0; s < SMALL; ++s) small[s] = (const bf16_t*)g.X + (16 * s + c < g.m ? 16 * s + c : g.m - 1) * g.ldx;
  f32x4 acc[8][SMALL];
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int s = 0; s < SMALL; ++s) acc[j][s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  if (g.T && blockIdx.y == 0 && 32 * wave < g.r) {
    const int r0 = 32 * wave + 8 * q;
#pragma unroll
    for (int s = 0; s < SMALL; ++s) {
      const bf16x8 sm = ln_rank_x(g, 16 * s + c < g.m ? 16 * s + c : g.m - 1, r0);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        acc[j][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ln_rank_w(g, col0 + j, r0), sm, acc[j][s], 0, 0, 0) * g.lora_scale;
    }
  }
  const int64_t k_beg0 = (int64_t)blockIdx.y * g.k_per_split, k_end0 = k_beg0 + g.k_per_split < g.k ? k_beg0 + g.k_per_split : g.k;
  const int64_t per = ((k_end0 - k_beg0 + 32 * LN_WAVES - 1) / (32 * LN_WAVES)) * 32;
  const int64_t k_beg = k_beg0 + wave * per, k_end = k_beg + per < k_end0 ? k_beg + per : k_end0;
  typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
  auto step = [&](const u32x4_t (&v)[8], const bf16x8 (&sm)[SMALL]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      u32x4_t f;
#pragma unroll
      for (int p = 0; p < 4; ++p)        // rows 2 p and 2 p + 1: their low or high halves of dword j / 2
        f[p] = __builtin_amdgcn_perm(v[2 * p + 1][j / 2], v[2 * p][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int s = 0; s < SMALL; ++s)
        acc[j][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), sm[s], acc[j][s], 0, 0, 0);
    }
  };
  auto load = [&](int64_t k0, u32x4_t (&v)[8], bf16x8 (&sm)[SMALL]) {
    const bool whole = k0 + 32 <= k_end;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t k = k0 + 8 * q + i;
      v[i] = *(const u32x4_t*)((const bf16_t*)g.W + (whole || k < k_end ? k : k_end - 1) * g.ldw + col0);
      if (!whole && k >= k_end) v[i] = (u32x4_t){0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int s = 0; s < SMALL; ++s) sm[s] = ln_load(small[s], k0 + 8 * q, k_end);
  };
  for (int64_t k0 = k_beg; k0 < k_end; k0 += 64) {
    u32x4_t v0[8], v1[8];
    bf16x8 s0[SMALL], s1[SMALL];
    load(k0, v0, s0);
    if (k0 + 32 < k_end) load(k0 + 32, v1, s1);
    step(v0, s0);
    if (k0 + 32 < k_end) step(v1, s1);
  }
  // the waves' sums: the upper four add theirs to the lower four's, these are added as above
  f32x4* const part = (f32x4*)smem;
#pragma unroll
  for (int h = 1; h >= 0; --h) {
    if (wave / (LN_WAVES / 2) == h)
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int s = 0; s < SMALL; ++s) {
          f32x4* at = part + wave % (LN_WAVES / 2) * QUADS + (j * SMALL + s) * 64 + lane;
          *at = h ? acc[j][s] : *at + acc[j][s];
        }
    __syncthreads();
  }
  // register u of lane l in product j: row l % 16, column 8 (4 (l / 16) + u) + j; four consecutive columns are four products'
  for (int i = threadIdx.x; i < QUADS; i += 64 * LN_WAVES) {
    const int half = i & 1, at16 = i / 2 % 16, m16 = i / 32 % 16, s = i / 512;
    const int l = 16 * (at16 >> 2) + m16, u = at16 & 3;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < LN_WAVES / 2; ++w)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += ((const float*)(part + w * QUADS + ((4 * half + j) * SMALL + s) * 64 + l))[u];
    const int64_t row = 16 * s + m16, col = first + 8 * at16 + 4 * half;
    if (gridDim.y == 1) lin_store4<bf16_t>(g.e, row, col, v, lin_load4<bf16_t>(g.e, row, col));
    else if (row < g.m && col < g.n_pad) *(f32x4*)(g.part + ((int64_t)blockIdx.y * g.m + row) * g.n_pad + col) = v;
  }
}

// Which of the forms: 0 none, 1 rows of W are streamed, 2 rows of X, 3 W as it lies.  Rows along K at multiples of 4 bytes, W as it
// lies in whole pieces: at 2 bytes the general tiles are faster (one token through 4095 -> 11007 44 us against 31, 8192 x 4095 -> 16 31
// against 21), at 8 they are not (one token through 4092 -> 11008 20 against 27); W as it lies at 8 bytes 53 against 32.
static int linear_thin_form(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw, bool w_kc) {
  if (k < 8 || m > (1 << 27) || n > (1 << 27)) return 0;    // (2^32 threads to a grid)
  if (ldx % 2 || (w_kc ? ldw % 2 : (ldw % 8 || n % 8))) return 0;
  if (m <= 32) return w_kc ? 1 : 3;
  // (33 to 64 outputs of many tokens: the tiles read W's columns once per 128 tokens; 8192 x 11008 -> 64 49 us against 67,
  // 2048 x 4096 -> 64 17 against 14)
  return n <= 32 || (n <= 64 && m <= 4096) ? 2 : 0;
}
static bool linear_thin_fits(const LinearArgs& g, bool w_kc) { return (uintptr_t)g.X % 4 == 0 && (uintptr_t)g.W % (w_kc ? 4 : 16) == 0; }
// Blocks of 16 streamed rows per wave: two where 32 rows still give every CU a workgroup, and for two blocks of tokens, whose X
// would otherwise be read by twice as many workgroups (32 tokens through 4096 -> 11008: 36 us with one block of W's rows, 34 with two).
static int linear_thin_blocks(int64_t m, int form) { return form == 1 ? (m > 16 ? 2 : 1) : (ceil_div64(m, 32) >= 256 ? 2 : 1); }
// K splits between workgroups: as many as make 256 of them, of at least 1024 of K (128 per wave).  More cost the launch that joins
// them (8192 x 4096 -> 16: 19 us with one split, 23 with two; one token through 11008 -> 4096: 20 and 23), but W as it lies, read by
// a third as many workgroups, takes four at up to 16 tokens (4096 -> 11008: 27 us with four splits, 31 with two; 32 tokens 35 and 29).
static int linear_thin_splits(int64_t m, int64_t n, int64_t k, int form) {
  const int64_t rows = 16 * linear_thin_blocks(m, form);
  const int64_t wgs = form == 1 ? ceil_div64(n, rows) : (form == 2 ? ceil_div64(m, rows) : ceil_div64(n, 128));
  const int64_t want = std::max<int64_t>(256 / wgs, form == 3 && m <= 16 ? 4 : 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, k / 1024), 64));
}
static size_t linear_thin_part_bytes(int64_t m, int64_t n, int64_t k, int form) {
  const int s = linear_thin_splits(m, n, k, form);
  return s > 1 ? align_up((size_t)s * m * align_up((size_t)n, 4) * 4, 256) : 0;
}

static int launch_linear_thin(hipStream_t s, LinearArgs g, bool w_kc, int form) {
  int splits = linear_thin_splits(g.m, g.n, g.k, form);
  g.k_per_split = ceil_div64(ceil_div64(g.k, splits), 256) * 256;
  splits = (int)ceil_div64(g.k, g.k_per_split);
  g.n_pad = (int64_t)align_up((size_t)g.n, 4);
  const dim3 block(64 * LN_WAVES);
#define LN_LAUNCH(...) LORACT_LAUNCH("linear_thin", s, (linear_thin_kernel<__VA_ARGS__>), grid, block, 0, g)
  if (form == 1) {
    const dim3 grid((unsigned)ceil_div64(g.n, 16 * linear_thin_blocks(g.m, form)), (unsigned)splits);
    if (g.m <= 16) LN_LAUNCH(true, true, 1, 1);
    else LN_LAUNCH(true, true, 2, 2);
  } else if (form == 2) {
    const int blocks = linear_thin_blocks(g.m, form);
    const dim3 grid((unsigned)ceil_div64(g.m, 16 * blocks), (unsigned)splits);
#define LN_SMALL(KC, B)                                                                 \
    {                                                                                   \
      if (g.n <= 16) LN_LAUNCH(false, KC, B, 1);                                         \
      else if (g.n <= 32) LN_LAUNCH(false, KC, B, 2);                                    \
      else LN_LAUNCH(false, KC, B, 4);                                                   \
    }
    if (w_kc) { if (blocks == 2) LN_SMALL(true, 2) else LN_SMALL(true, 1) }
    else { if (blocks == 2) LN_SMALL(false, 2) else LN_SMALL(false, 1) }
#undef LN_SMALL
  } else {
    const dim3 grid((unsigned)ceil_div64(g.n, 128), (unsigned)splits);
    if (g.m <= 16) LORACT_LAUNCH("linear_thin", s, linear_thin_t_kernel<1>, grid, block, 0, g);
    else LORACT_LAUNCH("linear_thin", s, linear_thin_t_kernel<2>, grid, block, 0, g);
  }
#undef LN_LAUNCH
  return splits > 1 ? launch_linear_join<bf16_t>(s, g, splits) : LORACT_OK;
}

// P = X W^T + s T B for maps with few tokens (a step of serving) or few outputs (T = X A): one large operand is read
// once, and everything else is small.
//
// Bound by reading the large operand.  It goes from memory straight into the registers that v_mfma_f32_16x16x32_bf16 takes: a lane
// holds eight consecutive k of one row (float32: four, one for each of four v_mfma_f32_16x16x4_f32).  The eight waves of a workgroup
// share its rows and split K, so that 16 rows are enough to keep a CU's share of the memory system busy; their sums are added in LDS
// in a fixed order, then comes the epilogue.
// One token through 4096 -> 11008 17.6 us (5.1 TB/s; a copy 5.1), with bias, 16 columns of B and SiLU 22, 8192 x 4096 -> 16 16 us (4.2), 65536 x
// 4096 -> 16 100 us (5.4): what a short pass loses is its start, and with 17 to 32 tokens half of a wave's loads are X (32 us).  A second trip's loads ahead of the products gave fewer waves and 31 us instead of 24.
// float32 (the general tiles before): one token through 4096 -> 11008 33 us (64; 5.4 TB/s), 8192 x 4096 -> 16 29 us (61), 8 tokens
// through 11008 -> 11008 112 (168); with 17 to 32 rows on both sides its products weigh as much as its reads: 32 tokens through
// 8192 -> 8192 74 (99), 12096 x 9920 -> 30 142 (161; 170 with twice the steps in flight, at half the waves).
// Accumulators start with the low-rank term (the first waves, one step of its rank each), scaled in float32.
#pragma once
#include "linear_large.h"

#define LN_WAVES 8

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
// A lane's k of a row, zero past the end of K (of at least 8).  Rows along K may start at any multiple of 4 bytes.
template <typename T>
__device__ inline typename Ln<T>::frag ln_load(const T* row, int64_t k, int64_t k_len) {
  constexpr int E = Ln<T>::E;
  typedef typename Ln<T>::frag frag;
  const frag v = *(const typename Ln<T>::frag_any*)(row + (k + E <= k_len ? k : k_len - E));
  const int64_t over = k + E - k_len;
  if (over <= 0) return v;
  if (over >= E) return (frag){};
  return __builtin_bit_cast(frag, __builtin_bit_cast(unsigned __int128, v) >> (8 * (int)sizeof(T) * (int)over));
}
// Fragment of T (row `row`) or of B (column `col`), one step of the rank from r0 on.
template <typename T>
__device__ inline typename Ln<T>::frag ln_rank_x(const LinearArgs& g, int64_t row, int r0) {
  typename Ln<T>::frag v = {};
#pragma unroll
  for (int e = 0; e < Ln<T>::E; ++e)
    if (r0 + e < g.r) v[e] = ((const T*)g.T)[row * g.r + r0 + e];
  return v;
}
template <typename T>
__device__ inline typename Ln<T>::frag ln_rank_w(const LinearArgs& g, int64_t col, int r0) {
  typename Ln<T>::frag v = {};
#pragma unroll
  for (int e = 0; e < Ln<T>::E; ++e)
    if (r0 + e < g.r) v[e] = ((const T*)g.B)[(r0 + e) * g.n + col];
  return v;
}

// Adds the waves' sums (part[wave][quads], four consecutive columns each) and finishes them; row and first column by place(quad).
template <typename T, typename Place>
__device__ inline void ln_finish(const LinearArgs& g, const f32x4* part, int quads, Place place) {
  for (int i = threadIdx.x; i < quads; i += 64 * LN_WAVES) {
    int64_t row, col;
    place(i, &row, &col);
    f32x4 s = part[i];
#pragma unroll
    for (int w = 1; w < LN_WAVES; ++w) s += part[w * quads + i];
    if (gridDim.y == 1) lin_store4<T>(g.e, row, col, s, lin_load4<T>(g.e, row, col));
    else if (row < g.m && col < g.n_pad) *(f32x4*)(g.part + ((int64_t)blockIdx.y * g.m + row) * g.n_pad + col) = s;
  }
}

// OF_W: the rows that are streamed are those of W (n_out x n_in), X is small (16 SMALL rows at most); else they are those of X, and W has
// 16 SMALL columns at most, stored either way (W_KC).  BLOCKS: 16 streamed rows per wave each.
template <typename T, bool OF_W, bool W_KC, int BLOCKS, int SMALL>
__global__ __launch_bounds__(64 * LN_WAVES) void linear_thin_kernel(LinearArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP;
  typedef typename Ln<T>::frag frag;
  typedef typename Ln<T>::frag_any frag_any;
  constexpr int U = SMALL == 1 ? 4 : 2;                  // steps in flight
  constexpr bool TURN = !OF_W && !W_KC;                  // the small operand passes through LDS to be transposed
  constexpr int QUADS = BLOCKS * SMALL * 64;
  constexpr int TURN_BYTES = TURN ? LN_WAVES * U * SMALL * 1024 : 0, PART_BYTES = LN_WAVES * QUADS * 16;
  __shared__ __attribute__((aligned(16))) unsigned char smem[TURN_BYTES > PART_BYTES ? TURN_BYTES : PART_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t first = (int64_t)blockIdx.x * (16 * BLOCKS);
  const int64_t rows = OF_W ? g.n : g.m, others = OF_W ? g.m : g.n;
  const T *stream[BLOCKS], *small[SMALL];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b) {
    const int64_t row = first + 16 * b + c < rows ? first + 16 * b + c : rows - 1;      // rows past the end are never stored
    stream[b] = OF_W ? (const T*)g.W + row * g.ldw : (const T*)g.X + row * g.ldx;
  }
#pragma unroll
  for (int b = 0; b < SMALL; ++b) {
    const int64_t row = 16 * b + c < others ? 16 * b + c : others - 1;
    const int turn_col = 16 * b + E * (lane % (16 / E));             // (n is a multiple of E then)
    if (TURN) small[b] = (const T*)g.W + (turn_col < g.n ? turn_col : 0);
    else small[b] = OF_W ? (const T*)g.X + row * g.ldx : (const T*)g.W + row * g.ldw;
  }
  f32x4 acc[BLOCKS][SMALL];
#pragma unroll
  for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
    for (int s = 0; s < SMALL; ++s) acc[b][s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  // the weights' fragment comes first: a lane holds four consecutive columns of one row of Y
  auto mfma = [&](frag st, frag sm, f32x4 a) { return OF_W ? ln_mfma(st, sm, a) : ln_mfma(sm, st, a); };
  if (g.T && blockIdx.y == 0 && STEP * wave < g.r) {
    const int r0 = STEP * wave + E * q;
    frag sm[SMALL];
#pragma unroll
    for (int s = 0; s < SMALL; ++s) {
      const int64_t row = 16 * s + c < others ? 16 * s + c : others - 1;
      sm[s] = OF_W ? ln_rank_x<T>(g, row, r0) : ln_rank_w<T>(g, row, r0);
    }
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
      const int64_t row = first + 16 * b + c < rows ? first + 16 * b + c : rows - 1;
      const frag st = OF_W ? ln_rank_w<T>(g, row, r0) : ln_rank_x<T>(g, row, r0);
#pragma unroll
      for (int s = 0; s < SMALL; ++s) acc[b][s] = mfma(st, sm[s], acc[b][s]) * g.lora_scale;
    }
  }
  const int64_t k_beg0 = (int64_t)blockIdx.y * g.k_per_split, k_end0 = k_beg0 + g.k_per_split < g.k ? k_beg0 + g.k_per_split : g.k;
  const int64_t per = ((k_end0 - k_beg0 + STEP * LN_WAVES - 1) / (STEP * LN_WAVES)) * STEP;
  const int64_t k_beg = k_beg0 + wave * per, k_end = k_beg + per < k_end0 ? k_beg + per : k_end0;
  unsigned char* const turn = smem + wave * (U * SMALL * 1024);
  for (int64_t k0 = k_beg; k0 < k_end; k0 += STEP * U) {
    frag st[U][BLOCKS], sm[U][SMALL];
    if (k0 + STEP * U <= k_end) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + STEP * u;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) st[u][b] = *(const frag_any*)(stream[b] + k + E * q);
#pragma unroll
        for (int s = 0; s < SMALL; ++s)
          sm[u][s] = TURN ? *(const frag*)(small[s] + (k + lane / (16 / E)) * g.ldw) : *(const frag_any*)(small[s] + k + E * q);
      }
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + STEP * u;
#pragma unroll
        for (int b = 0; b < BLOCKS; ++b) st[u][b] = ln_load<T>(stream[b], k + E * q, k_end);
#pragma unroll
        for (int s = 0; s < SMALL; ++s) {
          if (TURN) {
            const int64_t kr = k + lane / (16 / E);
            sm[u][s] = *(const frag*)(small[s] + (kr < k_end ? kr : k_end - 1) * g.ldw);
            if (kr >= k_end) sm[u][s] = (frag){};
          } else {
            sm[u][s] = ln_load<T>(small[s], k + E * q, k_end);
          }
        }
      }
    }
    if (TURN) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SMALL; ++s) *(frag*)(turn + (u * SMALL + s) * 1024 + lane * 16) = sm[u][s];
      sb_wave_sync();
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SMALL; ++s) {
          const unsigned char* at = turn + (u * SMALL + s) * 1024;
          if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) gb_s16x4* lds_ptr;
            at += (8 * q + (c >> 2)) * 32 + (c & 3) * 8;
            const gb_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
            const gb_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * 32));
            sm[u][s] = __builtin_bit_cast(frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) sm[u][s][e] = *(const T*)(at + (E * q + e) * 64 + c * 4);
          }
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
  ln_finish<T>(g, part, QUADS, [&](int i, int64_t* row, int64_t* col) {
    const int b = i / (64 * SMALL), s = i / 64 % SMALL, l = i & 63;      // register u of lane l: column 4 (l / 16) + u, row l % 16
    *row = (OF_W ? 16 * s : first + 16 * b) + (l & 15);
    *col = (OF_W ? first + 16 * b : 16 * s) + 4 * (l >> 4);
  });
}

// Few tokens with W stored n_in x n_out.  A lane reads an E x E block of W (E k, E columns: 8 or, of float32, 4; 16 lanes cover 256
// bytes of a row): the j-th product takes column E (l % 16) + j from every lane, whose k are the block's rows (bf16 rows are paired by
// byte permutations for it).  float32 through 4096 -> 11008: one token 42 us (70 with the general tiles), 32 tokens 60 (73).
template <typename T, int SMALL>
__global__ __launch_bounds__(64 * LN_WAVES) void linear_thin_t_kernel(LinearArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP, QUADS = SMALL * E * 64;
  typedef typename Ln<T>::frag frag;
  __shared__ __attribute__((aligned(16))) unsigned char smem[LN_WAVES / 2 * QUADS * 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t first = (int64_t)blockIdx.x * (16 * E), col0 = first + E * c < g.n ? first + E * c : g.n - E;   // (n is a multiple of E)
  const T* small[SMALL];
#pragma unroll
  for (int s = 0; s < SMALL; ++s) small[s] = (const T*)g.X + (16 * s + c < g.m ? 16 * s + c : g.m - 1) * g.ldx;
  f32x4 acc[E][SMALL];
#pragma unroll
  for (int j = 0; j < E; ++j)
#pragma unroll
    for (int s = 0; s < SMALL; ++s) acc[j][s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  if (g.T && blockIdx.y == 0 && STEP * wave < g.r) {
    const int r0 = STEP * wave + E * q;
#pragma unroll
    for (int s = 0; s < SMALL; ++s) {
      const frag sm = ln_rank_x<T>(g, 16 * s + c < g.m ? 16 * s + c : g.m - 1, r0);
#pragma unroll
      for (int j = 0; j < E; ++j) acc[j][s] = ln_mfma(ln_rank_w<T>(g, col0 + j, r0), sm, acc[j][s]) * g.lora_scale;
    }
  }
  const int64_t k_beg0 = (int64_t)blockIdx.y * g.k_per_split, k_end0 = k_beg0 + g.k_per_split < g.k ? k_beg0 + g.k_per_split : g.k;
  const int64_t per = ((k_end0 - k_beg0 + STEP * LN_WAVES - 1) / (STEP * LN_WAVES)) * STEP;
  const int64_t k_beg = k_beg0 + wave * per, k_end = k_beg + per < k_end0 ? k_beg + per : k_end0;
  auto step = [&](const frag (&v)[E], const frag (&sm)[SMALL]) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      frag f;
      if constexpr (sizeof(T) == 2) {
        typedef unsigned int words __attribute__((ext_vector_type(4)));
        words w;
#pragma unroll
        for (int p = 0; p < 4; ++p)        // rows 2 p and 2 p + 1: their low or high halves of dword j / 2
          w[p] = __builtin_amdgcn_perm(__builtin_bit_cast(words, v[2 * p + 1])[j / 2], __builtin_bit_cast(words, v[2 * p])[j / 2],
                                       j & 1 ? 0x07060302u : 0x05040100u);
        f = __builtin_bit_cast(frag, w);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = v[e][j];
      }
#pragma unroll
      for (int s = 0; s < SMALL; ++s) acc[j][s] = ln_mfma(f, sm[s], acc[j][s]);
    }
  };
  auto load = [&](int64_t k0, frag (&v)[E], frag (&sm)[SMALL]) {
    const bool whole = k0 + STEP <= k_end;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int64_t k = k0 + E * q + i;
      v[i] = *(const frag*)((const T*)g.W + (whole || k < k_end ? k : k_end - 1) * g.ldw + col0);
      if (!whole && k >= k_end) v[i] = (frag){};
    }
#pragma unroll
    for (int s = 0; s < SMALL; ++s) sm[s] = ln_load<T>(small[s], k0 + E * q, k_end);
  };
  for (int64_t k0 = k_beg; k0 < k_end; k0 += 2 * STEP) {
    frag v0[E], v1[E], s0[SMALL], s1[SMALL];
    load(k0, v0, s0);
    if (k0 + STEP < k_end) load(k0 + STEP, v1, s1);
    step(v0, s0);
    if (k0 + STEP < k_end) step(v1, s1);
  }
  // the waves' sums: the upper four add theirs to the lower four's, these are added as above
  f32x4* const part = (f32x4*)smem;
#pragma unroll
  for (int h = 1; h >= 0; --h) {
    if (wave / (LN_WAVES / 2) == h)
#pragma unroll
      for (int j = 0; j < E; ++j)
#pragma unroll
        for (int s = 0; s < SMALL; ++s) {
          f32x4* at = part + wave % (LN_WAVES / 2) * QUADS + (j * SMALL + s) * 64 + lane;
          *at = h ? acc[j][s] : *at + acc[j][s];
        }
    __syncthreads();
  }
  // register u of lane l in product j: row l % 16, column E (4 (l / 16) + u) + j; four consecutive columns are four products'
  for (int i = threadIdx.x; i < QUADS; i += 64 * LN_WAVES) {
    const int part4 = i % (E / 4), at16 = i / (E / 4) % 16, m16 = i / (4 * E) % 16, s = i / (64 * E);
    const int l = 16 * (at16 >> 2) + m16, u = at16 & 3;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < LN_WAVES / 2; ++w)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] += ((const float*)(part + w * QUADS + ((4 * part4 + j) * SMALL + s) * 64 + l))[u];
    const int64_t row = 16 * s + m16, col = first + E * at16 + 4 * part4;
    if (gridDim.y == 1) lin_store4<T>(g.e, row, col, v, lin_load4<T>(g.e, row, col));
    else if (row < g.m && col < g.n_pad) *(f32x4*)(g.part + ((int64_t)blockIdx.y * g.m + row) * g.n_pad + col) = v;
  }
}

// Which of the forms: 0 none, 1 rows of W are streamed, 2 rows of X, 3 W as it lies.  Rows along K at multiples of 4 bytes, W as it
// lies in whole pieces: at 2 bytes the general tiles are faster (one token through 4095 -> 11007 44 us against 31, 8192 x 4095 -> 16 31
// against 21), at 8 they are not (one token through 4092 -> 11008 20 against 27); W as it lies at 8 bytes 53 against 32.
static int linear_thin_form(int64_t m, int64_t n, int64_t k, int64_t ldx, int64_t ldw, bool w_kc, bool bf16) {
  if (k < 8 || m > (1 << 27) - 16 || n > (1 << 27) - 16) return 0;    // (fewer than 2^32 threads to a launch, 512 for 16 rows)
  const int e = bf16 ? 8 : 4;
  if ((bf16 && (ldx % 2 || (w_kc && ldw % 2))) || (!w_kc && (ldw % e || n % e))) return 0;
  if (m <= 32) return w_kc ? 1 : 3;
  // (33 to 64 outputs of many tokens: the tiles read W's columns once per 128 tokens; 8192 x 11008 -> 64 49 us against 67,
  // 2048 x 4096 -> 64 17 against 14; of float32 four blocks of products would outweigh the reads)
  return n <= 32 || (n <= 64 && m <= 4096 && bf16) ? 2 : 0;
}
static bool linear_thin_fits(const LinearArgs& g, bool w_kc) { return (uintptr_t)g.X % 4 == 0 && (uintptr_t)g.W % (w_kc ? 4 : 16) == 0; }
// Blocks of 16 streamed rows per wave: two where 32 rows still give every CU a workgroup, and for two blocks of tokens, whose X
// would otherwise be read by twice as many workgroups (32 tokens through 4096 -> 11008: 36 us with one block of W's rows, 34 with two).
static int linear_thin_blocks(int64_t m, int form) { return form == 1 ? (m > 16 ? 2 : 1) : (ceil_div64(m, 32) >= 256 ? 2 : 1); }
// K splits between workgroups: as many as make 256 of them, of at least 2 KB of K (256 bytes per wave).  More cost the launch that joins
// them (8192 x 4096 -> 16: 19 us with one split, 23 with two; one token through 11008 -> 4096: 20 and 23), but W as it lies, read by
// a third as many workgroups, takes four at up to 16 tokens (4096 -> 11008: 27 us with four splits, 31 with two; 32 tokens 35 and 29).
static int linear_thin_splits(int64_t m, int64_t n, int64_t k, int form, bool bf16) {
  const int64_t rows = 16 * linear_thin_blocks(m, form);
  const int64_t wgs = form == 1 ? ceil_div64(n, rows) : (form == 2 ? ceil_div64(m, rows) : ceil_div64(n, bf16 ? 128 : 64));
  const int64_t want = std::max<int64_t>(256 / wgs, form == 3 && m <= 16 ? 4 : 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, k / (bf16 ? 1024 : 512)), 64));
}
static size_t linear_thin_part_bytes(int64_t m, int64_t n, int64_t k, int form, bool bf16) {
  const int s = linear_thin_splits(m, n, k, form, bf16);
  return s > 1 ? align_up((size_t)s * m * align_up((size_t)n, 4) * 4, 256) : 0;
}

template <typename T>
static int launch_linear_thin(hipStream_t s, LinearArgs g, bool w_kc, int form) {
  constexpr bool BF = sizeof(T) == 2;
  int splits = linear_thin_splits(g.m, g.n, g.k, form, BF);
  g.k_per_split = ceil_div64(ceil_div64(g.k, splits), 256) * 256;
  splits = (int)ceil_div64(g.k, g.k_per_split);
  g.n_pad = (int64_t)align_up((size_t)g.n, 4);
  const dim3 block(64 * LN_WAVES);
#define LN_LAUNCH(...) LORACT_LAUNCH("linear_thin", s, (linear_thin_kernel<T, __VA_ARGS__>), grid, block, 0, g)
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
      else if constexpr (BF && B == 1) LN_LAUNCH(false, KC, B, 4);                       \
    }
    if (w_kc) { if (blocks == 2) LN_SMALL(true, 2) else LN_SMALL(true, 1) }
    else { if (blocks == 2) LN_SMALL(false, 2) else LN_SMALL(false, 1) }
#undef LN_SMALL
  } else {
    const dim3 grid((unsigned)ceil_div64(g.n, 16 * Ln<T>::E), (unsigned)splits);
    if (g.m <= 16) LORACT_LAUNCH("linear_thin", s, (linear_thin_t_kernel<T, 1>), grid, block, 0, g);
    else LORACT_LAUNCH("linear_thin", s, (linear_thin_t_kernel<T, 2>), grid, block, 0, g);
  }
#undef LN_LAUNCH
  return splits > 1 ? launch_linear_join<T>(s, g, splits) : LORACT_OK;
}

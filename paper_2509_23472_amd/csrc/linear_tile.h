// P = X W^T + s T B on tiles of 128 x 128 (128 x 64, 64 x 64): the form of loract_linear that takes every size, stride, alignment
// and type.
//
// The slabs (64 of K of bf16, 16 of float32) pass through registers into a double-buffered LDS tile, two
// slabs ahead of the one that is multiplied.
// The low-rank term comes first: acc = T B, acc *= s, then the slabs of X W^T on top of it, so that it costs one
// slab or two and its scale is applied in float32.  The products are formed transposed (the weights' fragment first), so that a lane holds
// four consecutive columns of a row: one group of the dropout generator, one 8- or 16-byte store.
// bf16 runs on v_mfma_f32_32x32x16_bf16, float32 on v_mfma_f32_32x32x2_f32 (a sixteenth of the rate): there a lane
// reads four consecutive k at once and the four products take one of them each, the same one for both operands.
//
// float32 is bound by its matrix instructions: 8192 x 1024 -> 4096 563 us, 122 TFLOP/s where a library's plain product reaches 144.
// bf16 comes here with rows that are no pieces or with sizes that are too small for copies to pay: 700 x 1030 -> 700 15 us.
#pragma once
#include "gemm_bf16.h"
#include "linear_epilogue.h"

struct LinearArgs {
  const void* X;
  int64_t ldx;
  const void* W;
  int64_t ldw;
  const void* T;         // m x r contiguous, or null
  const void* B;         // r x n_out contiguous (large tiles: rows of ldb)
  int64_t r;
  int64_t ldb, b_n8, w_n8;   // large tiles: columns of B and of W as it lies that can be read, multiples of 8
  float lora_scale;
  int64_t m, n, k;       // tokens, outputs, inputs
  float* part;           // [split][m][n_pad] when the K range is split
  int64_t n_pad;
  int64_t k_per_split;
  int splits;            // of K (general tiles)
  LinEpilogue e;
};

// One operand's share of a slab: R rows (or columns) of the output x BK of K, in pieces of 16 bytes at whatever address they have;
// K-strided operands lie in LDS as in memory and are read transposed (bf16) or element by element (float32).
// A piece that crosses the end of a row is loaded from the row's last whole piece and shifted, which also fills in the zeros.
// TINY: rows may be shorter than a piece; they are read element by element.  (As a choice at run time this puts a branch around
// every load, and the compiler a wait for the slabs in flight: 8192 x 1024 -> 4096 float32 608 us, without 568.)
template <typename T, bool KC, int R, bool TINY>
struct LinOperand {
  static constexpr int E = 16 / sizeof(T);
  static constexpr int BK = sizeof(T) == 2 ? 64 : 16, STEPS = sizeof(T) == 2 ? 4 : 2;
  static constexpr int CPR = KC ? BK / E : R / E;  // pieces per row of the slab
  static constexpr int BYTES = R * BK * (int)sizeof(T), NCH = BYTES / 16 / 256, RPP = 256 / CPR;      // rows per round of the 256 threads
  typedef T piece __attribute__((ext_vector_type(E)));
  typedef piece piece_any __attribute__((aligned(sizeof(T))));
  typedef piece frag_t;
  const T* base[KC ? NCH : 1];
  int64_t ld;
  int k_len, at, r0, len;                          // len: of a row

  __device__ void init(const T* P, int64_t ld_, int64_t first, int64_t count, int64_t K, int t) {
    ld = ld_;
    k_len = (int)K;
    r0 = t / CPR;
    if (KC) {
      at = t % CPR * E;
      len = (int)K;
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        int64_t g = first + r0 + RPP * i;
        if (g > count - 1) g = count - 1;          // rows past the end are never stored
        base[i] = P + g * ld;
      }
    } else {
      len = (int)count;
      at = (int)first + t % CPR * E;
      base[0] = P;
    }
  }
  __device__ static int place(int r, int c) {      // of piece c of row r in LDS
    if (sizeof(T) == 2) return KC ? r * 128 + ((c ^ (r & 7)) << 4) : r * (R * 2) + ((c ^ (2 * (r & 3))) << 4);
    return KC ? r * 64 + ((c ^ ((r >> 2) & 3)) << 4) : r * (R * 4) + (c << 4);
  }
  __device__ static piece load_piece(const T* row, int at, int len) {
    if (!TINY) return *(const piece_any*)(row + (at < len - E ? at : len - E));
    piece v;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = at + e < len ? row[at + e] : (T)0.0f;
    return v;
  }
  __device__ static piece shift(piece v, int at, int len) {
    if (TINY || at + E <= len) return v;
    const int over = at + E - len;
    if (over >= E) return (piece){};
    return __builtin_bit_cast(piece, __builtin_bit_cast(unsigned __int128, v) >> (8 * (int)sizeof(T) * over));
  }
  __device__ void load(piece* v, int k0) const {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int k = k0 + r0 + RPP * i;
      v[i] = KC ? load_piece(base[KC ? i : 0], k0 + at, len) : load_piece(base[0] + (int64_t)(k < k_len ? k : k_len - 1) * ld, at, len);
    }
  }
  // `edge`: the slab or the tile touches the end of the matrix (uniform)
  __device__ void put(const piece* v, unsigned char* lds, int k0, bool edge) const {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      piece w = v[i];
      if (edge) {
        w = shift(w, KC ? k0 + at : at, len);
        if (!KC && k0 + r0 + RPP * i >= k_len) w = (piece){};
      }
      *(piece*)(lds + place(r0 + RPP * i, KC ? at / E : threadIdx.x % CPR)) = w;
    }
  }
  // fragment address of a 32-wide group that starts at row (or column) `base` of the tile
  __device__ static int frag_off(int base, int lane) {
    if (KC) return (base + (lane & 31)) * (BK * (int)sizeof(T));
    if (sizeof(T) == 4) return 4 * (lane >> 5) * (R * 4) + (base + (lane & 31)) * 4;
    const int s16 = lane & 15, c = base + 16 * ((lane >> 4) & 1) + 4 * (s16 & 3);
    return (8 * (lane >> 5) + (s16 >> 2)) * (R * 2) + (((c >> 3) ^ (2 * (s16 >> 2))) << 4) + (c & 7) * 2;
  }
  // bf16: the eight k 16 ks + 8 (lane / 32) ..; float32: the four k 8 ks + 4 (lane / 32) ..
  __device__ static piece frag(const unsigned char* lds, int off, int ks, int lane) {
    if constexpr (KC) {
      return *(const piece*)(lds + off + (((2 * ks + (lane >> 5)) ^ (sizeof(T) == 2 ? lane & 7 : (lane >> 2) & 3)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) gb_s16x4* lds_ptr;
      const gb_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + off + 16 * ks * (R * 2)));
      const gb_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + off + (16 * ks + 4) * (R * 2)));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      piece v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const float*)(lds + off + (8 * ks + j) * (R * 4));
      return v;
    }
  }
};

// One step of a wave's MT x NT products.  float32: the k in turn for all of them, so that a product does not wait for the one before.
template <int MT, int NT>
__device__ inline void lin_multiply(const bf16x8 (&w)[NT], const bf16x8 (&x)[MT], f32x16 (&acc)[MT][NT]) {
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w[j], x[i], acc[i][j], 0, 0, 0);
}
template <int MT, int NT>
__device__ inline void lin_multiply(const f32x4 (&w)[NT], const f32x4 (&x)[MT], f32x16 (&acc)[MT][NT]) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[j][e], x[i][e], acc[i][j], 0, 0, 0);
}

// TINY: K, or the rows of W stored n_in x n_out, are shorter than a piece (the low-rank term's always may be).
// WKC: W is n_out x n_in (rows along K), else n_in x n_out.  BM x BN tile, four waves of BM/2 x BN/2.  blockIdx.x: row of tiles, blockIdx.y: column;
// blockIdx.z: split of K, or where K is whole and there are more than LT_MAX_Y columns, further columns.
#define LT_MAX_Y 65535
template <typename T, bool WKC, int BM, int BN, bool TINY>
__global__ __launch_bounds__(256) void linear_tile_kernel(LinearArgs g) {
  typedef LinOperand<T, true, BM, TINY> OpX;
  typedef LinOperand<T, WKC, BN, TINY> OpW;
  typedef LinOperand<T, true, BM, true> OpT;
  typedef LinOperand<T, false, BN, true> OpB;
  constexpr int MT = BM / 64, NT = BN / 64, BK = OpX::BK, STEPS = OpX::STEPS;
  typedef typename OpX::piece piece;
  typedef piece frag_t;
  constexpr int STAGE = OpX::BYTES + OpW::BYTES;
  constexpr int OUT = 4 * 32 * (BN / 2 + 4) * 4;     // staging of the output
  __shared__ __attribute__((aligned(16))) unsigned char smem[2 * STAGE > OUT ? 2 * STAGE : OUT];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  const int split = g.splits > 1 ? blockIdx.z : 0;
  const int64_t row0 = (int64_t)blockIdx.x * BM, col0 = ((g.splits > 1 ? 0 : (int64_t)blockIdx.z * gridDim.y) + blockIdx.y) * BN;
  if (col0 >= g.n) return;                           // (the last of several blockIdx.z may not be full)
  const int kbeg = (int)(split * g.k_per_split);
  const int kend = (int)(kbeg + g.k_per_split < g.k ? kbeg + g.k_per_split : g.k);
  const int nslab = (kend - kbeg + BK - 1) / BK;
  int x_off[MT], w_off[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) x_off[i] = OpX::frag_off(wm * (BM / 2) + 32 * i, lane);

  // TWO: odd and even steps of K have an accumulator each, which shortens the chain of roundings, where that costs nothing: 3001 x 1030 ->
  // 770 is 6.9 units of 2^-24 off (rms) instead of 9.7 in the same time; W as it lies 1024 x 256 -> 256 would take 11.6 us instead of 11.0, tiles of
  // 128 x 128 (8192 x 1024 -> 4096) 633 instead of 565.
  constexpr bool TWO = sizeof(T) == 4 && WKC && BM == 64 && BN == 64;
  f32x16 acc[MT][NT], odd[TWO ? MT : 1][TWO ? NT : 1];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        acc[i][j][r] = 0.0f;
        if (TWO) odd[i][j][r] = 0.0f;
      }

  if (g.T && split == 0) {
#pragma unroll
    for (int j = 0; j < NT; ++j) w_off[j] = OpX::BYTES + OpB::frag_off(wn * (BN / 2) + 32 * j, lane);
    OpT ot;
    OpB ob;
    ot.init((const T*)g.T, g.r, row0, g.m, g.r, t);
    ob.init((const T*)g.B, g.n, col0, g.n, g.r, t);
    for (int k0 = 0; k0 < (int)g.r; k0 += BK) {
      piece vt[OpT::NCH], vb[OpB::NCH];
      ot.load(vt, k0);
      ob.load(vb, k0);
      ot.put(vt, smem, k0, true);
      ob.put(vb, smem + OpX::BYTES, k0, true);
      sb_barrier_lds();
#pragma unroll
      for (int ks = 0; ks < STEPS; ++ks) {
        frag_t x[MT], w[NT];
#pragma unroll
        for (int i = 0; i < MT; ++i) x[i] = OpX::frag(smem, x_off[i], ks, lane);
#pragma unroll
        for (int j = 0; j < NT; ++j) w[j] = OpB::frag(smem, w_off[j], ks, lane);
        lin_multiply<MT, NT>(w, x, acc);
      }
      sb_barrier_lds();
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] *= g.lora_scale;
  }

  OpX ox;
  OpW ow;
  ox.init((const T*)g.X, g.ldx, row0, g.m, g.k, t);
  ow.init((const T*)g.W, g.ldw, col0, g.n, g.k, t);
#pragma unroll
  for (int j = 0; j < NT; ++j) w_off[j] = OpX::BYTES + OpW::frag_off(wn * (BN / 2) + 32 * j, lane);
  const bool tile_edge = !WKC && col0 + BN > g.n;
  piece vx[2][OpX::NCH], vw[2][OpW::NCH];
  auto fetch = [&](int p, int s) {                 // slabs past the last one repeat it and are not multiplied
    const int k0 = kbeg + (s < nslab ? s : nslab - 1) * BK;
    ox.load(vx[p], k0);
    ow.load(vw[p], k0);
  };
  auto step = [&](int p, int s) {
    const int k0 = kbeg + s * BK;
    unsigned char* st = smem + p * STAGE;
    const bool edge = tile_edge || k0 + BK > (int)g.k;
    ox.put(vx[p], st, k0, edge);
    ow.put(vw[p], st + OpX::BYTES, k0, edge);
    sb_barrier_lds();                              // (the half of slab s - 2 was left before slab s - 1's barrier)
    fetch(p, s + 2);
#pragma unroll
    for (int ks = 0; ks < STEPS; ++ks) {
      frag_t x[MT], w[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i) x[i] = OpX::frag(st, x_off[i], ks, lane);
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j] = OpW::frag(st, w_off[j], ks, lane);
      if constexpr (TWO) lin_multiply<MT, NT>(w, x, ks % 2 ? odd : acc);
      else lin_multiply<MT, NT>(w, x, acc);
    }
  };
  fetch(0, 0);
  fetch(1, 1);
  int s = 0;
  for (; s + 2 <= nslab; s += 2) { step(0, s); step(1, s + 1); }
  if (s < nslab) step(0, s);
  if constexpr (TWO) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] += odd[i][j];
  }

  // Accumulator register 4 q + u of lane l: column 8 q + 4 (l / 32) + u, row l % 32 of its tile.  They leave 32 rows at a time through LDS, so
  // that neighbouring lanes hold neighbouring columns, with all loads of the residual ahead.
  constexpr int PART = BN / 2, LDC = PART + 4, QPR = PART / 4, ROWS = 64 / QPR, N4 = 32 / ROWS;
  sb_barrier_lds();                                // the last slab has been read
  float* const cs = (float*)(smem + wave * (32 * LDC * 4));
  const int c4 = lane % QPR * 4, r0 = lane / QPR;
  const int64_t col = col0 + wn * PART + c4;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t row = row0 + wm * (BM / 2) + 32 * i + r0;
    f32x4 res[N4];
    if (g.splits == 1) {
#pragma unroll
      for (int q = 0; q < N4; ++q) res[q] = lin_load4<T>(g.e, row + ROWS * q, col);
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(f32x4*)(cs + (lane & 31) * LDC + 32 * j + 8 * q + 4 * (lane >> 5)) =
            (f32x4){acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    sb_wave_sync();
#pragma unroll
    for (int q = 0; q < N4; ++q) {
      const f32x4 v = *(const f32x4*)(cs + (r0 + ROWS * q) * LDC + c4);
      const int64_t at = row + ROWS * q;
      if (g.splits == 1) lin_store4<T>(g.e, at, col, v, res[q]);
      else if (at < g.m && col < g.n_pad) *(f32x4*)(g.part + ((int64_t)split * g.m + at) * g.n_pad + col) = v;
    }
    sb_wave_sync();
  }
}

// Tiles: 128 x 128 (64 in a direction that has no more), but 64 x 64 for float32 where the large ones leave CUs without work or
// need a second round for less than half of the card: a float32 tile of 128 x 128 is matrix instructions for 55 us per 1024 of K
// whatever feeds it, so small ones lose nothing but traffic and balance better (1024 x 256 -> 256 26 -> 10 us, 500 x 500 -> 500 44 -> 16,
// 12608 x 768 -> 768 168 -> 146; 4096 x 1024 -> 4096, which they do not take, 284 -> 293).
// K splits: as many as make 512 workgroups (1024 of the small float32 tiles), of at least 256 of K each, at most 64.
struct TilePlan {
  int bm, bn, splits;
};
static inline TilePlan linear_tile_plan(int64_t m, int64_t n, int64_t k, bool bf16) {
  TilePlan p;
  const int64_t large = ceil_div64(m, 128) * ceil_div64(n, 128);
  const bool fine = !bf16 && (large < 256 || (large > 512 && large < 768));
  p.bm = m <= 64 || fine ? 64 : 128;
  p.bn = m <= 64 || n <= 64 || fine ? 64 : 128;
  const int64_t tiles = ceil_div64(m, p.bm) * ceil_div64(n, p.bn);
  const int64_t s = std::min<int64_t>((fine ? 1024 : 512) / tiles, k / 256);
  p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(s, 64));
  return p;
}
static inline bool linear_tile_tiny(int64_t n, int64_t k, bool w_kc, bool bf16) {
  const int e = bf16 ? 8 : 4;
  return k < e || (!w_kc && n < e);
}
// A launch takes fewer than 2^32 threads in a direction.  (More than LT_MAX_Y columns leave K whole.)
static inline bool linear_tile_launches(int64_t m, int64_t n, int64_t k, bool w_kc, bool bf16) {
  return ceil_div64(m, linear_tile_tiny(n, k, w_kc, bf16) ? 64 : linear_tile_plan(m, n, k, bf16).bm) < 1 << 24;
}
static inline size_t linear_tile_part_bytes(int64_t m, int64_t n, int64_t k, bool bf16) {
  const int s = linear_tile_plan(m, n, k, bf16).splits;
  return s > 1 ? (size_t)s * m * align_up((size_t)n, 4) * 4 : 0;
}

template <typename T>
static int launch_linear_join(hipStream_t s, const LinearArgs& g, int splits) {
  const int64_t blocks = std::min<int64_t>(ceil_div64(g.m * (g.n_pad / 4), 256), 2048);
  LORACT_LAUNCH("linear_join", s, linear_join_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, (const float*)g.part, splits,
                g.n_pad, g.e);
  return LORACT_OK;
}

template <typename T>
static int launch_linear_tile(hipStream_t s, LinearArgs g, bool w_kc) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int BK = LinOperand<T, true, 64, false>::BK;
  const bool tiny = linear_tile_tiny(g.n, g.k, w_kc, BF);
  TilePlan p = linear_tile_plan(g.m, g.n, g.k, BF);
  if (tiny) p.bm = p.bn = 64;
  const int bm = p.bm, bn = p.bn;
  int splits = p.splits;
  g.k_per_split = ceil_div64(ceil_div64(g.k, splits), BK) * BK;
  splits = (int)ceil_div64(g.k, g.k_per_split);
  g.n_pad = (int64_t)align_up((size_t)g.n, 4);
  g.splits = splits;
  const int64_t columns = ceil_div64(g.n, bn), y = std::min<int64_t>(columns, LT_MAX_Y);
  const dim3 grid((unsigned)ceil_div64(g.m, bm), (unsigned)y, splits > 1 ? (unsigned)splits : (unsigned)ceil_div64(columns, y));
#define LT_LAUNCH(WKC, BM, BN, TINY) LORACT_LAUNCH("linear_tile", s, (linear_tile_kernel<T, WKC, BM, BN, TINY>), grid, dim3(256), 0, g)
  if (w_kc) {
    if (tiny) LT_LAUNCH(true, 64, 64, true);
    else if (bm == 64) LT_LAUNCH(true, 64, 64, false);
    else if (bn == 64) LT_LAUNCH(true, 128, 64, false);
    else LT_LAUNCH(true, 128, 128, false);
  } else {
    if (tiny) LT_LAUNCH(false, 64, 64, true);
    else if (bm == 64) LT_LAUNCH(false, 64, 64, false);
    else if (bn == 64) LT_LAUNCH(false, 128, 64, false);
    else LT_LAUNCH(false, 128, 128, false);
  }
#undef LT_LAUNCH
  return splits > 1 ? launch_linear_join<T>(s, g, splits) : LORACT_OK;
}

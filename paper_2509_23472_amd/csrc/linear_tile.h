// P = X W^T + s T B on tiles of 128 x 128 (128 x 64, 64 x 64): the form of loract_linear that takes every size, stride, alignment
// and type.
//
// The slabs (128 bytes of K per row: 64 bf16 or 32 float32) pass through registers into a double-buffered LDS tile, two
// slabs ahead of the one that is multiplied; the operands are those of gemm_bf16.h and their float32 counterparts below.
// The low-rank term comes first: acc = T B, acc *= s, then the slabs of X W^T on top of it, so that it costs one
// slab or two and its scale is applied in float32.  The products are formed transposed (the weights' fragment first), so that a lane holds
// four consecutive columns of a row: one group of the dropout generator, one 8- or 16-byte store.
// bf16 runs on v_mfma_f32_32x32x16_bf16, float32 on v_mfma_f32_32x32x2_f32 (a sixteenth of the rate): there a lane
// reads four consecutive k at once and the four products take one of them each, the same one for both operands.
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
  LinEpilogue e;
};

// The float32 counterpart of GbOperand: R rows (or columns) of the output x 32 of K.
__device__ inline f32x4 lf_load(const float* row, int64_t at, int64_t len) {
  typedef f32x4 any __attribute__((aligned(4)));
  if (len >= 4) return *(const any*)(row + (at + 4 <= len ? at : len - 4));
  f32x4 v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = at + e < len ? row[at + e] : 0.0f;
  return v;
}
__device__ inline f32x4 lf_shift(f32x4 v, int64_t at, int64_t len) {
  if (len < 4 || at + 4 <= len) return v;
  const int64_t over = at + 4 - len;
  f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  if (over == 1) { o[0] = v[1]; o[1] = v[2]; o[2] = v[3]; }
  if (over == 2) { o[0] = v[2]; o[1] = v[3]; }
  if (over == 3) o[0] = v[3];
  return o;
}

template <bool KC, int R>
struct LfOperand {
  static constexpr int NCH = R / 32;
  static constexpr int CPR = R / 4;                // K-strided: pieces per row of the slab
  static constexpr int BYTES = R * 128;
  const float* row[KC ? NCH : 1];
  int64_t ld, k_len, col, n_len;
  int lds_off[NCH], kr0;

  __device__ void init(const float* P, int64_t ld_, const int32_t*, int64_t first, int64_t count, int64_t K, int t) {
    ld = ld_;
    k_len = K;
    n_len = count;
    if (KC) {
      col = (t & 7) * 4;
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int r = (t >> 3) + 32 * i;
        int64_t g = first + r;
        if (g > count - 1) g = count - 1;          // rows past the end are never stored
        row[i] = P + g * ld;
        lds_off[i] = r * 128 + (((t & 7) ^ (r & 7)) << 4);
      }
    } else {
      const int c = t % CPR;
      kr0 = t / CPR;
      col = first + c * 4;
      row[0] = P;
#pragma unroll
      for (int i = 0; i < NCH; ++i) lds_off[i] = (kr0 + (256 / CPR) * i) * (R * 4) + c * 16;
    }
  }
  __device__ void load(f32x4* v, int64_t k0, bool) const {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      if (KC) {
        v[i] = lf_load(row[i], k0 + col, k_len);
      } else {
        int64_t k = k0 + kr0 + (256 / CPR) * i;
        if (k > k_len - 1) k = k_len - 1;
        v[i] = lf_load(row[0] + k * ld, col < n_len ? col : n_len, n_len);
      }
    }
  }
  __device__ void put(const f32x4* v, unsigned char* lds, int64_t k0, bool edge, bool) const {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      f32x4 w = v[i];
      if (edge) {
        if (KC) {
          w = lf_shift(w, k0 + col, k_len);
        } else {
          w = lf_shift(w, col < n_len ? col : n_len, n_len);
          if (k0 + kr0 + (256 / CPR) * i >= k_len) w = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
        }
      }
      *(f32x4*)(lds + lds_off[i]) = w;
    }
  }
  __device__ static int frag_off(int base, int lane) {
    if (KC) return (base + (lane & 31)) * 128;
    return 4 * (lane >> 5) * (R * 4) + (base + (lane & 31)) * 4;
  }
  // the four k of this lane in step ks: 8 ks + 4 (lane / 32) ..
  __device__ static f32x4 frag(const unsigned char* lds, int off, int ks, int lane) {
    if (KC) return *(const f32x4*)(lds + off + (((2 * ks + (lane >> 5)) ^ (lane & 7)) << 4));
    f32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = *(const float*)(lds + off + (8 * ks + j) * (R * 4));
    return v;
  }
};

template <typename T, bool KC, int R> struct LinOperand;
template <bool KC, int R> struct LinOperand<bf16_t, KC, R> {
  typedef GbOperand<KC, R> type;
  typedef gb_u32x4 piece;
  typedef bf16x8 frag;
};
template <bool KC, int R> struct LinOperand<float, KC, R> {
  typedef LfOperand<KC, R> type;
  typedef f32x4 piece;
  typedef f32x4 frag;
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

// WKC: W is n_out x n_in (rows along K), else n_in x n_out.  BM x BN tile, four waves of BM/2 x BN/2; blockIdx.z: split of K.
template <typename T, bool WKC, int BM, int BN>
__global__ __launch_bounds__(256) void linear_tile_kernel(LinearArgs g) {
  constexpr int MT = BM / 64, NT = BN / 64, BK = 128 / (int)sizeof(T);
  typedef typename LinOperand<T, true, BM>::type OpX;
  typedef typename LinOperand<T, WKC, BN>::type OpW;
  typedef typename LinOperand<T, false, BN>::type OpB;
  typedef typename LinOperand<T, true, BM>::piece piece;
  typedef typename LinOperand<T, true, BM>::frag frag_t;
  constexpr int STAGE = OpX::BYTES + OpW::BYTES;
  __shared__ __attribute__((aligned(16))) unsigned char smem[2 * STAGE];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int wm = wave >> 1, wn = wave & 1;
  const int64_t row0 = (int64_t)blockIdx.x * BM, col0 = (int64_t)blockIdx.y * BN;
  const int64_t kbeg = (int64_t)blockIdx.z * g.k_per_split;
  const int64_t kend = (kbeg + g.k_per_split < g.k) ? kbeg + g.k_per_split : g.k;
  const int nslab = (int)((kend - kbeg + BK - 1) / BK);
  int x_off[MT], w_off[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) x_off[i] = OpX::frag_off(wm * (BM / 2) + 32 * i, lane);

  f32x16 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  if (g.T && blockIdx.z == 0) {
#pragma unroll
    for (int j = 0; j < NT; ++j) w_off[j] = OpX::BYTES + OpB::frag_off(wn * (BN / 2) + 32 * j, lane);
    OpX ot;
    OpB ob;
    ot.init((const T*)g.T, g.r, nullptr, row0, g.m, g.r, t);
    ob.init((const T*)g.B, g.n, nullptr, col0, g.n, g.r, t);
    for (int64_t k0 = 0; k0 < g.r; k0 += BK) {
      piece vt[OpX::NCH], vb[OpB::NCH];
      ot.load(vt, k0, false);
      ob.load(vb, k0, false);
      ot.put(vt, smem, k0, true, false);
      ob.put(vb, smem + OpX::BYTES, k0, true, false);
      sb_barrier_lds();
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
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
  ox.init((const T*)g.X, g.ldx, nullptr, row0, g.m, g.k, t);
  ow.init((const T*)g.W, g.ldw, nullptr, col0, g.n, g.k, t);
#pragma unroll
  for (int j = 0; j < NT; ++j) w_off[j] = OpX::BYTES + OpW::frag_off(wn * (BN / 2) + 32 * j, lane);
  const bool tile_edge = !WKC && col0 + BN > g.n;
  piece vx[2][OpX::NCH], vw[2][OpW::NCH];
  auto fetch = [&](int p, int s) {                 // slabs past the last one repeat it and are not multiplied
    const int64_t k0 = kbeg + (int64_t)(s < nslab ? s : nslab - 1) * BK;
    ox.load(vx[p], k0, false);
    ow.load(vw[p], k0, false);
  };
  auto step = [&](int p, int s) {
    const int64_t k0 = kbeg + (int64_t)s * BK;
    unsigned char* st = smem + p * STAGE;
    const bool edge = tile_edge || k0 + BK > g.k;
    ox.put(vx[p], st, k0, edge, false);
    ow.put(vw[p], st + OpX::BYTES, k0, edge, false);
    sb_barrier_lds();                              // (the half of slab s - 2 was left before slab s - 1's barrier)
    fetch(p, s + 2);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      frag_t x[MT], w[NT];
#pragma unroll
      for (int i = 0; i < MT; ++i) x[i] = OpX::frag(st, x_off[i], ks, lane);
#pragma unroll
      for (int j = 0; j < NT; ++j) w[j] = OpW::frag(st, w_off[j], ks, lane);
      lin_multiply<MT, NT>(w, x, acc);
    }
  };
  fetch(0, 0);
  fetch(1, 1);
  int s = 0;
  for (; s + 2 <= nslab; s += 2) { step(0, s); step(1, s + 1); }
  if (s < nslab) step(0, s);

  // Accumulator register 4 q + u of lane l: column 8 q + 4 (l / 32) + u, row l % 32 of its tile.  They leave 32 rows at a time through LDS, so
  // that neighbouring lanes hold neighbouring columns, with all loads of the residual ahead.
  constexpr int PART = BN / 2, LDC = PART + 4, QPR = PART / 4, ROWS = 64 / QPR, N4 = 32 / ROWS;
  static_assert(4 * 32 * LDC * 4 <= 2 * STAGE, "staging of the output");
  sb_barrier_lds();                                // the last slab has been read
  float* const cs = (float*)(smem + wave * (32 * LDC * 4));
  const int c4 = lane % QPR * 4, r0 = lane / QPR;
  const int64_t col = col0 + wn * PART + c4;
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t row = row0 + wm * (BM / 2) + 32 * i + r0;
    f32x4 res[N4];
    if (gridDim.z == 1) {
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
      if (gridDim.z == 1) lin_store4<T>(g.e, at, col, v, res[q]);
      else if (at < g.m && col < g.n_pad) *(f32x4*)(g.part + ((int64_t)blockIdx.z * g.m + at) * g.n_pad + col) = v;
    }
    sb_wave_sync();
  }
}

// Tiles: 128 x 128 (64 in a direction that has no more), but 64 x 64 for float32 where the large ones leave CUs without work or
// need a second round for less than half of the card: a float32 tile of 128 x 128 is matrix instructions for 55 us per 1024 of K
// whatever feeds it, so small ones lose nothing but traffic and balance better (1024 x 256 -> 256 20 -> 13 us, 500 x 500 -> 500 26 -> 15,
// 12608 x 768 -> 768 210 -> 190; 4096 x 1024 -> 4096, which they do not take, 305 -> 339).
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
  constexpr int BK = 128 / (int)sizeof(T);
  const TilePlan p = linear_tile_plan(g.m, g.n, g.k, BF);
  const int bm = p.bm, bn = p.bn;
  int splits = p.splits;
  g.k_per_split = ceil_div64(ceil_div64(g.k, splits), BK) * BK;
  splits = (int)ceil_div64(g.k, g.k_per_split);
  g.n_pad = (int64_t)align_up((size_t)g.n, 4);
  const dim3 grid((unsigned)ceil_div64(g.m, bm), (unsigned)ceil_div64(g.n, bn), (unsigned)splits);
  if (grid.y > 65535) return LORACT_ERR_UNSUPPORTED;
#define LT_LAUNCH(WKC, BM, BN) LORACT_LAUNCH("linear_tile", s, (linear_tile_kernel<T, WKC, BM, BN>), grid, dim3(256), 0, g)
  if (w_kc) {
    if (bm == 64) LT_LAUNCH(true, 64, 64);
    else if (bn == 64) LT_LAUNCH(true, 128, 64);
    else LT_LAUNCH(true, 128, 128);
  } else {
    if (bm == 64) LT_LAUNCH(false, 64, 64);
    else if (bn == 64) LT_LAUNCH(false, 128, 64);
    else LT_LAUNCH(false, 128, 128);
  }
#undef LT_LAUNCH
  return splits > 1 ? launch_linear_join<T>(s, g, splits) : LORACT_OK;
}

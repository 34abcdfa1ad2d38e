// P = X W^T + s T B for large bf16 maps: tiles of 256 x 256 on v_mfma_f32_16x16x32_bf16.
//
// Slabs of 64 of K -- whole 128-byte lines of X and of W -- go from memory straight into LDS (asynchronous copies): three stages for
// X, fetched up to three slabs ahead, and two for W, 160 KB in all.  A stage holds 256 rows as [row][64] or, for W stored
// n_in x n_out, 64 rows of it as they lie ([k][256], read with the transposing LDS read).  A wave reads the fragments of the next 32 of K
// while it multiplies the present ones; there is one barrier per slab, behind the first products of its second half.
#pragma once
#include "linear_tile.h"

#include <type_traits>

#define LL_BK 64
#define LL_WAVES 8
#define LL_STAGE (256 * LL_BK * 2)    // bytes of one operand's slab
#define LL_X_STAGES 3
#define LL_W_STAGES 2

// XCD b % 8 takes a run of consecutive tiles; within it tiles go in bands of LL_BAND tile rows, so that the tiles that are in
// flight on one XCD share rows of X and of W in its L2.
#define LL_BAND 8
__device__ inline void ll_tile_of(int b, int tiles_m, int tiles_n, int* tm, int* tn) {
  const int total = tiles_m * tiles_n;
  const int xcd = b & 7, per = total >> 3, rest = total & 7;
  const int id = xcd * per + (xcd < rest ? xcd : rest) + (b >> 3);
  const int band = id / (LL_BAND * tiles_n), in = id - band * (LL_BAND * tiles_n);
  const int rows = tiles_m - band * LL_BAND < LL_BAND ? tiles_m - band * LL_BAND : LL_BAND;
  *tn = in / rows;
  *tm = band * LL_BAND + in - *tn * rows;
}

__device__ inline bf16x8 ll_read_tr(const unsigned char* lds, int off) {
  typedef __attribute__((address_space(3))) gb_s16x4* lds_ptr;
  const gb_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + off));
  const gb_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + off + 4 * 512));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Where the 16-byte chunks of a row lie: chunk c of row r (along K) at c ^ ll_turn(r), chunk c of row k of W as it lies at
// c ^ ll_turn_k(k).  The 16 lanes that LDS serves at a time (256 bytes) then read from 16 different groups of banks, whether these are 16
// neighbours or four runs of four (counted: no conflicts).
__device__ inline int ll_turn(int r) { return (r >> 1) & 7; }
__device__ inline int ll_turn_k(int k) { return 4 * (k & 3) + ((k >> 2) & 2); }

template <bool WKC>
__global__ __launch_bounds__(64 * LL_WAVES, 1) void linear_large_kernel(LinearArgs g, int tiles_m, int tiles_n) {
  constexpr int MT = 8, NT = 4, C = 32 / LL_WAVES;       // a wave: 8 x 4 products of 16 x 16; copies per operand and slab
  __shared__ __attribute__((aligned(16))) unsigned char smem[(LL_X_STAGES + LL_W_STAGES) * LL_STAGE];
  unsigned char* const smem_w = smem + LL_X_STAGES * LL_STAGE;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave >> 2, wn = wave & 3;
  int tm, tn;
  ll_tile_of(blockIdx.x, tiles_m, tiles_n, &tm, &tn);
  const int64_t row0 = (int64_t)tm * 256, col0 = (int64_t)tn * 256;
  const int k_len = (int)g.k, full = k_len / LL_BK, nslab = (k_len + LL_BK - 1) / LL_BK;

  const char* const xb = (const char*)((const bf16_t*)g.X + row0 * g.ldx);
  const char* const wb = (const char*)((const bf16_t*)g.W + (WKC ? col0 * g.ldw : col0));
  const int64_t w_step = WKC ? 2 * LL_BK : 2 * LL_BK * g.ldw;
  // copy c of a wave: 8 rows of 128 bytes along K, or two rows of 512 bytes of W as it lies
  const int copy_row = 8 * wave * C + (lane >> 3), copy_k = 2 * wave * C + (lane >> 5);
  auto chunk_of = [&](int c) { return (lane & 7) ^ ll_turn(copy_row + 8 * c); };
  auto col_of = [&](int c) {
    const int64_t col = ((lane & 31) ^ ll_turn_k(copy_k + 2 * c)) * 8;
    return col0 + col < g.n ? col : g.n - 8 - col0;                         // columns past the end are never stored
  };
  unsigned xo[C], wo[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int row = copy_row + 8 * c;
    const int64_t xr = row0 + row < g.m ? row : g.m - 1 - row0;            // (nor rows)
    xo[c] = (unsigned)(xr * g.ldx * 2) + chunk_of(c) * 16;
    if (WKC) {
      const int64_t wr = col0 + row < g.n ? row : g.n - 1 - col0;
      wo[c] = (unsigned)(wr * g.ldw * 2) + chunk_of(c) * 16;
    } else {
      wo[c] = (unsigned)((copy_k + 2 * c) * g.ldw * 2) + (unsigned)col_of(c) * 2;
    }
  }
  // Slabs are numbered through: the one of T and B, if there is a low-rank term, then those of X and W.
  const int r = g.T ? (int)g.r : 0, nlr = r ? 1 : 0, slabs = nlr + nslab;
  auto x_stage = [&](int v) { return smem + v % LL_X_STAGES * LL_STAGE; };
  auto w_stage = [&](int v) { return smem_w + v % LL_W_STAGES * LL_STAGE; };
  auto copy_x = [&](int v) {
    unsigned char* const st = x_stage(v) + wave * (C * 1024);
    if (v >= slabs) v = slabs - 1;                                         // (never multiplied)
    const int left = v < nlr ? r : k_len - (v - nlr) * LL_BK;              // of K in this slab
    const char* const xs = xb + (int64_t)(v - nlr) * (2 * LL_BK);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int chunk = chunk_of(c);
      const int back = chunk * 8 < left ? 0 : chunk * 16;                  // past the end of K: something that is there
      if (v < nlr) {
        const int64_t row = row0 + copy_row + 8 * c;
        sb_async16((const char*)g.T + (row < g.m ? row : g.m - 1) * r * 2 + chunk * 16 - back, st + c * 1024);
      } else {
        sb_async16_at(xs, xo[c] - back, st + c * 1024);
      }
    }
  };
  auto copy_w = [&](int v) {
    unsigned char* const st = w_stage(v) + wave * (C * 1024);
    if (v >= slabs) v = slabs - 1;
    const int left = v < nlr ? r : k_len - (v - nlr) * LL_BK;
    const char* const ws = wb + (v - nlr) * w_step;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int kr = copy_k + 2 * c, chunk = chunk_of(c);
      if (v < nlr)
        sb_async16((const bf16_t*)g.B + (int64_t)(kr < left ? kr : left - 1) * g.n + col0 + col_of(c), st + c * 1024);
      else if (WKC)
        sb_async16_at(ws, wo[c] - (chunk * 8 < left ? 0 : chunk * 16), st + c * 1024);
      else
        sb_async16_at(ws, wo[c] - (unsigned)((kr < left ? 0 : kr - left + 1) * g.ldw * 2), st + c * 1024);
    }
  };

  // fragments: 16 rows (columns), lane l holds row l % 16 and the eight k from 8 (l / 16) on of a half slab
  const int k_off[2] = {((lane >> 4) ^ ll_turn(lane & 15)) << 4, ((4 + (lane >> 4)) ^ ll_turn(lane & 15)) << 4};
  const int xr_off = (wm * 128 + (lane & 15)) * 128, wr_off = (wn * 64 + (lane & 15)) * 128;
  int tr_off[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int s16 = lane & 15, kr = 8 * (lane >> 4) + (s16 >> 2), c = wn * 64 + 16 * j + 4 * (s16 & 3);
    tr_off[j] = kr * 512 + (((c >> 3) ^ ll_turn_k(kr)) << 4) + (c & 7) * 2;
  }
  bf16x8 x[2][MT], w[2][NT];
  // fragment f of half h of a slab: those of W, then those of X
  auto read_one = [&](const unsigned char* xs, const unsigned char* ws, int h, bool w_kc, int f) {
    if (f < NT) w[h][f] = w_kc ? *(const bf16x8*)(ws + wr_off + k_off[h] + f * 2048) : ll_read_tr(ws, tr_off[f] + h * (32 * 512));
    else x[h][f - NT] = *(const bf16x8*)(xs + xr_off + k_off[h] + (f - NT) * 2048);
  };
  auto read = [&](int v, int h, bool w_kc) {
#pragma unroll
    for (int f = 0; f < MT + NT; ++f) read_one(x_stage(v), w_stage(v), h, w_kc, f);
  };
  f32x4 acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  auto multiply = [&](int h) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[h][j], x[h][i], acc[i][j], 0, 0, 0);
  };
  auto mask = [&](int h, int left) {                                        // zero past the end of K, in both operands
    const bool keep = 32 * h + 8 * (lane >> 4) < left;
#pragma unroll
    for (int i = 0; i < MT; ++i) x[h][i] = keep ? x[h][i] : (bf16x8){};
#pragma unroll
    for (int j = 0; j < NT; ++j) w[h][j] = keep ? w[h][j] : (bf16x8){};
  };

  copy_x(0);
  copy_w(0);
  copy_x(1);
  copy_w(1);
  copy_x(2);
  SB_WAIT_VMCNT(3 * C);                // slab 0 has landed
  sb_barrier_lds();
  if (r) {
    read(0, 0, false);
    mask(0, r);
    multiply(0);
    if (r > 32) {
      read(0, 1, false);
      mask(1, r);
      multiply(1);
    }
    sb_barrier_lds();                  // (its stages are free)
    copy_w(2);
    copy_x(3);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] *= g.lora_scale;
    SB_WAIT_VMCNT(3 * C);
    sb_barrier_lds();
  }
  read(nlr, 0, WKC);
  int v = nlr;
  // One instruction of another kind after a product at most: whatever keeps a wave from issuing the next product leaves its
  // matrix unit idle.
  for (; v + 3 < nlr + full; ++v) {
    const unsigned char *xs = x_stage(v), *ws = w_stage(v);
#pragma unroll
    for (int u = 0; u < MT * NT; ++u) {
      acc[u / NT][u % NT] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[0][u % NT], x[0][u / NT], acc[u / NT][u % NT], 0, 0, 0);
      if (u < 2 * (MT + NT) && u % 2 == 0) read_one(xs, ws, 1, WKC, u / 2);
      __builtin_amdgcn_sched_barrier(0);
    }
    xs = x_stage(v + 1);
    ws = w_stage(v + 1);
    const char* const x_src = xb + (int64_t)(v + 3 - nlr) * (2 * LL_BK);
    const char* const w_src = wb + (v + 2 - nlr) * w_step;
    unsigned char* const x_dst = x_stage(v) + wave * (C * 1024);
    unsigned char* const w_dst = w_stage(v) + wave * (C * 1024);
#pragma unroll
    for (int u = 0; u < MT * NT; ++u) {
      acc[u / NT][u % NT] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[1][u % NT], x[1][u / NT], acc[u / NT][u % NT], 0, 0, 0);
      if (u == 3) {
        SB_WAIT_VMCNT(C);              // slab v + 1 has landed (behind it: X of slab v + 2); everyone has read slab v
        sb_barrier_lds();
      }
      if (u >= 4 && u < 4 + 2 * (MT + NT) && u % 2 == 0) read_one(xs, ws, 0, WKC, (u - 4) / 2);
      if (u >= 4 && u < 4 + 3 * 2 * C && u % 3 == 1) {
        const int c = (u - 4) / 3;
        if (c < C) sb_async16_at(w_src, wo[c % C], w_dst + (c % C) * 1024);
        else sb_async16_at(x_src, xo[c % C], x_dst + (c % C) * 1024);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  for (; v < nlr + full; ++v) {
    read(v, 1, WKC);
    multiply(0);
    SB_WAIT_VMCNT(C);
    sb_barrier_lds();
    copy_w(v + 2);
    copy_x(v + 3);
    read(v + 1, 0, WKC);               // (past the last slab: not multiplied)
    multiply(1);
  }
  if (full < nslab) {
    const int left = k_len - full * LL_BK;
    mask(0, left);
    multiply(0);
    if (left > 32) {
      read(v, 1, WKC);
      mask(1, left);
      multiply(1);
    }
  }
  SB_WAIT_VMCNT(0);
  sb_barrier_lds();

  // 32 rows of the wave's part at a time through LDS, so that a lane holds eight consecutive columns (always the same ones) of
  // every ROWS-th row.  All of a block's loads are in flight at once, and every choice is made once per block.
  constexpr int PART = 64, LDC = PART + 4, LPR = PART / 8, ROWS = 64 / LPR, N8 = 32 / ROWS;
  const LinEpilogue& e = g.e;
  float* const cs = (float*)(smem + wave * (32 * LDC * 4));
  const int c8 = (lane % LPR) * 8, r8 = lane / LPR;
  const int64_t col = col0 + wn * PART + c8;
  const bool in = col < g.n;
  float bias[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) bias[u] = e.bias && in ? e.bias[col + u] : 0.0f;
#pragma unroll
  for (int i = 0; i < MT; i += 2) {
    const int64_t row = row0 + wm * 128 + 16 * i + r8;
    bf16x8 res[N8];
    if (e.R) {
#pragma unroll
      for (int q = 0; q < N8; ++q) {
        const int64_t at = row + ROWS * q < g.m ? row + ROWS * q : g.m - 1;
        res[q] = *(const bf16x8*)((const bf16_t*)e.R + at * e.ldr + (in ? col : 0));
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < NT; ++j) *(f32x4*)(cs + (16 * h + (lane & 15)) * LDC + 16 * j + 4 * (lane >> 4)) = acc[i + h][j];
    sb_wave_sync();
    float y[N8][8];
#pragma unroll
    for (int q = 0; q < N8; ++q) {
      const f32x4 lo = *(const f32x4*)(cs + (r8 + ROWS * q) * LDC + c8), hi = *(const f32x4*)(cs + (r8 + ROWS * q) * LDC + c8 + 4);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        y[q][u] = lo[u] + bias[u];
        y[q][4 + u] = hi[u] + bias[4 + u];
      }
    }
    sb_wave_sync();
    if (e.Z && in) {
#pragma unroll
      for (int q = 0; q < N8; ++q) {
        bf16x8 z;
#pragma unroll
        for (int u = 0; u < 8; ++u) z[u] = (bf16_t)y[q][u];
        if (row + ROWS * q < g.m) *(bf16x8*)((bf16_t*)e.Z + (row + ROWS * q) * e.ldz + col) = z;
      }
    }
    if (e.act != LORACT_ACT_NONE) {
#pragma unroll
      for (int q = 0; q < N8; ++q)
#pragma unroll
        for (int u = 0; u < 8; ++u) y[q][u] = lin_act<true>(e.act, y[q][u]);
    }
    if (e.d.thr) {
#pragma unroll
      for (int q = 0; q < N8; ++q) {
        const uint64_t w0 = drop_word(e.d, row + ROWS * q, col / 4), w1 = drop_word(e.d, row + ROWS * q, col / 4 + 1);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          y[q][u] = drop_one(e.d, w0, u, y[q][u]);
          y[q][4 + u] = drop_one(e.d, w1, u, y[q][4 + u]);
        }
      }
    }
    if (e.R) {
#pragma unroll
      for (int q = 0; q < N8; ++q)
#pragma unroll
        for (int u = 0; u < 8; ++u) y[q][u] += (float)res[q][u];
    }
#pragma unroll
    for (int q = 0; q < N8; ++q) {
      if (!in || row + ROWS * q >= g.m) continue;
      if (e.y_f32) {
        float* out = (float*)e.Y + (row + ROWS * q) * e.ldy + col;
        *(f32x4*)out = (f32x4){y[q][0], y[q][1], y[q][2], y[q][3]};
        *(f32x4*)(out + 4) = (f32x4){y[q][4], y[q][5], y[q][6], y[q][7]};
      } else {
        bf16x8 o;
#pragma unroll
        for (int u = 0; u < 8; ++u) o[u] = (bf16_t)y[q][u];
        *(bf16x8*)((bf16_t*)e.Y + (row + ROWS * q) * e.ldy + col) = o;
      }
    }
  }
}

// What the tiles of 256 x 256 need: 16-byte pieces of everything, and 32 bits for the byte offsets within a tile.
static bool linear_large_fits(const LinearArgs& g, bool w_kc) {
  auto rows = [](const void* p, int64_t ld) { return !p || ((uintptr_t)p % 16 == 0 && ld % 8 == 0); };
  return g.k % 8 == 0 && g.n % 8 == 0 && rows(g.X, g.ldx) && rows(g.W, g.ldw) && rows(g.e.R, g.e.ldr) &&
         rows(g.e.Y, g.e.ldy) && rows(g.e.Z, g.e.ldz) && g.ldx < (1 << 22) && g.ldw < (w_kc ? 1 << 22 : 1 << 25) &&
         ceil_div64(g.m, 256) * ceil_div64(g.n, 256) < (1 << 24);
}
static bool linear_large_pays(int64_t m, int64_t n, int64_t k) {
  return ceil_div64(m, 256) * ceil_div64(n, 256) >= 128 && m >= 192 && n >= 192 && k >= 128;
}

// T and B where their rows are not 16-byte pieces: copies with the rank rounded up to a multiple of 8, zeros in between.
__global__ __launch_bounds__(256) void linear_pad_kernel(const bf16_t* T, const bf16_t* B, int64_t m, int64_t n, int r, int rp, bf16_t* Tp, bf16_t* Bp) {
  const int64_t step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t e = first; e < m * rp; e += step) {
    const int64_t row = e / rp;
    const int c = (int)(e - row * rp);
    Tp[e] = c < r ? T[row * r + c] : (bf16_t)0.0f;
  }
  for (int64_t e = first; e < rp * n; e += step) Bp[e] = e < r * n ? B[e] : (bf16_t)0.0f;
}
static int64_t linear_pad_rank(int64_t r) { return (r + 7) / 8 * 8; }
static size_t linear_large_ws_bytes(int64_t m, int64_t n, int64_t r) { return r ? align_up((size_t)(m + n) * linear_pad_rank(r) * 2, 256) : 0; }

static int launch_linear_large(hipStream_t s, LinearArgs g, bool w_kc) {
  if (g.T && (g.r % 8 || (uintptr_t)g.T % 16 || (uintptr_t)g.B % 16)) {
    const int rp = (int)linear_pad_rank(g.r);
    bf16_t* const tp = (bf16_t*)g.part;
    bf16_t* const bp = tp + g.m * rp;                  // (m rp elements are a multiple of 16 bytes)
    const int64_t blocks = std::min<int64_t>(ceil_div64(std::max(g.m, g.n) * rp, 256), 1024);
    LORACT_LAUNCH("linear_pad", s, linear_pad_kernel, dim3((unsigned)blocks), dim3(256), 0, (const bf16_t*)g.T, (const bf16_t*)g.B, g.m, g.n,
                  (int)g.r, rp, tp, bp);
    g.T = tp; g.B = bp; g.r = rp;
  }
  const int tm = (int)ceil_div64(g.m, 256), tn = (int)ceil_div64(g.n, 256);
  if (w_kc) LORACT_LAUNCH("linear_large", s, (linear_large_kernel<true>), dim3((unsigned)(tm * tn)), dim3(64 * LL_WAVES), 0, g, tm, tn);
  else LORACT_LAUNCH("linear_large", s, (linear_large_kernel<false>), dim3((unsigned)(tm * tn)), dim3(64 * LL_WAVES), 0, g, tm, tn);
  return LORACT_OK;
}

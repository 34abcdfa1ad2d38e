// P = X W^T + s T B for bf16 maps whose rows are 16-byte pieces: tiles of 256 x 256 or 128 x 128 on v_mfma_f32_16x16x32_bf16.
//
// Slabs of 64 of K -- whole 128-byte lines of X and of W -- go from memory straight into LDS (asynchronous copies): three stages for
// X, fetched up to three slabs ahead, and two for W, 160 KB in all (80 KB for the smaller tiles, of which a CU holds two).  A
// stage holds the tile's rows as [row][64] or, for W stored n_in x n_out, 64 rows of it as they lie ([k][columns], read with the transposing LDS read).  A wave reads the fragments of the next 32 of K
// while it multiplies the present ones; there is one barrier per slab, behind the first products of its second half.
//
// Bound by power, then by the issue of the products: the matrix units of a busy CU work 60 to 70 % of the time at a clock that has
// fallen to 1.6 to 1.9 of 2.4 GHz.  What lowers the energy of a product raised the rate: whole lines (slabs of 32 of K, half a line of X and
// of W per row: 8192 x 8192 -> 2048 203 us against 194), products of 16 x 16 x 32 rather than 32 x 32 x 16, which move half the
// accumulators (218 against 205 of W as it lies).  Four waves of 128 x 128 with all accumulators in 256 accumulation registers
// read a third less from LDS and were no faster (225): alone on its matrix unit, a wave that waits for the issue of a copy leaves it idle.
// 8192 x 4096 -> 4096 199 to 214 us from one program to another (1384 to 1284 TFLOP/s), 8192 x 4096 -> 11008 605 (1221: 1376 tiles are 5.4 rounds), 8192 x 11008 -> 4096 of W as it
// lies 556 (1329); a library's plain products take 177, 636 and 537 us beside 199, 605 and 556.
#pragma once
#include "linear_tile.h"

#include <type_traits>

typedef bf16x8 bf16x8_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

#define LL_BK 64
#define LL_X_STAGES 3
#define LL_W_STAGES 2

// XCD b % 8 takes a run of consecutive tiles; within it tiles go in bands of LL_BAND tile rows, so that the tiles that are in
// flight on one XCD share rows of X and of W in its L2.
#define LL_BAND 4
__device__ inline void ll_tile_of(int b, int tiles_m, int tiles_n, int* tm, int* tn) {
  const int total = tiles_m * tiles_n;
  const int xcd = b & 7, per = total >> 3, rest = total & 7;
  const int id = xcd * per + (xcd < rest ? xcd : rest) + (b >> 3);
  const int band = id / (LL_BAND * tiles_n), in = id - band * (LL_BAND * tiles_n);
  const int rows = tiles_m - band * LL_BAND < LL_BAND ? tiles_m - band * LL_BAND : LL_BAND;
  *tn = in / rows;
  *tm = band * LL_BAND + in - *tn * rows;
}

template <int PITCH>
__device__ inline bf16x8 ll_read_tr(const unsigned char* lds, int off) {
  typedef __attribute__((address_space(3))) gb_s16x4* lds_ptr;
  const gb_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + off));
  const gb_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(lds + off + 4 * PITCH));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
// Where the 16-byte chunks of a row lie: chunk c of row r (along K) at c ^ ll_turn(r), chunk c of row k of W as it lies at
// c ^ ll_turn_k(k).  The 16 lanes that LDS serves at a time (256 bytes) then read from 16 different groups of banks, whether these are 16
// neighbours or four runs of four (counted: no conflicts).
__device__ inline int ll_turn(int r) { return (r >> 1) & 7; }
__device__ inline int ll_turn_k(int k) { return 4 * (k & 3) + ((k >> 2) & 2); }

// Waves of a tile (TILE / 2 x 64 each), in two rows.
constexpr int ll_waves(int tile) { return tile / 32; }

// blockIdx.x: tile, blockIdx.y: split of K.  Y_F32: Y is float32, and its activations the refined ones.
template <bool WKC, int TILE, bool Y_F32>
__global__ __launch_bounds__(64 * ll_waves(TILE), TILE == 256 ? 1 : 2) void linear_large_kernel(LinearArgs g, int tiles_m, int tiles_n) {
  constexpr int WAVES = ll_waves(TILE), WN = TILE / 64, MT = TILE / 32, NT = 4;      // a wave: MT x NT products of 16 x 16
  constexpr int C = TILE / 8 / WAVES;                    // copies of 1 KB per operand and slab
  constexpr int STAGE = TILE * LL_BK * 2, PITCH = TILE * 2, LPK = PITCH / 16, KPC = 64 / LPK;      // W as it lies: lanes to a row, rows to a copy
  __shared__ __attribute__((aligned(16))) unsigned char smem[(LL_X_STAGES + LL_W_STAGES) * STAGE];
  unsigned char* const smem_w = smem + LL_X_STAGES * STAGE;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int wm = wave / WN, wn = wave % WN;
  int tm, tn;
  ll_tile_of(blockIdx.x, tiles_m, tiles_n, &tm, &tn);
  const int64_t row0 = (int64_t)tm * TILE, col0 = (int64_t)tn * TILE;
  const int64_t k_beg = (int64_t)blockIdx.y * g.k_per_split;
  const int k_len = (int)(k_beg + g.k_per_split < g.k ? g.k_per_split : g.k - k_beg), full = k_len / LL_BK, nslab = (k_len + LL_BK - 1) / LL_BK;

  const char* const xb = (const char*)((const bf16_t*)g.X + row0 * g.ldx + k_beg);
  const char* const wb = (const char*)((const bf16_t*)g.W + (WKC ? col0 * g.ldw + k_beg : col0 + k_beg * g.ldw));
  const int64_t w_step = WKC ? 2 * LL_BK : 2 * LL_BK * g.ldw;
  // copy c of a wave: 8 rows of 128 bytes along K, or KPC whole rows of W as it lies
  const int copy_row = 8 * wave * C + (lane >> 3), copy_k = KPC * wave * C + lane / LPK;
  auto chunk_of = [&](int c) { return (lane & 7) ^ ll_turn(copy_row + 8 * c); };
  auto col_of = [&](int c, int64_t n8) {
    const int64_t col = ((lane % LPK) ^ ll_turn_k(copy_k + KPC * c)) * 8;
    return col0 + col < n8 ? col : n8 - 8 - col0;                           // columns past the end are never stored
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
      wo[c] = (unsigned)((copy_k + KPC * c) * g.ldw * 2) + (unsigned)col_of(c, g.w_n8) * 2;
    }
  }
  // Slabs are numbered through: the one of T and B, if there is a low-rank term, then those of X and W.
  const int r = g.T && blockIdx.y == 0 ? (int)g.r : 0, nlr = r ? 1 : 0, slabs = nlr + nslab;
  auto x_stage = [&](int v) { return smem + v % LL_X_STAGES * STAGE; };
  auto w_stage = [&](int v) { return smem_w + v % LL_W_STAGES * STAGE; };
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
      const int kr = copy_k + KPC * c, chunk = chunk_of(c);
      if (v < nlr)
        sb_async16((const bf16_t*)g.B + (int64_t)(kr < left ? kr : left - 1) * g.ldb + col0 + col_of(c, g.b_n8), st + c * 1024);
      else if (WKC)
        sb_async16_at(ws, wo[c] - (chunk * 8 < left ? 0 : chunk * 16), st + c * 1024);
      else
        sb_async16_at(ws, wo[c] - (unsigned)((kr < left ? 0 : kr - left + 1) * g.ldw * 2), st + c * 1024);
    }
  };

  // fragments: 16 rows (columns), lane l holds row l % 16 and the eight k from 8 (l / 16) on of a half slab
  const int k_off[2] = {((lane >> 4) ^ ll_turn(lane & 15)) << 4, ((4 + (lane >> 4)) ^ ll_turn(lane & 15)) << 4};
  const int xr_off = (wm * (TILE / 2) + (lane & 15)) * 128, wr_off = (wn * 64 + (lane & 15)) * 128;
  int tr_off[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int s16 = lane & 15, kr = 8 * (lane >> 4) + (s16 >> 2), c = wn * 64 + 16 * j + 4 * (s16 & 3);
    tr_off[j] = kr * PITCH + (((c >> 3) ^ ll_turn_k(kr)) << 4) + (c & 7) * 2;
  }
  bf16x8 x[2][MT], w[2][NT];
  // fragment f of half h of a slab: those of W, then those of X
  auto read_one = [&](const unsigned char* xs, const unsigned char* ws, int h, bool w_kc, int f) {
    if (f < NT) w[h][f] = w_kc ? *(const bf16x8*)(ws + wr_off + k_off[h] + f * 2048) : ll_read_tr<PITCH>(ws, tr_off[f] + h * (32 * PITCH));
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
      if (u % 2 == 0 && u / 2 < MT + NT) read_one(xs, ws, 1, WKC, u / 2);
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
      constexpr int RS = TILE == 256 ? 2 : 1, CS = TILE == 256 ? 3 : 1;      // products from one read or copy to the next
      if (u >= 4 && (u - 4) % RS == 0 && (u - 4) / RS < MT + NT) read_one(xs, ws, 0, WKC, (u - 4) / RS);
      if (u >= 4 && (u - 4) % CS == 0 && (u - 4) / CS < 2 * C) {
        const int c = (u - 4) / CS;
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
  // (pieces of R, Z and Y at any address; the last one of a row whose length is no multiple of 8 goes element by element)
  const bool in = col < g.n, whole = col + 8 <= g.n, split = gridDim.y > 1;
  auto store = [&](bf16_t* out, const float (&v)[8]) {
    bf16x8 o;
#pragma unroll
    for (int u = 0; u < 8; ++u) o[u] = (bf16_t)v[u];
    if (whole) {
      *(bf16x8_any*)out = o;
    } else {
#pragma unroll
      for (int u = 0; u < 8; ++u)
        if (col + u < g.n) out[u] = o[u];
    }
  };
  float bias[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) bias[u] = e.bias && col + u < g.n && !split ? e.bias[col + u] : 0.0f;
#pragma unroll
  for (int i = 0; i < MT; i += 2) {
    const int64_t row = row0 + wm * (TILE / 2) + 16 * i + r8;
    bf16x8 res[N8];
    if (e.R && !split) {
#pragma unroll
      for (int q = 0; q < N8; ++q) {
        const int64_t at = row + ROWS * q < g.m ? row + ROWS * q : g.m - 1;
        const bf16_t* const src = (const bf16_t*)e.R + at * e.ldr + col;
        if (whole) {
          res[q] = *(const bf16x8_any*)src;
        } else {
#pragma unroll
          for (int u = 0; u < 8; ++u) res[q][u] = col + u < g.n ? src[u] : (bf16_t)0.0f;
        }
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
    if (split) {
#pragma unroll
      for (int q = 0; q < N8; ++q) {
        if (!in || row + ROWS * q >= g.m) continue;
        float* out = g.part + ((int64_t)blockIdx.y * g.m + row + ROWS * q) * g.n_pad + col;       // (n_pad: a multiple of 8)
        *(f32x4*)out = (f32x4){y[q][0], y[q][1], y[q][2], y[q][3]};
        *(f32x4*)(out + 4) = (f32x4){y[q][4], y[q][5], y[q][6], y[q][7]};
      }
      continue;
    }
    if (e.Z && in) {
#pragma unroll
      for (int q = 0; q < N8; ++q)
        if (row + ROWS * q < g.m) store((bf16_t*)e.Z + (row + ROWS * q) * e.ldz + col, y[q]);
    }
#pragma unroll
    for (int q = 0; q < N8; ++q) lin_act<Y_F32>(e.act, y[q]);
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
      if (!Y_F32) {
        store((bf16_t*)e.Y + (row + ROWS * q) * e.ldy + col, y[q]);
        continue;
      }
      float* const out = (float*)e.Y + (row + ROWS * q) * e.ldy + col;
      if (whole) {
        *(f32x4_any*)out = (f32x4){y[q][0], y[q][1], y[q][2], y[q][3]};
        *(f32x4_any*)(out + 4) = (f32x4){y[q][4], y[q][5], y[q][6], y[q][7]};
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (col + u < g.n) out[u] = y[q][u];
      }
    }
  }
}

// Tile (0: another form) and K splits.
//
// Costs in hundredths of a round of 256 tiles of 256 x 256, one per CU: a last round of few of them takes two thirds of one; 512
// tiles of 128 x 128, two per CU, take 62 (a quarter of the work at 40 % of the rate: half the products per byte fetched), 256
// 35.  Measured (256 / 128 x 128): 2048 x 2048 -> 2048 46 / 26 us, 8192 x 4096 -> 1024 92 / 70, 6000 x 4096 -> 3000 177 / 165, 2048 x
// 4096 -> 11008 195 / 195, 5000 x 2048 -> 2048 48 / 52, 4096 x 4096 -> 4096 123 / 155, 8192 x 4096 -> 11008 619 / 725.
// Where even the smaller tiles leave CUs without work, K is split in parts of at least 512: 256 x 4096 -> 4096 36 -> 24 us, 128 x
// 11008 -> 4096 124 -> 33; more than one workgroup per CU loses to the join (2048 x 2048 -> 2048 26 -> 39).  What this leaves: 256 x 4096 ->
// 4096 is at 3.5 times its floor of bytes (a library's product 22 us), 128 x 11008 -> 4096 at 1.7 (56), 1024 x 4096 -> 4096 50 us (41).
struct LargePlan {
  int tile, splits;
};
static LargePlan linear_large_plan(int64_t m, int64_t n, int64_t k) {
  LargePlan p = {0, 1};
  if (m <= 64 || n <= 64 || k < 64) return p;
  const int64_t t256 = ceil_div64(m, 256) * ceil_div64(n, 256), t128 = ceil_div64(m, 128) * ceil_div64(n, 128);
  if (t128 >= 1 << 23) return p;
  const int64_t last256 = t256 % 256, last128 = t128 % 512;
  const int64_t cost256 = t256 / 256 * 100 + (last256 ? 66 + 34 * last256 / 256 : 0);
  const int64_t cost128 = t128 / 512 * 62 + (last128 > 256 ? 60 : (last128 ? 35 : 0));
  p.tile = cost256 <= cost128 ? 256 : 128;
  if (p.tile == 128) p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(256 / t128, k / 512));
  return p;
}
// Operands whose rows are not 16-byte pieces are copied first: rows x cols into rows_p x cols_p (a multiple of 8), zeros in between.
struct PadArgs {
  const bf16_t* src;
  int64_t ld, rows, cols;
  bf16_t* dst;
  int64_t rows_p, cols_p;
};
__global__ __launch_bounds__(256) void linear_pad_kernel(PadArgs a, PadArgs b) {
  const PadArgs& p = blockIdx.y ? b : a;
  const int64_t per_row = p.cols_p / 8, step = (int64_t)gridDim.x * 256;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < p.rows_p * per_row; e += step) {
    const int64_t row = e / per_row, c = (e - row * per_row) * 8;
    const bf16_t* src = p.src + row * p.ld + c;
    bf16x8 v = {};
    if (row < p.rows) {
      if (c + 8 <= p.cols) {
        v = *(const bf16x8_any*)src;
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (c + u < p.cols) v[u] = src[u];
      }
    }
    *(bf16x8*)(p.dst + e * 8) = v;
  }
}
static int launch_linear_pad(hipStream_t s, PadArgs a, PadArgs b) {
  if (!a.src && !b.src) return LORACT_OK;
  if (!a.src) a = b;
  const int64_t pieces = std::max(a.rows_p * a.cols_p, b.src ? b.rows_p * b.cols_p : 0) / 8;
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div64(pieces, 256), 2048), b.src && b.dst != a.dst ? 2 : 1);
  LORACT_LAUNCH("linear_pad", s, linear_pad_kernel, grid, dim3(256), 0, a, b);
  return LORACT_OK;
}

// What a call copies, by sizes and strides alone, so that the workspace can be told in advance.
struct LargeSpace {
  bool pad_x, pad_w;
  int64_t k8, n8, r8;
  size_t off_t, off_b, off_x, off_w, off_part, total;
};
static LargeSpace linear_large_space(const LargePlan& p, int64_t m, int64_t n, int64_t k, int64_t r, int64_t ldx, int64_t ldw, bool w_kc) {
  LargeSpace q;
  auto up8 = [](int64_t v) { return (v + 7) / 8 * 8; };
  q.k8 = up8(k); q.n8 = up8(n); q.r8 = up8(r);
  q.pad_x = k % 8 || ldx % 8;
  q.pad_w = ldw % 8 || k % 8 || (!w_kc && n % 8);
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, 256); return o; };
  q.off_t = take((size_t)m * q.r8 * 2);
  q.off_b = take((size_t)q.r8 * q.n8 * 2);
  q.off_x = take(q.pad_x ? (size_t)m * q.k8 * 2 : 0);
  q.off_w = take(q.pad_w ? (size_t)(w_kc ? n * q.k8 : q.k8 * q.n8) * 2 : 0);
  q.off_part = take(p.splits > 1 ? (size_t)p.splits * m * q.n8 * 4 : 0);
  q.total = off;
  return q;
}
// The copies read and write X and W once, the general tiles take twice the time: 8192 x 4095 -> 4096 248 us against 444, 2001 x 501 ->
// 2001 19 / 23, 513 x 3001 -> 2001 30 / 32; 700 x 1030 -> 700 20 / 16, 100 x 4001 -> 4001 31 / 23.
static bool linear_large_pays(const LargeSpace& q, int64_t m, int64_t n) {
  return (!q.pad_x && !q.pad_w) || m * n >= (m + n) * 400;
}
// 32 bits have to do for the byte offsets within a tile; an operand that is not copied has to start on 16 bytes.
static bool linear_large_fits(const LinearArgs& g, bool w_kc, const LargeSpace& q) {
  return (q.pad_x || ((uintptr_t)g.X % 16 == 0 && g.ldx < (1 << 22))) && q.k8 < (1 << 22) && q.n8 < (1 << 24) &&
         (q.pad_w || ((uintptr_t)g.W % 16 == 0 && g.ldw < (w_kc ? 1 << 22 : 1 << 24)));
}

static int launch_linear_large(hipStream_t s, LinearArgs g, bool w_kc, LargePlan p, const LargeSpace& q) {
  char* const ws = (char*)g.part;
  g.part = (float*)(ws + q.off_part);
  PadArgs pt{}, pb{}, px{}, pw{};
  g.ldb = g.n;
  g.b_n8 = g.n;
  if (g.T && (g.r % 8 || (uintptr_t)g.T % 16 || (uintptr_t)g.B % 16 || g.n % 8)) {
    pt = {(const bf16_t*)g.T, g.r, g.m, g.r, (bf16_t*)(ws + q.off_t), g.m, q.r8};
    pb = {(const bf16_t*)g.B, g.n, g.r, g.n, (bf16_t*)(ws + q.off_b), q.r8, q.n8};
    g.T = pt.dst; g.B = pb.dst; g.r = q.r8; g.ldb = g.b_n8 = q.n8;
  }
  g.w_n8 = g.n;
  if (q.pad_x) {
    px = {(const bf16_t*)g.X, g.ldx, g.m, g.k, (bf16_t*)(ws + q.off_x), g.m, q.k8};
    g.X = px.dst; g.ldx = q.k8;
  }
  if (q.pad_w) {
    pw = {(const bf16_t*)g.W, g.ldw, w_kc ? g.n : g.k, w_kc ? g.k : g.n, (bf16_t*)(ws + q.off_w), w_kc ? g.n : q.k8, w_kc ? q.k8 : q.n8};
    g.W = pw.dst; g.ldw = w_kc ? q.k8 : q.n8; g.w_n8 = q.n8;
  }
  LORACT_TRY(launch_linear_pad(s, pt, pb));
  LORACT_TRY(launch_linear_pad(s, px, pw));
  // (an operand that is not copied has whole pieces along K, or is the one that decides that neither is)
  g.k = q.pad_x && q.pad_w ? q.k8 : g.k;
  g.k_per_split = ceil_div64(ceil_div64(g.k, p.splits), LL_BK) * LL_BK;
  p.splits = (int)ceil_div64(g.k, g.k_per_split);
  g.n_pad = q.n8;
  const int tm = (int)ceil_div64(g.m, p.tile), tn = (int)ceil_div64(g.n, p.tile);
  const dim3 grid((unsigned)(tm * tn), (unsigned)p.splits), block(64 * ll_waves(p.tile));
#define LL_LAUNCH(KC, TILE)                                                                                                          \
  {                                                                                                                                 \
    if (g.e.y_f32) LORACT_LAUNCH("linear_large", s, (linear_large_kernel<KC, TILE, true>), grid, block, 0, g, tm, tn);                \
    else LORACT_LAUNCH("linear_large", s, (linear_large_kernel<KC, TILE, false>), grid, block, 0, g, tm, tn);                         \
  }
  if (p.tile == 256) { if (w_kc) LL_LAUNCH(true, 256) else LL_LAUNCH(false, 256) }
  else { if (w_kc) LL_LAUNCH(true, 128) else LL_LAUNCH(false, 128) }
#undef LL_LAUNCH
  return p.splits > 1 ? launch_linear_join<bf16_t>(s, g, p.splits) : LORACT_OK;
}

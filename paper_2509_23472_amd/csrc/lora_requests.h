// The low-rank adapters of many requests beside a projection that they share: Y_i = R_i + s_a (X_i A_a) B_a, a = ids_i, in two launches.
//
//   down   T = X A: tokens in tiles, in order; a tile goes over the different adapters of its tokens (found by ballots: no sorting, no plan
//          on the host) and takes from each product the columns of the tokens that it belongs to.  An adapter's infinities and NaN thus reach its own
//          tokens only.  K is split between the eight waves of a workgroup, whose sums are added in LDS, and between workgroups, whose
//          parts the second launch adds as it reads them (no third launch, no atomics).
//   up     Y = R + s T B: a wave has 16 E columns and a tile of tokens; the same walk, rows of Y written as their adapter comes.
//
// bf16 T enters the second product as the sum of two bf16 numbers: 16 bits of it for one more matrix instruction, where one rounding
// would weigh as much as the output's own.
//
// Bound by memory: single tokens by A and B, prompts by X, R and Y.  Few tokens with an adapter each: the walk is shared out over workgroups too.
#pragma once
#include "common.h"
#include "frag.h"

#include <algorithm>

#define LQ_WAVES 8                                   // of the first launch
#define LQ_UP_WAVES 4

struct LqArgs {
  const void* X;
  int64_t ldx;
  const void *A, *B;     // adapters x k x r, adapters x r x n
  const int32_t* ids;
  const float* scales;   // or null
  const void* R;
  int64_t ldr;
  void* Y;
  int64_t ldy;
  int64_t m, k, n, adapters;
  int r;
  bool a_pieces, b_pieces;           // rows of A and B are whole 16-byte pieces
  bool in_place;
  float* part;           // splits x m x ldt
  int ldt, splits, shares;           // shares: workgroups (z) that share the adapters of a tile
  int64_t k_per_split;
};

// Walks over the different adapters of a tile: f(adapter, lanes whose tokens have it) for those that are the share's.
template <typename F>
__device__ inline void lq_adapters(const LqArgs& g, int id, bool live, int share, F f) {
  uint64_t left = __ballot(live && id >= 0 && (int64_t)id < g.adapters);
  for (int rank = 0; left; ++rank) {
    const int d = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
    const uint64_t same = __ballot(live && id == d);
    left &= ~same;
    if (rank % g.shares == share) f(d, same);
  }
}

// E elements from `at` on, of which `left` are there; zeros behind.
template <typename T>
__device__ inline typename Ln<T>::frag lq_load(const T* at, int64_t left) {
  constexpr int E = Ln<T>::E;
  if (left >= E) return *(const typename Ln<T>::frag_any*)at;
  typename Ln<T>::frag v = {};
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (e < left) v[e] = at[e];
  return v;
}

// TB: blocks of 16 tokens per tile.  SB: blocks of 16 columns of A.
template <typename T, int TB, int SB>
__global__ __launch_bounds__(64 * LQ_WAVES) void lora_down_kernel(LqArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP, U = SB == 1 ? 4 : 2, QUADS = TB * SB * 64, PER = 16 / E;
  typedef typename Ln<T>::frag frag;
  constexpr int TURN_BYTES = LQ_WAVES * U * SB * 1024, PART_BYTES = LQ_WAVES * QUADS * 16;
  __shared__ __attribute__((aligned(16))) unsigned char smem[TURN_BYTES > PART_BYTES ? TURN_BYTES : PART_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t first = (int64_t)blockIdx.x * (16 * TB);
  const int64_t mine = first + (lane < 16 * TB ? lane : 0);
  const bool live = lane < 16 * TB && mine < g.m;
  const int id = live ? g.ids[mine] : -1;
  const int64_t k_beg0 = (int64_t)blockIdx.y * g.k_per_split, k_end0 = k_beg0 + g.k_per_split < g.k ? k_beg0 + g.k_per_split : g.k;
  const int64_t per = ((k_end0 - k_beg0 + STEP * LQ_WAVES - 1) / (STEP * LQ_WAVES)) * STEP;
  const int64_t k_beg = k_beg0 + wave * per, k_end = k_beg + per < k_end0 ? k_beg + per : k_end0;
  const T* x[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) x[b] = (const T*)g.X + (first + 16 * b + c < g.m ? first + 16 * b + c : g.m - 1) * g.ldx;
  f32x4 total[TB][SB];
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int s = 0; s < SB; ++s) total[b][s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  unsigned char* const turn = smem + wave * (U * SB * 1024);
  uint64_t done = 0;
  lq_adapters(g, id, live, blockIdx.z, [&](int d, uint64_t same) {
    done |= same;
    const T* const a = (const T*)g.A + (int64_t)d * g.k * g.r;
    f32x4 acc[TB][SB];
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
      for (int s = 0; s < SB; ++s) acc[b][s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t k0 = k_beg; k0 < k_end; k0 += STEP * U) {
      frag st[U][TB], sm[U][SB];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + STEP * u + E * q, row = k0 + STEP * u + lane / PER;
#pragma unroll
        for (int b = 0; b < TB; ++b) st[u][b] = lq_load<T>(x[b] + k, k_end - k);
#pragma unroll
        for (int s = 0; s < SB; ++s) {
          const int col = 16 * s + E * (lane % PER);
          if (g.a_pieces) {
            sm[u][s] = (frag){};
            if (row < k_end && col < g.r) sm[u][s] = *(const frag*)(a + row * g.r + col);
          } else {
            sm[u][s] = lq_load<T>(a + row * g.r + col, row < k_end ? g.r - col : 0);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SB; ++s) *(frag*)(turn + (u * SB + s) * 1024 + lane * 16) = sm[u][s];
      sb_wave_sync();
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SB; ++s) {
          const unsigned char* at = turn + (u * SB + s) * 1024;
          if constexpr (sizeof(T) == 2) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4* lds_ptr;
            at += (8 * q + (c >> 2)) * 32 + (c & 3) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * 32));
            sm[u][s] = __builtin_bit_cast(frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) sm[u][s][e] = *(const T*)(at + (E * q + e) * 64 + c * 4);
          }
        }
      sb_wave_sync();
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int b = 0; b < TB; ++b)
#pragma unroll
          for (int s = 0; s < SB; ++s) acc[b][s] = ln_mfma(sm[u][s], st[u][b], acc[b][s]);
    }
#pragma unroll
    for (int b = 0; b < TB; ++b) {                   // a lane's column is token c of the block
      const bool own = same >> (16 * b + c) & 1;
#pragma unroll
      for (int s = 0; s < SB; ++s)
#pragma unroll
        for (int u = 0; u < 4; ++u) total[b][s][u] = own ? acc[b][s][u] : total[b][s][u];
    }
  });
  if (!done) return;                                 // (the same for all waves)
  __syncthreads();
  f32x4* const part = (f32x4*)smem;
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int s = 0; s < SB; ++s) part[wave * QUADS + (b * SB + s) * 64 + lane] = total[b][s];
  __syncthreads();
  for (int i = threadIdx.x; i < QUADS; i += 64 * LQ_WAVES) {
    const int b = i / (64 * SB), s = i / 64 % SB, l = i & 63;
    f32x4 v = part[i];
#pragma unroll
    for (int w = 1; w < LQ_WAVES; ++w) v += part[w * QUADS + i];
    if (done >> (16 * b + (l & 15)) & 1)
      *(f32x4*)(g.part + ((int64_t)blockIdx.y * g.m + first + 16 * b + (l & 15)) * g.ldt + 16 * s + 4 * (l >> 4)) = v;
  }
}

template <typename O, int E>
struct LqOut {
  typedef O vec __attribute__((ext_vector_type(E)));
  typedef vec any __attribute__((aligned(sizeof(O))));
};
// RS: steps of the rank.  TB: blocks of 16 tokens per wave.
template <typename T, typename O, int TB, int RS>
__global__ __launch_bounds__(64 * LQ_UP_WAVES) void lora_up_kernel(LqArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP;
  typedef typename Ln<T>::frag frag;
  typedef typename LqOut<O, E>::any out_any;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t col = ((int64_t)blockIdx.y * LQ_UP_WAVES + wave) * (16 * E) + E * c;       // of this lane's E columns
  if (col - E * c >= g.n) return;
  const int64_t first = (int64_t)blockIdx.x * (16 * TB);
  const int64_t mine = first + (lane < 16 * TB ? lane : 0);
  const bool live = lane < 16 * TB && mine < g.m;
  const int id = live ? g.ids[mine] : -1;
  const float scale = live && id >= 0 && id < g.adapters ? (g.scales ? g.scales[id] : 1.0f) : 0.0f;
  const int here = g.n - col < E ? (int)(g.n - col < 0 ? 0 : g.n - col) : E;                // columns that exist
  auto put = [&](int64_t token, const float (&v)[E]) {
    const O* const rp = (const O*)g.R + token * g.ldr + col;
    O* const yp = (O*)g.Y + token * g.ldy + col;
    if (here == E) {
      typename LqOut<O, E>::vec y;
      if (g.R) {
        y = *(const out_any*)rp;
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = (O)((float)y[e] + v[e]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = (O)v[e];
      }
      *(out_any*)yp = y;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < here) yp[e] = (O)((g.R ? (float)rp[e] : 0.0f) + v[e]);
    }
  };
  lq_adapters(g, id, live, blockIdx.z, [&](int d, uint64_t same) {
    // the lane's E x E blocks of B, turned: f[s][j] has column E c + j, rows STEP s + E q ..
    frag f[RS][E];
    const T* const b0 = (const T*)g.B + (int64_t)d * g.r * g.n + col;
#pragma unroll
    for (int s = 0; s < RS; ++s) {
      frag v[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int row = STEP * s + E * q + i;
        if (g.b_pieces) {
          v[i] = (frag){};
          if (row < g.r && here == E) v[i] = *(const frag*)(b0 + (int64_t)row * g.n);
        } else {
          v[i] = lq_load<T>(b0 + (int64_t)row * g.n, row < g.r ? here : 0);
        }
      }
#pragma unroll
      for (int j = 0; j < E; ++j) {
        if constexpr (sizeof(T) == 2) {
          typedef unsigned int words __attribute__((ext_vector_type(4)));
          words w;
#pragma unroll
          for (int p = 0; p < 4; ++p)
            w[p] = __builtin_amdgcn_perm(__builtin_bit_cast(words, v[2 * p + 1])[j / 2], __builtin_bit_cast(words, v[2 * p])[j / 2],
                                         j & 1 ? 0x07060302u : 0x05040100u);
          f[s][j] = __builtin_bit_cast(frag, w);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) f[s][j][e] = v[e][j];
        }
      }
    }
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const unsigned rows = (unsigned)(same >> (16 * b)) & 0xffffu;
      if (!rows) continue;
      const int64_t token = first + 16 * b + c < g.m ? first + 16 * b + c : g.m - 1;
      const float by = __shfl(scale, 16 * b + c);
      f32x4 acc[E];
#pragma unroll
      for (int j = 0; j < E; ++j) acc[j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int s = 0; s < RS; ++s) {
        float t[E];
#pragma unroll
        for (int e = 0; e < E; ++e) t[e] = 0.0f;
        const int k = STEP * s + E * q;
        if ((rows >> c & 1) && k < g.r) {            // (rows of other adapters may not be written at all)
          for (int p = 0; p < g.splits; ++p) {
            const float* at = g.part + ((int64_t)p * g.m + token) * g.ldt + k;
#pragma unroll
            for (int h = 0; h < E / 4; ++h) {
              const f32x4 v = *(const f32x4*)(at + 4 * h);
#pragma unroll
              for (int e = 0; e < 4; ++e) t[4 * h + e] += v[e];
            }
          }
        }
        frag hi, lo;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float v = k + e < g.r ? t[e] * by : 0.0f;
          hi[e] = (T)v;
          if constexpr (sizeof(T) == 2) {
            const float rest = v - (float)hi[e];
            lo[e] = (T)(fabsf(rest) < __builtin_inff() ? rest : 0.0f);
          }
        }
#pragma unroll
        for (int j = 0; j < E; ++j) {
          acc[j] = ln_mfma(hi, f[s][j], acc[j]);
          if constexpr (sizeof(T) == 2) acc[j] = ln_mfma(lo, f[s][j], acc[j]);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (here && (rows >> (4 * q + i) & 1)) {
          float v[E];
#pragma unroll
          for (int j = 0; j < E; ++j) v[j] = acc[j][i];
          put(first + 16 * b + 4 * q + i, v);
        }
    }
  });
  if (blockIdx.z) return;
  // tokens without an adapter, and with one that is not there (asked of all lanes, also those without columns: they hold tokens)
  const uint64_t past = __ballot(live && (int64_t)id >= g.adapters), none = __ballot(live && id < 0);
  if (!here) return;
  for (uint64_t left = g.in_place ? past : past | none; left; left &= left - 1) {
    const int t = __builtin_ctzll(left);
    if ((t & 3) != q) continue;                      // (rows in turn: the lanes of a quarter hold all of the wave's columns)
    float v[E];
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = past >> t & 1 ? __builtin_nanf("") : 0.0f;
    put(first + t, v);
  }
}

struct LqPlan {
  int tb, splits, shares, up_tb, up_shares, ldt;
  int64_t k_per_split;
};
static LqPlan lora_requests_plan(int64_t m, int64_t k, int64_t n, int r, int64_t adapters, bool bf16) {
  LqPlan p;
  const int e = bf16 ? 8 : 4, step = 4 * e * LQ_WAVES;
  p.ldt = r <= 16 ? 16 : (r <= 32 ? 32 : 64);
  p.tb = ceil_div64(m, 32) >= 256 ? 2 : 1;
  const int64_t tiles = ceil_div64(m, 16 * p.tb), most = std::min<int64_t>(16 * p.tb, adapters);
  p.shares = (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, most));
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / (tiles * p.shares), ceil_div64(k, step)), 16));
  p.k_per_split = ceil_div64(ceil_div64(k, splits), step) * step;
  p.splits = (int)ceil_div64(k, p.k_per_split);
  const int64_t cols = ceil_div64(n, 16 * e);
  p.up_tb = cols * ceil_div64(m, 64) >= 2048 ? 4 : 1;
  const int64_t up_tiles = ceil_div64(m, 16 * p.up_tb);
  p.up_shares = (int)std::max<int64_t>(1, std::min<int64_t>(2048 / (cols * up_tiles), std::min<int64_t>(16 * p.up_tb, adapters)));
  return p;
}
static size_t lora_requests_part_bytes(const LqPlan& p, int64_t m) { return (size_t)p.splits * m * p.ldt * 4; }
// Fewer than 2^32 threads to a launch.
static bool lora_requests_launches(const LqPlan& p, int64_t m, int64_t n, bool bf16) {
  const int64_t down = ceil_div64(m, 16 * p.tb) * p.splits * p.shares, cols = ceil_div64(n, (bf16 ? 128 : 64) * LQ_UP_WAVES);
  return down < (1ll << 32) / (64 * LQ_WAVES) && cols < 65536 && ceil_div64(m, 16 * p.up_tb) * cols * p.up_shares < (1ll << 32) / (64 * LQ_UP_WAVES);
}

template <typename T, typename O, int TB>
static int launch_lora_up(hipStream_t s, const LqArgs& g, dim3 grid) {
  const dim3 block(64 * LQ_UP_WAVES);
  const int steps = (g.r + Ln<T>::STEP - 1) / Ln<T>::STEP;
  if (steps == 1) LORACT_LAUNCH("lora_requests_up", s, (lora_up_kernel<T, O, TB, 1>), grid, block, 0, g);
  else if (steps == 2) LORACT_LAUNCH("lora_requests_up", s, (lora_up_kernel<T, O, TB, 2>), grid, block, 0, g);
  else if constexpr (sizeof(T) == 4) LORACT_LAUNCH("lora_requests_up", s, (lora_up_kernel<T, O, TB, 4>), grid, block, 0, g);
  return LORACT_OK;
}
template <typename T, int TB>
static int launch_lora_down(hipStream_t s, const LqArgs& g, dim3 grid) {
  const dim3 block(64 * LQ_WAVES);
  if (g.ldt == 16) LORACT_LAUNCH("lora_requests_down", s, (lora_down_kernel<T, TB, 1>), grid, block, 0, g);
  else if (g.ldt == 32) LORACT_LAUNCH("lora_requests_down", s, (lora_down_kernel<T, TB, 2>), grid, block, 0, g);
  else LORACT_LAUNCH("lora_requests_down", s, (lora_down_kernel<T, TB, 4>), grid, block, 0, g);
  return LORACT_OK;
}
template <typename T, typename O>
static int launch_lora_requests(hipStream_t s, LqArgs g, const LqPlan& p) {
  g.ldt = p.ldt; g.splits = p.splits; g.k_per_split = p.k_per_split;
  g.shares = p.shares;
  const dim3 down((unsigned)ceil_div64(g.m, 16 * p.tb), (unsigned)p.splits, (unsigned)p.shares);
  if (p.tb == 2) LORACT_TRY((launch_lora_down<T, 2>(s, g, down)));
  else LORACT_TRY((launch_lora_down<T, 1>(s, g, down)));
  g.shares = p.up_shares;
  const dim3 up((unsigned)ceil_div64(g.m, 16 * p.up_tb), (unsigned)ceil_div64(g.n, 16 * Ln<T>::E * LQ_UP_WAVES), (unsigned)p.up_shares);
  if (p.up_tb == 4) return launch_lora_up<T, O, 4>(s, g, up);
  return launch_lora_up<T, O, 1>(s, g, up);
}

// The low-rank adapters of many requests beside a projection that they share: Y_i = R_i + s_a (X_i A_a) B_a, a = ids_i.
//
//   down   T = X A.  K is split between the eight waves of a workgroup, whose sums are added in LDS, and between workgroups, whose parts the
//          next launch adds as it reads them.
//   up     Y = R + s T B.
//
// Up to 64 tokens: two launches.  Tokens in tiles, in order; a tile goes over the different adapters of its tokens (found by ballots) and takes
// from each product what belongs to their tokens.  An adapter's infinities and NaN thus reach its own tokens only.
// More tokens: a first launch orders them by adapter, in tiles of 64 that have one adapter each.  (In the order they come, a tile of single tokens of 22
// requests walks over 22 adapters while others have one: 8192 tokens, the last hundred of them single ones, took 1040 us at rank 64 and 11008
// columns, 330 without those.)  The places of an adapter's tokens among each other depend on an atomic counter, but no result depends on them.
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
  int *tiles, *order;                // ordered tokens: their number, then group and size of each tile; the tokens, 64 to a tile
};
#define LQ_TILE 64
#define LQ_SORTED 8192                               // adapters that are counted in LDS

// Orders the tokens by adapter.  Groups: the adapters, tokens without one (none where Y is R), tokens whose adapter is not there.
__global__ __launch_bounds__(1024) void lora_sort_kernel(LqArgs g) {
  __shared__ int count[LQ_SORTED + 2];
  __shared__ int sums[16];
  const int tid = threadIdx.x, lane = tid & 63, groups = (int)g.adapters + 2;
  auto group = [&](int64_t i) {
    if (i >= g.m) return -1;
    const int id = g.ids[i];
    return id < 0 ? (g.in_place ? -1 : groups - 2) : ((int64_t)id < g.adapters ? id : groups - 1);
  };
  // Place of each lane's token among those of its group so far: a wave of one group, as prompts make them, by one atomic.
  auto place = [&](int mine) {
    const int d = __builtin_amdgcn_readfirstlane(mine);
    if (__all(mine == d)) {
      int at = 0;
      if (lane == 0 && d >= 0) at = atomicAdd(&count[d], 64);
      return __builtin_amdgcn_readfirstlane(at) + lane;
    }
    return mine >= 0 ? atomicAdd(&count[mine], 1) : 0;
  };
  for (int i = tid; i < groups; i += 1024) count[i] = 0;
  __syncthreads();
  for (int64_t i0 = tid; i0 - tid < g.m; i0 += 4096) {         // (every lane comes as often)
    int mine[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) mine[u] = group(i0 + 1024 * u);
#pragma unroll
    for (int u = 0; u < 4; ++u) place(mine[u]);
  }
  __syncthreads();
  // first tile of every group: a thread has consecutive groups
  const int per = (groups + 1023) / 1024, from = tid * per, to = from + per < groups ? from + per : groups;
  int mine = 0;
  for (int i = from; i < to; ++i) mine += (count[i] + LQ_TILE - 1) / LQ_TILE;
  int up_to = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int other = __shfl_up(up_to, d);
    if (lane >= d) up_to += other;
  }
  if (lane == 63) sums[tid >> 6] = up_to;
  __syncthreads();
  int tile = up_to - mine;
  for (int w = 0; w < (tid >> 6); ++w) tile += sums[w];
  if (tid == 1023) g.tiles[0] = tile + mine;
  for (int i = from; i < to; ++i) {
    const int n = count[i];
    count[i] = tile * LQ_TILE;
    for (int at = 0; at < n; at += LQ_TILE, ++tile) {
      g.tiles[2 + 2 * tile] = i;
      g.tiles[3 + 2 * tile] = n - at < LQ_TILE ? n - at : LQ_TILE;
    }
  }
  __syncthreads();
  for (int64_t i0 = tid; i0 - tid < g.m; i0 += 4096) {
    int mine4[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) mine4[u] = group(i0 + 1024 * u);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = place(mine4[u]);
      if (mine4[u] >= 0) g.order[at] = (int)(i0 + 1024 * u);
    }
  }
}

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

// TB: blocks of 16 tokens per tile.  SB: blocks of 16 columns of A.  SORTED: halves of the ordered tiles.
template <typename T, int TB, int SB, bool SORTED>
__global__ __launch_bounds__(64 * LQ_WAVES) void lora_down_kernel(LqArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP, U = SB == 1 ? 4 : 2, QUADS = TB * SB * 64, PER = 16 / E;
  typedef typename Ln<T>::frag frag;
  constexpr int TURN_BYTES = LQ_WAVES * U * SB * 1024, PART_BYTES = LQ_WAVES * QUADS * 16;
  __shared__ __attribute__((aligned(16))) unsigned char smem[TURN_BYTES > PART_BYTES ? TURN_BYTES : PART_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  int64_t token[TB];                                 // token c of each block
  int id = -1, blocks = TB;
  bool live = false;
  uint64_t done = 0;                                 // tokens whose T is written
  if constexpr (SORTED) {
    const int tile = blockIdx.x / (LQ_TILE / (16 * TB)), part = blockIdx.x % (LQ_TILE / (16 * TB));
    if (tile >= g.tiles[0]) return;
    id = g.tiles[2 + 2 * tile];
    const int left = g.tiles[3 + 2 * tile] - part * (16 * TB);
    if (left <= 0 || (int64_t)id >= g.adapters) return;
    blocks = left > 16 ? TB : 1;
    done = left >= 16 * TB ? ~0ull >> (64 - 16 * TB) : (1ull << left) - 1;
#pragma unroll
    for (int b = 0; b < TB; ++b) token[b] = g.order[tile * LQ_TILE + part * (16 * TB) + (done >> (16 * b + c) & 1 ? 16 * b + c : 0)];
  } else {
    const int64_t first = (int64_t)blockIdx.x * (16 * TB), mine = first + (lane < 16 * TB ? lane : 0);
    live = lane < 16 * TB && mine < g.m;
    id = live ? g.ids[mine] : -1;
#pragma unroll
    for (int b = 0; b < TB; ++b) token[b] = first + 16 * b + c < g.m ? first + 16 * b + c : g.m - 1;
  }
  const int64_t k_beg0 = (int64_t)blockIdx.y * g.k_per_split, k_end0 = k_beg0 + g.k_per_split < g.k ? k_beg0 + g.k_per_split : g.k;
  const int64_t per = ((k_end0 - k_beg0 + STEP * LQ_WAVES - 1) / (STEP * LQ_WAVES)) * STEP;
  const int64_t k_beg = k_beg0 + wave * per, k_end = k_beg + per < k_end0 ? k_beg + per : k_end0;
  const T* x[TB];
#pragma unroll
  for (int b = 0; b < TB; ++b) x[b] = (const T*)g.X + token[b] * g.ldx;
  f32x4 total[TB][SB];
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int s = 0; s < SB; ++s) total[b][s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  unsigned char* const turn = smem + wave * (U * SB * 1024);
  auto product = [&](int d, uint64_t same) {
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
        for (int b = 0; b < TB; ++b) st[u][b] = lq_load<T>(x[b] + k, b < blocks ? k_end - k : 0);
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
  };
  if constexpr (SORTED) product(id, done);
  else lq_adapters(g, id, live, blockIdx.z, product);
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
    if (done >> (16 * b + c) & 1)                    // (l is the lane)
      *(f32x4*)(g.part + ((int64_t)blockIdx.y * g.m + (b ? token[TB - 1] : token[0])) * g.ldt + 16 * s + 4 * (l >> 4)) = v;
  }
}

// E consecutive numbers of a token's T summed over W of its parts from p0 on, in their order and all in flight.
template <int E, int W>
__device__ inline void lq_sum(const LqArgs& g, int64_t token, int k, int p0, float (&t)[E]) {
  f32x4 v[W][E / 4];
#pragma unroll
  for (int p = 0; p < W; ++p) {
    const float* at = g.part + ((int64_t)(p0 + p < g.splits ? p0 + p : p0) * g.m + token) * g.ldt + k;
#pragma unroll
    for (int h = 0; h < E / 4; ++h) v[p][h] = *(const f32x4*)(at + 4 * h);
  }
#pragma unroll
  for (int p = 0; p < W; ++p)
    if (p0 + p < g.splits) {
#pragma unroll
      for (int e = 0; e < E; ++e) t[e] += v[p][e / 4][e % 4];
    }
}
// The same over all parts, times the scale.
template <int E>
__device__ inline void lq_t(const LqArgs& g, int64_t token, int k, float by, float (&t)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) t[e] = 0.0f;
  if (g.splits == 1) lq_sum<E, 1>(g, token, k, 0, t);
  else if (g.splits == 2) lq_sum<E, 2>(g, token, k, 0, t);
  else for (int p0 = 0; p0 < g.splits; p0 += 8) lq_sum<E, 8>(g, token, k, p0, t);
#pragma unroll
  for (int e = 0; e < E; ++e) t[e] = k + e < g.r ? t[e] * by : 0.0f;
}
// The operand of that: hi, and for bf16 what it leaves.
template <typename T, int E>
__device__ inline void lq_parts(const float (&t)[E], typename Ln<T>::frag& hi, typename Ln<T>::frag& lo) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    hi[e] = (T)t[e];
    if constexpr (sizeof(T) == 2) {
      const float rest = t[e] - (float)hi[e];
      lo[e] = (T)(fabsf(rest) < __builtin_inff() ? rest : 0.0f);
    }
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
        float t[E] = {};
        const int k = STEP * s + E * q;
        if ((rows >> c & 1) && k < g.r) lq_t<E>(g, token, k, by, t);            // (rows of other adapters may not be written at all)
        frag hi, lo;
        lq_parts<T>(t, hi, lo);
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

// Ordered tokens: a tile of 64, 16 to each wave, and 16 E columns, whose part of B passes through LDS.  B gives the rows of the product, in an
// order that leaves a lane with E consecutive columns of its token: the transposing reads take chunks of four columns 2 E bytes apart.
template <typename T, typename O, int RS>
__global__ __launch_bounds__(64 * LQ_UP_WAVES) void lora_up_sorted_kernel(LqArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP, PITCH = 256 + 64, J = 4;
  typedef typename Ln<T>::frag frag;
  typedef typename LqOut<O, E>::any out_any;
  __shared__ __attribute__((aligned(16))) unsigned char smem[RS * STEP * PITCH];
  const int cols = (int)((g.n + 16 * E - 1) / (16 * E)), tile = blockIdx.x / cols;       // (the columns of a tile one after the other)
  if (tile >= g.tiles[0]) return;
  const int d = g.tiles[2 + 2 * tile], size = g.tiles[3 + 2 * tile];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t first = (int64_t)(blockIdx.x - tile * cols) * (16 * E);
  const bool there = (int64_t)d < g.adapters;
  if (there) {
    const T* const b = (const T*)g.B + (int64_t)d * g.r * g.n;
    constexpr int TRIPS = RS * STEP / 16;            // 16 rows of 16 pieces at a time
    frag v[TRIPS];
    const int64_t col = first + E * (threadIdx.x & 15);
#pragma unroll
    for (int i = 0; i < TRIPS; ++i) {
      const int row = 16 * i + (threadIdx.x >> 4);
      v[i] = (frag){};
      if (row < g.r && col < g.n) v[i] = g.b_pieces ? *(const frag*)(b + (int64_t)row * g.n + col) : lq_load<T>(b + (int64_t)row * g.n + col, g.n - col);
    }
#pragma unroll
    for (int i = 0; i < TRIPS; ++i) *(frag*)(smem + (16 * i + (threadIdx.x >> 4)) * PITCH + 16 * (threadIdx.x & 15)) = v[i];
  }
  const bool live = 16 * wave + c < size;
  const int64_t token = g.order[tile * LQ_TILE + (live ? 16 * wave + c : 0)];
  frag hi[RS], lo[RS];
  if (there) {
    const float by = g.scales ? g.scales[d] : 1.0f;
#pragma unroll
    for (int s = 0; s < RS; ++s) {
      float t[E] = {};
      const int k = STEP * s + E * q;
      if (live && k < g.r) lq_t<E>(g, token, k, by, t);
      lq_parts<T>(t, hi[s], lo[s]);
    }
  }
  const O* const rp = (const O*)g.R + token * g.ldr;
  O* const yp = (O*)g.Y + token * g.ldy;
  typename LqOut<O, E>::vec res[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int64_t col = first + 4 * E * j + E * q;
    if (g.R && live && col + E <= g.n) res[j] = *(const out_any*)(rp + col);
  }
  __syncthreads();
  if (16 * wave >= size) return;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    f32x4 acc[E / 4];
#pragma unroll
    for (int h = 0; h < E / 4; ++h) acc[h] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    if (there) {
#pragma unroll
      for (int s = 0; s < RS; ++s)
#pragma unroll
        for (int h = 0; h < E / 4; ++h) {
          frag f;
          if constexpr (sizeof(T) == 2) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s16x4* lds_ptr;
            const unsigned char* at = smem + (STEP * s + 8 * q + (c >> 2)) * PITCH + 64 * j + 16 * (c & 3) + 8 * h;
            const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
            const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * PITCH));
            f = __builtin_bit_cast(frag, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) f[e] = *(const T*)(smem + (STEP * s + E * q + e) * PITCH + 64 * j + 4 * c);
          }
          acc[h] = ln_mfma(f, hi[s], acc[h]);
          if constexpr (sizeof(T) == 2) acc[h] = ln_mfma(f, lo[s], acc[h]);
        }
    } else if ((int64_t)d > g.adapters) {
#pragma unroll
      for (int h = 0; h < E / 4; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[h][e] = __builtin_nanf("");
    }
    const int64_t col = first + 4 * E * j + E * q;
    if (!live || col >= g.n) continue;
    if (col + E <= g.n) {
      typename LqOut<O, E>::vec y;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = (O)((g.R ? (float)res[j][e] : 0.0f) + acc[e / 4][e % 4]);
      *(out_any*)(yp + col) = y;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (col + e < g.n) yp[col + e] = (O)((g.R ? (float)rp[col + e] : 0.0f) + acc[e / 4][e % 4]);
    }
  }
}

struct LqPlan {
  bool sorted;
  int64_t tiles;         // at most
  size_t part_bytes, tile_bytes, bytes;
  int tb, splits, shares, up_tb, up_shares, ldt;
  int64_t k_per_split;
};
static LqPlan lora_requests_plan(int64_t m, int64_t k, int64_t n, int r, int64_t adapters, bool bf16) {
  LqPlan p;
  const int e = bf16 ? 8 : 4, step = 4 * e * LQ_WAVES;
  p.sorted = m > 64 && adapters <= LQ_SORTED;
  p.tiles = p.sorted ? ceil_div64(m, LQ_TILE) + std::min<int64_t>(adapters + 2, m) : 0;
  p.ldt = r <= 16 ? 16 : (r <= 32 ? 32 : 64);
  p.tb = p.sorted || ceil_div64(m, 32) >= 256 ? 2 : 1;
  const int64_t tiles = ceil_div64(m, 16 * p.tb), most = p.sorted ? 1 : std::min<int64_t>(16 * p.tb, adapters);
  p.shares = (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, most));
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(512 / (tiles * p.shares), ceil_div64(k, step)), 16));
  p.k_per_split = ceil_div64(ceil_div64(k, splits), step) * step;
  p.splits = (int)ceil_div64(k, p.k_per_split);
  const int64_t cols = ceil_div64(n, 16 * e);
  p.up_tb = cols * ceil_div64(m, 64) >= 2048 ? 4 : 1;
  const int64_t up_tiles = ceil_div64(m, 16 * p.up_tb);
  p.up_shares = (int)std::max<int64_t>(1, std::min<int64_t>(2048 / (cols * up_tiles), std::min<int64_t>(16 * p.up_tb, adapters)));
  p.part_bytes = (size_t)p.splits * m * p.ldt * 4;
  p.tile_bytes = p.sorted ? align_up(8 + (size_t)p.tiles * 8, 16) : 0;
  p.bytes = p.part_bytes + p.tile_bytes + (size_t)p.tiles * LQ_TILE * 4;
  return p;
}
// Fewer than 2^32 threads to a launch, and than 65536 rows of workgroups.
static bool lora_requests_launches(const LqPlan& p, int64_t m, int64_t n, bool bf16) {
  const int64_t wide = bf16 ? 128 : 64, limit = (1ll << 32) / 512;
  if (p.sorted) {
    const int64_t cols = ceil_div64(n, wide);
    return 2 * p.tiles * p.splits < limit && p.tiles * cols < 2 * limit && p.tiles < (1ll << 31) / LQ_TILE;
  }
  const int64_t cols = ceil_div64(n, wide * LQ_UP_WAVES);
  return ceil_div64(m, 16 * p.tb) * p.splits * p.shares < limit && cols < 65536 && ceil_div64(m, 16 * p.up_tb) * cols * p.up_shares < 2 * limit;
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
template <typename T, int TB, bool SORTED>
static int launch_lora_down(hipStream_t s, const LqArgs& g, dim3 grid) {
  const dim3 block(64 * LQ_WAVES);
  if (g.ldt == 16) LORACT_LAUNCH("lora_requests_down", s, (lora_down_kernel<T, TB, 1, SORTED>), grid, block, 0, g);
  else if (g.ldt == 32) LORACT_LAUNCH("lora_requests_down", s, (lora_down_kernel<T, TB, 2, SORTED>), grid, block, 0, g);
  else LORACT_LAUNCH("lora_requests_down", s, (lora_down_kernel<T, TB, 4, SORTED>), grid, block, 0, g);
  return LORACT_OK;
}
template <typename T, typename O>
static int launch_lora_requests(hipStream_t s, LqArgs g, const LqPlan& p) {
  g.ldt = p.ldt; g.splits = p.splits; g.k_per_split = p.k_per_split;
  g.shares = p.shares;
  if (p.sorted) {
    g.tiles = (int*)((char*)g.part + p.part_bytes);
    g.order = (int*)((char*)g.tiles + p.tile_bytes);
    LORACT_LAUNCH("lora_requests_sort", s, lora_sort_kernel, dim3(1), dim3(1024), 0, g);
    LORACT_TRY((launch_lora_down<T, 2, true>(s, g, dim3((unsigned)(2 * p.tiles), (unsigned)p.splits))));
    const dim3 grid((unsigned)(p.tiles * ceil_div64(g.n, 16 * Ln<T>::E))), block(64 * LQ_UP_WAVES);
    const int steps = (g.r + Ln<T>::STEP - 1) / Ln<T>::STEP;
    if (steps == 1) LORACT_LAUNCH("lora_requests_up", s, (lora_up_sorted_kernel<T, O, 1>), grid, block, 0, g);
    else if (steps == 2) LORACT_LAUNCH("lora_requests_up", s, (lora_up_sorted_kernel<T, O, 2>), grid, block, 0, g);
    else if constexpr (sizeof(T) == 4) LORACT_LAUNCH("lora_requests_up", s, (lora_up_sorted_kernel<T, O, 4>), grid, block, 0, g);
    return LORACT_OK;
  }
  const dim3 down((unsigned)ceil_div64(g.m, 16 * p.tb), (unsigned)p.splits, (unsigned)p.shares);
  if (p.tb == 2) LORACT_TRY((launch_lora_down<T, 2, false>(s, g, down)));
  else LORACT_TRY((launch_lora_down<T, 1, false>(s, g, down)));
  g.shares = p.up_shares;
  const dim3 up((unsigned)ceil_div64(g.m, 16 * p.up_tb), (unsigned)ceil_div64(g.n, 16 * Ln<T>::E * LQ_UP_WAVES), (unsigned)p.up_shares);
  if (p.up_tb == 4) return launch_lora_up<T, O, 4>(s, g, up);
  return launch_lora_up<T, O, 1>(s, g, up);
}

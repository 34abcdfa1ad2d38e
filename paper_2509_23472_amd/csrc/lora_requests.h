// The low-rank adapters of many requests beside a projection that they share: Y_i = R_i + s_a (X_i A_a) B_a, a = ids_i.
//
//   down   T = X A.  K is split between the eight waves of a workgroup, whose sums are added in LDS, and between workgroups, whose parts the
//          next launch adds as it reads them.
//   up     Y = R + s T B.
//
// Few tokens and adapters: two launches.  Tokens in tiles, in order; a tile goes over the different adapters of its tokens (found by ballots) and takes
// from each product what belongs to their tokens.  An adapter's infinities and NaN thus reach its own tokens only.
// Else a first launch orders them by adapter, in tiles of 64 that have one adapter each.  (In the order they come, a tile of single tokens of 22
// requests walks over 22 adapters while others have one: 8192 tokens, the last hundred of them single ones, took 1040 us at rank 64 and 11008
// columns, 330 without those.)  The places of an adapter's tokens among each other depend on an atomic counter, but no result depends on them.
//
// T of bf16 operands enters the second product as the sum of three bf16 numbers, which hold all of its 24 digits: float32 results are off by 1.0e-7 to 1.3e-7 of
// the norm, as those of float32 operands are (with two numbers, 16 digits, by 2.5e-6, and the second launch takes 1 to 2 % less: 101 against 102 us at 8192 tokens of 24
// adapters, 4096 -> 11008, rank 64).
//
// Bound by memory: single tokens by A and B, prompts by X, R and Y.  Few tokens with an adapter each: the walk is shared out over workgroups too.
// 8192 tokens of 24 adapters, 4096 -> 11008, rank 64: ordering 10 us, down 43 (rank 16: 24), up 102 (87, 4.1 TB/s; float32 results, whose R and Y are 721 MB, 226 together);
// one token, rank 16, 4.6 and 6.8, where each launch is a chain of three reads.
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
  int trips, groups;                 // ordered tokens, second launch: times 16 E columns per workgroup, workgroups to a tile
  int *tiles, *order;                // ordered tokens: their number, then group and size of each tile; the tokens, 64 to a tile
};
#define LQ_TILE 64
#define LQ_SORTED 8192                               // adapters that are counted in LDS

// Orders the tokens by adapter.  Groups: the adapters, tokens without one (none where Y is R), tokens whose adapter is not there.
__global__ __launch_bounds__(1024) void lora_sort_kernel(LqArgs g) {
  constexpr int HELD = 8;                            // groups of a thread's first tokens that stay in registers
  __shared__ int next[LQ_SORTED + 2], start[LQ_SORTED + 2];      // tokens counted, or placed; first tile
  __shared__ int sums[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, groups = (int)g.adapters + 2;
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
      if (lane == 0 && d >= 0) at = atomicAdd(&next[d], 64);
      return __builtin_amdgcn_readfirstlane(at) + lane;
    }
    return mine >= 0 ? atomicAdd(&next[mine], 1) : 0;
  };
  int held[HELD];
#pragma unroll
  for (int u = 0; u < HELD; ++u) held[u] = group(tid + 1024 * u);
  for (int i = tid; i < groups; i += 1024) next[i] = 0;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < HELD; ++u)
    if (1024 * u < g.m) place(held[u]);
  for (int64_t i = tid + 1024 * HELD; i - tid < g.m; i += 4096) {       // (every lane comes as often)
    int more[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) more[u] = group(i + 1024 * u);
#pragma unroll
    for (int u = 0; u < 4; ++u) place(more[u]);
  }
  __syncthreads();
  // first tile of every group: a thread has consecutive groups
  const int per = (groups + 1023) / 1024, from = tid * per < groups ? tid * per : groups, to = from + per < groups ? from + per : groups;
  int mine = 0;
  for (int i = from; i < to; ++i) mine += (next[i] + LQ_TILE - 1) / LQ_TILE;
  int up_to = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int other = __shfl_up(up_to, d);
    if (lane >= d) up_to += other;
  }
  if (lane == 63) sums[wave] = up_to;
  __syncthreads();
  int tile = up_to - mine, total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    const int s = sums[w];
    tile += w < wave ? s : 0;
    total += s;
  }
  for (int i = from; i < to; ++i) {
    start[i] = tile;
    tile += (next[i] + LQ_TILE - 1) / LQ_TILE;
  }
  __syncthreads();
  if (tid == 0) g.tiles[0] = total;
  for (int t = tid; t < total; t += 1024) {          // its group: the last that begins at it or before
    int lo = 0, hi = groups;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (start[mid] <= t) lo = mid;
      else hi = mid;
    }
    const int left = next[lo] - (t - start[lo]) * LQ_TILE;
    g.tiles[2 + 2 * t] = lo;
    g.tiles[3 + 2 * t] = left < LQ_TILE ? left : LQ_TILE;
  }
  __syncthreads();
  for (int i = tid; i < groups; i += 1024) next[i] = start[i] * LQ_TILE;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < HELD; ++u)
    if (1024 * u < g.m) {
      const int at = place(held[u]);
      if (held[u] >= 0) g.order[at] = tid + 1024 * u;
    }
  for (int64_t i = tid + 1024 * HELD; i - tid < g.m; i += 4096) {
    int more[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) more[u] = group(i + 1024 * u);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = place(more[u]);
      if (more[u] >= 0) g.order[at] = (int)(i + 1024 * u);
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

// The transposed fragment of 16 columns of A: k from E q on, column c, of rows `pitch` bytes apart that start at `at`.
template <typename T>
__device__ inline typename Ln<T>::frag lq_turned(const unsigned char* at, int pitch, int c, int q) {
  constexpr int E = Ln<T>::E;
  typename Ln<T>::frag f;
  if constexpr (sizeof(T) == 2) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    at += (8 * q + (c >> 2)) * pitch + (c & 3) * 8;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * pitch));
    f = __builtin_bit_cast(typename Ln<T>::frag, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = *(const T*)(at + (E * q + e) * pitch + c * 4);
  }
  return f;
}
// A piece of a row of A: columns col .. col + E - 1 of row k, zeros where there is none.
template <typename T>
__device__ inline typename Ln<T>::frag lq_piece(const LqArgs& g, const T* a, int64_t k, int64_t k_end, int col) {
  const bool here = k < k_end && col < g.r;
  if (!g.a_pieces) return lq_load<T>(a + k * g.r + col, here ? g.r - col : 0);
  typename Ln<T>::frag v = {};
  if (here) v = *(const typename Ln<T>::frag*)(a + k * g.r + col);
  return v;
}

// Few tokens: tiles of 16 in the order they come.  SB: blocks of 16 columns of A.
template <typename T, int SB>
__global__ __launch_bounds__(64 * LQ_WAVES) void lora_down_kernel(LqArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP, U = SB == 1 ? 4 : 2, QUADS = SB * 64, PER = 16 / E;
  typedef typename Ln<T>::frag frag;
  constexpr int TURN_BYTES = LQ_WAVES * U * SB * 1024, PART_BYTES = LQ_WAVES * QUADS * 16;
  __shared__ __attribute__((aligned(16))) unsigned char smem[TURN_BYTES > PART_BYTES ? TURN_BYTES : PART_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t first = (int64_t)blockIdx.x * 16, mine = first + (lane < 16 ? lane : 0);
  const bool live = lane < 16 && mine < g.m;
  const int id = live ? g.ids[mine] : -1;
  const int64_t token = first + c < g.m ? first + c : g.m - 1;
  const int64_t k_beg0 = (int64_t)blockIdx.y * g.k_per_split, k_end0 = k_beg0 + g.k_per_split < g.k ? k_beg0 + g.k_per_split : g.k;
  const int64_t per = ((k_end0 - k_beg0 + STEP * LQ_WAVES - 1) / (STEP * LQ_WAVES)) * STEP;
  const int64_t k_beg = k_beg0 + wave * per, k_end = k_beg + per < k_end0 ? k_beg + per : k_end0;
  const T* const x = (const T*)g.X + token * g.ldx;
  f32x4 total[SB];
#pragma unroll
  for (int s = 0; s < SB; ++s) total[s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  unsigned char* const turn = smem + wave * (U * SB * 1024);
  uint64_t done = 0;                                 // tokens whose T is written
  lq_adapters(g, id, live, blockIdx.z, [&](int d, uint64_t same) {
    done |= same;
    const T* const a = (const T*)g.A + (int64_t)d * g.k * g.r;
    f32x4 acc[SB];
#pragma unroll
    for (int s = 0; s < SB; ++s) acc[s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t k0 = k_beg; k0 < k_end; k0 += STEP * U) {
      frag st[U], sm[U][SB];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + STEP * u + E * q;
        st[u] = lq_load<T>(x + k, k_end - k);
#pragma unroll
        for (int s = 0; s < SB; ++s) sm[u][s] = lq_piece<T>(g, a, k0 + STEP * u + lane / PER, k_end, 16 * s + E * (lane % PER));
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SB; ++s) *(frag*)(turn + (u * SB + s) * 1024 + lane * 16) = sm[u][s];
      sb_wave_sync();
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SB; ++s) sm[u][s] = lq_turned<T>(turn + (u * SB + s) * 1024, 16 * (int)sizeof(T), c, q);
      sb_wave_sync();
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SB; ++s) acc[s] = ln_mfma(sm[u][s], st[u], acc[s]);
    }
    const bool own = same >> c & 1;                  // a lane's column is token c
#pragma unroll
    for (int s = 0; s < SB; ++s)
#pragma unroll
      for (int u = 0; u < 4; ++u) total[s][u] = own ? acc[s][u] : total[s][u];
  });
  if (!done) return;                                 // (the same for all waves)
  __syncthreads();
  f32x4* const part = (f32x4*)smem;
#pragma unroll
  for (int s = 0; s < SB; ++s) part[wave * QUADS + s * 64 + lane] = total[s];
  __syncthreads();
  for (int i = threadIdx.x; i < QUADS; i += 64 * LQ_WAVES) {
    f32x4 v = part[i];
#pragma unroll
    for (int w = 1; w < LQ_WAVES; ++w) v += part[w * QUADS + i];
    if (done >> c & 1) *(f32x4*)(g.part + ((int64_t)blockIdx.y * g.m + token) * g.ldt + 16 * (i / 64) + 4 * q) = v;
  }
}

// Ordered tokens: a tile of 64; four groups of waves share K, in each 16 tokens to a wave.  A passes through LDS in slabs that the waves of a group
// read, the next one (and the next part of X) on its way while one is multiplied.  The groups' sums are added in LDS: parts of T that only the next
// launch adds cost it a reading of each per 512 columns (8192 tokens, 11008 columns, rank 64: 97 us with one part, 124 with four).
#define LQ_K_GROUPS 4
template <typename T, int SB>
__global__ __launch_bounds__(256 * LQ_K_GROUPS) void lora_down_sorted_kernel(LqArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP, U = 4, SLAB = U * STEP, PITCH = 16 * SB * (int)sizeof(T) + (SB == 4 ? 16 : 0);
  constexpr int PER = 16 * SB / E, TRIPS = SLAB * PER / 256;                     // pieces to a row, and of a slab to a thread
  constexpr int SLABS = LQ_K_GROUPS * 2 * SLAB * PITCH, PARTS = (LQ_K_GROUPS - 1) * 4 * SB * 1024;
  static_assert(SLAB * PER % 256 == 0, "whole trips");
  typedef typename Ln<T>::frag frag;
  __shared__ __attribute__((aligned(16))) unsigned char smem[SLABS > PARTS ? SLABS : PARTS];
  const int tile = blockIdx.x;
  if (tile >= g.tiles[0]) return;
  const int d = g.tiles[2 + 2 * tile], size = g.tiles[3 + 2 * tile];
  if ((int64_t)d >= g.adapters) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 3, group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  const int tid = threadIdx.x & 255, c = lane & 15, q = lane >> 4;
  const int64_t k_beg0 = (int64_t)blockIdx.y * g.k_per_split, k_end0 = k_beg0 + g.k_per_split < g.k ? k_beg0 + g.k_per_split : g.k;
  const int64_t per = (g.k_per_split + LQ_K_GROUPS * SLAB - 1) / (LQ_K_GROUPS * SLAB) * SLAB;      // (as many slabs for every group)
  const int64_t k_beg = k_beg0 + group * per, k_end = k_beg + per < k_end0 ? k_beg + per : k_end0;
  const bool work = 16 * wave < size, live = 16 * wave + c < size;
  const int64_t token = g.order[tile * LQ_TILE + (live ? 16 * wave + c : 0)];
  const T* const x = (const T*)g.X + token * g.ldx;
  const T* const a = (const T*)g.A + (int64_t)d * g.k * g.r;
  unsigned char* const slabs = smem + group * (2 * SLAB * PITCH);
  frag xs[U], as[TRIPS];
  auto load = [&](int64_t k0) {
#pragma unroll
    for (int i = 0; i < TRIPS; ++i) {
      const int at = tid + i * 256;
      as[i] = lq_piece<T>(g, a, k0 + at / PER, k_end, E * (at % PER));
    }
    if (work) {
#pragma unroll
      for (int u = 0; u < U; ++u) xs[u] = lq_load<T>(x + k0 + STEP * u + E * q, k_end - (k0 + STEP * u + E * q));
    }
  };
  f32x4 acc[SB];
#pragma unroll
  for (int s = 0; s < SB; ++s) acc[s] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
  load(k_beg);
  int turn = 0;
  for (int64_t at_k = 0; at_k < per; at_k += SLAB, turn ^= 1) {
    unsigned char* const slab = slabs + turn * (SLAB * PITCH);
    frag now[U];
#pragma unroll
    for (int u = 0; u < U; ++u) now[u] = xs[u];
#pragma unroll
    for (int i = 0; i < TRIPS; ++i) {
      const int at = tid + i * 256;
      *(frag*)(slab + at / PER * PITCH + at % PER * 16) = as[i];
    }
    if (at_k + SLAB < per) load(k_beg + at_k + SLAB);
    sb_barrier_lds();                                // (two slabs: who writes one has passed the barrier behind its last reading)
    if (work) {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int s = 0; s < SB; ++s) acc[s] = ln_mfma(lq_turned<T>(slab + STEP * u * PITCH + 16 * s * (int)sizeof(T), PITCH, c, q), now[u], acc[s]);
    }
  }
  __syncthreads();
  f32x4* const part = (f32x4*)smem;
  if (group) {
#pragma unroll
    for (int s = 0; s < SB; ++s) part[((group - 1) * 4 + wave) * (SB * 64) + s * 64 + lane] = acc[s];
  }
  __syncthreads();
  if (group || !live) return;
#pragma unroll
  for (int s = 0; s < SB; ++s) {
#pragma unroll
    for (int h = 1; h < LQ_K_GROUPS; ++h) acc[s] += part[((h - 1) * 4 + wave) * (SB * 64) + s * 64 + lane];
    *(f32x4*)(g.part + ((int64_t)blockIdx.y * g.m + token) * g.ldt + 16 * s + 4 * q) = acc[s];
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
// The operand of that: T itself, or three bf16 numbers whose sum is T.  Each takes eight of the 24 digits, and what it leaves is exact.  A number that eight digits
// hold gives its predecessor towards zero, so that something is left: all three have T's sign, and an infinite element of B meets no zero and no
// opposite sign (T inf is T's infinity whatever its digits, as of float32 operands; an infinite T has the largest number twice, then infinity).
template <typename T>
struct LqParts {
  static constexpr int N = sizeof(T) == 2 ? 3 : 1;
  typename Ln<T>::frag part[N];
};
template <typename T, int E>
__device__ inline LqParts<T> lq_parts(const float (&t)[E]) {
  constexpr int N = LqParts<T>::N;
  LqParts<T> f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    float left = t[e];
#pragma unroll
    for (int p = 0; p < N - 1; ++p) {
      const float cut = __uint_as_float((__float_as_uint(left) - (left != 0.0f)) & 0xffff0000u);
      f.part[p][e] = (T)cut;
      left -= cut;
    }
    f.part[N - 1][e] = (T)left;
  }
  return f;
}

template <typename O, int E>
struct LqOut {
  typedef O vec __attribute__((ext_vector_type(E)));
  typedef vec any __attribute__((aligned(sizeof(O))));
};
// Few tokens: tiles of 16 in the order they come; a wave has 16 E columns.  RS: steps of the rank.  (The conditions around its loads and stores are more than the scalar
// registers hold: 157 of them pass through vector registers for bf16 and rank up to 32, 319 beyond, 35 to 180 for float32.  They are part of its 9 us at 64 tokens,
// 4096 -> 4096, rank 16.)
template <typename T, typename O, int RS>
__global__ __launch_bounds__(64 * LQ_UP_WAVES) void lora_up_kernel(LqArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP;
  typedef typename Ln<T>::frag frag;
  typedef typename LqOut<O, E>::any out_any;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t col = ((int64_t)blockIdx.y * LQ_UP_WAVES + wave) * (16 * E) + E * c;       // of this lane's E columns
  if (col - E * c >= g.n) return;
  const int64_t first = (int64_t)blockIdx.x * 16;
  const int64_t mine = first + (lane < 16 ? lane : 0);
  const bool live = lane < 16 && mine < g.m;
  const int id = live ? g.ids[mine] : -1;
  const int64_t token = first + c < g.m ? first + c : g.m - 1;
  const int here = g.n - col < E ? (int)(g.n - col < 0 ? 0 : g.n - col) : E;                // columns that exist
  // R and Y of the lane's columns, in turn: read early, written when the product is there
  auto get = [&](int64_t row, float (&v)[E]) {
    const O* const rp = (const O*)g.R + row * g.ldr + col;
    if (g.R && here == E) {
      const typename LqOut<O, E>::vec y = *(const out_any*)rp;
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = (float)y[e];
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = g.R && e < here ? (float)rp[e] : 0.0f;
    }
  };
  auto put = [&](int64_t row, const float (&v)[E]) {
    O* const yp = (O*)g.Y + row * g.ldy + col;
    if (here == E) {
      typename LqOut<O, E>::vec y;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = (O)v[e];
      *(out_any*)yp = y;
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (e < here) yp[e] = (O)v[e];
    }
  };
  lq_adapters(g, id, live, blockIdx.z, [&](int d, uint64_t same) {
    const unsigned rows = (unsigned)same;
    const float by = g.scales ? g.scales[d] : 1.0f;
    float res[4][E];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (rows >> (4 * q + i) & 1) get(first + 4 * q + i, res[i]);
    f32x4 acc[E];
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    const T* const b0 = (const T*)g.B + (int64_t)d * g.r * g.n + col;
    frag v[RS][E];                                   // the lane's E x E blocks of B
#pragma unroll
    for (int s = 0; s < RS; ++s)
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int row = STEP * s + E * q + i;
        if (g.b_pieces) {
          v[s][i] = (frag){};
          if (row < g.r && here == E) v[s][i] = *(const frag*)(b0 + (int64_t)row * g.n);
        } else {
          v[s][i] = lq_load<T>(b0 + (int64_t)row * g.n, row < g.r ? here : 0);
        }
      }
#pragma unroll
    for (int s = 0; s < RS; ++s) {
      float t[E] = {};
      const int k = STEP * s + E * q;
      if ((rows >> c & 1) && k < g.r) lq_t<E>(g, token, k, by, t);            // (rows of other adapters may not be written at all)
      const LqParts<T> ts = lq_parts<T>(t);
#pragma unroll
      for (int j = 0; j < E; ++j) {                  // turned: column E c + j, rows STEP s + E q ..
        frag f;
        if constexpr (sizeof(T) == 2) {
          typedef unsigned int words __attribute__((ext_vector_type(4)));
          words w;
#pragma unroll
          for (int p = 0; p < 4; ++p)
            w[p] = __builtin_amdgcn_perm(__builtin_bit_cast(words, v[s][2 * p + 1])[j / 2], __builtin_bit_cast(words, v[s][2 * p])[j / 2],
                                         j & 1 ? 0x07060302u : 0x05040100u);
          f = __builtin_bit_cast(frag, w);
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) f[e] = v[s][e][j];
        }
#pragma unroll
        for (int p = 0; p < LqParts<T>::N; ++p) acc[j] = ln_mfma(ts.part[p], f, acc[j]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (rows >> (4 * q + i) & 1) {
        float y[E];
#pragma unroll
        for (int j = 0; j < E; ++j) y[j] = res[i][j] + acc[j][i];
        put(first + 4 * q + i, y);
      }
  });
  if (blockIdx.z) return;
  // tokens without an adapter, and with one that is not there (asked of all lanes, also those without columns: they hold tokens)
  const uint64_t past = __ballot(live && (int64_t)id >= g.adapters), none = __ballot(live && id < 0);
  for (uint64_t left = g.in_place ? past : past | none; left; left &= left - 1) {
    const int t = __builtin_ctzll(left);
    if ((t & 3) != q) continue;                      // (rows in turn: the lanes of a quarter hold all of the wave's columns)
    float v[E];
    get(first + t, v);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = past >> t & 1 ? __builtin_nanf("") : v[e];
    put(first + t, v);
  }
}

// Ordered tokens: a tile of 64, 16 to each wave, and `trips` times 16 E columns.  T is read once; the part of B for 16 E columns passes through LDS,
// the next one (and R) on its way meanwhile.  B gives the rows of the product, in an order that leaves a lane with E consecutive columns of its
// token: the transposing reads take chunks of four columns 2 E bytes apart.
template <typename T, typename O, int RS>
__global__ __launch_bounds__(64 * LQ_UP_WAVES) void lora_up_sorted_kernel(LqArgs g) {
  constexpr int E = Ln<T>::E, STEP = Ln<T>::STEP, PITCH = 256 + 64, J = 4, PIECES = RS * STEP / 16;      // (16 rows of 16 pieces at a time)
  typedef typename Ln<T>::frag frag;
  typedef typename LqOut<O, E>::any out_any;
  typedef typename LqOut<O, E>::vec out_vec;
  __shared__ __attribute__((aligned(16))) unsigned char smem[2][RS * STEP * PITCH];
  const int tile = blockIdx.x / g.groups;            // (the columns of a tile one after the other)
  if (tile >= g.tiles[0]) return;
  const int d = g.tiles[2 + 2 * tile], size = g.tiles[3 + 2 * tile];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int64_t first = (int64_t)(blockIdx.x - tile * g.groups) * g.trips * (16 * E);
  const int64_t end = first + (int64_t)g.trips * (16 * E) < g.n ? first + (int64_t)g.trips * (16 * E) : g.n;
  const bool there = (int64_t)d < g.adapters, work = 16 * wave < size, live = 16 * wave + c < size;
  const int64_t token = g.order[tile * LQ_TILE + (live ? 16 * wave + c : 0)];
  const T* const b = (const T*)g.B + (int64_t)(there ? d : 0) * g.r * g.n;
  const O* const rp = (const O*)g.R + token * g.ldr;
  O* const yp = (O*)g.Y + token * g.ldy;
  frag v[PIECES];
  out_vec res[J];
  auto load = [&](int64_t at) {
    const int64_t col = at + E * (threadIdx.x & 15);
    if (there) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int row = 16 * i + (threadIdx.x >> 4);
        v[i] = (frag){};
        if (row < g.r && col < g.n) v[i] = g.b_pieces ? *(const frag*)(b + (int64_t)row * g.n + col) : lq_load<T>(b + (int64_t)row * g.n + col, g.n - col);
      }
    }
    if (g.R && live) {
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (at + 4 * E * j + E * q + E <= g.n) res[j] = *(const out_any*)(rp + at + 4 * E * j + E * q);
    }
  };
  load(first);
  LqParts<T> ts[RS];
  if (there && work) {
    const float by = g.scales ? g.scales[d] : 1.0f;
#pragma unroll
    for (int s = 0; s < RS; ++s) {
      float t[E] = {};
      const int k = STEP * s + E * q;
      if (live && k < g.r) lq_t<E>(g, token, k, by, t);
      ts[s] = lq_parts<T>(t);
    }
  }
  int turn = 0;
  for (int64_t at = first; at < end; at += 16 * E, turn ^= 1) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) *(frag*)(smem[turn] + (16 * i + (threadIdx.x >> 4)) * PITCH + 16 * (threadIdx.x & 15)) = v[i];
    out_vec now[J];
#pragma unroll
    for (int j = 0; j < J; ++j) now[j] = res[j];
    if (at + 16 * E < end) load(at + 16 * E);
    sb_barrier_lds();                                // (two parts: who writes one has passed the barrier behind its last reading)
    if (!work) continue;
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
              const unsigned char* from = smem[turn] + (STEP * s + 8 * q + (c >> 2)) * PITCH + 64 * j + 16 * (c & 3) + 8 * h;
              const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)from);
              const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(from + 4 * PITCH));
              f = __builtin_bit_cast(frag, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
            } else {
#pragma unroll
              for (int e = 0; e < E; ++e) f[e] = *(const T*)(smem[turn] + (STEP * s + E * q + e) * PITCH + 64 * j + 4 * c);
            }
#pragma unroll
            for (int p = 0; p < LqParts<T>::N; ++p) acc[h] = ln_mfma(f, ts[s].part[p], acc[h]);
          }
      } else if ((int64_t)d > g.adapters) {
#pragma unroll
        for (int h = 0; h < E / 4; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[h][e] = __builtin_nanf("");
      }
      const int64_t col = at + 4 * E * j + E * q;
      if (!live || col >= g.n) continue;
      if (col + E <= g.n) {
        out_vec y;
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = (O)((g.R ? (float)now[j][e] : 0.0f) + acc[e / 4][e % 4]);
        *(out_any*)(yp + col) = y;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (col + e < g.n) yp[col + e] = (O)((g.R ? (float)rp[col + e] : 0.0f) + acc[e / 4][e % 4]);
      }
    }
  }
}

struct LqPlan {
  bool sorted;
  int64_t tiles;         // at most
  size_t part_bytes, tile_bytes, bytes;
  int splits, shares, up_shares, ldt, trips;
  int64_t k_per_split, groups;
};
static LqPlan lora_requests_plan(int64_t m, int64_t k, int64_t n, int r, int64_t adapters, bool bf16) {
  LqPlan p;
  const int e = bf16 ? 8 : 4;
  // Ordering costs a launch (4 us), which the walk's serial turns cost too where there are many adapters: 64 tokens of as many, 4096 -> 4096 at rank 16
  // (17 MB of A and B) 14 us in the order they come, 18 ordered; 4096 -> 11008 (31 MB) 27 both ways; at rank 64 (124 MB) 77 and 43.  More than 64 tokens are ordered
  // because the identifiers, which are not known here, may be mixed: 4096 -> 4096, rank 16, 128 tokens of 24 adapters in any order 20 us in the order they come, 13.5 ordered (5
  // adapters 14.1 and 12.6), 512 tokens 41 and 16, 1000 tokens 74 and 20.  Where they are not, that costs up to 4 us: 128 tokens of one adapter 10.3 and 13.4,
  // 1000 tokens 17 and 18.5; float32 1030 -> 770 of one adapter 8.5 and 13, of 24 mixed ones 12.6 and 13.3, 1000 tokens 38 and 17.
  const int64_t wide = 16 * e, cols = ceil_div64(n, wide), own = std::min(adapters, m);
  p.sorted = adapters <= LQ_SORTED && (m > 64 || r > 32 || (double)own * r * (double)(k + n) * (16 / e) > (double)(32 << 20));
  p.ldt = r <= 16 ? 16 : (r <= 32 ? 32 : 64);
  // K splits: 256 workgroups, of a slab (a step) for each group (wave) at least.  More parts of T cost the second launch more than they give the first: 64
  // tokens of as many adapters, 4096 -> 4096 at rank 16, 13.4 us with 256, 14.7 with 512, 20 with 1024.  Eight parts at most, which that launch has in
  // flight: one token 4096 -> 11008 9.6 us in a graph, 10.8 with sixteen parts, 9.2 with four; at rank 64, ordered, 14.5, 14.5 and 15.9.
  const int64_t tiles = p.sorted ? std::max(ceil_div64(m, LQ_TILE), own) : ceil_div64(m, 16), step = (p.sorted ? 16 * LQ_K_GROUPS : 4 * LQ_WAVES) * e;
  const int64_t most = std::min<int64_t>(16, adapters);
  p.shares = p.sorted ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, most));
  const int64_t splits = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(256 / (tiles * p.shares), ceil_div64(k, step)), 8));
  p.k_per_split = ceil_div64(ceil_div64(k, splits), step) * step;
  p.splits = (int)ceil_div64(k, p.k_per_split);
  // Second launch: in the order they come, 2048 waves (64 tokens as above 14.7 us, with 1024 of them 16.7, with 4096 14.7); ordered, up to four times
  // 16 E columns per workgroup, for T's sake (8192 tokens, 11008 columns, rank 64, four parts of T: once 217 us, twice 149, four times 124).
  p.up_shares = (int)std::max<int64_t>(1, std::min<int64_t>(2048 / (cols * tiles), most));
  p.trips = (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(tiles * cols / 1024, 4), cols));
  p.groups = ceil_div64(cols, p.trips);
  p.tiles = p.sorted ? ceil_div64(m, LQ_TILE) + std::min<int64_t>(adapters + 2, m) : 0;
  p.part_bytes = (size_t)p.splits * m * p.ldt * 4;
  p.tile_bytes = p.sorted ? align_up(8 + (size_t)p.tiles * 8, 16) : 0;
  p.bytes = p.part_bytes + p.tile_bytes + (size_t)p.tiles * LQ_TILE * 4;
  return p;
}
// Fewer than 2^32 threads to a launch, and than 65536 rows of workgroups.
static bool lora_requests_launches(const LqPlan& p, int64_t m, int64_t n, bool bf16) {
  const int64_t limit = (1ll << 32) / 512;
  if (p.sorted) return p.tiles * p.splits < limit / LQ_K_GROUPS * 2 && p.tiles * p.groups < 2 * limit && p.tiles < (1ll << 31) / LQ_TILE;
  const int64_t cols = ceil_div64(n, (bf16 ? 128 : 64) * LQ_UP_WAVES), tiles = ceil_div64(m, 16);
  return tiles * p.splits * p.shares < limit && cols < 65536 && tiles * cols * p.up_shares < 2 * limit;
}

template <typename T, typename O>
static int launch_lora_requests(hipStream_t s, LqArgs g, const LqPlan& p) {
  g.ldt = p.ldt; g.splits = p.splits; g.k_per_split = p.k_per_split; g.shares = p.shares; g.trips = p.trips; g.groups = (int)p.groups;
  const int steps = (g.r + Ln<T>::STEP - 1) / Ln<T>::STEP;
  const dim3 up_block(64 * LQ_UP_WAVES);
#define LQ_DOWN(KERNEL, GRID, BLOCK)                                                                 \
  do {                                                                                               \
    if (g.ldt == 16) LORACT_LAUNCH("lora_requests_down", s, (KERNEL<T, 1>), GRID, BLOCK, 0, g);       \
    else if (g.ldt == 32) LORACT_LAUNCH("lora_requests_down", s, (KERNEL<T, 2>), GRID, BLOCK, 0, g);  \
    else LORACT_LAUNCH("lora_requests_down", s, (KERNEL<T, 4>), GRID, BLOCK, 0, g);                   \
  } while (0)
#define LQ_UP(KERNEL, GRID)                                                                                                     \
  do {                                                                                                                          \
    if (steps == 1) LORACT_LAUNCH("lora_requests_up", s, (KERNEL<T, O, 1>), GRID, up_block, 0, g);                               \
    else if (steps == 2) LORACT_LAUNCH("lora_requests_up", s, (KERNEL<T, O, 2>), GRID, up_block, 0, g);                          \
    else if constexpr (sizeof(T) == 4) LORACT_LAUNCH("lora_requests_up", s, (KERNEL<T, O, 4>), GRID, up_block, 0, g);            \
  } while (0)
  if (p.sorted) {
    g.tiles = (int*)((char*)g.part + p.part_bytes);
    g.order = (int*)((char*)g.tiles + p.tile_bytes);
    LORACT_LAUNCH("lora_requests_sort", s, lora_sort_kernel, dim3(1), dim3(1024), 0, g);
    const dim3 down((unsigned)p.tiles, (unsigned)p.splits), up((unsigned)(p.tiles * p.groups));
    LQ_DOWN(lora_down_sorted_kernel, down, dim3(256 * LQ_K_GROUPS));
    LQ_UP(lora_up_sorted_kernel, up);
    return LORACT_OK;
  }
  const dim3 down((unsigned)ceil_div64(g.m, 16), (unsigned)p.splits, (unsigned)p.shares);
  LQ_DOWN(lora_down_kernel, down, dim3(64 * LQ_WAVES));
  g.shares = p.up_shares;
  const dim3 up((unsigned)ceil_div64(g.m, 16), (unsigned)ceil_div64(g.n, 16 * Ln<T>::E * LQ_UP_WAVES), (unsigned)p.up_shares);
  LQ_UP(lora_up_kernel, up);
#undef LQ_DOWN
#undef LQ_UP
  return LORACT_OK;
}

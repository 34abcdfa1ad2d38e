// RMS norm of every head of queries and keys and the rotation by position, in one pass, forward and backward.
//
//   forward   xh = x / sqrt(mean_d x_d^2 + eps),  y = Rot(xh * gamma)
//             Rot turns the pairs (a_i, b_i), i < rot / 2, of the first `rot` elements by the angle of (position, i):
//             (a c - b s, a s + b c); a_i, b_i are elements i and i + rot / 2, or 2 i and 2 i + 1 (interleaved)
//   backward  t = Rot^T dy,  dgamma = sum t xh,  u = t gamma,  dx = (u - xh mean(u xh)) / rms
//             from x itself: the statistics are two sums over a row that is in registers, cheaper than reading them
//
// Bound by memory: x is read and y written once (backward: x and dy read, dx written).  A head is held by L lanes of
// a wave, a 16-byte piece each; sums go over these lanes, and where the partner of an element is in another
// lane it comes by a lane exchange.  A wave keeps to one token while it walks over the heads, so that cos, sin and gamma
// stay in registers: the table is 2 to 4 times the bytes of a bf16 head, and would otherwise pass through L1 for each.
// gamma's gradients are summed in registers over the rows of a wave, then over the waves in LDS and over the
// workgroups through partial sums, in a fixed order.  8192 tokens of 32 + 8 heads of 128 bf16: forward 38 us (4.4 TB/s; a copy 5.1),
// backward 52 us with its join (4.8); float32 62 and 104.
#pragma once
#include "common.h"

#include <algorithm>

struct QkStream {
  const void* x;         // token t, head h, element d at x + t ldt + h ldh + d
  int64_t ldt, ldh;
  const void* dy;        // backward: gradient of the forward's output
  int64_t dy_ldt, dy_ldh;
  void* out;             // y, or dx
  int64_t out_ldt, out_ldh;
  const float* gamma;    // d, or null (ones)
  int heads;
  int chunk;             // heads that a wave takes at a time
  int per_token;         // chunks per token
  int blocks;            // workgroups
  float* part;           // backward: [block][d_pad] partial sums of dgamma, or null
};
struct QkArgs {
  QkStream q, k;         // k.heads may be 0
  int64_t m;
  int d, rot;
  int d_pad;
  const int32_t* pos;    // null: the token's own index
  int64_t n_pos;
  const float* table;    // position, cos then sin, rot / 2 each
  float eps;
};

#define QK_WAVES 4
// Where a token has no position (negative) its rows are zero, forward and backward; past the table they are NaN.
enum { QK_LIVE = 0, QK_PAD = 1, QK_PAST = 2 };
__device__ inline int qk_position(const QkArgs& g, int64_t token, int64_t* row) {
  const int64_t p = g.pos ? (int64_t)g.pos[token] : token;
  *row = p < 0 ? 0 : (p < g.n_pos ? p : g.n_pos - 1);
  return p < 0 ? QK_PAD : (p < g.n_pos ? QK_LIVE : QK_PAST);
}

// a c + b s.  For float32 gradients to one rounding of the whole: what the rounding of b s left is added, so that a difference of nearly
// equal terms keeps its digits (b s may be infinite, then what it left is no number and must not count).  A bf16 gradient has none to keep,
// and its pass of 8192 x (32 + 8) x 128 would take 55.7 us instead of 51.8 (float32: 104.2, 102.9).
template <typename T>
__device__ inline float qk_turn_back(float a, float c, float b, float s) {
  if (sizeof(T) < 4) return a * c + b * s;
  const float p = b * s;
  return fmaf(a, c, p) + fmaxf(fmaf(b, s, -p), -1e30f);
}

// T: element type.  E: elements per piece.  L: lanes per head (a power of two, L E >= d).  INTER: interleaved pairs.  d, rot and
// (unless INTER) rot / 2 are multiples of E.
template <typename T, int E, int L, bool INTER, bool BWD>
__global__ __launch_bounds__(64 * QK_WAVES) void qknorm_rope_kernel(QkArgs g) {
  constexpr int HPW = 64 / L;                        // heads of a wave at a time
  constexpr int U = BWD ? 2 : 4;                     // head groups in flight
  typedef T piece __attribute__((ext_vector_type(E)));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool is_k = (int)blockIdx.x >= g.q.blocks;
  const QkStream& st = is_k ? g.k : g.q;
  const int block = is_k ? (int)blockIdx.x - g.q.blocks : (int)blockIdx.x;
  const int p = lane & (L - 1), sub = lane / L;      // piece of the head, head of the group
  const int at = p * E;
  const bool on = at < g.d;
  const int half = g.rot / 2, hp = half / E;         // pieces of a half
  const bool turn = at < g.rot;
  const int partner = INTER || !turn ? lane : (p < hp ? lane + hp : lane - hp);
  const float sign = p < hp ? -1.0f : 1.0f;          // of the partner's share (not INTER)
  float gm[E], dg[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    gm[e] = on ? (st.gamma ? st.gamma[at + e] : 1.0f) : 0.0f;
    dg[e] = 0.0f;
  }
  const float inv_d = 1.0f / (float)g.d;
  const int64_t items = g.m * st.per_token;
  for (int64_t item = (int64_t)block * QK_WAVES + wave; item < items; item += (int64_t)st.blocks * QK_WAVES) {
    const int64_t token = item / st.per_token;
    const int h_beg = (int)(item - token * st.per_token) * st.chunk;
    const int h_end = h_beg + st.chunk < st.heads ? h_beg + st.chunk : st.heads;
    int64_t trow;
    const int state = qk_position(g, token, &trow);
    // c, s: of this lane's elements (INTER: of its pairs, in the first E / 2)
    float c[E], s[E];
    const float* tab = g.table + trow * g.rot;
#pragma unroll
    for (int e = 0; e < E; ++e) { c[e] = 1.0f; s[e] = 0.0f; }
    if (turn && on) {
      if (INTER) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) { c[e] = tab[at / 2 + e]; s[e] = tab[half + at / 2 + e]; }
      } else {
        const int i0 = (p < hp ? p : p - hp) * E;
#pragma unroll
        for (int e = 0; e < E; ++e) { c[e] = tab[i0 + e]; s[e] = tab[half + i0 + e]; }
      }
    }
    for (int h0 = h_beg; h0 < h_end; h0 += U * HPW) {
      piece x[U], dy[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h0 + u * HPW >= h_end) break;            // (uniform)
        int h = h0 + u * HPW + sub;
        if (h > h_end - 1) h = h_end - 1;            // heads past the end repeat the last one and are not stored
        const int a = on ? at : 0;
        x[u] = *(const piece*)((const T*)st.x + token * st.ldt + h * st.ldh + a);
        if (BWD) dy[u] = *(const piece*)((const T*)st.dy + token * st.dy_ldt + h * st.dy_ldh + a);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h0 + u * HPW >= h_end) break;
        const int h = h0 + u * HPW + sub;
        const bool store = on && h < h_end;
        float v[E], t[E];
        float ss = 0.0f, in = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          v[e] = on ? (float)x[u][e] : 0.0f;
          ss += v[e] * v[e];
        }
        if (BWD) {                                   // t = Rot^T dy
#pragma unroll
          for (int e = 0; e < E; ++e) t[e] = (float)dy[u][e];
          if (INTER) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
              const float a = t[2 * e], b = t[2 * e + 1];
              t[2 * e] = qk_turn_back<T>(a, c[e], b, s[e]);
              t[2 * e + 1] = qk_turn_back<T>(b, c[e], a, -s[e]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float o = __shfl(t[e], partner);
              if (sizeof(T) == 4) t[e] = turn ? qk_turn_back<T>(t[e], c[e], o, -sign * s[e]) : t[e];
              else t[e] = turn ? t[e] * c[e] - sign * (o * s[e]) : t[e];
            }
          }
#pragma unroll
          for (int e = 0; e < E; ++e) {
            if (state != QK_LIVE || !on) t[e] = state == QK_PAST && on ? NAN : 0.0f;
            in += t[e] * gm[e] * v[e];
          }
        }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) {
          ss += __shfl_xor(ss, o);
          if (BWD) in += __shfl_xor(in, o);
        }
        const float inv = 1.0f / sqrtf(ss * inv_d + g.eps);
        piece out;
        if (!BWD) {
          float y[E];
#pragma unroll
          for (int e = 0; e < E; ++e) y[e] = v[e] * inv * gm[e];
          if (INTER) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
              const float a = y[2 * e], b = y[2 * e + 1];
              y[2 * e] = a * c[e] - b * s[e];
              y[2 * e + 1] = a * s[e] + b * c[e];
            }
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float o = __shfl(y[e], partner);
              y[e] = turn ? y[e] * c[e] + sign * (o * s[e]) : y[e];
            }
          }
#pragma unroll
          for (int e = 0; e < E; ++e) out[e] = (T)(state == QK_LIVE ? y[e] : (state == QK_PAD ? 0.0f : NAN));
        } else {
          const float inner = in * inv * inv_d;      // mean(u xh)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float xh = v[e] * inv;
            if (state == QK_PAD) {
              out[e] = (T)0.0f;
            } else {
              if (store) dg[e] += t[e] * xh;
              out[e] = (T)((t[e] * gm[e] - xh * inner) * inv);
            }
          }
        }
        if (store) *(piece*)((T*)st.out + token * st.out_ldt + h * st.out_ldh + at) = out;
      }
    }
  }
  if (!BWD || !st.part) return;
  // heads of the wave, then the waves one after the other
  __shared__ float red[64 * E];
#pragma unroll
  for (int e = 0; e < E; ++e)
#pragma unroll
    for (int o = L; o < 64; o <<= 1) dg[e] += __shfl_xor(dg[e], o);
  for (int w = 0; w < QK_WAVES; ++w) {
    if (wave == w && sub == 0)
#pragma unroll
      for (int e = 0; e < E; ++e) red[at + e] = (w ? red[at + e] : 0.0f) + dg[e];
    __syncthreads();
  }
  for (int i = threadIdx.x; i < g.d; i += 64 * QK_WAVES) st.part[(int64_t)block * g.d_pad + i] = red[i];
}

// Any head size (up to LORACT_MAX_HEAD), alignment and pairing: a wave per head and token, element by element in two sweeps.
template <typename T, bool BWD>
__global__ __launch_bounds__(64 * QK_WAVES) void qknorm_rope_any_kernel(QkArgs g, int interleaved) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const bool is_k = (int)blockIdx.x >= g.q.blocks;
  const QkStream& st = is_k ? g.k : g.q;
  const int block = is_k ? (int)blockIdx.x - g.q.blocks : (int)blockIdx.x;
  __shared__ float acc[BWD ? QK_WAVES : 1][BWD ? LORACT_MAX_HEAD : 1];
  if (BWD)
    for (int i = lane; i < g.d; i += 64) acc[wave][i] = 0.0f;
  __syncthreads();                                   // (from here on an element belongs to one lane)
  const int half = g.rot / 2, units = half + (g.d - g.rot);        // pairs, then single elements
  const int64_t items = g.m * st.heads;
  for (int64_t item = (int64_t)block * QK_WAVES + wave; item < items; item += (int64_t)st.blocks * QK_WAVES) {
    const int64_t token = item / st.heads, h = item - token * st.heads;
    int64_t trow;
    const int state = qk_position(g, token, &trow);
    const float* tab = g.table + trow * g.rot;
    const T* x = (const T*)st.x + token * st.ldt + h * st.ldh;
    const T* dy = (const T*)st.dy + token * st.dy_ldt + h * st.dy_ldh;
    T* out = (T*)st.out + token * st.out_ldt + h * st.out_ldh;
    float ss = 0.0f, in = 0.0f, inv = 0.0f, inner = 0.0f;
    for (int sweep = 0; sweep < 2; ++sweep) {
      for (int i = lane; i < units; i += 64) {
        const bool pair = i < half;
        const int ia = pair ? (interleaved ? 2 * i : i) : i + half, ib = pair ? (interleaved ? 2 * i + 1 : i + half) : ia;
        const float xa = (float)x[ia], xb = pair ? (float)x[ib] : 0.0f;
        const float c = pair ? tab[i] : 1.0f, s = pair ? tab[half + i] : 0.0f;
        const float ga = st.gamma ? st.gamma[ia] : 1.0f, gb = pair ? (st.gamma ? st.gamma[ib] : 1.0f) : 0.0f;
        float ta = 0.0f, tb = 0.0f;
        if (BWD) {
          const float da = (float)dy[ia], db = pair ? (float)dy[ib] : 0.0f;
          ta = qk_turn_back<T>(da, c, db, s);
          tb = qk_turn_back<T>(db, c, da, -s);
          if (state != QK_LIVE) { ta = tb = state == QK_PAST ? NAN : 0.0f; }
        }
        if (sweep == 0) {
          ss += xa * xa + xb * xb;
          if (BWD) in += ta * ga * xa + (pair ? tb * gb * xb : 0.0f);
          continue;
        }
        const float ha = xa * inv, hb = xb * inv;
        float oa, ob;
        if (BWD) {
          oa = (ta * ga - ha * inner) * inv;
          ob = (tb * gb - hb * inner) * inv;
          if (state != QK_PAD) {
            acc[wave][ia] += ta * ha;
            if (pair) acc[wave][ib] += tb * hb;
          }
        } else {
          const float ya = ha * ga, yb = hb * gb;
          oa = pair ? ya * c - yb * s : ya;
          ob = ya * s + yb * c;
          if (state == QK_PAST) oa = ob = NAN;
        }
        if (state == QK_PAD) oa = ob = 0.0f;
        out[ia] = (T)oa;
        if (pair) out[ib] = (T)ob;
      }
      if (sweep == 0) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          ss += __shfl_xor(ss, o);
          if (BWD) in += __shfl_xor(in, o);
        }
        inv = 1.0f / sqrtf(ss / (float)g.d + g.eps);
        inner = in * inv / (float)g.d;
      }
    }
  }
  if (!BWD || !st.part) return;
  __syncthreads();
  for (int i = threadIdx.x; i < g.d; i += 64 * QK_WAVES) {
    float s = acc[0][i];
    for (int w = 1; w < QK_WAVES; ++w) s += acc[w][i];
    st.part[(int64_t)block * g.d_pad + i] = s;
  }
}

// dgamma of both streams (blockIdx.x) from the workgroups' partial sums.  Sixteen elements per workgroup, 64 threads to each of
// them: a thread takes every 64th partial sum in order, sixteen of them in flight, then 64 sums are added pair by pair.
struct QkJoin {
  const float* part[2];
  int blocks[2];
  float* out[2];
  int d, d_pad;
};
__global__ __launch_bounds__(1024) void qknorm_join_kernel(QkJoin g) {
  __shared__ float red[64][17];
  const int which = blockIdx.x, c = threadIdx.x & 15, i = blockIdx.y * 16 + c, w = threadIdx.x >> 4;
  if (!g.out[which]) return;
  const float* src = g.part[which] + i;              // (rows are padded past d)
  const int blocks = g.blocks[which];
  float s = 0.0f;
  for (int b0 = w; b0 < blocks; b0 += 1024) {
    float v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = src[(int64_t)(b0 + 64 * u < blocks ? b0 + 64 * u : b0) * g.d_pad];
#pragma unroll
    for (int u = 0; u < 16; ++u)
      if (b0 + 64 * u < blocks) s += v[u];
  }
  red[w][c] = s;
  for (int h = 32; h > 0; h >>= 1) {
    __syncthreads();
    if (w < h) red[w][c] += red[w + h][c];
  }
  if (w == 0 && i < g.d) g.out[which][i] = red[0][c];
}

// cos and sin of position * theta^(-2 i / rot), the angle in float64.
__global__ __launch_bounds__(256) void rope_table_kernel(float* table, int64_t n_pos, int half, double theta, int64_t first) {
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < n_pos * half; e += (int64_t)gridDim.x * 256) {
    const int64_t p = e / half;
    const int i = (int)(e - p * half);
    const double angle = (double)(first + p) * pow(theta, -(double)i / (double)half);
    double s, c;
    sincos(angle, &s, &c);
    table[p * 2 * half + i] = (float)c;
    table[p * 2 * half + half + i] = (float)s;
  }
}

// How a call is laid out: lanes per head and pieces, or the kernel that takes anything.
struct QkPlan {
  int e, l;              // l = 0: qknorm_rope_any_kernel
  int q_blocks, k_blocks, q_chunk, k_chunk;
  int d_pad;
  size_t part_bytes;
};
static QkPlan qknorm_plan(int64_t m, int hq, int hk, int d, int rot, bool inter, bool bf16, bool aligned16, bool aligned8, bool bwd) {
  QkPlan p;
  auto fits = [&](int e) { return d % e == 0 && rot % e == 0 && (inter || (rot / 2) % e == 0) && d / e <= 64; };
  p.e = bf16 ? (aligned16 && fits(8) ? 8 : (aligned8 && fits(4) ? 4 : 0)) : (aligned16 && fits(4) ? 4 : 0);
  p.l = 0;
  if (p.e) {
    p.l = 4;
    while (p.l * p.e < d) p.l *= 2;
  }
  // A wave takes all heads of a token where that leaves 2048 waves; else as few as one group of them.
  const int hpw = p.l ? 64 / p.l : 1;
  const int total = 2048;
  auto shape = [&](int heads, int* chunk, int* blocks) {
    if (!heads) { *chunk = 1; *blocks = 0; return; }
    const int groups = (heads + hpw - 1) / hpw;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(groups, ceil_div64(total, m)));
    *chunk = p.l ? (int)((groups + parts - 1) / parts) * hpw : 1;
    const int64_t items = m * ceil_div64(heads, *chunk);
    // backward sums gamma's gradient over a wave's items: no more workgroups than fill the card a few times
    *blocks = (int)std::min<int64_t>(ceil_div64(items, QK_WAVES), bwd ? 1024 : 4096);
  };
  shape(hq, &p.q_chunk, &p.q_blocks);
  shape(hk, &p.k_chunk, &p.k_blocks);
  p.d_pad = (d + 63) / 64 * 64;
  p.part_bytes = bwd ? (size_t)(p.q_blocks + p.k_blocks) * p.d_pad * 4 : 0;
  return p;
}

template <typename T, int E, bool BWD>
static int launch_qknorm_pieces(hipStream_t s, const QkArgs& g, int l, bool inter, const char* name) {
  const dim3 grid((unsigned)(g.q.blocks + g.k.blocks));
#define QK_CASE(L)                                                                                                       \
  case L:                                                                                                                \
    if (inter) LORACT_LAUNCH(name, s, (qknorm_rope_kernel<T, E, L, true, BWD>), grid, dim3(64 * QK_WAVES), 0, g);          \
    else LORACT_LAUNCH(name, s, (qknorm_rope_kernel<T, E, L, false, BWD>), grid, dim3(64 * QK_WAVES), 0, g);               \
    break;
  switch (l) {
    QK_CASE(4)
    QK_CASE(8)
    QK_CASE(16)
    QK_CASE(32)
    QK_CASE(64)
    default: return LORACT_ERR_UNSUPPORTED;
  }
#undef QK_CASE
  return LORACT_OK;
}

template <bool BWD>
static int launch_qknorm(hipStream_t s, QkArgs g, const QkPlan& p, bool bf16, bool inter) {
  const char* name = BWD ? "qknorm_rope_backward" : "qknorm_rope_forward";
  g.d_pad = p.d_pad;
  g.q.blocks = p.q_blocks; g.q.chunk = p.q_chunk; g.q.per_token = (int)ceil_div64(g.q.heads, p.q_chunk);
  g.k.blocks = p.k_blocks; g.k.chunk = p.k_chunk; g.k.per_token = (int)ceil_div64(g.k.heads, p.k_chunk);
  if (p.e == 8) return launch_qknorm_pieces<bf16_t, 8, BWD>(s, g, p.l, inter, name);
  if (p.e == 4 && bf16) return launch_qknorm_pieces<bf16_t, 4, BWD>(s, g, p.l, inter, name);
  if (p.e == 4) return launch_qknorm_pieces<float, 4, BWD>(s, g, p.l, inter, name);
  const dim3 grid((unsigned)(p.q_blocks + p.k_blocks));
  if (bf16) LORACT_LAUNCH(name, s, (qknorm_rope_any_kernel<bf16_t, BWD>), grid, dim3(64 * QK_WAVES), 0, g, (int)inter);
  else LORACT_LAUNCH(name, s, (qknorm_rope_any_kernel<float, BWD>), grid, dim3(64 * QK_WAVES), 0, g, (int)inter);
  return LORACT_OK;
}

// libloract: the operators of the sub-layer around a compressed activation -- linear maps with their epilogue and its
// backward pass, dropout, norm and rotation of queries and keys.  See include/loract.h.
#include "common.h"
#include "dropout.h"
#include "linear_backward.h"
#include "linear_large.h"
#include "linear_thin.h"
#include "linear_tile.h"
#include "overlap.h"
#include "qknorm.h"

#include <algorithm>
#include <cmath>

// Sizes are limited so that grids and 32-bit tile indexes hold; strides and offsets are 64 bits.
static bool extent_ok(int64_t v) { return v >= 1 && v <= (1ll << 30); }

static bool aligned_rows(const void* p, int64_t ld, int64_t elems, size_t bytes) {
  return !p || (((uintptr_t)p) % bytes == 0 && ld % elems == 0);
}

static int check_linear(const loract_linear_params* p) {
  if (!p) return LORACT_ERR_INVALID_ARG;
  if (p->m < 1 || p->n_out < 1 || p->r_lora < 0) return LORACT_ERR_INVALID_ARG;
  if (!dtype_ok(p->dtype) || p->act < LORACT_ACT_NONE || p->act > LORACT_ACT_SILU) return LORACT_ERR_INVALID_ARG;
  if (!(p->p_drop >= 0.0 && p->p_drop < 1.0)) return LORACT_ERR_INVALID_ARG;
  if (!extent_ok(p->m) || !extent_ok(p->n_out) || p->r_lora > LORACT_MAX_LORA_RANK) return LORACT_ERR_UNSUPPORTED;
  return LORACT_OK;
}
static int check_linear_forward(const loract_linear_params* p) {
  LORACT_TRY(check_linear(p));
  if (p->n_in < 1 || !dtype_ok(p->out_dtype)) return LORACT_ERR_INVALID_ARG;
  if (p->w_layout != LORACT_W_OUT_IN && p->w_layout != LORACT_W_IN_OUT) return LORACT_ERR_INVALID_ARG;
  if (!extent_ok(p->n_in) || (p->dtype == LORACT_F32 && p->out_dtype != LORACT_F32)) return LORACT_ERR_UNSUPPORTED;
  if (!linear_tile_launches(p->m, p->n_out, p->n_in, p->w_layout == LORACT_W_OUT_IN, p->dtype == LORACT_BF16)) return LORACT_ERR_UNSUPPORTED;
  return LORACT_OK;
}

// Outputs of the linear map within what it reads, but the residual in place, or within each other.
static bool linear_outputs_meet(const loract_linear_params* p, const void* X, const void* W, const float* bias, const void* T, const void* B, const void* R,
                                const void* Y, const void* Z, const void* ws, size_t ws_bytes) {
  const int64_t size = p->dtype == LORACT_BF16 ? 2 : 4, y_size = p->out_dtype == LORACT_BF16 ? 2 : 4;
  const bool w_kc = p->w_layout == LORACT_W_OUT_IN;
  const Extent y = extent_rows(Y, p->m, p->ldy, p->n_out, y_size), z = extent_rows(Z, p->m, p->ldz, p->n_out, size);
  const Extent r = extent_rows(R, p->m, p->ldr, p->n_out, size);
  const Extent in[] = {extent_rows(X, p->m, p->ldx, p->n_in, size),
                       extent_rows(W, w_kc ? p->n_out : p->n_in, p->ldw, w_kc ? p->n_in : p->n_out, size), extent_bytes(bias, p->n_out * 4),
                       extent_bytes(p->r_lora ? T : nullptr, p->m * p->r_lora * size),
                       extent_bytes(p->r_lora ? B : nullptr, p->n_out * p->r_lora * size), extent_bytes(ws_bytes ? ws : nullptr, ws_bytes)};
  for (const Extent& e : in)
    if (extents_meet(y, e) || extents_meet(z, e)) return true;
  return extents_meet(y, z) || extents_meet(z, r) || meets_but_in_place(y, r);
}
// The same of its backward pass: dP in place of dY or Z.
static bool linear_backward_outputs_meet(const loract_linear_params* p, const void* dY, const void* Z, const void* T, const void* dP, const float* dbias,
                                         const float* dB, const void* ws, size_t ws_bytes) {
  const int64_t size = p->dtype == LORACT_BF16 ? 2 : 4;
  const Extent dy = extent_rows(dY, p->m, p->ldy, p->n_out, size), z = extent_rows(Z, p->m, p->ldz, p->n_out, size);
  const Extent dp = extent_rows(dP, p->m, p->ldp, p->n_out, size), t = extent_bytes(dB ? T : nullptr, p->m * p->r_lora * size);
  const Extent db = extent_bytes(dbias, p->n_out * 4), d_b = extent_bytes(dB, p->n_out * p->r_lora * 4);
  const Extent scratch = extent_bytes(dbias || dB ? ws : nullptr, ws_bytes);
  for (const Extent& e : {dy, z, dp, t, scratch})
    if (extents_meet(db, e) || extents_meet(d_b, e)) return true;
  return extents_meet(db, d_b) || meets_but_in_place(dp, dy) || meets_but_in_place(dp, z) || extents_meet(dp, t) || extents_meet(dp, scratch);
}

extern "C" {

int loract_dropout(const void* X_dev, int64_t ldx, const void* R_dev, int64_t ldr, int64_t m, int64_t n, int32_t dtype,
                   double p, uint64_t seed, void* Y_dev, int64_t ldy, void* stream) {
  if (!X_dev || !Y_dev || m < 1 || n < 1 || ldx < n || ldy < n || (R_dev && ldr < n)) return LORACT_ERR_INVALID_ARG;
  if (!dtype_ok(dtype) || !(p >= 0.0 && p < 1.0)) return LORACT_ERR_INVALID_ARG;
  if (!extent_ok(m) || !extent_ok(n)) return LORACT_ERR_UNSUPPORTED;
  const int64_t size = dtype == LORACT_BF16 ? 2 : 4;
  const Extent y = extent_rows(Y_dev, m, ldy, n, size);
  if (meets_but_in_place(y, extent_rows(X_dev, m, ldx, n, size)) || meets_but_in_place(y, extent_rows(R_dev, m, ldr, n, size))) return LORACT_ERR_INVALID_ARG;
  DropoutArgs g;
  g.X = X_dev; g.ldx = ldx; g.R = R_dev; g.ldr = R_dev ? ldr : 0; g.Y = Y_dev; g.ldy = ldy; g.m = m; g.n = n;
  g.d = drop_args(p, seed, n);
  const int64_t e = dtype == LORACT_BF16 ? 8 : 4;
  const bool vec = n % e == 0 && aligned_rows(X_dev, ldx, e, 16) && aligned_rows(R_dev, ldr, e, 16) && aligned_rows(Y_dev, ldy, e, 16);
  return dtype == LORACT_BF16 ? launch_dropout<bf16_t>((hipStream_t)stream, g, vec) : launch_dropout<float>((hipStream_t)stream, g, vec);
}

int loract_linear_workspace_bytes(const loract_linear_params* p, size_t* bytes) {
  if (!bytes) return LORACT_ERR_INVALID_ARG;
  LORACT_TRY(check_linear_forward(p));
  const bool bf16 = p->dtype == LORACT_BF16;
  *bytes = align_up(linear_tile_part_bytes(p->m, p->n_out, p->n_in, bf16), 256);
  const bool w_kc = p->w_layout == LORACT_W_OUT_IN;                   // (whichever form the call's addresses allow)
  const int form = linear_thin_form(p->m, p->n_out, p->n_in, p->ldx, p->ldw, w_kc, bf16);
  if (form) *bytes = std::max(*bytes, linear_thin_part_bytes(p->m, p->n_out, p->n_in, form, bf16));
  if (form || !bf16) return LORACT_OK;
  const LargePlan plan = linear_large_plan(p->m, p->n_out, p->n_in);
  const LargeSpace space = linear_large_space(plan, p->m, p->n_out, p->n_in, p->r_lora, p->ldx, p->ldw, w_kc);
  if (plan.tile && linear_large_pays(space, p->m, p->n_out)) *bytes = std::max(*bytes, space.total);
  return LORACT_OK;
}

int loract_linear(const void* X_dev, const void* W_dev, const float* bias_dev, const void* T_dev, const void* Blora_dev,
                  const void* R_dev, const loract_linear_params* p, void* Y_dev, void* Z_dev, void* ws_dev,
                  size_t ws_bytes, void* stream) {
  LORACT_TRY(check_linear_forward(p));
  const bool w_kc = p->w_layout == LORACT_W_OUT_IN, bf16 = p->dtype == LORACT_BF16;
  if (!X_dev || !W_dev || !Y_dev || (p->r_lora && (!T_dev || !Blora_dev))) return LORACT_ERR_INVALID_ARG;
  if (p->ldx < p->n_in || p->ldw < (w_kc ? p->n_in : p->n_out) || p->ldy < p->n_out) return LORACT_ERR_INVALID_ARG;
  if ((R_dev && p->ldr < p->n_out) || (Z_dev && p->ldz < p->n_out)) return LORACT_ERR_INVALID_ARG;
  size_t need = 0;
  LORACT_TRY(loract_linear_workspace_bytes(p, &need));
  if (need && (!ws_dev || ws_bytes < need)) return LORACT_ERR_WORKSPACE_TOO_SMALL;
  if (need && ((uintptr_t)ws_dev) % 16 != 0) return LORACT_ERR_INVALID_ARG;
  if (linear_outputs_meet(p, X_dev, W_dev, bias_dev, T_dev, Blora_dev, R_dev, Y_dev, Z_dev, ws_dev, need)) return LORACT_ERR_INVALID_ARG;
  LinearArgs g;
  g.X = X_dev; g.ldx = p->ldx; g.W = W_dev; g.ldw = p->ldw; g.r = p->r_lora; g.lora_scale = p->lora_scale;
  g.T = p->r_lora ? T_dev : nullptr; g.B = p->r_lora ? Blora_dev : nullptr;
  g.m = p->m; g.n = p->n_out; g.k = p->n_in; g.part = (float*)ws_dev; g.n_pad = 0; g.k_per_split = 0; g.splits = 1;
  LinEpilogue& e = g.e;
  e.bias = bias_dev; e.R = R_dev; e.ldr = R_dev ? p->ldr : 0; e.Y = Y_dev; e.ldy = p->ldy; e.Z = Z_dev; e.ldz = Z_dev ? p->ldz : 0;
  e.m = p->m; e.n = p->n_out; e.act = p->act; e.y_f32 = p->out_dtype == LORACT_F32;
  e.d = drop_args(p->p_drop, p->seed, p->n_out);
  const size_t quad = bf16 ? 8 : 16;
  e.vec = p->n_out % 4 == 0 && aligned_rows(R_dev, p->ldr, 4, quad) && aligned_rows(Z_dev, p->ldz, 4, quad) &&
          aligned_rows(Y_dev, p->ldy, 4, e.y_f32 ? 16 : 8);
  const int form = linear_thin_form(g.m, g.n, g.k, g.ldx, g.ldw, w_kc, bf16);
  if (form && linear_thin_fits(g, w_kc))
    return bf16 ? launch_linear_thin<bf16_t>((hipStream_t)stream, g, w_kc, form) : launch_linear_thin<float>((hipStream_t)stream, g, w_kc, form);
  if (bf16 && !form) {
    const LargePlan plan = linear_large_plan(g.m, g.n, g.k);
    const LargeSpace space = linear_large_space(plan, g.m, g.n, g.k, p->r_lora, g.ldx, g.ldw, w_kc);
    if (plan.tile && linear_large_pays(space, g.m, g.n) && linear_large_fits(g, w_kc, space))
      return launch_linear_large((hipStream_t)stream, g, w_kc, plan, space);
  }
  return bf16 ? launch_linear_tile<bf16_t>((hipStream_t)stream, g, w_kc) : launch_linear_tile<float>((hipStream_t)stream, g, w_kc);
}

int loract_linear_backward_workspace_bytes(const loract_linear_params* p, size_t* bytes) {
  if (!bytes) return LORACT_ERR_INVALID_ARG;
  LORACT_TRY(check_linear(p));
  *bytes = align_up(linear_backward_plan(p->m, p->n_out, p->r_lora, p->dtype == LORACT_BF16).bytes, 256);
  return LORACT_OK;
}

int loract_linear_backward(const void* dY_dev, const void* Z_dev, const void* T_dev, const loract_linear_params* p,
                           void* dP_dev, float* dbias_dev, float* dB_dev, void* ws_dev, size_t ws_bytes, void* stream) {
  LORACT_TRY(check_linear(p));
  const bool bf16 = p->dtype == LORACT_BF16, act = p->act != LORACT_ACT_NONE;
  if (!dY_dev || !dP_dev || (act && !Z_dev) || (dB_dev && (!T_dev || !p->r_lora))) return LORACT_ERR_INVALID_ARG;
  if (p->ldy < p->n_out || p->ldp < p->n_out || (act && p->ldz < p->n_out)) return LORACT_ERR_INVALID_ARG;
  const LinBackPlan plan = linear_backward_plan(p->m, p->n_out, dB_dev ? p->r_lora : 0, bf16);
  const bool sums = dbias_dev || dB_dev;
  if (sums && (!ws_dev || ws_bytes < plan.bytes)) return LORACT_ERR_WORKSPACE_TOO_SMALL;
  if (sums && ((uintptr_t)ws_dev) % 16 != 0) return LORACT_ERR_INVALID_ARG;
  if (linear_backward_outputs_meet(p, dY_dev, act ? Z_dev : nullptr, T_dev, dP_dev, dbias_dev, dB_dev, ws_dev, plan.bytes)) return LORACT_ERR_INVALID_ARG;
  LinBackArgs g;
  g.dY = dY_dev; g.lddy = p->ldy; g.Z = act ? Z_dev : nullptr; g.ldz = act ? p->ldz : 0; g.T = dB_dev ? T_dev : nullptr;
  g.r = dB_dev ? p->r_lora : 0; g.dP = dP_dev; g.lddp = p->ldp; g.m = p->m; g.n = p->n_out; g.act = p->act;
  g.part = sums ? (float*)ws_dev : nullptr; g.chunk = 0; g.n_pad = 0;
  g.d = drop_args(p->p_drop, p->seed, p->n_out);
  const int64_t e = bf16 ? 8 : 4;
  const bool vec = p->n_out % e == 0 && aligned_rows(dY_dev, p->ldy, e, 16) && aligned_rows(g.Z, g.ldz, e, 16) &&
                   aligned_rows(dP_dev, p->ldp, e, 16);
  return bf16 ? launch_linear_backward<bf16_t>((hipStream_t)stream, g, plan, vec, p->lora_scale, dbias_dev, dB_dev)
              : launch_linear_backward<float>((hipStream_t)stream, g, plan, vec, p->lora_scale, dbias_dev, dB_dev);
}

int loract_rope_table(float* table_dev, int64_t n_pos, int32_t rot, double theta, int64_t first, void* stream) {
  if (!table_dev || n_pos < 1 || rot < 2 || rot % 2 || !(theta > 0.0) || first < 0) return LORACT_ERR_INVALID_ARG;
  if (!extent_ok(n_pos) || rot > LORACT_MAX_HEAD) return LORACT_ERR_UNSUPPORTED;
  const int64_t blocks = std::min<int64_t>(ceil_div64(n_pos * (rot / 2), 256), 4096);
  LORACT_LAUNCH("rope_table", (hipStream_t)stream, rope_table_kernel, dim3((unsigned)blocks), dim3(256), 0, table_dev, n_pos,
                rot / 2, theta, first);
  return LORACT_OK;
}

static int check_qk(const loract_qk_params* p) {
  if (!p) return LORACT_ERR_INVALID_ARG;
  if (p->m < 1 || p->heads_q < 1 || p->heads_k < 0 || p->d < 1 || p->rot < 0 || p->rot % 2 || p->rot > p->d) return LORACT_ERR_INVALID_ARG;
  if (!dtype_ok(p->dtype) || !(p->eps >= 0.0f) || (p->rot && p->n_pos < 1)) return LORACT_ERR_INVALID_ARG;
  if (!extent_ok(p->m) || p->d > LORACT_MAX_HEAD || p->heads_q > 65536 || p->heads_k > 65536) return LORACT_ERR_UNSUPPORTED;
  return LORACT_OK;
}
static Extent qk_extent(const loract_qk_params* p, const void* at, int heads, int64_t token, int64_t head) {
  return extent_heads(heads ? at : nullptr, p->m, token, heads, head, p->d, p->dtype == LORACT_BF16 ? 2 : 4);
}
// Whether the outputs (written) share memory with what is read, but one in place of the inputs of its own stream, or with each other.
struct QkOperands {
  Extent q, k, dq_out, dk_out;
  const float *gamma_q, *gamma_k, *table;
  const int32_t* pos;
};
static bool qk_outputs_meet(const loract_qk_params* p, const QkOperands& in, const Extent& oq, const Extent& ok, const Extent& scratch, const float* dgq,
                            const float* dgk) {
  const Extent read[] = {extent_bytes(in.gamma_q, p->d * 4), extent_bytes(in.gamma_k, p->d * 4), extent_bytes(in.pos, p->m * 4), scratch,
                         extent_bytes(p->rot ? in.table : nullptr, (wide_t)p->n_pos * p->rot * 4)};
  const Extent g[] = {extent_bytes(dgq, p->d * 4), extent_bytes(dgk, p->d * 4)};
  for (const Extent& e : read)
    if (extents_meet(oq, e) || extents_meet(ok, e) || extents_meet(g[0], e) || extents_meet(g[1], e)) return true;
  for (const Extent& e : {in.q, in.k, in.dq_out, in.dk_out, oq, ok})
    if (extents_meet(g[0], e) || extents_meet(g[1], e)) return true;
  return !extent_distinct(oq) || (ok.at && !extent_distinct(ok)) || extents_meet(oq, ok) || extents_meet(g[0], g[1]) || meets_but_in_place(oq, in.q) ||
         meets_but_in_place(oq, in.dq_out) || meets_but_in_place(ok, in.k) || meets_but_in_place(ok, in.dk_out) || extents_meet(oq, in.k) ||
         extents_meet(oq, in.dk_out) || extents_meet(ok, in.q) || extents_meet(ok, in.dq_out);
}
static bool qk_strides(const void* p, int64_t token, int64_t head, int elems, size_t bytes) {
  return ((uintptr_t)p) % bytes == 0 && token % elems == 0 && head % elems == 0;
}

int loract_qknorm_rope_workspace_bytes(const loract_qk_params* p, size_t* bytes) {
  if (!bytes) return LORACT_ERR_INVALID_ARG;
  LORACT_TRY(check_qk(p));
  size_t most = 0;                                   // whatever alignment the call turns out to have
  const bool bf16 = p->dtype == LORACT_BF16, inter = p->interleaved != 0;
  for (int a = 0; a < 3; ++a)
    most = std::max(most, qknorm_plan(p->m, p->heads_q, p->heads_k, p->d, p->rot, inter, bf16, a == 0, a < 2, true).part_bytes);
  *bytes = align_up(most, 256);
  return LORACT_OK;
}

int loract_qknorm_rope_forward(const void* q_dev, const void* k_dev, const loract_qk_params* p, const float* gamma_q_dev,
                               const float* gamma_k_dev, const float* table_dev, const int32_t* pos_dev, void* q_out_dev,
                               void* k_out_dev, void* stream) {
  LORACT_TRY(check_qk(p));
  const bool keys = p->heads_k > 0;
  if (!q_dev || !q_out_dev || (keys && (!k_dev || !k_out_dev)) || (p->rot && !table_dev)) return LORACT_ERR_INVALID_ARG;
  const QkOperands in = {qk_extent(p, q_dev, p->heads_q, p->q_token, p->q_head), qk_extent(p, k_dev, p->heads_k, p->k_token, p->k_head), {}, {},
                         gamma_q_dev, gamma_k_dev, table_dev, pos_dev};
  if (qk_outputs_meet(p, in, qk_extent(p, q_out_dev, p->heads_q, p->qo_token, p->qo_head), qk_extent(p, k_out_dev, p->heads_k, p->ko_token, p->ko_head), {},
                      nullptr, nullptr))
    return LORACT_ERR_INVALID_ARG;
  const bool bf16 = p->dtype == LORACT_BF16;
  auto aligned = [&](int elems) {
    const size_t b = (size_t)elems * (bf16 ? 2 : 4);
    return qk_strides(q_dev, p->q_token, p->q_head, elems, b) && qk_strides(q_out_dev, p->qo_token, p->qo_head, elems, b) &&
           (!keys || (qk_strides(k_dev, p->k_token, p->k_head, elems, b) && qk_strides(k_out_dev, p->ko_token, p->ko_head, elems, b)));
  };
  const QkPlan plan = qknorm_plan(p->m, p->heads_q, p->heads_k, p->d, p->rot, p->interleaved != 0, bf16, aligned(bf16 ? 8 : 4), aligned(4), false);
  QkArgs g{};
  g.m = p->m; g.d = p->d; g.rot = p->rot; g.pos = pos_dev; g.n_pos = p->rot ? p->n_pos : INT64_MAX; g.table = table_dev; g.eps = p->eps;
  g.q.x = q_dev; g.q.ldt = p->q_token; g.q.ldh = p->q_head; g.q.out = q_out_dev; g.q.out_ldt = p->qo_token; g.q.out_ldh = p->qo_head;
  g.k.x = k_dev; g.k.ldt = p->k_token; g.k.ldh = p->k_head; g.k.out = k_out_dev; g.k.out_ldt = p->ko_token; g.k.out_ldh = p->ko_head;
  g.q.gamma = gamma_q_dev; g.k.gamma = gamma_k_dev; g.q.heads = p->heads_q; g.k.heads = p->heads_k;
  return launch_qknorm<false>((hipStream_t)stream, g, plan, bf16, p->interleaved != 0);
}

int loract_qknorm_rope_backward(const void* q_dev, const void* k_dev, const loract_qk_params* p, const float* gamma_q_dev,
                                const float* gamma_k_dev, const float* table_dev, const int32_t* pos_dev,
                                const void* dq_out_dev, const void* dk_out_dev, void* dq_dev, void* dk_dev,
                                float* dgamma_q_dev, float* dgamma_k_dev, void* ws_dev, size_t ws_bytes, void* stream) {
  LORACT_TRY(check_qk(p));
  const bool keys = p->heads_k > 0;
  if (!q_dev || !dq_out_dev || !dq_dev || (keys && (!k_dev || !dk_out_dev || !dk_dev)) || (p->rot && !table_dev) ||
      (dgamma_k_dev && !keys))
    return LORACT_ERR_INVALID_ARG;
  const bool bf16 = p->dtype == LORACT_BF16;
  auto aligned = [&](int elems) {
    const size_t b = (size_t)elems * (bf16 ? 2 : 4);
    return qk_strides(q_dev, p->q_token, p->q_head, elems, b) && qk_strides(dq_dev, p->qo_token, p->qo_head, elems, b) &&
           qk_strides(dq_out_dev, p->dq_token, p->dq_head, elems, b) &&
           (!keys || (qk_strides(k_dev, p->k_token, p->k_head, elems, b) && qk_strides(dk_dev, p->ko_token, p->ko_head, elems, b) &&
                      qk_strides(dk_out_dev, p->dk_token, p->dk_head, elems, b)));
  };
  const QkPlan plan = qknorm_plan(p->m, p->heads_q, p->heads_k, p->d, p->rot, p->interleaved != 0, bf16, aligned(bf16 ? 8 : 4), aligned(4), true);
  const bool sums = dgamma_q_dev || dgamma_k_dev;
  if (sums && (!ws_dev || ws_bytes < plan.part_bytes)) return LORACT_ERR_WORKSPACE_TOO_SMALL;
  if (sums && ((uintptr_t)ws_dev) % 16 != 0) return LORACT_ERR_INVALID_ARG;
  const QkOperands in = {qk_extent(p, q_dev, p->heads_q, p->q_token, p->q_head), qk_extent(p, k_dev, p->heads_k, p->k_token, p->k_head),
                         qk_extent(p, dq_out_dev, p->heads_q, p->dq_token, p->dq_head), qk_extent(p, dk_out_dev, p->heads_k, p->dk_token, p->dk_head),
                         gamma_q_dev, gamma_k_dev, table_dev, pos_dev};
  if (qk_outputs_meet(p, in, qk_extent(p, dq_dev, p->heads_q, p->qo_token, p->qo_head), qk_extent(p, dk_dev, p->heads_k, p->ko_token, p->ko_head),
                      extent_bytes(sums ? ws_dev : nullptr, plan.part_bytes), dgamma_q_dev, dgamma_k_dev))
    return LORACT_ERR_INVALID_ARG;
  QkArgs g{};
  g.m = p->m; g.d = p->d; g.rot = p->rot; g.pos = pos_dev; g.n_pos = p->rot ? p->n_pos : INT64_MAX; g.table = table_dev; g.eps = p->eps;
  g.q.x = q_dev; g.q.ldt = p->q_token; g.q.ldh = p->q_head; g.q.out = dq_dev; g.q.out_ldt = p->qo_token; g.q.out_ldh = p->qo_head;
  g.k.x = k_dev; g.k.ldt = p->k_token; g.k.ldh = p->k_head; g.k.out = dk_dev; g.k.out_ldt = p->ko_token; g.k.out_ldh = p->ko_head;
  g.q.dy = dq_out_dev; g.q.dy_ldt = p->dq_token; g.q.dy_ldh = p->dq_head;
  g.k.dy = dk_out_dev; g.k.dy_ldt = p->dk_token; g.k.dy_ldh = p->dk_head;
  g.q.gamma = gamma_q_dev; g.k.gamma = gamma_k_dev; g.q.heads = p->heads_q; g.k.heads = p->heads_k;
  float* const parts = (float*)ws_dev;
  g.q.part = dgamma_q_dev ? parts : nullptr;
  g.k.part = dgamma_k_dev ? parts + (size_t)plan.q_blocks * plan.d_pad : nullptr;
  LORACT_TRY(launch_qknorm<true>((hipStream_t)stream, g, plan, bf16, p->interleaved != 0));
  if (!sums) return LORACT_OK;
  QkJoin j;
  j.part[0] = g.q.part; j.part[1] = g.k.part; j.blocks[0] = plan.q_blocks; j.blocks[1] = plan.k_blocks;
  j.out[0] = dgamma_q_dev; j.out[1] = dgamma_k_dev; j.d = p->d; j.d_pad = plan.d_pad;
  LORACT_LAUNCH("qknorm_rope_join", (hipStream_t)stream, qknorm_join_kernel, dim3(2, (unsigned)(plan.d_pad / 16)), dim3(1024), 0, j);
  return LORACT_OK;
}

}  // extern "C"

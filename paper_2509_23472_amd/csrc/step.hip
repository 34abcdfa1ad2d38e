// libloract: what a fine-tuning step ends with -- the loss and its gradient, the update of its parameters -- and
// the adapters of many requests that it serves.  See include/loract.h.
#include "common.h"
#include "adamw.h"
#include "logprobs.h"
#include "lora_requests.h"
#include "overlap.h"
#include "spans.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <new>

// ---------------------------------------------------------------------------------------------
// AdamW.

static int64_t adamw_padded(int64_t n) { return (int64_t)align_up((size_t)n, LORACT_ADAMW_BLOCK); }

static bool in_unit(double v) { return v >= 0.0 && v < 1.0; }
static bool at_least_zero(double v) { return v >= 0.0 && v <= 1.7e308; }
// (to the hardware's reciprocal a denominator below 2^-126 is zero: a parameter without a gradient would become 0 / 0)
static bool eps_ok(double v) { return v == 0.0 || (v >= 0x1p-126 && v <= 1.7e308); }

extern "C" {

int loract_adamw(void* const* p, const void* const* g, void* const* copy, const int64_t* n, int64_t count,
                 const loract_adamw_params* params, void* m_dev, void* v_dev, uint8_t* exps_dev, const float* lr_dev,
                 const int64_t* step_dev, const float* grad_scale_dev, void* stream) {
  if (!params || count < 0 || (count && (!p || !g || !n))) return LORACT_ERR_INVALID_ARG;
  if (!dtype_ok(params->p_dtype) || !dtype_ok(params->g_dtype) || (params->state_bits != 32 && params->state_bits != 8)) return LORACT_ERR_INVALID_ARG;
  if (!in_unit(params->beta1) || !in_unit(params->beta2) || !eps_ok(params->eps) || !at_least_zero(params->weight_decay)) return LORACT_ERR_INVALID_ARG;
  if ((!lr_dev && !at_least_zero(params->lr)) || (!step_dev && params->step < 1)) return LORACT_ERR_INVALID_ARG;
  if (count > (1 << 24)) return LORACT_ERR_UNSUPPORTED;
  const bool narrow = params->state_bits == 8, p_bf16 = params->p_dtype == LORACT_BF16, g_bf16 = params->g_dtype == LORACT_BF16;
  int64_t total = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (n[i] < 0 || (n[i] && (!p[i] || !g[i])) || (p_bf16 && copy && copy[i])) return LORACT_ERR_INVALID_ARG;
    if (n[i] && ((uintptr_t)p[i] % (p_bf16 ? 2 : 4) || (uintptr_t)g[i] % (g_bf16 ? 2 : 4) || (copy && (uintptr_t)copy[i] % 2))) return LORACT_ERR_INVALID_ARG;
    if (n[i] > (1ll << 33)) return LORACT_ERR_UNSUPPORTED;
    total += adamw_padded(n[i]);
    if (total > (1ll << 39)) return LORACT_ERR_UNSUPPORTED;
  }
  if (!total) return LORACT_OK;
  if (!m_dev || !v_dev || (narrow && !exps_dev)) return LORACT_ERR_INVALID_ARG;
  if ((uintptr_t)m_dev % 16 || (uintptr_t)v_dev % 16 || (narrow && (uintptr_t)exps_dev % 2)) return LORACT_ERR_INVALID_ARG;
  if ((uintptr_t)lr_dev % 4 || (uintptr_t)step_dev % 8 || (uintptr_t)grad_scale_dev % 4) return LORACT_ERR_INVALID_ARG;
  const uintptr_t m0 = (uintptr_t)m_dev, v0 = (uintptr_t)v_dev, e0 = (uintptr_t)exps_dev;
  const uintptr_t state_bytes = (uintptr_t)total * (narrow ? 1 : 4);
  const Span state[3] = {{m0, m0 + state_bytes}, {v0, v0 + state_bytes}, {e0, narrow ? e0 + (uintptr_t)total / LORACT_ADAMW_BLOCK * 2 : e0}};
  const Span scalars[3] = {{(uintptr_t)lr_dev, (uintptr_t)lr_dev + (lr_dev ? 4 : 0)}, {(uintptr_t)step_dev, (uintptr_t)step_dev + (step_dev ? 8 : 0)},
                           {(uintptr_t)grad_scale_dev, (uintptr_t)grad_scale_dev + (grad_scale_dev ? 4 : 0)}};
  const int meets = adamw_meets(p, g, copy, n, count, p_bf16 ? 2 : 4, g_bf16 ? 2 : 4, state, scalars);
  if (meets < 0) {
    g_host.last_hip_error = "no host memory to look the tensors over";
    return LORACT_ERR_HIP;
  }
  if (meets) return LORACT_ERR_INVALID_ARG;
  AdamwArgs a;
  a.m = m_dev; a.v = v_dev; a.exps = exps_dev; a.lr_dev = lr_dev; a.step_dev = step_dev; a.grad_scale_dev = grad_scale_dev;
  a.lr = params->lr; a.log2_beta1 = log2(params->beta1); a.log2_beta2 = log2(params->beta2); a.weight_decay = params->weight_decay;
  a.beta1 = (float)params->beta1; a.one_beta1 = (float)(1.0 - params->beta1);
  a.beta2 = (float)params->beta2; a.one_beta2 = (float)(1.0 - params->beta2);
  a.eps = (float)params->eps; a.seed = params->seed; a.step = params->step; a.rate = a.inv = a.decay = 0.0f;
  if (!lr_dev && !step_dev) adamw_rates(a, params->lr, pow(params->beta1, (double)params->step), pow(params->beta2, (double)params->step));
  const hipStream_t s = (hipStream_t)stream;
#define LORACT_ADAMW(P, G, COPY) launch_adamw<P, G, COPY>(s, a, narrow, p, g, copy, n, count)
  if (p_bf16) return g_bf16 ? LORACT_ADAMW(bf16_t, bf16_t, false) : LORACT_ADAMW(bf16_t, float, false);
  if (copy) return g_bf16 ? LORACT_ADAMW(float, bf16_t, true) : LORACT_ADAMW(float, float, true);
  return g_bf16 ? LORACT_ADAMW(float, bf16_t, false) : LORACT_ADAMW(float, float, false);
#undef LORACT_ADAMW
}

}  // extern "C"

// ---------------------------------------------------------------------------------------------
// Log probabilities.

static int check_logprobs(const loract_logprob_params* p, bool top) {
  if (!p || p->m < 1 || p->n < 1 || p->ld < p->n || !dtype_ok(p->dtype) || (p->target_bits != 32 && p->target_bits != 64)) return LORACT_ERR_INVALID_ARG;
  if (!(p->temperature > 0.0) || !std::isfinite((float)p->temperature) || !std::isfinite((float)(1.5 / p->temperature)) || p->reserved) return LORACT_ERR_INVALID_ARG;
  if (top && (p->top < 0 || p->top > p->n)) return LORACT_ERR_INVALID_ARG;
  if (p->m > (1 << 30) || p->n > (1 << 30) || (top && p->top > LORACT_MAX_TOP)) return LORACT_ERR_UNSUPPORTED;
  return LORACT_OK;
}
struct LpOperands {
  Extent x, targets, d_logp, d_entropy, logp, stats, top_logp, top_ids, grad, ws;
};
// Whether what is written shares memory with what is read or written beside it, but the gradient in place of the logits.
static bool logprobs_meet(const LpOperands& o) {
  const Extent out[] = {o.logp, o.stats, o.top_logp, o.top_ids, o.ws, o.grad};
  for (int i = 0; i < 6; ++i) {
    for (int j = i + 1; j < 6; ++j)
      if (extents_meet(out[i], out[j])) return true;
    for (const Extent& e : {o.targets, o.d_logp, o.d_entropy})
      if (extents_meet(out[i], e)) return true;
    if (i < 5 ? extents_meet(out[i], o.x) : meets_but_in_place(out[i], o.x)) return true;
  }
  return false;
}
static LpArgs logprob_args(const void* x, const void* targets, const loract_logprob_params* p) {
  LpArgs g{};
  g.x = x; g.ld = p->ld; g.m = p->m; g.n = p->n; g.targets = targets; g.target_64 = p->target_bits == 64;
  g.inv_t = (float)(1.0 / p->temperature); g.c = (float)(1.4426950408889634 / p->temperature); g.splits = 1;
  return g;
}
static bool at_multiple(const void* p, size_t bytes) { return (uintptr_t)p % bytes == 0; }
static bool logprobs_aligned(const void* x, const void* targets, const loract_logprob_params* p, std::initializer_list<const void*> words) {
  for (const void* w : words)
    if (!at_multiple(w, 4)) return false;
  return at_multiple(x, p->dtype == LORACT_BF16 ? 2 : 4) && at_multiple(targets, p->target_bits / 8);
}

extern "C" {

int loract_token_logprobs_workspace_bytes(const loract_logprob_params* p, size_t* bytes) {
  if (!bytes) return LORACT_ERR_INVALID_ARG;
  LORACT_TRY(check_logprobs(p, true));
  *bytes = align_up(lp_part_bytes(p->m, p->n, p->top, p->dtype == LORACT_BF16), 256);
  return LORACT_OK;
}

int loract_token_logprobs(const void* x_dev, const void* targets_dev, const loract_logprob_params* p, float* logp_dev,
                          float* stats_dev, float* top_logp_dev, int32_t* top_ids_dev, void* ws_dev, size_t ws_bytes, void* stream) {
  LORACT_TRY(check_logprobs(p, true));
  if (!x_dev || !stats_dev || (logp_dev && !targets_dev) || (p->top && (!top_logp_dev || !top_ids_dev))) return LORACT_ERR_INVALID_ARG;
  if (!logprobs_aligned(x_dev, targets_dev, p, {logp_dev, stats_dev, p->top ? top_logp_dev : nullptr, p->top ? top_ids_dev : nullptr})) return LORACT_ERR_INVALID_ARG;
  const size_t need = lp_part_bytes(p->m, p->n, p->top, p->dtype == LORACT_BF16);
  if (need && (!ws_dev || ws_bytes < need)) return LORACT_ERR_WORKSPACE_TOO_SMALL;
  if (need && !at_multiple(ws_dev, 16)) return LORACT_ERR_INVALID_ARG;
  const int64_t size = p->dtype == LORACT_BF16 ? 2 : 4;
  const LpOperands o = {extent_rows(x_dev, p->m, p->ld, p->n, size), extent_bytes(targets_dev, p->m * p->target_bits / 8), {}, {},
                        extent_bytes(logp_dev, p->m * 4), extent_bytes(stats_dev, p->m * 12), extent_bytes(p->top ? top_logp_dev : nullptr, p->m * p->top * 4),
                        extent_bytes(p->top ? top_ids_dev : nullptr, p->m * p->top * 4), {}, extent_bytes(need ? ws_dev : nullptr, need)};
  if (logprobs_meet(o)) return LORACT_ERR_INVALID_ARG;
  LpArgs g = logprob_args(x_dev, targets_dev, p);
  g.logp = logp_dev; g.stats = stats_dev; g.top = p->top; g.top_logp = top_logp_dev; g.top_ids = top_ids_dev;
  g.part = (float*)ws_dev;
  g.part_top = need ? (uint64_t*)((char*)ws_dev + (size_t)p->m * lp_splits(p->m, p->n, p->dtype == LORACT_BF16) * 16) : nullptr;
  return size == 2 ? launch_logprobs<bf16_t>((hipStream_t)stream, g) : launch_logprobs<float>((hipStream_t)stream, g);
}

int loract_token_logprobs_backward(const void* x_dev, const void* targets_dev, const loract_logprob_params* p, const float* stats_dev,
                                   const float* d_logp_dev, const float* d_entropy_dev, void* grad_dev, void* stream) {
  LORACT_TRY(check_logprobs(p, false));
  if (!x_dev || !stats_dev || !grad_dev || p->ldg < p->n || (!d_logp_dev && !d_entropy_dev) || (d_logp_dev && !targets_dev)) return LORACT_ERR_INVALID_ARG;
  const int64_t size = p->dtype == LORACT_BF16 ? 2 : 4;
  if (!logprobs_aligned(x_dev, targets_dev, p, {stats_dev, d_logp_dev, d_entropy_dev}) || !at_multiple(grad_dev, size)) return LORACT_ERR_INVALID_ARG;
  LpOperands o = {extent_rows(x_dev, p->m, p->ld, p->n, size), extent_bytes(targets_dev, p->m * p->target_bits / 8), extent_bytes(d_logp_dev, p->m * 4),
                  extent_bytes(d_entropy_dev, p->m * 4), {}, {}, {}, {}, extent_rows(grad_dev, p->m, p->ldg, p->n, size), {}};
  if (logprobs_meet(o) || extents_meet(o.grad, extent_bytes(stats_dev, p->m * 12))) return LORACT_ERR_INVALID_ARG;
  LpArgs g = logprob_args(x_dev, targets_dev, p);
  g.stats = (float*)stats_dev; g.d_logp = d_logp_dev; g.d_entropy = d_entropy_dev; g.grad = grad_dev; g.ldg = p->ldg;
  return size == 2 ? launch_logprobs_backward<bf16_t>((hipStream_t)stream, g) : launch_logprobs_backward<float>((hipStream_t)stream, g);
}

int loract_token_logprobs_grad(const void* x_dev, const void* targets_dev, const loract_logprob_params* p, const float* d_logp_dev,
                               const float* d_entropy_dev, float* logp_dev, float* stats_dev, void* grad_dev, void* ws_dev, size_t ws_bytes,
                               void* stream) {
  LORACT_TRY(check_logprobs(p, false));
  if (!x_dev || !stats_dev || !grad_dev || p->ldg < p->n || (!d_logp_dev && !d_entropy_dev)) return LORACT_ERR_INVALID_ARG;
  if ((d_logp_dev || logp_dev) && !targets_dev) return LORACT_ERR_INVALID_ARG;
  const int64_t size = p->dtype == LORACT_BF16 ? 2 : 4;
  if (!logprobs_aligned(x_dev, targets_dev, p, {logp_dev, stats_dev, d_logp_dev, d_entropy_dev}) || !at_multiple(grad_dev, size)) return LORACT_ERR_INVALID_ARG;
  const size_t need = lp_part_bytes(p->m, p->n, 0, p->dtype == LORACT_BF16);
  if (need && (!ws_dev || ws_bytes < need)) return LORACT_ERR_WORKSPACE_TOO_SMALL;
  if (need && !at_multiple(ws_dev, 16)) return LORACT_ERR_INVALID_ARG;
  const LpOperands o = {extent_rows(x_dev, p->m, p->ld, p->n, size), extent_bytes(targets_dev, p->m * p->target_bits / 8), extent_bytes(d_logp_dev, p->m * 4),
                        extent_bytes(d_entropy_dev, p->m * 4), extent_bytes(logp_dev, p->m * 4), extent_bytes(stats_dev, p->m * 12), {}, {},
                        extent_rows(grad_dev, p->m, p->ldg, p->n, size), extent_bytes(need ? ws_dev : nullptr, need)};
  if (logprobs_meet(o)) return LORACT_ERR_INVALID_ARG;
  LpArgs g = logprob_args(x_dev, targets_dev, p);
  g.logp = logp_dev; g.stats = stats_dev; g.d_logp = d_logp_dev; g.d_entropy = d_entropy_dev; g.grad = grad_dev; g.ldg = p->ldg; g.part = (float*)ws_dev;
  return size == 2 ? launch_logprobs_grad<bf16_t>((hipStream_t)stream, g) : launch_logprobs_grad<float>((hipStream_t)stream, g);
}

}  // extern "C"

// ---------------------------------------------------------------------------------------------
// Adapters of many requests.

static int check_requests(const loract_requests_params* p, LqPlan* plan) {
  if (!p || p->m < 1 || p->n_in < 1 || p->n_out < 1 || p->adapters < 1 || p->r < 1 || p->reserved) return LORACT_ERR_INVALID_ARG;
  if (!dtype_ok(p->dtype) || !dtype_ok(p->out_dtype) || p->ldx < p->n_in || p->ldy < p->n_out) return LORACT_ERR_INVALID_ARG;
  if (p->m > (1 << 27) || p->n_in > (1 << 30) || p->n_out > (1 << 24) || p->adapters > (1 << 30) || p->r > LORACT_MAX_LORA_RANK) return LORACT_ERR_UNSUPPORTED;
  const bool bf16 = p->dtype == LORACT_BF16;
  if (!bf16 && p->out_dtype == LORACT_BF16) return LORACT_ERR_UNSUPPORTED;
  *plan = lora_requests_plan(p->m, p->n_in, p->n_out, p->r, p->adapters, bf16);
  return lora_requests_launches(*plan, p->m, p->n_out, bf16) ? LORACT_OK : LORACT_ERR_UNSUPPORTED;
}

extern "C" {

int loract_lora_requests_workspace_bytes(const loract_requests_params* p, size_t* bytes) {
  LqPlan plan;
  if (!bytes) return LORACT_ERR_INVALID_ARG;
  LORACT_TRY(check_requests(p, &plan));
  *bytes = align_up(plan.bytes, 256);
  return LORACT_OK;
}

int loract_lora_requests(const void* X_dev, const void* A_dev, const void* B_dev, const int32_t* ids_dev, const float* scales_dev,
                         const void* R_dev, const loract_requests_params* p, void* Y_dev, void* ws_dev, size_t ws_bytes, void* stream) {
  LqPlan plan;
  LORACT_TRY(check_requests(p, &plan));
  if (!X_dev || !A_dev || !B_dev || !ids_dev || !Y_dev || (R_dev && p->ldr < p->n_out)) return LORACT_ERR_INVALID_ARG;
  const int64_t size = p->dtype == LORACT_BF16 ? 2 : 4, y_size = p->out_dtype == LORACT_BF16 ? 2 : 4;
  for (const void* at : {X_dev, A_dev, B_dev})
    if (!at_multiple(at, size)) return LORACT_ERR_INVALID_ARG;
  if (!at_multiple(ids_dev, 4) || !at_multiple(scales_dev, 4) || !at_multiple(R_dev, y_size) || !at_multiple(Y_dev, y_size)) return LORACT_ERR_INVALID_ARG;
  const size_t need = plan.bytes;
  if (!ws_dev || ws_bytes < need) return LORACT_ERR_WORKSPACE_TOO_SMALL;
  if (!at_multiple(ws_dev, 16)) return LORACT_ERR_INVALID_ARG;
  const Extent y = extent_rows(Y_dev, p->m, p->ldy, p->n_out, y_size), r = extent_rows(R_dev, p->m, p->ldr, p->n_out, y_size), ws = extent_bytes(ws_dev, need);
  for (const Extent& e : {extent_rows(X_dev, p->m, p->ldx, p->n_in, size), extent_bytes(A_dev, (wide_t)p->adapters * p->n_in * p->r * size),
                          extent_bytes(B_dev, (wide_t)p->adapters * p->n_out * p->r * size), extent_bytes(ids_dev, p->m * 4),
                          extent_bytes(scales_dev, p->adapters * 4)})
    if (extents_meet(y, e) || extents_meet(ws, e)) return LORACT_ERR_INVALID_ARG;
  if (extents_meet(y, ws) || extents_meet(r, ws) || meets_but_in_place(y, r)) return LORACT_ERR_INVALID_ARG;
  LqArgs g{};
  g.X = X_dev; g.ldx = p->ldx; g.A = A_dev; g.B = B_dev; g.ids = ids_dev; g.scales = scales_dev; g.R = R_dev; g.ldr = R_dev ? p->ldr : 0;
  g.Y = Y_dev; g.ldy = p->ldy; g.m = p->m; g.k = p->n_in; g.n = p->n_out; g.adapters = p->adapters; g.r = p->r; g.part = (float*)ws_dev;
  const int64_t e = 16 / size;
  g.a_pieces = p->r % e == 0 && at_multiple(A_dev, 16);
  g.b_pieces = p->n_out % e == 0 && at_multiple(B_dev, 16);
  g.in_place = R_dev == Y_dev;
  const hipStream_t s = (hipStream_t)stream;
  if (size == 4) return launch_lora_requests<float, float>(s, g, plan);
  return y_size == 2 ? launch_lora_requests<bf16_t, bf16_t>(s, g, plan) : launch_lora_requests<bf16_t, float>(s, g, plan);
}

}  // extern "C"

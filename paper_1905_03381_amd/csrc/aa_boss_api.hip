// C ABI of the operators of a Boss block of experts: argument checks and the choice of kernels.
#include "../../include/autoassist.h"

#include "aa_experts.hpp"
#include "aa_route.hpp"
#include "aa_rows.hpp"

#include <math.h>

using namespace aa;

namespace {

constexpr int32_t kMaxWidth = 1 << 24;           // row widths
constexpr int64_t kMaxPairs = (1ll << 31) - 4096;  // n_max * top_k

int32_t hip_status(hipError_t e) { return e == hipSuccess ? AA_OK : AA_ERR_HIP; }

hipStream_t as_stream(void *s) { return static_cast<hipStream_t>(s); }

bool on(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// 0 for an unknown type
int type_bytes(int32_t dtype) { return dtype == AA_F32 ? 4 : dtype == AA_BF16 || dtype == AA_F16 ? 2 : 0; }

// A matrix of `rows` rows: present (unless it has none), of a legal stride, on its type's alignment.
int32_t check_rows(const void *p, int64_t rows, int64_t ld, int64_t width, int bytes) {
  if (ld < width || ld > (1ll << 40)) return AA_ERR_SHAPE;
  if (rows > 0 && !p) return AA_ERR_NULL;
  return on(p, (size_t)bytes) ? AA_OK : AA_ERR_ALIGN;
}

// int32 / float arrays
int32_t check_words(const void *p, bool needed) {
  if (needed && !p) return AA_ERR_NULL;
  return on(p, 4) ? AA_OK : AA_ERR_ALIGN;
}

#define AA_TRY(expr)                    \
  do {                                  \
    const int32_t rc_ = (expr);         \
    if (rc_ != AA_OK) return rc_;       \
  } while (0)

// Rows of `width` elements can be moved 16 bytes at a time, but for a shorter end.
bool rows_on_16(const void *p, int64_t ld, int bytes) { return on(p, 16) && ld * bytes % 16 == 0; }

// What the kernels that move 16 bytes at a time address with 32 bits a lane: rows by their place in units of 16
// bytes (gathered ones, of which there may be more than rows_max, by 64 bits); rows that run along the result by their place
// among 31.
bool in_reach(const void *p, int64_t rows, int64_t ld) {
  return rows_on_16(p, ld, 2) && (rows == 0 || ld / 8 < (1ll << 32) / rows);
}
bool columns_in_reach(const void *p, int64_t ld) { return rows_on_16(p, ld, 2) && ld < (1ll << 25); }

size_t plan_bytes(int64_t n_max, int32_t top_k, int32_t n_experts) {
  return align_up(plan_table_ints(n_max, top_k, n_experts) * sizeof(int32_t), 256);
}

int32_t check_ws(const void *ws, size_t ws_bytes, size_t need) {
  return !ws || !on(ws, 256) || ws_bytes < need ? AA_ERR_WORKSPACE : AA_OK;
}

int32_t check_pairs(int32_t n_max, int32_t top_k, int32_t n_experts) {
  if (n_max < 0 || top_k < 1 || top_k > AA_MAX_CHOICES || n_experts < 1 || n_experts > AA_MAX_EXPERTS)
    return AA_ERR_SHAPE;
  return (int64_t)n_max * top_k <= kMaxPairs ? AA_OK : AA_ERR_SHAPE;
}

int32_t check_route_config(const aa_route_config *c, int32_t n_max, int32_t n_experts) {
  if (!c) return AA_ERR_NULL;
  AA_TRY(check_pairs(n_max, c->top_k, n_experts));
  if (c->score != AA_SCORE_SOFTMAX && c->score != AA_SCORE_SIGMOID) return AA_ERR_SHAPE;
  if (c->n_groups < 1 || n_experts % c->n_groups != 0) return AA_ERR_SHAPE;
  if (c->top_groups < 1 || c->top_groups > c->n_groups) return AA_ERR_SHAPE;
  if (c->top_k > c->top_groups * (n_experts / c->n_groups)) return AA_ERR_SHAPE;
  if (c->group_best != 1 && c->group_best != 2) return AA_ERR_SHAPE;
  return isfinite(c->scale) ? AA_OK : AA_ERR_SHAPE;
}

PlanArgs plan_args(const int32_t *ids, const int32_t *count, int32_t n_max, int32_t top_k, int32_t n_experts,
                   int32_t *offsets, int32_t *order, int32_t *slot, void *ws) {
  return {ids, count, n_max, top_k, n_experts, offsets, order, slot,
          reinterpret_cast<int32_t *>(static_cast<char *>(ws) + 256)};
}

int32_t check_plan(int32_t n_max, const int32_t *offsets, const int32_t *order, const int32_t *slot) {
  AA_TRY(check_words(offsets, true));
  AA_TRY(check_words(order, n_max > 0));
  return check_words(slot, n_max > 0);
}

// p in [0, 1]: the draws' limit and the scale of what is kept
bool drop_key(float p, uint64_t seed, uint64_t step, DropKey *k) {
  if (!(p >= 0.0f && p <= 1.0f)) return false;
  const DrawKey d = make_draw_key(seed, step);
  k->k0 = d.k0;
  k->k1 = d.k1;
  k->s0 = d.s0;
  k->s1 = d.s1;
  k->limit = (uint32_t)lrint(65536.0 * (1.0 - (double)p));
  k->scale = k->limit ? 65536.0f / (float)k->limit : 0.0f;
  return true;
}

int32_t check_product(int32_t dtype, const int32_t *offsets, int32_t rows_max, int32_t n_experts, int32_t d_in,
                      int32_t d_out) {
  if (dtype != AA_BF16 && dtype != AA_F16) return AA_ERR_SHAPE;
  if (rows_max < 0 || rows_max > kMaxPairs || n_experts < 1 || n_experts > AA_MAX_EXPERTS) return AA_ERR_SHAPE;
  if (d_in < 1 || d_in > kMaxWidth || d_out < 1 || d_out > kMaxWidth) return AA_ERR_SHAPE;
  return check_words(offsets, true);
}

int32_t check_order(const int32_t *order, int32_t top_k) {
  if (order && (top_k < 1 || top_k > AA_MAX_CHOICES)) return AA_ERR_SHAPE;
  return check_words(order, false);
}

bool is_act(int32_t act) { return act == AA_ACT_NONE || act == AA_ACT_RELU || act == AA_ACT_GATED; }

}  // namespace

extern "C" {

size_t aa_expert_workspace_bytes(int32_t n_max, int32_t top_k, int32_t n_experts) {
  const int64_t n = n_max > 0 ? n_max : 0;
  const size_t plan = plan_bytes(n, top_k > 0 ? top_k : 1, n_experts > 0 ? n_experts : 1);
  return 256 + (plan > kGradWeightPartialBytes ? plan : kGradWeightPartialBytes);
}

int32_t aa_route(const void *logits, int32_t dtype, int64_t ld, const int32_t *count, int32_t n_max,
                 int32_t n_experts, const float *bias, const aa_route_config *cfg, int32_t *ids, float *weights,
                 int32_t *offsets, int32_t *order, int32_t *slot, void *ws, size_t ws_bytes, void *stream) {
  AA_TRY(check_route_config(cfg, n_max, n_experts));
  const int bytes = type_bytes(dtype);
  if (bytes == 0) return AA_ERR_SHAPE;
  AA_TRY(check_rows(logits, n_max, ld, n_experts, bytes));
  AA_TRY(check_words(count, false));
  AA_TRY(check_words(bias, false));
  AA_TRY(check_words(ids, n_max > 0));
  AA_TRY(check_words(weights, n_max > 0));
  const bool plan = offsets || order || slot;
  if (plan) {
    AA_TRY(check_plan(n_max, offsets, order, slot));
    AA_TRY(check_ws(ws, ws_bytes, 256 + plan_bytes(n_max, cfg->top_k, n_experts)));
  }
  const RouteArgs r = {logits, dtype, 0, ld, count, n_max, n_experts, bias, *cfg, ids, weights};
  if (!plan) return hip_status(launch_route(r, nullptr, as_stream(stream)));
  const PlanArgs p = plan_args(ids, count, n_max, cfg->top_k, n_experts, offsets, order, slot, ws);
  return hip_status(launch_route(r, &p, as_stream(stream)));
}

int32_t aa_route_grad(const void *logits, int32_t dtype, int64_t ld, const int32_t *count, int32_t n_max,
                      int32_t n_experts, const aa_route_config *cfg, const int32_t *ids, const float *dweights,
                      void *dlogits, int64_t ld_out, void *stream) {
  AA_TRY(check_route_config(cfg, n_max, n_experts));
  const int bytes = type_bytes(dtype);
  if (bytes == 0) return AA_ERR_SHAPE;
  AA_TRY(check_rows(logits, n_max, ld, n_experts, bytes));
  AA_TRY(check_rows(dlogits, n_max, ld_out, n_experts, bytes));
  AA_TRY(check_words(count, false));
  AA_TRY(check_words(ids, n_max > 0));
  AA_TRY(check_words(dweights, n_max > 0));
  const RouteGradArgs r = {logits, dtype, 0, ld, count, n_max, n_experts, *cfg, ids, dweights, dlogits, ld_out};
  return hip_status(launch_route_grad(r, as_stream(stream)));
}

int32_t aa_expert_plan(const int32_t *ids, const int32_t *count, int32_t n_max, int32_t top_k, int32_t n_experts,
                       int32_t *offsets, int32_t *order, int32_t *slot, void *ws, size_t ws_bytes, void *stream) {
  AA_TRY(check_pairs(n_max, top_k, n_experts));
  AA_TRY(check_words(ids, n_max > 0));
  AA_TRY(check_words(count, false));
  AA_TRY(check_plan(n_max, offsets, order, slot));
  AA_TRY(check_ws(ws, ws_bytes, 256 + plan_bytes(n_max, top_k, n_experts)));
  return hip_status(launch_expert_plan(plan_args(ids, count, n_max, top_k, n_experts, offsets, order, slot, ws),
                                       as_stream(stream)));
}

int32_t aa_expert_forward(const void *x, int32_t dtype, int64_t ldx, const int32_t *order, int32_t top_k,
                          const int32_t *offsets, int32_t rows_max, int32_t n_experts, int32_t d_in, int32_t d_out,
                          const void *w, int32_t act, void *out, int64_t ldo, void *pre, int64_t ldpre,
                          void *stream) {
  AA_TRY(check_product(dtype, offsets, rows_max, n_experts, d_in, d_out));
  if (!is_act(act) || (pre && act != AA_ACT_GATED)) return AA_ERR_SHAPE;
  AA_TRY(check_order(order, top_k));
  AA_TRY(check_rows(x, rows_max, ldx, d_in, 2));
  AA_TRY(check_rows(out, rows_max, ldo, d_out, 2));
  if (pre) AA_TRY(check_rows(pre, rows_max, ldpre, 2 * (int64_t)d_out, 2));
  AA_TRY(check_rows(w, 1, d_in, d_in, 2));
  ProductArgs a{};
  a.rows = x;
  a.ld_rows = ldx;
  a.mat = w;
  a.order = order;
  a.top_k = order ? top_k : 1;
  a.offsets = offsets;
  a.rows_max = rows_max;
  a.n_experts = n_experts;
  a.d_in = d_in;
  a.d_out = d_out;
  a.out = out;
  a.ldo = ldo;
  a.pre = pre;
  a.ldpre = ldpre;
  a.act = act;
  a.aligned = d_in % 8 == 0 && (order ? rows_on_16(x, ldx, 2) : in_reach(x, rows_max, ldx)) &&
              in_reach(w, 2 * (int64_t)d_out, d_in);
  return hip_status(launch_expert_forward(a, dtype == AA_F16, as_stream(stream)));
}

int32_t aa_expert_grad_input(const void *dout, int32_t dtype, int64_t lddo, const int32_t *offsets, int32_t rows_max,
                             int32_t n_experts, int32_t d_in, int32_t d_out, const void *w, int32_t act,
                             const void *saved, int64_t lds, void *dx, int64_t lddx, void *stream) {
  AA_TRY(check_product(dtype, offsets, rows_max, n_experts, d_in, d_out));
  if (!is_act(act)) return AA_ERR_SHAPE;
  const int64_t wide = act == AA_ACT_GATED ? 2 * (int64_t)d_in : d_in;
  AA_TRY(check_rows(dout, rows_max, lddo, d_out, 2));
  AA_TRY(check_rows(dx, rows_max, lddx, wide, 2));
  if (act != AA_ACT_NONE) AA_TRY(check_rows(saved, rows_max, lds, wide, 2));
  AA_TRY(check_rows(w, 1, d_in, d_in, 2));
  ProductArgs a{};
  a.rows = dout;
  a.ld_rows = lddo;
  a.mat = w;
  a.top_k = 1;
  a.offsets = offsets;
  a.rows_max = rows_max;
  a.n_experts = n_experts;
  a.d_in = d_in;
  a.d_out = d_out;
  a.out = dx;
  a.ldo = lddx;
  a.saved = saved;
  a.lds = lds;
  a.act = act;
  a.aligned = d_in % 8 == 0 && d_out % 8 == 0 && in_reach(dout, rows_max, lddo) && columns_in_reach(w, d_in);
  return hip_status(launch_expert_grad_input(a, dtype == AA_F16, as_stream(stream)));
}

int32_t aa_expert_grad_weight(const void *dout, int32_t dtype, int64_t lddo, const void *x, int64_t ldx,
                              const int32_t *order, int32_t top_k, const int32_t *offsets, int32_t rows_max,
                              int32_t n_experts, int32_t d_in, int32_t d_out, void *dw, int32_t out_dtype,
                              int32_t accumulate, void *ws, size_t ws_bytes, void *stream) {
  AA_TRY(check_product(dtype, offsets, rows_max, n_experts, d_in, d_out));
  if (out_dtype != dtype && out_dtype != AA_F32) return AA_ERR_SHAPE;
  AA_TRY(check_order(order, top_k));
  AA_TRY(check_rows(dout, rows_max, lddo, d_out, 2));
  AA_TRY(check_rows(x, rows_max, ldx, d_in, 2));
  AA_TRY(check_rows(dw, 1, d_in, d_in, type_bytes(out_dtype)));
  AA_TRY(check_ws(ws, ws_bytes, 256 + kGradWeightPartialBytes));
  ProductArgs a{};
  a.rows = dout;
  a.ld_rows = lddo;
  a.mat = x;
  a.ld_mat = ldx;
  a.order = order;
  a.top_k = order ? top_k : 1;
  a.offsets = offsets;
  a.rows_max = rows_max;
  a.n_experts = n_experts;
  a.d_in = d_in;
  a.d_out = d_out;
  a.out = dw;
  a.ldo = d_in;
  a.out_f32 = out_dtype == AA_F32;
  a.accumulate = accumulate != 0;
  a.aligned = d_in % 8 == 0 && d_out % 8 == 0 && columns_in_reach(dout, lddo) && columns_in_reach(x, ldx);
  a.partial = reinterpret_cast<float *>(static_cast<char *>(ws) + 256);
  a.partial_bytes = kGradWeightPartialBytes;
  return hip_status(launch_expert_grad_weight(a, dtype == AA_F16, as_stream(stream)));
}

int32_t aa_dropout(const void *x, int32_t dtype, int64_t ldx, const int32_t *count, int32_t n_max, int32_t d,
                   const void *residual, int64_t ldr, float p, uint64_t seed, uint64_t step, void *out, int64_t ldo,
                   void *stream) {
  const int bytes = type_bytes(dtype);
  DropoutArgs a{};
  if (bytes == 0 || n_max < 0 || d < 1 || d > kMaxWidth || !drop_key(p, seed, step, &a.key)) return AA_ERR_SHAPE;
  AA_TRY(check_rows(x, n_max, ldx, d, bytes));
  AA_TRY(check_rows(out, n_max, ldo, d, bytes));
  if (residual) AA_TRY(check_rows(residual, n_max, ldr, d, bytes));
  AA_TRY(check_words(count, false));
  a.x = x;
  a.ldx = ldx;
  a.count = count;
  a.n_max = n_max;
  a.d = d;
  a.residual = residual;
  a.ldr = ldr;
  a.out = out;
  a.ldo = ldo;
  return hip_status(launch_dropout(a, dtype, as_stream(stream)));
}

int32_t aa_expert_combine(const void *y, int32_t dtype, int64_t ldy, const int32_t *slot, const float *weights,
                          const int32_t *count, int32_t n_max, int32_t top_k, int32_t d, const void *residual,
                          int64_t ldr, float p, uint64_t seed, uint64_t step, void *out, int64_t ldo, void *stream) {
  const int bytes = type_bytes(dtype);
  CombineArgs a{};
  if (bytes == 0 || d < 1 || d > kMaxWidth || !drop_key(p, seed, step, &a.key)) return AA_ERR_SHAPE;
  AA_TRY(check_pairs(n_max, top_k, 1));
  AA_TRY(check_rows(y, n_max, ldy, d, bytes));
  AA_TRY(check_rows(out, n_max, ldo, d, bytes));
  if (residual) AA_TRY(check_rows(residual, n_max, ldr, d, bytes));
  AA_TRY(check_words(slot, n_max > 0));
  AA_TRY(check_words(weights, false));
  AA_TRY(check_words(count, false));
  a.y = y;
  a.ldy = ldy;
  a.slot = slot;
  a.weights = weights;
  a.count = count;
  a.n_max = n_max;
  a.top_k = top_k;
  a.d = d;
  a.residual = residual;
  a.ldr = ldr;
  a.out = out;
  a.ldo = ldo;
  return hip_status(launch_expert_combine(a, dtype, as_stream(stream)));
}

int32_t aa_expert_combine_grad(const void *dout, int32_t dtype, int64_t lddo, const void *y, int64_t ldy,
                               const int32_t *slot, const float *weights, const int32_t *count, int32_t n_max,
                               int32_t top_k, int32_t d, float p, uint64_t seed, uint64_t step, void *dy,
                               int64_t lddy, float *dweights, void *stream) {
  const int bytes = type_bytes(dtype);
  CombineArgs a{};
  if (bytes == 0 || d < 1 || d > kMaxWidth || !drop_key(p, seed, step, &a.key)) return AA_ERR_SHAPE;
  AA_TRY(check_pairs(n_max, top_k, 1));
  AA_TRY(check_rows(dout, n_max, lddo, d, bytes));
  AA_TRY(check_rows(dy, n_max, lddy, d, bytes));
  if (dweights) AA_TRY(check_rows(y, n_max, ldy, d, bytes));
  AA_TRY(check_words(slot, n_max > 0));
  AA_TRY(check_words(weights, false));
  AA_TRY(check_words(dweights, false));
  AA_TRY(check_words(count, false));
  a.dout = dout;
  a.lddo = lddo;
  a.y = y;
  a.ldy = ldy;
  a.slot = slot;
  a.weights = weights;
  a.count = count;
  a.n_max = n_max;
  a.top_k = top_k;
  a.d = d;
  a.out = dy;
  a.ldo = lddy;
  a.dweights = dweights;
  return hip_status(launch_expert_combine_grad(a, dtype, as_stream(stream)));
}

}  // extern "C"

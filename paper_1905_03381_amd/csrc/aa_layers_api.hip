// C ABI of the operators around a Boss block of experts: argument checks and the choice of kernels.
#include "../../include/autoassist.h"

#include "aa_adamw.hpp"
#include "aa_checks.hpp"
#include "aa_linear.hpp"
#include "aa_norm.hpp"
#include "aa_route.hpp"

#include <math.h>

#include <algorithm>
#include <new>

using namespace aa;

namespace {

float *body(void *ws) { return reinterpret_cast<float *>(static_cast<char *>(ws) + kLayerHead); }

// Rows that a layer norm reads or writes.
int32_t check_norm(int32_t dtype, int32_t n_max, int32_t d, const int32_t *count) {
  if (type_bytes(dtype) == 0 || n_max < 0 || d < 1 || d > kMaxWidth) return AA_ERR_SHAPE;
  return check_words(count, false);
}

bool is_dense_act(int32_t act) { return act >= AA_ACT_NONE && act <= AA_ACT_GELU; }

// Results of so many bytes, half of the cache that all of the chip shares, are not there any more when they are read.  (Rows
// off 16-byte boundaries fill lines in parts, which the caches put together: 4422 x 1024 -> 8018 with pre 89 us, past them 124.)
constexpr int64_t kPassingBytes = 128ll << 20;

// Rows of a dense layer.
int32_t check_linear(int32_t dtype, const int32_t *count, int32_t n_max, int32_t d_out, int32_t act) {
  if (dtype != AA_BF16 && dtype != AA_F16) return AA_ERR_SHAPE;
  if (n_max < 0 || n_max > kMaxPairs || d_out < 1 || d_out > kMaxWidth || !is_dense_act(act)) return AA_ERR_SHAPE;
  return check_words(count, false);
}

// What both directions of the balance loss are asked about.
int32_t check_balance(const void *logits, int32_t dtype, int64_t ld, const int32_t *count, int32_t n_max,
                      int32_t n_experts, const aa_route_config *cfg, float coef, float z_coef) {
  AA_TRY(check_route_config(cfg, n_max, n_experts));
  if (type_bytes(dtype) == 0 || !isfinite(coef) || !isfinite(z_coef)) return AA_ERR_SHAPE;
  AA_TRY(check_rows(logits, n_max, ld, n_experts, type_bytes(dtype)));
  return check_words(count, false);
}

// One tensor of an update.
int32_t check_tensor(const aa_adamw_tensor &t) {
  if (t.n < 0 || t.n > (1ll << 35) || type_bytes(t.grad_dtype) == 0 || !isfinite(t.decay)) return AA_ERR_SHAPE;
  if (t.state_bits != 32 && t.state_bits != 8) return AA_ERR_SHAPE;
  if (t.copy && t.copy_dtype != AA_BF16 && t.copy_dtype != AA_F16) return AA_ERR_SHAPE;
  if (t.n > 0 && (!t.param || !t.grad || !t.m || !t.v)) return AA_ERR_NULL;
  if (t.n > 0 && t.state_bits == 8 && (!t.m_scale || !t.v_scale)) return AA_ERR_NULL;
  const size_t state = t.state_bits / 8;
  const bool fits = on(t.param, 4) && on(t.grad, type_bytes(t.grad_dtype)) && on(t.copy, 2) && on(t.m, state) &&
                    on(t.v, state) && on(t.m_scale, 4) && on(t.v_scale, 4);
  return fits ? AA_OK : AA_ERR_ALIGN;
}

// Memory that a tensor of an update reads, or writes, too.
struct Stretch {
  uintptr_t from, to;
  bool written;
};

// Whether any memory that is written is another tensor's, or the same tensor's, under another name: AA_ERR_SHAPE.
int32_t check_apart(const aa_adamw_tensor *tensors, int32_t n) {
  Stretch *all = new (std::nothrow) Stretch[(size_t)n * 7];
  if (!all) return AA_ERR_HIP;
  size_t k = 0;
  const auto add = [&](const void *p, int64_t bytes, bool written) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(p);
    if (p && bytes > 0) all[k++] = {from, from + (uintptr_t)bytes, written};
  };
  for (int32_t i = 0; i < n; ++i) {
    const aa_adamw_tensor &t = tensors[i];
    const int64_t scales = t.state_bits == 8 ? (t.n + kStateBlock - 1) / kStateBlock * 4 : 0;
    add(t.param, t.n * 4, true);
    add(t.grad, t.n * type_bytes(t.grad_dtype), false);
    add(t.copy, t.n * 2, true);
    add(t.m, t.n * (t.state_bits / 8), true);
    add(t.v, t.n * (t.state_bits / 8), true);
    add(t.m_scale, scales, true);
    add(t.v_scale, scales, true);
  }
  std::sort(all, all + k, [](const Stretch &x, const Stretch &y) { return x.from < y.from; });
  uintptr_t written = 0, any = 0;  // where what has been seen ends
  bool apart = true;
  for (size_t i = 0; i < k; ++i) {
    apart = apart && all[i].from >= (all[i].written ? any : written);
    any = std::max(any, all[i].to);
    if (all[i].written) written = std::max(written, all[i].to);
  }
  delete[] all;
  return apart ? AA_OK : AA_ERR_SHAPE;
}

// A table as aa_adamw_table made it.
int32_t check_table(const void *table, size_t bytes, int32_t n_tensors, int64_t n_chunks) {
  if (n_tensors < 1 || n_tensors > 65536 || n_chunks < 0 || n_chunks > kMaxPairs) return AA_ERR_SHAPE;
  return check_ws(table, bytes, table_bytes(n_tensors, n_chunks));
}

}  // namespace

extern "C" {

size_t aa_layer_workspace_bytes(int32_t d_max) { return layer_bytes(d_max > 0 ? d_max : 1); }

int32_t aa_layer_norm(const void *x, int32_t dtype, int64_t ldx, const int32_t *count, int32_t n_max, int32_t d,
                      const float *gamma, const float *beta, float eps, void *out, int64_t ldo, float *mean,
                      float *rstd, void *stream) {
  AA_TRY(check_norm(dtype, n_max, d, count));
  if (!(eps >= 0.0f) || !isfinite(eps)) return AA_ERR_SHAPE;
  AA_TRY(check_rows(x, n_max, ldx, d, type_bytes(dtype)));
  AA_TRY(check_rows(out, n_max, ldo, d, type_bytes(dtype)));
  AA_TRY(check_words(gamma, false));
  AA_TRY(check_words(beta, false));
  AA_TRY(check_words(mean, false));
  AA_TRY(check_words(rstd, false));
  NormArgs a{};
  a.x = x;
  a.ldx = ldx;
  a.count = count;
  a.n_max = n_max;
  a.d = d;
  a.gamma = gamma;
  a.beta = beta;
  a.eps = eps;
  a.out = out;
  a.ldo = ldo;
  a.mean = mean;
  a.rstd = rstd;
  return hip_status(launch_layer_norm(a, dtype, as_stream(stream)));
}

int32_t aa_layer_norm_grad(const void *dout, int32_t dtype, int64_t lddo, const void *x, int64_t ldx,
                           const int32_t *count, int32_t n_max, int32_t d, const float *gamma, const float *mean,
                           const float *rstd, const void *residual, int64_t ldr, void *dx, int64_t lddx,
                           float *dgamma, float *dbeta, int32_t accumulate, void *ws, size_t ws_bytes, void *stream) {
  AA_TRY(check_norm(dtype, n_max, d, count));
  const int bytes = type_bytes(dtype);
  AA_TRY(check_rows(dout, n_max, lddo, d, bytes));
  AA_TRY(check_rows(x, n_max, ldx, d, bytes));
  AA_TRY(check_rows(dx, n_max, lddx, d, bytes));
  if (residual) AA_TRY(check_rows(residual, n_max, ldr, d, bytes));
  AA_TRY(check_words(gamma, false));
  AA_TRY(check_words(mean, n_max > 0));
  AA_TRY(check_words(rstd, n_max > 0));
  AA_TRY(check_words(dgamma, false));
  AA_TRY(check_words(dbeta, false));
  if (dgamma || dbeta) AA_TRY(check_ws(ws, ws_bytes, layer_need(d)));
  NormArgs a{};
  a.x = x;
  a.ldx = ldx;
  a.count = count;
  a.n_max = n_max;
  a.d = d;
  a.gamma = gamma;
  a.out = dx;
  a.ldo = lddx;
  a.mean = const_cast<float *>(mean);
  a.rstd = const_cast<float *>(rstd);
  a.dout = dout;
  a.lddo = lddo;
  a.residual = residual;
  a.ldr = ldr;
  a.dgamma = dgamma;
  a.dbeta = dbeta;
  a.accumulate = accumulate != 0;
  a.part = dgamma || dbeta ? body(ws) : nullptr;
  return hip_status(launch_layer_norm_grad(a, dtype, as_stream(stream)));
}

int32_t aa_linear(const void *x, int32_t dtype, int64_t ldx, const int32_t *count, int32_t n_max, int32_t d_in,
                  int32_t d_out, const void *w, const float *bias, int32_t act, const void *residual, int64_t ldr,
                  void *out, int64_t ldo, void *pre, int64_t ldpre, void *stream) {
  AA_TRY(check_linear(dtype, count, n_max, d_out, act));
  if (d_in < 1 || d_in > kMaxWidth) return AA_ERR_SHAPE;
  const int64_t wide = act == AA_ACT_GATED ? 2 * (int64_t)d_out : d_out;
  AA_TRY(check_rows(x, n_max, ldx, d_in, 2));
  AA_TRY(check_rows(out, n_max, ldo, d_out, 2));
  if (residual) AA_TRY(check_rows(residual, n_max, ldr, d_out, 2));
  if (pre) AA_TRY(check_rows(pre, n_max, ldpre, wide, 2));
  AA_TRY(check_rows(w, 1, d_in, d_in, 2));
  AA_TRY(check_words(bias, false));
  ProductArgs a{};
  a.rows = x;
  a.ld_rows = ldx;
  a.mat = w;
  a.top_k = 1;
  a.rows_max = n_max;
  a.n_experts = 1;
  a.d_in = d_in;
  a.d_out = d_out;
  a.out = out;
  a.ldo = ldo;
  a.pre = pre;
  a.ldpre = ldpre;
  a.act = act;
  a.aligned = d_in % 8 == 0 && in_reach(x, n_max, ldx) && in_reach(w, wide, d_in);
  a.count = count;
  a.bias = bias;
  a.residual = residual;
  a.ldres = ldr;
  a.passing = rows_on_16(out, ldo, 2) && (int64_t)n_max * d_out * 2 >= kPassingBytes;
  a.passing_pre = pre && rows_on_16(pre, ldpre, 2) && (int64_t)n_max * wide * 2 >= kPassingBytes;
  return hip_status(launch_linear(a, dtype == AA_F16, as_stream(stream)));
}

int32_t aa_linear_grad(const void *dout, int32_t dtype, int64_t lddo, const int32_t *count, int32_t n_max,
                       int32_t d_out, int32_t act, const void *pre, int64_t ldpre, void *dpre, int64_t lddp,
                       float *dbias, int32_t accumulate, void *ws, size_t ws_bytes, void *stream) {
  AA_TRY(check_linear(dtype, count, n_max, d_out, act));
  if (!dpre && !dbias) return AA_ERR_NULL;
  const int64_t wide = act == AA_ACT_GATED ? 2 * (int64_t)d_out : d_out;
  AA_TRY(check_rows(dout, n_max, lddo, d_out, 2));
  if (act != AA_ACT_NONE) AA_TRY(check_rows(pre, n_max, ldpre, wide, 2));
  if (dpre) AA_TRY(check_rows(dpre, n_max, lddp, wide, 2));
  AA_TRY(check_words(dbias, false));
  if (dbias) AA_TRY(check_ws(ws, ws_bytes, layer_need(wide)));
  ActGradArgs a{};
  a.dout = dout;
  a.lddo = lddo;
  a.count = count;
  a.n_max = n_max;
  a.d = d_out;
  a.act = act;
  a.pre = pre;
  a.ldpre = ldpre;
  a.dpre = dpre;
  a.lddp = lddp;
  a.dbias = dbias;
  a.accumulate = accumulate != 0;
  a.part = dbias ? body(ws) : nullptr;
  return hip_status(launch_linear_grad(a, dtype == AA_F16, as_stream(stream)));
}

int32_t aa_balance(const void *logits, int32_t dtype, int64_t ld, const int32_t *count, int32_t n_max,
                   int32_t n_experts, const aa_route_config *cfg, const int32_t *ids, float coef, float z_coef,
                   int32_t *counts, float *share, float *loss, void *ws, size_t ws_bytes, void *stream) {
  AA_TRY(check_balance(logits, dtype, ld, count, n_max, n_experts, cfg, coef, z_coef));
  AA_TRY(check_words(ids, n_max > 0));
  AA_TRY(check_words(counts, true));
  AA_TRY(check_words(share, false));
  AA_TRY(check_words(loss, false));
  AA_TRY(check_ws(ws, ws_bytes, layer_need(n_experts)));
  BalanceArgs a{};
  a.logits = logits;
  a.dtype = dtype;
  a.ld = ld;
  a.count = count;
  a.n_max = n_max;
  a.n_experts = n_experts;
  a.cfg = *cfg;
  a.ids = ids;
  a.coef = coef;
  a.z_coef = z_coef;
  a.counts = counts;
  a.share = share;
  a.loss = loss;
  static_assert(256 + kBalanceTerms * sizeof(double) + kBalanceBlocks * sizeof(float) <= kLayerHead, "");
  a.done = static_cast<int32_t *>(ws);
  a.terms = reinterpret_cast<double *>(static_cast<char *>(ws) + 256);
  a.z_part = reinterpret_cast<float *>(a.terms + kBalanceTerms);
  a.part = body(ws);
  return hip_status(launch_balance(a, as_stream(stream)));
}

int32_t aa_balance_grad(const void *logits, int32_t dtype, int64_t ld, const int32_t *count, int32_t n_max,
                        int32_t n_experts, const aa_route_config *cfg, const int32_t *ids, const float *dweights,
                        const int32_t *counts, float coef, float z_coef, const float *dloss, void *dlogits,
                        int64_t ld_out, void *stream) {
  AA_TRY(check_balance(logits, dtype, ld, count, n_max, n_experts, cfg, coef, z_coef));
  AA_TRY(check_words(ids, dweights && n_max > 0));
  AA_TRY(check_words(dweights, false));
  AA_TRY(check_words(counts, true));
  AA_TRY(check_words(dloss, false));
  AA_TRY(check_rows(dlogits, n_max, ld_out, n_experts, type_bytes(dtype)));
  RouteGradArgs a{};
  a.logits = logits;
  a.dtype = dtype;
  a.ld = ld;
  a.count = count;
  a.n_max = n_max;
  a.n_experts = n_experts;
  a.cfg = *cfg;
  a.ids = ids;
  a.dweights = dweights;
  a.dlogits = dlogits;
  a.ld_out = ld_out;
  a.counts = counts;
  a.coef = coef;
  a.z_coef = z_coef;
  a.dloss = dloss;
  return hip_status(launch_balance_grad(a, as_stream(stream)));
}

int64_t aa_adamw_chunks(const aa_adamw_tensor *tensors, int32_t n_tensors) {
  if (n_tensors < 1 || n_tensors > 65536) return AA_ERR_SHAPE;
  if (!tensors) return AA_ERR_NULL;
  int64_t chunks = 0;
  for (int32_t k = 0; k < n_tensors; ++k) {
    AA_TRY(check_tensor(tensors[k]));
    chunks += (tensors[k].n + kChunk - 1) / kChunk;
  }
  return chunks <= kMaxPairs ? chunks : (int64_t)AA_ERR_SHAPE;
}

size_t aa_adamw_table_bytes(int32_t n_tensors, int64_t n_chunks) {
  return table_bytes(n_tensors > 0 ? n_tensors : 1, n_chunks > 0 ? n_chunks : 0);
}

int32_t aa_adamw_table(const aa_adamw_tensor *tensors, int32_t n_tensors, void *table, size_t table_bytes_,
                       void *stream) {
  const int64_t chunks = aa_adamw_chunks(tensors, n_tensors);
  if (chunks < 0) return (int32_t)chunks;
  AA_TRY(check_table(table, table_bytes_, n_tensors, chunks));
  AA_TRY(check_apart(tensors, n_tensors));
  return hip_status(launch_adamw_table(tensors, n_tensors, static_cast<char *>(table), as_stream(stream)));
}

int32_t aa_grad_norm(void *table, size_t table_bytes_, int32_t n_tensors, int64_t n_chunks, float max_norm,
                     const float *scale, float *out, void *stream) {
  AA_TRY(check_table(table, table_bytes_, n_tensors, n_chunks));
  if (!(max_norm > 0.0f)) return AA_ERR_SHAPE;
  AA_TRY(check_words(scale, false));
  AA_TRY(check_words(out, true));
  AdamWArgs a{};
  a.table = static_cast<char *>(table);
  a.map = (int64_t)table_map(n_tensors);
  a.n_tensors = n_tensors;
  a.n_chunks = n_chunks;
  a.max_norm = max_norm;
  a.scale = scale;
  a.out = out;
  return hip_status(launch_grad_norm(a, as_stream(stream)));
}

int32_t aa_adamw_step(void *table, size_t table_bytes_, int32_t n_tensors, int64_t n_chunks,
                      const aa_adamw_config *cfg, const float *lr_factor, const float *grad_factor,
                      const int32_t *count, int32_t *t, void *stream) {
  if (!cfg) return AA_ERR_NULL;
  AA_TRY(check_table(table, table_bytes_, n_tensors, n_chunks));
  const auto beta = [](float b) { return b >= 0.0f && b < 1.0f; };
  const auto size = [](float v) { return v >= 0.0f && isfinite(v); };
  if (!beta(cfg->beta1) || !beta(cfg->beta2) || !size(cfg->lr) || !size(cfg->weight_decay)) return AA_ERR_SHAPE;
  if (!size(cfg->eps) || cfg->eps < 0x1p-126f) return AA_ERR_SHAPE;  // (a normal number: it is divided by)
  AA_TRY(check_words(lr_factor, false));
  AA_TRY(check_words(grad_factor, false));
  AA_TRY(check_words(count, false));
  AA_TRY(check_words(t, true));
  AdamWArgs a{};
  a.table = static_cast<char *>(table);
  a.map = (int64_t)table_map(n_tensors);
  a.n_tensors = n_tensors;
  a.n_chunks = n_chunks;
  a.cfg = *cfg;
  a.log_beta1 = (float)log((double)cfg->beta1);
  a.log_beta2 = (float)log((double)cfg->beta2);
  a.lr_factor = lr_factor;
  a.grad_factor = grad_factor;
  a.count = count;
  a.t = t;
  return hip_status(launch_adamw_step(a, as_stream(stream)));
}

}  // extern "C"

// C ABI of the operators around a Boss block of experts: argument checks and the choice of kernels.
#include "../../include/autoassist.h"

#include "aa_checks.hpp"
#include "aa_norm.hpp"
#include "aa_route.hpp"

#include <math.h>

using namespace aa;

namespace {

float *body(void *ws) { return reinterpret_cast<float *>(static_cast<char *>(ws) + kLayerHead); }

// Rows that a layer norm reads or writes.
int32_t check_norm(int32_t dtype, int32_t n_max, int32_t d, const int32_t *count) {
  if (type_bytes(dtype) == 0 || n_max < 0 || d < 1 || d > kMaxWidth) return AA_ERR_SHAPE;
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
  if (dgamma || dbeta) AA_TRY(check_ws(ws, ws_bytes, layer_bytes(d)));
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

int32_t aa_balance(const void *logits, int32_t dtype, int64_t ld, const int32_t *count, int32_t n_max,
                   int32_t n_experts, const aa_route_config *cfg, const int32_t *ids, float coef, float z_coef,
                   int32_t *counts, float *share, float *loss, void *ws, size_t ws_bytes, void *stream) {
  AA_TRY(check_balance(logits, dtype, ld, count, n_max, n_experts, cfg, coef, z_coef));
  AA_TRY(check_words(ids, n_max > 0));
  AA_TRY(check_words(counts, true));
  AA_TRY(check_words(share, false));
  AA_TRY(check_words(loss, false));
  AA_TRY(check_ws(ws, ws_bytes, layer_bytes(n_experts)));
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
  a.z_part = reinterpret_cast<float *>(static_cast<char *>(ws) + 256);
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

}  // extern "C"

// C ABI of the operators around a Boss block of experts: argument checks and the choice of kernels.
#include "../../include/autoassist.h"

#include "aa_checks.hpp"
#include "aa_norm.hpp"

#include <math.h>

using namespace aa;

namespace {

float *body(void *ws) { return reinterpret_cast<float *>(static_cast<char *>(ws) + 256); }

// Rows that a layer norm reads or writes.
int32_t check_norm(int32_t dtype, int32_t n_max, int32_t d, const int32_t *count) {
  if (type_bytes(dtype) == 0 || n_max < 0 || d < 1 || d > kMaxWidth) return AA_ERR_SHAPE;
  return check_words(count, false);
}

}  // namespace

extern "C" {

size_t aa_layer_workspace_bytes(int32_t d_max) {
  const size_t need = 256 + column_bytes(d_max > 0 ? d_max : 1);
  return need > kWsBody ? need : align_up(kWsBody, 256);  // (what aa_workspace_init prepares)
}

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
  if (dgamma || dbeta) AA_TRY(check_ws(ws, ws_bytes, 256 + column_bytes(d)));
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

}  // extern "C"

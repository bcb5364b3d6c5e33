// Host-side launch interface of the layer norm and of the sums over columns (aa_norm.hip).
#pragma once

#include "aa_common.hpp"

namespace aa {

struct NormArgs {
  const void *x;
  int64_t ldx;
  const int32_t *count;
  int32_t n_max, d;
  const float *gamma, *beta;  // (NULL: 1, 0)
  float eps;
  void *out;  // forward: out; gradient: dx
  int64_t ldo;
  float *mean, *rstd;  // forward (may be NULL); gradient: read
  const void *dout;    // gradient
  int64_t lddo;
  const void *residual;
  int64_t ldr;
  float *dgamma, *dbeta;  // (may be NULL)
  int32_t accumulate;
  float *part;  // [column_parts(d)][2][d]
};

// Parts that a sum over rows comes in, of `d` columns: what the workspace holds.
constexpr int kColumnPartsMost = 512;
__host__ __device__ inline int column_parts(int64_t d) {
  const int64_t p = (4ll << 20) / (d > 0 ? d : 1);
  return (int)(p < 1 ? 1 : p > kColumnPartsMost ? kColumnPartsMost : p);
}
// The workspace: control words, kLayerHead bytes of what blocks have one of, then the columns' parts.  What rows of d columns
// need of it, and what rows of up to d_max do (a number of columns may need more than a larger one: parts are whole).
constexpr size_t kLayerHead = 4096;
inline size_t layer_need(int64_t d) {
  const size_t parts = (size_t)column_parts(d) * 2 * d * sizeof(float);
  return kLayerHead + (parts > 16384 ? parts : 16384);
}
inline size_t layer_bytes(int64_t d_max) {
  const int64_t most = (4ll << 20) * 2 * (int64_t)sizeof(float);  // of columns that the parts are limited for
  const int64_t parts = (int64_t)kColumnPartsMost * 2 * d_max * (int64_t)sizeof(float);
  const int64_t one = 2 * d_max * (int64_t)sizeof(float), need = parts < most ? parts : one > most ? one : most;
  return kLayerHead + align_up(need > 16384 ? (size_t)need : 16384, 256);
}

// first[c], second[c] (+)= the sum over the parts, `stride` floats apart, of their columns c and d + c (either may be NULL);
// zeros.
hipError_t launch_join_columns(const float *part, int parts, int64_t stride, int32_t d, float *first, float *second,
                               int32_t accumulate, hipStream_t st);
hipError_t launch_clear_columns(float *first, float *second, int32_t d, hipStream_t st);

hipError_t launch_layer_norm(const NormArgs &a, int32_t dtype, hipStream_t st);
hipError_t launch_layer_norm_grad(const NormArgs &a, int32_t dtype, hipStream_t st);

}  // namespace aa

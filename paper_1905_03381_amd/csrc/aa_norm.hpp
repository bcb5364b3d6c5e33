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
// The workspace: control words, kLayerHead bytes of what blocks have one of, then the columns' parts.
constexpr size_t kLayerHead = 4096;
inline size_t layer_bytes(int64_t d) {
  const size_t parts = align_up((size_t)column_parts(d) * 2 * d * sizeof(float), 256);
  return kLayerHead + (parts > 16384 ? parts : 16384);
}

// first[c], second[c] (+)= the sum over the parts, `stride` floats apart, of their columns c and d + c (either may be NULL);
// zeros.
hipError_t launch_join_columns(const float *part, int parts, int64_t stride, int32_t d, float *first, float *second,
                               int32_t accumulate, hipStream_t st);
hipError_t launch_clear_columns(float *first, float *second, int32_t d, hipStream_t st);

hipError_t launch_layer_norm(const NormArgs &a, int32_t dtype, hipStream_t st);
hipError_t launch_layer_norm_grad(const NormArgs &a, int32_t dtype, hipStream_t st);

}  // namespace aa

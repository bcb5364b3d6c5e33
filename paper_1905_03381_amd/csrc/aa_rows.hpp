// Host-side launch interface of the row operators of a block of experts: dropout and the weighted
// combination of the experts' rows (aa_rows.hip).
#pragma once

#include "aa_common.hpp"

namespace aa {

struct DropKey {
  uint32_t k0, k1, s0, s1;
  uint32_t limit;  // an element is kept if its 16-bit draw is below (65536: all are, no draws are made)
  float scale;     // 65536 / limit
};

struct DropoutArgs {
  const void *x;
  int64_t ldx;
  const int32_t *count;
  int32_t n_max, d;
  const void *residual;
  int64_t ldr;
  DropKey key;
  void *out;
  int64_t ldo;
};

struct CombineArgs {
  const void *y;
  int64_t ldy;
  const int32_t *slot;
  const float *weights;
  const int32_t *count;
  int32_t n_max, top_k, d;
  const void *residual;  // combine
  int64_t ldr;
  const void *dout;  // combine_grad
  int64_t lddo;
  DropKey key;
  void *out;  // combine: out; combine_grad: dy
  int64_t ldo;
  float *dweights;
};

hipError_t launch_dropout(const DropoutArgs &a, int32_t dtype, hipStream_t st);
hipError_t launch_expert_combine(const CombineArgs &a, int32_t dtype, hipStream_t st);
hipError_t launch_expert_combine_grad(const CombineArgs &a, int32_t dtype, hipStream_t st);

}  // namespace aa

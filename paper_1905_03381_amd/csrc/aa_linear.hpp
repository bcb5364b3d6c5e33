// Host-side launch interface of the dense layer (aa_linear.hip).
#pragma once

#include "aa_experts.hpp"

namespace aa {

struct ActGradArgs {
  const void *dout;
  int64_t lddo;
  const int32_t *count;
  int32_t n_max, d;  // d: columns of dout
  int32_t act;
  const void *pre;
  int64_t ldpre;
  void *dpre;  // (may be NULL)
  int64_t lddp;
  float *dbias;  // (may be NULL)
  int32_t accumulate;
  float *part;
  int32_t parts;  // (chosen at launch)
};

hipError_t launch_linear(const ProductArgs &a, bool f16, hipStream_t st);
hipError_t launch_linear_grad(const ActGradArgs &a, bool f16, hipStream_t st);

}  // namespace aa

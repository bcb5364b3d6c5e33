// Host-side launch interface of the experts' products (aa_experts.hip).
#pragma once

#include "aa_common.hpp"

namespace aa {

struct ProductArgs {
  const void *rows;  // forward: x; the gradients: dout
  int64_t ld_rows;
  const void *mat;  // forward, grad_input: w; grad_weight: x
  int64_t ld_mat;   // grad_weight: leading dimension of x
  const int32_t *order;
  int32_t top_k;
  const int32_t *offsets;
  int32_t rows_max, n_experts, d_in, d_out;
  void *out;
  int64_t ldo;
  void *pre;
  int64_t ldpre;
  const void *saved;
  int64_t lds;
  int32_t act;
  int32_t out_f32, accumulate;
  int32_t aligned;  // 16-byte chunks of the operands are whole and on 16-byte boundaries
  float *partial;   // grad_weight: room for the parts of a split sum
  size_t partial_bytes;
  int32_t parts;    // (chosen at launch) parts a tile's sum over rows comes in
};

hipError_t launch_expert_forward(const ProductArgs &a, bool f16, hipStream_t st);
hipError_t launch_expert_grad_input(const ProductArgs &a, bool f16, hipStream_t st);
hipError_t launch_expert_grad_weight(const ProductArgs &a, bool f16, hipStream_t st);

constexpr size_t kGradWeightPartialBytes = 64u << 20;

}  // namespace aa

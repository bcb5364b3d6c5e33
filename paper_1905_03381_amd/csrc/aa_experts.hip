// The experts' products: matrix products over ragged groups of rows (aa_product.hpp).
#include "aa_product.hpp"

namespace aa {

namespace {

template <typename T, int MODE>
hipError_t launch_act(const ProductArgs &a, hipStream_t st) {
  switch (a.act) {
    case AA_ACT_RELU: return launch_product<T, MODE, AA_ACT_RELU>(a, st);
    case AA_ACT_GATED: return launch_product<T, MODE, AA_ACT_GATED>(a, st);
    default: return launch_product<T, MODE, AA_ACT_NONE>(a, st);
  }
}

}  // namespace

hipError_t launch_expert_forward(const ProductArgs &a, bool f16, hipStream_t st) {
  return f16 ? launch_act<_Float16, kForward>(a, st) : launch_act<__bf16, kForward>(a, st);
}

hipError_t launch_expert_grad_input(const ProductArgs &a, bool f16, hipStream_t st) {
  return f16 ? launch_act<_Float16, kGradInput>(a, st) : launch_act<__bf16, kGradInput>(a, st);
}

hipError_t launch_expert_grad_weight(const ProductArgs &a, bool f16, hipStream_t st) {
  return f16 ? launch_product<_Float16, kGradWeight, AA_ACT_NONE>(a, st)
             : launch_product<__bf16, kGradWeight, AA_ACT_NONE>(a, st);
}

}  // namespace aa

// The dense layer: a product with bias, activation and residual in its epilogue, and the gradient through them.
//
// The product is that of aa_product.hpp with one group; its sums start from the bias.  The gradient of what goes into the
// activation is one pass over the rows, bound by memory: a thread takes eight columns of the rows of its part and adds up the
// bias' gradient on the way, in 32 bits, before anything is rounded.
#include "aa_linear.hpp"

#include "aa_lines.hpp"
#include "aa_norm.hpp"
#include "aa_product.hpp"

namespace aa {

namespace {

// d with the activation's slope at h (gated: at the gate h and with up; *du gets up's gradient).
template <int ACT>
__device__ __forceinline__ float through(float d, float h, float up, float *du) {
  if (ACT == AA_ACT_RELU) return h > 0.f ? d : 0.f;
  if (ACT == AA_ACT_SILU || ACT == AA_ACT_GATED) {
    const float z = sigmoid_fast(h);
    if (ACT == AA_ACT_GATED) {
      *du = d * h * z;
      d *= up;
    }
    return d * (z + h * z * (1.f - z));
  }
  if (ACT == AA_ACT_GELU) {
    // (beyond 20 the sigmoid is 0 or 1 in 32 bits, and h^2 no concern)
    constexpr float k = 1.5957691216057308f;
    h = fminf(fmaxf(h, -20.f), 20.f);
    const float z = sigmoid_fast(gelu_argument(h));
    return d * (z + h * z * (1.f - z) * (k + 3.f * k * 0.044715f * h * h));
  }
  return d;
}

// CL lanes along the columns, 256 / CL rows at a time; blockIdx.y: the part.
template <typename T, int ACT, int CL>
__global__ __launch_bounds__(256) void k_act_grad(const ActGradArgs a) {
  constexpr int kRows = 256 / CL, kHalves = ACT == AA_ACT_GATED ? 2 : 1;
  __shared__ float room[kHalves][kRows][CL * 8];
  const int rows = rows_in_use(a.count, a.n_max), d = a.d;
  const int in_row = (int)threadIdx.x % CL, r0 = (int)threadIdx.x / CL;
  const int64_t c = ((int64_t)blockIdx.x * CL + in_row) * 8;
  Eight sum, sum_up;
#pragma unroll
  for (int i = 0; i < 8; ++i) sum.v[i] = sum_up.v[i] = 0.f;
  if (c < d) {
    const int n = d - (int)c;
    for (int64_t row = (int64_t)blockIdx.y * kRows + r0; row < rows; row += (int64_t)a.parts * kRows) {
      Eight g = load8(static_cast<const T *>(a.dout) + row * a.lddo + c, n), h, up;
      if (ACT != AA_ACT_NONE) h = load8(static_cast<const T *>(a.pre) + row * a.ldpre + c, n);
      if (ACT == AA_ACT_GATED) up = load8(static_cast<const T *>(a.pre) + row * a.ldpre + d + c, n);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float du = 0.f;
        g.v[i] = through<ACT>(g.v[i], ACT != AA_ACT_NONE ? h.v[i] : 0.f, ACT == AA_ACT_GATED ? up.v[i] : 0.f, &du);
        sum.v[i] += g.v[i];
        if (ACT == AA_ACT_GATED) {
          up.v[i] = du;
          sum_up.v[i] += du;
        }
      }
      if (a.dpre) {
        T *out = static_cast<T *>(a.dpre) + row * a.lddp + c;
        store8(out, g, n);
        if (ACT == AA_ACT_GATED) store8(out + d, up, n);
      }
    }
  }
  if (!a.dbias) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    room[0][r0][in_row * 8 + i] = sum.v[i];
    if (ACT == AA_ACT_GATED) room[kHalves - 1][r0][in_row * 8 + i] = sum_up.v[i];
  }
  __syncthreads();
#pragma unroll
  for (int half = 0; half < kHalves; ++half)
    for (int k = threadIdx.x; k < CL * 8; k += 256) {
      const int64_t at = (int64_t)blockIdx.x * CL * 8 + k;
      if (at >= d) continue;
      float all = 0.f;
#pragma unroll
      for (int r = 0; r < kRows; ++r) all += room[half][r][k];
      a.part[((int64_t)blockIdx.y * kHalves + half) * d + at] = all;
    }
}

template <typename T, int ACT, int CL>
hipError_t act_grad(ActGradArgs a, hipStream_t st) {
  constexpr int kRows = 256 / CL, kHalves = ACT == AA_ACT_GATED ? 2 : 1;
  // parts: eight blocks a compute unit, no more than there are rows or the workspace has room for
  const int64_t stripes = ((int64_t)a.d + CL * 8 - 1) / (CL * 8), fill = 2048 / stripes, turns = ((int64_t)a.n_max + kRows - 1) / kRows;
  const int64_t room = column_parts((int64_t)a.d * kHalves);
  int64_t parts = fill < turns ? fill : turns;
  parts = parts < room ? parts : room;
  a.parts = (int32_t)(parts > 1 ? parts : 1);
  hipLaunchKernelGGL((k_act_grad<T, ACT, CL>), dim3((uint32_t)stripes, (uint32_t)a.parts), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dbias) return e;
  return launch_join_columns(a.part, a.parts, (int64_t)a.d * kHalves, a.d, a.dbias, kHalves == 2 ? a.dbias + a.d : nullptr,
                             a.accumulate, st);
}

template <typename T, int ACT>
hipError_t by_columns(const ActGradArgs &a, hipStream_t st) {
  return a.d <= 128 ? act_grad<T, ACT, 16>(a, st) : act_grad<T, ACT, 64>(a, st);
}

template <typename T>
hipError_t by_act(const ActGradArgs &a, hipStream_t st) {
  switch (a.act) {
    case AA_ACT_RELU: return by_columns<T, AA_ACT_RELU>(a, st);
    case AA_ACT_GATED: return by_columns<T, AA_ACT_GATED>(a, st);
    case AA_ACT_SILU: return by_columns<T, AA_ACT_SILU>(a, st);
    case AA_ACT_GELU: return by_columns<T, AA_ACT_GELU>(a, st);
    default: return by_columns<T, AA_ACT_NONE>(a, st);
  }
}

template <typename T>
hipError_t linear(const ProductArgs &a, hipStream_t st) {
  switch (a.act) {
    case AA_ACT_RELU: return launch_product<T, kForward, AA_ACT_RELU, true>(a, st);
    case AA_ACT_GATED: return launch_product<T, kForward, AA_ACT_GATED, true>(a, st);
    case AA_ACT_SILU: return launch_product<T, kForward, AA_ACT_SILU, true>(a, st);
    case AA_ACT_GELU: return launch_product<T, kForward, AA_ACT_GELU, true>(a, st);
    default: return launch_product<T, kForward, AA_ACT_NONE, true>(a, st);
  }
}

}  // namespace

hipError_t launch_linear(const ProductArgs &a, bool f16, hipStream_t st) {
  return f16 ? linear<_Float16>(a, st) : linear<__bf16>(a, st);
}

hipError_t launch_linear_grad(const ActGradArgs &a, bool f16, hipStream_t st) {
  if (a.n_max == 0) {
    if (a.accumulate) return hipSuccess;
    return launch_clear_columns(a.dbias, a.act == AA_ACT_GATED && a.dbias ? a.dbias + a.d : nullptr, a.d, st);
  }
  return f16 ? by_act<_Float16>(a, st) : by_act<__bf16>(a, st);
}

}  // namespace aa

// Device helpers of the kernels that hold a row of logits in the registers of 16 or 64 lanes, neighbouring experts in a lane.
#pragma once

#include "aa_route.hpp"

#include <type_traits>

namespace aa {

namespace {

constexpr float kNegInf = -__builtin_inff();

// What the lanes of a wave wrote to LDS before is read by its other lanes after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Largest value and sum over aligned groups of LPR (16 or 64) lanes, every lane gets it: inside a row of 16 lanes
// quad swaps, half mirror, mirror; across rows exchanges with the lanes 16 and 32 away.  No LDS.
template <int CTRL>
__device__ __forceinline__ float lane_move(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ double lane_move(double v) {
  const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, true);
  const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, true);
  return __hiloint2double(hi, lo);
}

template <bool FAR>  // the lane 16 or (FAR) 32 away and this one, in some order
__device__ __forceinline__ void exchange(uint32_t v, uint32_t *x, uint32_t *y) {
  const auto r = FAR ? __builtin_amdgcn_permlane32_swap(v, v, false, false)
                     : __builtin_amdgcn_permlane16_swap(v, v, false, false);
  *x = r[0];
  *y = r[1];
}
template <bool FAR>
__device__ __forceinline__ void exchange(float v, float *x, float *y) {
  uint32_t a, b;
  exchange<FAR>(__float_as_uint(v), &a, &b);
  *x = __uint_as_float(a);
  *y = __uint_as_float(b);
}
template <bool FAR>
__device__ __forceinline__ void exchange(double v, double *x, double *y) {
  uint32_t al, bl, ah, bh;
  exchange<FAR>((uint32_t)__double2loint(v), &al, &bl);
  exchange<FAR>((uint32_t)__double2hiint(v), &ah, &bh);
  *x = __hiloint2double((int)ah, (int)al);
  *y = __hiloint2double((int)bh, (int)bl);
}

__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ double larger(double a, double b) { return fmax(a, b); }

template <int LPR, typename V>
__device__ __forceinline__ V lanes_max(V v) {
  static_assert(LPR == 16 || LPR == 64, "");
  v = larger(v, lane_move<0xB1>(v));
  v = larger(v, lane_move<0x4E>(v));
  v = larger(v, lane_move<0x141>(v));
  v = larger(v, lane_move<0x140>(v));
  if (LPR == 64) {
    V x, y;
    exchange<false>(v, &x, &y);
    exchange<true>(larger(x, y), &x, &y);
    v = larger(x, y);
  }
  return v;
}

template <int LPR, typename V>
__device__ __forceinline__ V lanes_sum(V v) {
  static_assert(LPR == 16 || LPR == 64, "");
  v += lane_move<0xB1>(v);
  v += lane_move<0x4E>(v);
  v += lane_move<0x141>(v);
  v += lane_move<0x140>(v);
  if (LPR == 64) {
    V x, y;
    exchange<false>(v, &x, &y);
    exchange<true>(x + y, &x, &y);
    v = x + y;
  }
  return v;
}

// N neighbouring logits of a row, -inf for those at or past E and for NaN.  vec: they exist whole or not at all, and can
// be moved at once.
template <typename T, int N>
__device__ __forceinline__ void load_logits(const T *row, int e0, int E, bool vec, float *x) {
  constexpr int kOn = N * sizeof(T) < 16 ? N * sizeof(T) : 16;
  typedef T Line __attribute__((ext_vector_type(N), aligned(kOn)));
  if (vec) {
    if (e0 < E) {
      const Line v = *reinterpret_cast<const Line *>(row + e0);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = (float)v[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (float)row[min(e0 + i, E - 1)];
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (e0 + i >= E || !(x[i] > kNegInf)) x[i] = kNegInf;
}

template <int N>
__device__ __forceinline__ void load_logits(const void *logits, int dtype, int64_t at, int e0, int E, bool vec, float *x) {
  if (dtype == AA_BF16) load_logits<__bf16, N>(static_cast<const __bf16 *>(logits) + at, e0, E, vec, x);
  else if (dtype == AA_F16) load_logits<_Float16, N>(static_cast<const _Float16 *>(logits) + at, e0, E, vec, x);
  else load_logits<float, N>(static_cast<const float *>(logits) + at, e0, E, vec, x);
}

template <typename T, int N>
__device__ __forceinline__ void store_logits(T *row, int e0, int E, bool vec, const float *x) {
  constexpr int kOn = N * sizeof(T) < 16 ? N * sizeof(T) : 16;
  typedef T Line __attribute__((ext_vector_type(N), aligned(kOn)));
  if (vec) {
    if (e0 >= E) return;
    Line v;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (T)x[i];
    *reinterpret_cast<Line *>(row + e0) = v;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (e0 + i < E) row[e0 + i] = (T)x[i];
  }
}

constexpr float kNoScore = -745.1332f;  // ln 2^-1075: from there down exp_below is 0

// Whether every lane's EPL logits exist whole or not at all and can be moved at once.
bool whole_lanes(const void *p, int64_t ld, int32_t E, int epl, int32_t dtype) {
  const int bytes = dtype == AA_F32 ? 4 : 2, on = epl * bytes < 16 ? epl * bytes : 16;
  return E % epl == 0 && ld * bytes % on == 0 && reinterpret_cast<uintptr_t>(p) % on == 0;
}

dim3 blocks_for(int32_t n_max, int rows_a_block) {
  const int64_t want = ((int64_t)n_max + rows_a_block - 1) / rows_a_block;
  return dim3((uint32_t)(want < (1 << 22) ? want : 1 << 22));  // (blocks take turns)
}

// The lanes of a row: 16 for up to most16 experts where they hold the choices too, else the wave (65,536 rows, 4 choices,
// sigmoid, without and with a bias: 32 experts 10.4 / 16.2 us, a wave a row 31.3 / 41.3).
template <typename Launch>
hipError_t by_width(int32_t E, int32_t K, int32_t most16, Launch launch) {
  using std::integral_constant;
  if (K <= 16 && E <= most16) {
    const integral_constant<int, 16> lpr;
    if (E <= 16) return launch(lpr, integral_constant<int, 1>());
    if (E <= 32) return launch(lpr, integral_constant<int, 2>());
    if (E <= 64) return launch(lpr, integral_constant<int, 4>());
    if (E <= 128) return launch(lpr, integral_constant<int, 8>());
    return launch(lpr, integral_constant<int, 16>());
  }
  const integral_constant<int, 64> lpr;
  if (E <= 64) return launch(lpr, integral_constant<int, 1>());
  if (E <= 128) return launch(lpr, integral_constant<int, 2>());
  if (E <= 256) return launch(lpr, integral_constant<int, 4>());
  if (E <= 512) return launch(lpr, integral_constant<int, 8>());
  return launch(lpr, integral_constant<int, 16>());
}

}  // namespace

}  // namespace aa

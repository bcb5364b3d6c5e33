// The dense layer: a product with bias, activation and residual in its epilogue, and the gradient through them.
//
// The product is that of aa_product.hpp with one group; its sums start from the bias.  The gradient of what goes into the
// activation is one pass over the rows, bound by memory: a thread takes eight columns of the rows of its part and adds up the
// bias' gradient on the way, in 32 bits, before anything is rounded.
#include "aa_linear.hpp"

#include "aa_checks.hpp"
#include "aa_lines.hpp"
#include "aa_norm.hpp"
#include "aa_product.hpp"

#include <math.h>

namespace aa {

namespace {

// d with the activation's slope at h (gated: at the gate h and with up; *du gets up's gradient).
template <int ACT>
__device__ __forceinline__ float through(float d, float h, float up, float *du) {
  if (ACT == AA_ACT_RELU) return h > 0.f ? d : 0.f;
  if (ACT == AA_ACT_SILU || ACT == AA_ACT_GATED) {
    const float z = sigmoid_near(h);
    if (ACT == AA_ACT_GATED) {
      *du = d * h * z;
      d *= up;
    }
    return d * (z + h * z * (1.f - z));
  }
  if (ACT == AA_ACT_GELU) {
    // (beyond 20 the sigmoid is 0 or 1 in 32 bits, and h^2 no concern; a NaN stays one)
    constexpr float k = 1.5957691216057308f;
    h = h < -20.f ? -20.f : h > 20.f ? 20.f : h;
    const float z = sigmoid_near(gelu_argument(h));
    return d * (z + h * z * (1.f - z) * (k + 3.f * k * 0.044715f * h * h));
  }
  return d;
}

// CL lanes along the columns, 256 / CL rows at a time; blockIdx.y: the part.  6001 x 1544 f16, silu: 15.6 us, 3.6 TB/s.
// dpre is rounded to the rows' 16 bits (without an activation it is dout, and nothing is rounded): it is what the matrix
// instructions of the gradients of rows and matrix take, and as much as dout itself holds.  Each of their terms is then off by
// half a step (6001 x 1000 -> 1544 silu f16: results furthest from 64 bits by 2.9e-4 of them, from a dpre of 32 bits 2.1e-4).
// What the rounding takes away, multiplied as well, would be the products' work a second time.
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
  const bool words = d % 8 != 0;
  const auto load = [&](const T *p, int n) __attribute__((always_inline)) {
    return words && n >= 8 ? to_eight<T>(load_words(p)) : load8(p, n);
  };
  const auto store = [&](T *p, const Eight &v, int n) __attribute__((always_inline)) {
    if (words && n >= 8) {
      Line<T> t;
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = (T)v.v[i];
      store_words(p, t);
    } else {
      store8(p, v, n);
    }
  };
  if (c < d) {
    const int n = d - (int)c;
    for (int64_t row = (int64_t)blockIdx.y * kRows + r0; row < rows; row += (int64_t)a.parts * kRows) {
      Eight g = load(static_cast<const T *>(a.dout) + row * a.lddo + c, n), h, up;
      if (ACT != AA_ACT_NONE) h = load(static_cast<const T *>(a.pre) + row * a.ldpre + c, n);
      if (ACT == AA_ACT_GATED) up = load(static_cast<const T *>(a.pre) + row * a.ldpre + d + c, n);
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
        store(out, g, n);
        if (ACT == AA_ACT_GATED) store(out + d, up, n);
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
      if (gridDim.y > 1) {
        a.part[((int64_t)blockIdx.y * kHalves + half) * d + at] = all;
      } else {  // (a part that is alone)
        float *to = a.dbias + (int64_t)half * d + at;
        *to = a.accumulate ? *to + all : all;
      }
    }
}

template <typename T, int ACT, int CL>
hipError_t act_grad(ActGradArgs a, hipStream_t st) {
  constexpr int kRows = 256 / CL, kHalves = ACT == AA_ACT_GATED ? 2 : 1;
  // Parts: eight blocks a compute unit, four where each still has much to do (bf16: 16,384 x 8192 gelu 166 us by eight, 155 by
  // four, 30,000 x 5000 139 and 129; 6001 x 1536 13.6 and 14.9; of lines off 16 bytes 50,000 x 1100 82 and 104), no more than
  // there are rows or the workspace has room for, and one where eight turns have them all (32 x 1024 6.6 us, in parts 9.3;
  // sixteen turns 11.2 and 9.2), of 16 lanes four (64 x 100 6.2 and 9.2, eight turns 10.4 and 9.1).
  const bool much = a.d % 8 == 0 && (int64_t)a.n_max * a.d >= 16ll << 20;
  const int64_t stripes = ((int64_t)a.d + CL * 8 - 1) / (CL * 8), fill = (much ? 1024 : 2048) / stripes;
  const int64_t turns = ((int64_t)a.n_max + kRows - 1) / kRows;
  const int64_t room = column_parts((int64_t)a.d * kHalves);
  int64_t parts = fill < turns ? fill : turns;
  parts = parts < room ? parts : room;
  a.parts = (int32_t)(parts > 1 && turns > (CL == 16 ? 4 : 8) ? parts : 1);
  hipLaunchKernelGGL((k_act_grad<T, ACT, CL>), dim3((uint32_t)stripes, (uint32_t)a.parts), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.dbias || a.parts == 1) return e;
  return launch_join_columns(a.part, a.parts, (int64_t)a.d * kHalves, a.d, a.dbias, kHalves == 2 ? a.dbias + a.d : nullptr,
                             a.accumulate, st);
}

// 64 lanes cover 512 columns (60,000 x 333 silu: 61 us, by 16 lanes 34; 50,000 x 1100: 82, 92).
template <typename T, int ACT>
hipError_t by_columns(const ActGradArgs &a, hipStream_t st) {
  return a.d <= 384 ? act_grad<T, ACT, 16>(a, st) : act_grad<T, ACT, 64>(a, st);
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

// The layer of a few rows: what is moved is the matrix, once.  A block takes 16 columns (with AA_ACT_GATED the gate's and
// up's) of 16 MF rows; its waves share the summed dimension out in chunks of 64, straight from memory into the matrix
// instructions' registers, kAhead of them on their way, and join their sums in LDS.  Rows are asked for whether they are in use
// or not: the count would be waited for first.  ODD: rows that may begin inside a word of four bytes.
// Four waves; eight or sixteen were slower (one row 4096 -> 136: 6.6, 7.2, 8.2 us).  One row 2048 -> 4096, 17 MB: 5.2 to 7.6 us;
// its waves wait for 75 % of that: each has eight chunks, of which kAhead are asked for before the first is there, so that memory is
// waited for twice in turn, and then the join.
constexpr int kFewWaves = 4;

// Sixteen bytes of a row at any address.  A load that begins inside a word of four bytes takes as long as four (9 rows 4781 ->
// 128: 20.7 us, 4782 8.3): with ODD the words that hold them are loaded, five of them, and shifted where they are used.
template <bool ODD>
struct Chunk {
  s16x8 v;
  __device__ __forceinline__ void ask(const char *row, int, int at, bool there) { v = *there_or_zeros(row + at, there); }
  __device__ __forceinline__ s16x8 get(int) const { return v; }
};
template <>
struct Chunk<true> {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  s16x8 v;
  uint32_t next;
  // row: where its first word begins; odd: 1 if the row begins inside it
  __device__ __forceinline__ void ask(const char *row, int odd, int at, bool there) {
    v = *there_or_zeros(row + at, there);
    next = *(const __attribute__((address_space(1))) uint32_t *)(there ? row + at + 12 + odd * 4 : (const char *)&kZeros);
  }
  __device__ __forceinline__ s16x8 get(int odd) const {
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_alignbit(i < 3 ? w[i < 3 ? i + 1 : 3] : next, w[i], odd * 16);
    return __builtin_bit_cast(s16x8, o);
  }
};

template <typename T, int ACT, int MF, bool ODD>
__global__ __launch_bounds__(kFewWaves *kWave) void k_dense_few(const ProductArgs a) {
  constexpr bool GATED = ACT == AA_ACT_GATED;
  constexpr int WAVES = kFewWaves, NF = GATED ? 2 : 1, kAhead = 4, kTurn = WAVES * kStep;
  __shared__ f4 sums[WAVES - 1][NF][MF][kWave];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int q0 = blockIdx.y * (16 * MF), j0 = blockIdx.x * 16, K = a.d_in & ~7, rest = a.d_in & 7;
  const T *wr[NF], *xr[MF];
  const char *w_at[NF], *x_at[MF];  // (ODD: the words' beginnings)
  int w_odd[NF], x_odd[MF];
  const auto begin = [](const T *row, const char **at, int *odd) {
    *odd = ODD ? (int)(reinterpret_cast<uintptr_t>(row) >> 1) & 1 : 0;
    *at = reinterpret_cast<const char *>(row) - *odd * 2;
  };
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    wr[f] = static_cast<const T *>(a.mat) + ((size_t)min(j0 + (lane & 15), a.d_out - 1) + (f > 0 ? a.d_out : 0)) * a.d_in + (lane >> 4) * 8;
    begin(wr[f], &w_at[f], &w_odd[f]);
  }
#pragma unroll
  for (int m = 0; m < MF; ++m) {
    xr[m] = static_cast<const T *>(a.rows) + (int64_t)min(q0 + m * 16 + (lane & 15), a.rows_max - 1) * a.ld_rows + (lane >> 4) * 8;
    begin(xr[m], &x_at[m], &x_odd[m]);
  }
  f4 acc[NF][MF];
#pragma unroll
  for (int f = 0; f < NF; ++f)
#pragma unroll
    for (int m = 0; m < MF; ++m) acc[f][m] = f4{0.f, 0.f, 0.f, 0.f};
  Chunk<ODD> fw[kAhead][NF][2], fx[kAhead][MF][2];
  const auto ask = [&](int slot, int k) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = k + h * 32;
      const bool there = at + (lane >> 4) * 8 < K;
#pragma unroll
      for (int f = 0; f < NF; ++f) fw[slot][f][h].ask(w_at[f], w_odd[f], at * 2, there);
#pragma unroll
      for (int m = 0; m < MF; ++m) fx[slot][m][h].ask(x_at[m], x_odd[m], at * 2, there);
    }
  };
  int k = wave * kStep;
#pragma unroll
  for (int s = 0; s < kAhead; ++s) ask(s, k + s * kTurn);
  const int rows = rows_in_use(a.count, a.rows_max);
  if (q0 >= rows) return;
  while (k < K) {
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
          for (int m = 0; m < MF; ++m) acc[f][m] = mfma16(fw[s][f][h].get(w_odd[f]), fx[s][m][h].get(x_odd[m]), acc[f][m], T());
      ask(s, k + kAhead * kTurn);
      k += kTurn;
    }
  }
  if (rest != 0 && wave == WAVES - 1) {  // what is left of a chunk of eight: the first lanes of four hold it, the others zeros
    const auto ends = [&](const T *row) {
      s16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
      const short *p = reinterpret_cast<const short *>(row + K);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < rest && lane < 16) v[i] = p[i];
      return v;
    };
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const s16x8 w = ends(wr[f]);
#pragma unroll
      for (int m = 0; m < MF; ++m) acc[f][m] = mfma16(w, ends(xr[m]), acc[f][m], T());
    }
  }
  if (wave > 0) {
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int m = 0; m < MF; ++m) sums[wave - 1][f][m][lane] = acc[f][m];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int o = 0; o < WAVES - 1; ++o)
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int m = 0; m < MF; ++m) acc[f][m] += sums[o][f][m][lane];
  const int c = j0 + (lane >> 4) * 4;
  if (c >= a.d_out) return;
  if (a.bias) {
#pragma unroll
    for (int f = 0; f < NF; ++f) {
      const f4 b = bias_of(a, c, f > 0 ? a.d_out : 0);
#pragma unroll
      for (int m = 0; m < MF; ++m) acc[f][m] += b;
    }
  }
#pragma unroll
  for (int m = 0; m < MF; ++m) {
    const int q = q0 + m * 16 + (lane & 15);
    if (q < rows) finish<T, kForward, ACT, true, false>(a, q, c, four_columns(acc[0][m]), four_columns(acc[NF - 1][m]));
  }
}

template <typename T, int ACT, int MF>
hipError_t dense_few(const ProductArgs &a, hipStream_t st) {
  const dim3 grid((a.d_out + 15) / 16, (a.rows_max + 16 * MF - 1) / (16 * MF)), block(kFewWaves * kWave);
  const bool words = on(a.rows, 4) && on(a.mat, 4) && a.d_in % 2 == 0 && a.ld_rows % 2 == 0;
  if (words) hipLaunchKernelGGL((k_dense_few<T, ACT, MF, false>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_dense_few<T, ACT, MF, true>), grid, block, 0, st, a);
  return hipGetLastError();
}

// Few rows or tiles, by what they take (us; bf16, 1 to 1065 rows, sums over 64 to 8192; few: blocks of 16 columns and up to
// 32 rows, one a compute unit at a time, steps of 256 of the sum; tiles as in launch_product, with what those of 32 x 64 and
// those through registers were measured at):
//   128 rows 4096 -> 256: few 13.5, tiles 19.2; 64 rows 8192 -> 1024: 24.5, 35.7; 128 rows 1024 -> 1024: 5.9, 7.1;
//   64 rows 1024 -> 4096: 9.0, 7.1; 128 rows 2048 -> 4096: 26.6, 12.2; 1065 rows 4096 -> 232: 25.5, 19.9
//   through registers: 72 rows 7319 -> 253: 56, 133 (few by words); 300 rows 1125 -> 217: 11, 26; 2000 rows 1002 -> 1000: 44, 24
template <typename T, int ACT>
hipError_t dense(const ProductArgs &a, hipStream_t st) {
  if (a.rows_max == 0) return hipSuccess;
  const double wide = (double)a.d_out * (ACT == AA_ACT_GATED ? 2 : 1), rows = a.rows_max, k = a.d_in;
  const auto cut = [](double v, double by) { return ceil(v / by); };
  const double blocks = cut(a.d_out, 16) * cut(rows, rows <= 16 ? 16 : 32), steps = cut(k, kStep);
  const double few = 3.0 + cut(k, 256) * (ACT == AA_ACT_GATED ? 0.9 : 0.7) * fmax(1.0, blocks / kUnits);
  const double tiles128 = cut(rows, 128) * cut(wide, 128);
  const double tiles = a.aligned ? fmin(cut(cut(rows, 32) * cut(wide, 64), 2 * kUnits) * (steps * 0.25 + 3.5),
                                        cut(tiles128, 2 * kUnits) * (steps * (tiles128 <= kUnits ? 0.6 : 1.05) + 3.0))
                                 : cut(tiles128, 2 * kUnits) * (steps * 1.15 + 3.0);
  if (few > tiles || cut(rows, 32) > 65535) return launch_product<T, kForward, ACT, true>(a, st);
  return rows <= 16 ? dense_few<T, ACT, 1>(a, st) : dense_few<T, ACT, 2>(a, st);
}

template <typename T>
hipError_t linear(const ProductArgs &a, hipStream_t st) {
  switch (a.act) {
    case AA_ACT_RELU: return dense<T, AA_ACT_RELU>(a, st);
    case AA_ACT_GATED: return dense<T, AA_ACT_GATED>(a, st);
    case AA_ACT_SILU: return dense<T, AA_ACT_SILU>(a, st);
    case AA_ACT_GELU: return dense<T, AA_ACT_GELU>(a, st);
    default: return dense<T, AA_ACT_NONE>(a, st);
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

// Layer norm, its gradient, and sums over columns of many rows.
//
// A row is held in registers by the TPR threads that take it, eight neighbouring columns at a time: it crosses the memory
// once.  mean = sum x / d; the squares are summed around it, so that no digits cancel.  With xh = (x - mean) rstd and
// g = dy gamma:
//   dx = residual + rstd (g - sum g / d - xh sum (g xh) / d),   dgamma = sum over rows of dy xh,   dbeta = of dy.
// The sums over rows: each block adds up the rows it takes in registers, and what the blocks have is added up in their
// order by a second launch, so that the same call gives the same bits.  Bound by memory.
#include "aa_norm.hpp"

#include "aa_lines.hpp"

#include <type_traits>

namespace aa {

namespace {

constexpr int kUnits = 256;  // compute units

// Row of this thread among the block's NT / TPR; the wave has one if TPR is a wave or more.
template <int TPR>
__device__ __forceinline__ uint32_t row_of(int64_t base) {
  const uint32_t row = (uint32_t)base + threadIdx.x / TPR;
  return TPR >= kWave ? (uint32_t)__builtin_amdgcn_readfirstlane((int)row) : row;
}

template <int TPR>
constexpr int kThreads = TPR > 256 ? TPR : 256;

// Sums of two values over the TPR threads of a row.  Rows of several waves meet in LDS: room is one of two that
// the block's turns take alternately, so that one barrier a turn is enough.
template <int TPR>
__device__ __forceinline__ void row_sums(float &a, float &b, int lane, float (*room)[2]) {
  constexpr int W = TPR < kWave ? TPR : kWave;
  a = lanes_sum<W>(a, lane);
  b = lanes_sum<W>(b, lane);
  if constexpr (TPR > kWave) {
    const int wave = threadIdx.x / kWave, first = wave / (TPR / kWave) * (TPR / kWave);  // (of the row's waves)
    if (lane == 0) {
      room[wave][0] = a;
      room[wave][1] = b;
    }
    __syncthreads();
    const int w = lane & 15;  // (each 16 lanes add up the waves', at most 16)
    a = lanes_sum<16>(w < TPR / kWave ? room[first + w][0] : 0.f, lane);
    b = lanes_sum<16>(w < TPR / kWave ? room[first + w][1] : 0.f, lane);
  }
}

// Mean of a row of d columns and the sum of the squares around it.  Rows of several waves: each wave's squares are
// summed around its own mean, and moved to the row's when they are joined (n_w (mean_w - mean)^2 more).
template <int TPR, int NV>
__device__ __forceinline__ void row_moments(const Eight (&x)[NV], int d, int c0, int lane, float (*room)[2], float *mean,
                                            float *squares) {
  constexpr int W = TPR < kWave ? TPR : kWave;
  float s = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[v].v[i];  // (columns past the row's end hold 0)
  s = lanes_sum<W>(s, lane);
  // columns of this wave
  int n = d;
  if (TPR > kWave) {
    n = 0;
    const int first = (int)threadIdx.x / kWave * kWave * 8;
#pragma unroll
    for (int v = 0; v < NV; ++v) n += min(max(d - (v * TPR * 8 + first), 0), kWave * 8);
  }
  const float mu = n > 0 ? s / (float)n : 0.f;
  float q = 0.f;
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = x[v].v[i] - mu;
      q += c0 + v * TPR * 8 + i < d ? t * t : 0.f;
    }
  q = lanes_sum<W>(q, lane);
  *mean = mu;
  *squares = q;
  if constexpr (TPR > kWave) {
    const int wave = threadIdx.x / kWave;
    if (lane == 0) {
      room[wave][0] = s;
      room[wave][1] = q;
    }
    __syncthreads();
    const int w = lane & 15;  // (each 16 lanes join the waves, at most 16)
    const bool there = w < TPR / kWave;
    s = there ? room[w][0] : 0.f;
    q = there ? room[w][1] : 0.f;
    const float m = lanes_sum<16>(s, lane) / (float)d;
    int nw = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v) nw += min(max(d - (v * TPR + w * kWave) * 8, 0), kWave * 8);
    const float off = there && nw > 0 ? s / (float)nw - m : 0.f;
    const float all = lanes_sum<16>(q + (float)nw * off * off, lane);
    *mean = m;
    *squares = all;
  }
}

// NV lines of a row, `step` columns apart, from column c0 on; 0 past its end.  NARROW: the row may hold fewer than eight
// columns.  PASSING: past the caches.
template <bool NARROW, bool PASSING = false, typename T, int NV>
__device__ __forceinline__ void load_row(const T *row, int c0, int step, int d, Eight (&x)[NV]) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = c0 + v * step;
    Line<T> t = {};
    if (c < d) {
      if (d % 8 != 0) t = NARROW ? load_line(row + c, d - c) : load_line_early(row + c, d - c);
      else if (PASSING) t = __builtin_nontemporal_load(reinterpret_cast<const Line<T> *>(row + c));
      else t = *reinterpret_cast<const Line<T> *>(row + c);
    }
    x[v] = to_eight<T>(t);
  }
}

template <bool PASSING, typename T>
__device__ __forceinline__ void store_line(T *p, const Eight &o, int n) {
  if (PASSING && n >= 8) {
    Line<T> t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)o.v[i];
    __builtin_nontemporal_store(t, reinterpret_cast<Line<T> *>(p));
  } else {
    store8(p, o, n);
  }
}

template <bool NARROW, int NV>
__device__ __forceinline__ void load_vector(const float *p, float none, int c0, int step, int d, Eight (&x)[NV]) {
  if (p) {
    load_row<NARROW>(p, c0, step, d, x);
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[v].v[i] = none;
  }
}

// 30,000 x 4096 bf16 94 us, 5.2 TB/s.
template <typename T, int TPR, int NV, bool PASSING>
__global__ __launch_bounds__(kThreads<TPR>) void k_layer_norm(const NormArgs a) {
  constexpr int kRows = kThreads<TPR> / TPR, kStepC = TPR * 8;
  constexpr bool kNarrow = TPR == 16 && NV == 1;
  __shared__ float room[2][kThreads<TPR> / kWave][2];
  const int rows = rows_in_use(a.count, a.n_max), d = a.d;
  const int lane = threadIdx.x & 63, c0 = (int)threadIdx.x % TPR * 8;
  Eight gamma[NV], beta[NV];
  load_vector<kNarrow>(a.gamma, 1.f, c0, kStepC, d, gamma);
  load_vector<kNarrow>(a.beta, 0.f, c0, kStepC, d, beta);
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < rows; base += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const uint32_t row = row_of<TPR>(base);
    if (row >= (uint32_t)rows) return;  // (a block of several rows has no barrier)
    Eight x[NV];
    load_row<kNarrow>(static_cast<const T *>(a.x) + (int64_t)row * a.ldx, c0, kStepC, d, x);
    float mean, squares;
    row_moments<TPR, NV>(x, d, c0, lane, room[turn], &mean, &squares);
    const float rstd = 1.0f / sqrtf(squares / (float)d + a.eps);
    if (c0 == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    T *out = static_cast<T *>(a.out) + (int64_t)row * a.ldo;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * kStepC;
      if (c >= d) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[v].v[i] = (x[v].v[i] - mean) * rstd * gamma[v].v[i] + beta[v].v[i];
      store_line<PASSING>(out + c, x[v], d - c);
    }
  }
}

// Sum over the block, in 64 bits; every thread gets it.
__device__ __forceinline__ double block_sum(double v, double *room) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  __syncthreads();  // (the room has been read)
  if ((threadIdx.x & 63) == 0) room[threadIdx.x / kWave] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < (int)blockDim.x / kWave; ++w) v += room[w];
  return v;
}

constexpr int kLongThreads = 1024;

// Rows that no block holds: read once for the mean, once for the squares, once for the result.  Nothing here has such rows, and
// they were left at this: 6710 x 20,000 bf16 201 us (2.7 TB/s by what has to move), of 20,001 274; 128 x 1,048,576 384.
template <typename T>
__global__ __launch_bounds__(kLongThreads) void k_layer_norm_long(const NormArgs a) {
  __shared__ double room[kLongThreads / kWave];
  const int rows = rows_in_use(a.count, a.n_max), d = a.d;
  for (int row = blockIdx.x; row < rows; row += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.ldx;
    T *out = static_cast<T *>(a.out) + (int64_t)row * a.ldo;
    double s = 0.0;
    for (int c = threadIdx.x * 8; c < d; c += kLongThreads * 8) {
      const Eight v = load8(x + c, d - c);
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) t += v.v[i];
      s += (double)t;
    }
    const float mean = (float)(block_sum(s, room) / d);
    double q = 0.0;
    for (int c = threadIdx.x * 8; c < d; c += kLongThreads * 8) {
      const Eight v = load8(x + c, d - c);
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) t += c + i < d ? (v.v[i] - mean) * (v.v[i] - mean) : 0.f;
      q += (double)t;
    }
    const float rstd = 1.0f / sqrtf((float)(block_sum(q, room) / d) + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    for (int c = threadIdx.x * 8; c < d; c += kLongThreads * 8) {
      Eight v = load8(x + c, d - c), one[1], zero[1];
      load_vector<false>(a.gamma, 1.f, c, 0, d, one);
      load_vector<false>(a.beta, 0.f, c, 0, d, zero);
#pragma unroll
      for (int i = 0; i < 8; ++i) v.v[i] = (v.v[i] - mean) * rstd * one[0].v[i] + zero[0].v[i];
      store8(out + c, v, d - c);
    }
  }
}

// Threads of a block of the gradient: there are as many blocks as the sums have parts, two a compute unit, and 16 waves there
// are needed (19,960 x 1688 bf16: 82 us with 8).
constexpr int kGradThreads = 512;

// 16,384 x 8192 bf16 with a residual 184 us, 5.8 TB/s, and 6.6 for the sums' parts.
template <typename T, int TPR, int NV, bool PASSING>
__global__ __launch_bounds__(kGradThreads) void k_layer_norm_grad(const NormArgs a) {
  constexpr int NT = kGradThreads, kRows = NT / TPR, kStepC = TPR * 8;
  constexpr bool kNarrow = TPR == 16 && NV == 1;
  __shared__ float room[2][NT / kWave][2];
  __shared__ float joined[kRows > 1 ? kRows : 1][kRows > 1 ? NV * kStepC : 1];
  const int rows = rows_in_use(a.count, a.n_max), d = a.d;
  const int lane = threadIdx.x & 63, c0 = (int)threadIdx.x % TPR * 8;
  const bool sums = a.dgamma || a.dbeta;
  Eight gamma[NV], dg[NV], db[NV];
  load_vector<kNarrow>(a.gamma, 1.f, c0, kStepC, d, gamma);
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[v].v[i] = db[v].v[i] = 0.f;
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < rows; base += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const uint32_t row = row_of<TPR>(base);
    // (threads whose row is past the last go along: with a dy of 0 they add nothing)
    const bool live = row < (uint32_t)rows;
    Eight x[NV], dy[NV];
    float mean = 0.f, rstd = 0.f;
    if (live) {
      load_row<kNarrow, PASSING>(static_cast<const T *>(a.x) + (int64_t)row * a.ldx, c0, kStepC, d, x);
      load_row<kNarrow, PASSING>(static_cast<const T *>(a.dout) + (int64_t)row * a.lddo, c0, kStepC, d, dy);
      mean = a.mean[row];
      rstd = a.rstd[row];
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[v].v[i] = dy[v].v[i] = 0.f;
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float xh = (x[v].v[i] - mean) * rstd, g = dy[v].v[i] * gamma[v].v[i];
        x[v].v[i] = xh;
        dg[v].v[i] += dy[v].v[i] * xh;
        db[v].v[i] += dy[v].v[i];
        dy[v].v[i] = g;
        s1 += g;  // (dy is 0 past the row's end)
        s2 += g * xh;
      }
    row_sums<TPR>(s1, s2, lane, room[turn]);
    if (!live) continue;
    s1 /= (float)d;
    s2 /= (float)d;
    T *out = static_cast<T *>(a.out) + (int64_t)row * a.ldo;
    const T *res = static_cast<const T *>(a.residual) + (a.residual ? (int64_t)row * a.ldr : 0);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = c0 + v * kStepC;
      if (c >= d) continue;
      Eight r;
#pragma unroll
      for (int i = 0; i < 8; ++i) r.v[i] = rstd * (dy[v].v[i] - s1 - x[v].v[i] * s2);
      if (a.residual) {
        Eight add[1];
        load_row<kNarrow, PASSING>(res, c, 0, d, add);
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] += add[0].v[i];
      }
      store_line<PASSING>(out + c, r, d - c);
    }
  }
  if (!sums) return;
  // a block that is alone has the sums, the others a part of them each
  const bool alone = gridDim.x == 1, add = alone && a.accumulate;
  float *part = a.part + (int64_t)blockIdx.x * 2 * d;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const Eight(&s)[NV] = which == 0 ? dg : db;
    float *to = alone ? (which == 0 ? a.dgamma : a.dbeta) : part + (int64_t)which * d;
    if (!to) continue;
    if constexpr (kRows == 1) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = c0 + v * kStepC;
        if (c >= d) continue;
        Eight all = s[v];
        if (add) {
          const Eight old = load8(to + c, d - c);
#pragma unroll
          for (int i = 0; i < 8; ++i) all.v[i] += old.v[i];
        }
        store8(to + c, all, d - c);
      }
    } else {  // the rows that the block took at once
      __syncthreads();
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) joined[threadIdx.x / TPR][c0 + v * kStepC + i] = s[v].v[i];
      __syncthreads();
      for (int c = threadIdx.x; c < d; c += NT) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) sum += joined[r][c];
        to[c] = add ? to[c] + sum : sum;
      }
    }
  }
}

// Rows that no block holds: read once for the two sums, once for the result, and before that for the sums over rows.  6710 x
// 20,000 bf16 343 us in all (2.3 TB/s), of 20,001 475; 128 x 1,048,576 575.
template <typename T>
__global__ __launch_bounds__(kLongThreads) void k_layer_norm_grad_long(const NormArgs a) {
  __shared__ double room[kLongThreads / kWave];
  const int rows = rows_in_use(a.count, a.n_max), d = a.d;
  for (int row = blockIdx.x; row < rows; row += gridDim.x) {
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.ldx;
    const T *dy = static_cast<const T *>(a.dout) + (int64_t)row * a.lddo;
    const T *res = static_cast<const T *>(a.residual) + (a.residual ? (int64_t)row * a.ldr : 0);
    T *out = static_cast<T *>(a.out) + (int64_t)row * a.ldo;
    const float mean = a.mean[row], rstd = a.rstd[row];
    const auto terms = [&](int c, Eight &xh, Eight &g) {
      Eight gamma[1];
      load_vector<false>(a.gamma, 1.f, c, 0, d, gamma);
      xh = load8(x + c, d - c);
      g = load8(dy + c, d - c);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xh.v[i] = (xh.v[i] - mean) * rstd;
        g.v[i] *= gamma[0].v[i];
      }
    };
    double p = 0.0, q = 0.0;
    for (int c = threadIdx.x * 8; c < d; c += kLongThreads * 8) {
      Eight xh, g;
      terms(c, xh, g);
      float t = 0.f, u = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        t += g.v[i];
        u += g.v[i] * xh.v[i];
      }
      p += (double)t;
      q += (double)u;
    }
    const float s1 = (float)(block_sum(p, room) / d), s2 = (float)(block_sum(q, room) / d);
    for (int c = threadIdx.x * 8; c < d; c += kLongThreads * 8) {
      Eight xh, g;
      terms(c, xh, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) g.v[i] = rstd * (g.v[i] - s1 - xh.v[i] * s2);
      if (a.residual) {
        const Eight add = load8(res + c, d - c);
#pragma unroll
        for (int i = 0; i < 8; ++i) g.v[i] += add.v[i];
      }
      store8(out + c, g, d - c);
    }
  }
}

// The sums over rows for rows that no block holds: a wave takes 512 columns of the rows of its part.
template <typename T>
__global__ __launch_bounds__(256) void k_layer_norm_columns(const NormArgs a, int parts) {
  const int rows = rows_in_use(a.count, a.n_max), d = a.d;
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8, part = blockIdx.y;
  if (c >= d) return;
  const int each = (rows + parts - 1) / parts, from = min(part * (int64_t)each, (int64_t)rows), to = min(from + each, rows);
  Eight dg, db;
#pragma unroll
  for (int i = 0; i < 8; ++i) dg.v[i] = db.v[i] = 0.f;
  for (int row = from; row < to; ++row) {
    const Eight x = load8(static_cast<const T *>(a.x) + (int64_t)row * a.ldx + c, d - c);
    const Eight dy = load8(static_cast<const T *>(a.dout) + (int64_t)row * a.lddo + c, d - c);
    const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      dg.v[i] += dy.v[i] * ((x.v[i] - mean) * rstd);
      db.v[i] += dy.v[i];
    }
  }
  store8(a.part + (int64_t)part * 2 * d + c, dg, d - c);
  store8(a.part + (int64_t)part * 2 * d + d + c, db, d - c);
}

// first[c], second[c] (+)= the sum over the parts (`stride` apart) of their columns c and d + c: 64 columns a block, 16
// shares of the parts, joined in their order.  512 parts of 8192 columns 6.6 us, of 1021 3.9.
constexpr int kJoinShares = 16;

__global__ __launch_bounds__(kJoinShares *kWave) void k_join_columns(const float *part, int parts, int64_t stride, int d,
                                                                      float *first, float *second, int accumulate) {
  __shared__ float sums[kJoinShares][kWave];
  float *out = blockIdx.y == 0 ? first : second;
  if (!out) return;
  const int lane = threadIdx.x & 63, share = threadIdx.x / kWave;
  const int64_t c = (int64_t)blockIdx.x * kWave + lane;
  const float *p = part + (int64_t)blockIdx.y * d + min(c, (int64_t)d - 1);
  const int each = (parts + kJoinShares - 1) / kJoinShares, from = min(share * each, parts), to = min(from + each, parts);
  float sum = 0.f;
#pragma unroll 8
  for (int i = from; i < to; ++i) sum += p[i * stride];
  sums[share][lane] = sum;
  __syncthreads();
  if (share > 0 || c >= d) return;
  float all = accumulate ? out[c] : 0.f;
  sum = 0.f;
#pragma unroll
  for (int s = 0; s < kJoinShares; ++s) sum += sums[s][lane];
  out[c] = all + sum;
}

hipError_t join_columns(const NormArgs &a, int parts, hipStream_t st) {
  return launch_join_columns(a.part, parts, 2 * (int64_t)a.d, a.d, a.dgamma, a.dbeta, a.accumulate, st);
}

// Threads of a row and lines of eight columns each of them holds.  Few threads with many lines share a sum with few and have
// much on its way; many threads leave registers for more waves, which the gradient with its sums needs more.  (us, bf16:
//   671,088 x 200: 16 threads of 2 lines forward 108, gradient 185; 64 of 1 169, 242
//   262,144 x 512: 16 of 4 forward 86, gradient 151; 64 of 1 95, 141
//   65,536 x 2048: 64 of 4 87, 157; 256 of 1 105, 142
//   16,384 x 8192: 256 of 4 85, 164 (2000 rows 16.3, 35); 512 of 2 93, 142 (13.9, 28)
//   14,913 x 9000: 512 of 3 88, 202; 1024 of 2 139, 199.  8388 x 16,000: 512 of 4 98, 257; 1024 of 2 110, 272.  The gradient
//   holds x, dy, gamma and both sums of a thread's 32 columns in registers there, 223 of them: one block a compute unit)
template <bool GRAD, typename Launch, typename Long>
hipError_t by_row_width(int32_t d, Launch launch, Long long_rows) {
  using std::integral_constant;
#define AA_ROW(T, V) launch(integral_constant<int, T>(), integral_constant<int, V>())
  if (d <= 128) return AA_ROW(16, 1);
  if (d <= 256) return AA_ROW(16, 2);
  if (d <= 512) {
    if constexpr (GRAD) return AA_ROW(64, 1);
    else return AA_ROW(16, 4);
  }
  if (d <= 1024) return AA_ROW(64, 2);
  if (d <= 2048) {
    if constexpr (GRAD) return AA_ROW(256, 1);
    else return AA_ROW(64, 4);
  }
  if (d <= 4096) return AA_ROW(256, 2);
  if (d <= 8192) return AA_ROW(512, 2);
  if (d <= 12288) return AA_ROW(512, 3);
  if (d <= 16384) return AA_ROW(512, 4);
#undef AA_ROW
  return long_rows();
}

// Results of so many bytes, half of the cache that all of the chip shares, are not there any more when they are read: they pass
// it by, and in the gradient so do the rows (16,384 x 8192 bf16 with a residual 203 -> 186 us; 30,000 x 4096 96 -> 94, its rows
// too 97; 8191 x 1021 f32, 33 MB, 25.1 and 26.6).
template <typename T>
bool passing(const NormArgs &a) {
  return (int64_t)a.n_max * a.d * (int64_t)sizeof(T) >= 128ll << 20;
}

template <typename T>
hipError_t layer_norm(const NormArgs &a, hipStream_t st) {
  return by_row_width<false>(
      a.d,
      [&](auto tpr, auto nv) {
        constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, kRows = kThreads<TPR> / TPR;
        const int64_t want = ((int64_t)a.n_max + kRows - 1) / kRows, most = (int64_t)kUnits * 2048 / kThreads<TPR>;
        const dim3 grid((uint32_t)(want < most ? want : most)), block(kThreads<TPR>);
        if (passing<T>(a)) hipLaunchKernelGGL((k_layer_norm<T, TPR, NV, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((k_layer_norm<T, TPR, NV, false>), grid, block, 0, st, a);
        return hipGetLastError();
      },
      [&] {
        hipLaunchKernelGGL(k_layer_norm_long<T>, dim3(a.n_max < 512 ? a.n_max : 512), dim3(kLongThreads), 0, st, a);
        return hipGetLastError();
      });
}

template <typename T>
hipError_t layer_norm_grad(const NormArgs &a, hipStream_t st) {
  const int most = column_parts(a.d);
  return by_row_width<true>(
      a.d,
      [&](auto tpr, auto nv) {
        constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value, kRows = kGradThreads / TPR;
        const int64_t want = ((int64_t)a.n_max + kRows - 1) / kRows;
        // (a block that is alone takes four turns in less than a second launch does: 32 rows of 1024 7.9 us, in parts 10.9; eight
        // turns 12.8 and 10.8)
        const int parts = want <= 4 ? 1 : (int)(want < most ? want : most);
        const dim3 grid(parts), block(kGradThreads);
        if (passing<T>(a)) hipLaunchKernelGGL((k_layer_norm_grad<T, TPR, NV, true>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((k_layer_norm_grad<T, TPR, NV, false>), grid, block, 0, st, a);
        const hipError_t e = hipGetLastError();
        return e != hipSuccess || parts == 1 ? e : join_columns(a, parts, st);
      },
      [&] {
        if (a.dgamma || a.dbeta) {  // (first: dx may be dout or x)
          const int parts = a.n_max < most ? a.n_max : most;
          const dim3 grid((uint32_t)(((int64_t)a.d + 2047) / 2048), (uint32_t)parts);
          hipLaunchKernelGGL(k_layer_norm_columns<T>, grid, dim3(256), 0, st, a, parts);
          hipError_t e = hipGetLastError();
          if (e == hipSuccess) e = join_columns(a, parts, st);
          if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(k_layer_norm_grad_long<T>, dim3(a.n_max < 512 ? a.n_max : 512), dim3(kLongThreads), 0, st, a);
        return hipGetLastError();
      });
}

// Sums of no rows.
__global__ void k_clear_columns(float *first, float *second, int d) {
  const int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= d) return;
  if (first) first[c] = 0.f;
  if (second) second[c] = 0.f;
}

}  // namespace

hipError_t launch_clear_columns(float *first, float *second, int32_t d, hipStream_t st) {
  if (!first && !second) return hipSuccess;
  hipLaunchKernelGGL(k_clear_columns, dim3((uint32_t)(((int64_t)d + 255) / 256)), dim3(256), 0, st, first, second, d);
  return hipGetLastError();
}

hipError_t launch_join_columns(const float *part, int parts, int64_t stride, int32_t d, float *first, float *second,
                               int32_t accumulate, hipStream_t st) {
  if (!first && !second) return hipSuccess;
  const dim3 grid((uint32_t)(((int64_t)d + kWave - 1) / kWave), 2);
  hipLaunchKernelGGL(k_join_columns, grid, dim3(kJoinShares * kWave), 0, st, part, parts, stride, d, first, second, accumulate);
  return hipGetLastError();
}

hipError_t launch_layer_norm(const NormArgs &a, int32_t dtype, hipStream_t st) {
  if (a.n_max == 0) return hipSuccess;
  switch (dtype) {
    case AA_BF16: return layer_norm<__bf16>(a, st);
    case AA_F16: return layer_norm<_Float16>(a, st);
    default: return layer_norm<float>(a, st);
  }
}

hipError_t launch_layer_norm_grad(const NormArgs &a, int32_t dtype, hipStream_t st) {
  if (a.n_max == 0) return a.accumulate ? hipSuccess : launch_clear_columns(a.dgamma, a.dbeta, a.d, st);
  switch (dtype) {
    case AA_BF16: return layer_norm_grad<__bf16>(a, st);
    case AA_F16: return layer_norm_grad<_Float16>(a, st);
    default: return layer_norm_grad<float>(a, st);
  }
}

}  // namespace aa

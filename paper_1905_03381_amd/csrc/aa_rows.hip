// Row operators of a block of experts: dropout whose mask is drawn again wherever it is needed, and the
// weighted combination of the experts' rows with its gradient.  All are one pass over their rows, bound
// by memory: eight neighbouring columns a thread (the eight draws of one Philox call), 16-byte
// accesses.  Rates of what has to move (a 4 GiB device copy reaches 4.8 TB/s read and written): dropout with
// residual of 65,536 x 2048 bf16 135 us, 6.0 TB/s; combination of 8192 rows of 8 x 2048 bf16 65 us, 5.1 TB/s; its
// gradient 117 us, 4.9 TB/s.
#include "aa_rows.hpp"

#include "aa_lines.hpp"

#include <type_traits>

namespace aa {

namespace {

// Columns c .. c + 7 (c a multiple of 8) of a row; what is dropped is 0 whatever it was.
__device__ __forceinline__ void drop8(const DropKey &k, int row, int c, Eight &x) {
  if (k.limit >= 65536u) return;
  const uint4 w = philox_words((uint32_t)c >> 3, (uint32_t)row + 1u, k.s0, k.s1, k.k0, k.k1);
  const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t draw = i & 1 ? word[i >> 1] >> 16 : word[i >> 1] & 0xFFFFu;
    x.v[i] = draw < k.limit ? x.v[i] * k.scale : 0.f;
  }
}

constexpr int kBatch = 8;  // choices of a row whose lines are asked for together

// TPR threads a row, 256 / TPR rows a turn of the block.  A wave that has one row knows it for all its lanes.
template <int TPR>
__device__ __forceinline__ int row_of(int base) {
  const int row = base + (int)threadIdx.x / TPR;
  return TPR >= kWave ? __builtin_amdgcn_readfirstlane(row) : row;
}

template <typename T, int TPR>
__global__ __launch_bounds__(256) void k_dropout(const DropoutArgs a) {
  const int rows = rows_in_use(a.count, a.n_max);
  for (int64_t base = (int64_t)blockIdx.x * (256 / TPR); base < rows; base += (int64_t)gridDim.x * (256 / TPR)) {
    const int row = row_of<TPR>((int)base);
    if (row >= rows) return;
    const T *x = static_cast<const T *>(a.x) + (int64_t)row * a.ldx;
    const T *r = static_cast<const T *>(a.residual) + (a.residual ? (int64_t)row * a.ldr : 0);
    T *o = static_cast<T *>(a.out) + (int64_t)row * a.ldo;
    for (int c = (threadIdx.x % TPR) * 8; c < a.d; c += TPR * 8) {
      const int n = a.d - c;
      Eight v = load8(x + c, n), add;
      if (a.residual) add = load8(r + c, n);
      drop8(a.key, row, c, v);
      if (a.residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v.v[i] += add.v[i];
      }
      store8(o + c, v, n);
    }
  }
}

// out = residual + dropout(sum_k w_k y_k).  The lines of eight choices are asked for before the first is used: one at
// a time left most of the memory's latency in the row (8192 rows of 8 x 2048 bf16: 80 us).
template <typename T, int TPR>
__global__ __launch_bounds__(256) void k_combine(const CombineArgs a) {
  const int rows = rows_in_use(a.count, a.n_max), K = a.top_k;
  for (int64_t base = (int64_t)blockIdx.x * (256 / TPR); base < rows; base += (int64_t)gridDim.x * (256 / TPR)) {
    const int row = row_of<TPR>((int)base);
    if (row >= rows) return;
    const T *y = static_cast<const T *>(a.y);
    const int32_t *slot = a.slot + (int64_t)row * K;
    const float *w = a.weights + (a.weights ? (int64_t)row * K : 0);
    const T *r = static_cast<const T *>(a.residual) + (a.residual ? (int64_t)row * a.ldr : 0);
    T *o = static_cast<T *>(a.out) + (int64_t)row * a.ldo;
    for (int c = (threadIdx.x % TPR) * 8; c < a.d; c += TPR * 8) {
      const int n = a.d - c;
      Eight sum = {{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}};
      Line<T> add;
      if (a.residual) add = load_line(r + c, n);
      for (int k0 = 0; k0 < K; k0 += kBatch) {
        Line<T> line[kBatch];
        int q[kBatch];
        float f[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          q[j] = k0 + j < K ? slot[k0 + j] : -1;
          f[j] = k0 + j < K && a.weights ? w[k0 + j] : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (q[j] >= 0) line[j] = load_line(y + (int64_t)q[j] * a.ldy + c, n);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          if (q[j] < 0) continue;
#pragma unroll
          for (int i = 0; i < 8; ++i) sum.v[i] = __fmaf_rn(f[j], (float)line[j][i], sum.v[i]);
        }
      }
      drop8(a.key, row, c, sum);
      if (a.residual) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum.v[i] += (float)add[i];
      }
      store8(o + c, sum, n);
    }
  }
}

// g = dropout(dout), dy_k = w_k g, dw_k = y_k . g.
template <typename T, int TPR>
__global__ __launch_bounds__(256) void k_combine_grad(const CombineArgs a) {
  constexpr int kWavesPerRow = TPR > kWave ? TPR / kWave : 1;
  __shared__ float s_part[256 / TPR][kWavesPerRow][kBatch];
  const int in_block = threadIdx.x / TPR, t = threadIdx.x % TPR, lane = threadIdx.x & 63;
  const int rows = rows_in_use(a.count, a.n_max), K = a.top_k;
  const T *y = static_cast<const T *>(a.y);
  T *dy = static_cast<T *>(a.out);
  for (int64_t base = (int64_t)blockIdx.x * (256 / TPR); base < rows; base += (int64_t)gridDim.x * (256 / TPR)) {
    const int row = row_of<TPR>((int)base);
    const bool live = row < rows;
    for (int k0 = 0; k0 < K; k0 += kBatch) {
      float part[kBatch], f[kBatch];
      int q[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        part[j] = 0.f;
        const bool there = live && k0 + j < K;
        q[j] = there ? a.slot[(int64_t)row * K + k0 + j] : -1;
        f[j] = there && a.weights ? a.weights[(int64_t)row * K + k0 + j] : 1.0f;
      }
      if (live) {
        const T *g_row = static_cast<const T *>(a.dout) + (int64_t)row * a.lddo;
        for (int c = t * 8; c < a.d; c += TPR * 8) {
          const int n = a.d - c;
          Eight g = load8(g_row + c, n);
          Line<T> line[kBatch];
          if (a.dweights) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j)
              if (q[j] >= 0) line[j] = load_line(y + (int64_t)q[j] * a.ldy + c, n);
          }
          drop8(a.key, row, c, g);
#pragma unroll
          for (int j = 0; j < kBatch; ++j) {
            if (q[j] < 0) continue;
            Eight d;
#pragma unroll
            for (int i = 0; i < 8; ++i) d.v[i] = f[j] * g.v[i];
            store8(dy + (int64_t)q[j] * a.ldo + c, d, n);
          }
          if (a.dweights) {
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
              if (q[j] < 0) continue;
#pragma unroll
              for (int i = 0; i < 8; ++i) part[j] = __fmaf_rn((float)line[j][i], g.v[i], part[j]);
            }
          }
        }
      }
      if (!a.dweights) continue;
#pragma unroll
      for (int j = 0; j < kBatch; ++j) part[j] = lanes_sum<(TPR < kWave ? TPR : kWave)>(part[j], lane);
      if (TPR > kWave) {
        __syncthreads();  // (the sums of the batch before are read)
        if (lane == 0) {
#pragma unroll
          for (int j = 0; j < kBatch; ++j) s_part[in_block][t >> 6][j] = part[j];
        }
        __syncthreads();
        if (t < kBatch) {
          part[0] = 0.f;
          for (int w = 0; w < kWavesPerRow; ++w) part[0] += s_part[in_block][w][t];
          if (live && k0 + t < K) a.dweights[(int64_t)row * K + k0 + t] = part[0];
        }
      } else if (live && t == 0) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (k0 + j < K) a.dweights[(int64_t)row * K + k0 + j] = part[j];
      }
    }
  }
}

// Threads a row: the smallest power of two that covers it eight columns a thread, 8 to 256.  (Rows of 2048 with 256, 128
// or 64 threads and as many more rows a block: combination 65, 77, 84 us, its gradient 117, 123, 130, dropout 137, 139,
// 143: more short waves end evenly and ask for more at once than fewer long ones.)
template <typename Launch>
hipError_t by_width(int32_t n_max, int32_t d, Launch launch) {
  if (n_max == 0) return hipSuccess;
  if (d <= 64) launch(std::integral_constant<int, 8>());
  else if (d <= 128) launch(std::integral_constant<int, 16>());
  else if (d <= 256) launch(std::integral_constant<int, 32>());
  else if (d <= 512) launch(std::integral_constant<int, 64>());
  else if (d <= 1024) launch(std::integral_constant<int, 128>());
  else launch(std::integral_constant<int, 256>());
  return hipGetLastError();
}

// Blocks for n_max rows, `per` a turn; a launch holds fewer than 2^32 threads, past that blocks take more turns.
dim3 blocks_for(int32_t n_max, int per) {
  const int64_t want = ((int64_t)n_max + per - 1) / per;
  return dim3((uint32_t)(want < (1 << 22) ? want : 1 << 22));
}

template <typename T>
hipError_t dropout_rows(const DropoutArgs &a, hipStream_t st) {
  return by_width(a.n_max, a.d, [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value, per = 256 / TPR;
    hipLaunchKernelGGL((k_dropout<T, TPR>), blocks_for(a.n_max, per), dim3(256), 0, st, a);
  });
}

template <typename T>
hipError_t combine_rows(const CombineArgs &a, hipStream_t st) {
  return by_width(a.n_max, a.d, [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value, per = 256 / TPR;
    hipLaunchKernelGGL((k_combine<T, TPR>), blocks_for(a.n_max, per), dim3(256), 0, st, a);
  });
}

template <typename T>
hipError_t combine_grad_rows(const CombineArgs &a, hipStream_t st) {
  return by_width(a.n_max, a.d, [&](auto tpr) {
    constexpr int TPR = decltype(tpr)::value, per = 256 / TPR;
    hipLaunchKernelGGL((k_combine_grad<T, TPR>), blocks_for(a.n_max, per), dim3(256), 0, st, a);
  });
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs &a, int32_t dtype, hipStream_t st) {
  if (dtype == AA_BF16) return dropout_rows<__bf16>(a, st);
  if (dtype == AA_F16) return dropout_rows<_Float16>(a, st);
  return dropout_rows<float>(a, st);
}

hipError_t launch_expert_combine(const CombineArgs &a, int32_t dtype, hipStream_t st) {
  if (dtype == AA_BF16) return combine_rows<__bf16>(a, st);
  if (dtype == AA_F16) return combine_rows<_Float16>(a, st);
  return combine_rows<float>(a, st);
}

hipError_t launch_expert_combine_grad(const CombineArgs &a, int32_t dtype, hipStream_t st) {
  if (dtype == AA_BF16) return combine_grad_rows<__bf16>(a, st);
  if (dtype == AA_F16) return combine_grad_rows<_Float16>(a, st);
  return combine_grad_rows<float>(a, st);
}

}  // namespace aa

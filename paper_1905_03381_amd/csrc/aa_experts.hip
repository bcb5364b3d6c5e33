// The experts' products: matrix products over ragged groups of rows, on the matrix cores.
//
// A block owns one tile of one group's result and walks the summed dimension in steps of 64.  Both
// operands' slices go from memory to LDS directly (16 bytes a lane, no registers between) while the step before
// is multiplied.  An operand whose rows run along the summed dimension is stored as rows of 128 bytes whose 16-byte
// chunks are permuted by the row (chunk ^ row % 8), so that the 16 rows a wave reads at once lie in different
// banks; one that runs along the result (the matrices in grad_input, both operands in grad_weight) is stored as it
// comes, in 32-byte units permuted by the row, and is transposed by the LDS read itself.  The matrix operand goes
// first into the matrix instruction, so that a lane ends with four neighbouring columns of one result row.
#include "aa_experts.hpp"

namespace aa {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int kStep = 64;  // summed dimension of one LDS tile

enum Mode { kForward, kGradInput, kGradWeight };

__device__ __forceinline__ f4 mfma16(const s16x8 a, const s16x8 b, const f4 c, __bf16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}
__device__ __forceinline__ f4 mfma16(const s16x8 a, const s16x8 b, const f4 c, _Float16) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// What is read where the summed dimension has ended.
__device__ const uint4 kZeros = {0u, 0u, 0u, 0u};

__device__ __forceinline__ void load_lds16(const void *src, char *dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                   (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
}

// Permutation of the 32-byte units of a transposed operand's row r: the rows that one half of a wave
// reads at once (r % 4 and r / 8 % 2 vary) fall into different banks.
template <int ROWS>
__device__ __forceinline__ int unit_swizzle(int r) {
  return ROWS >= 128 ? (r & 3) | ((r >> 1) & 4) : ((r >> 1) & 1) | ((r >> 2) & 2);
}

// Moves one operand's slices into LDS.  ROWS: of the result that the tile covers; TR: the operand's
// rows run along the result.
template <typename T, int ROWS, int NT, bool TR, bool ALIGNED>
struct Stage {
  static constexpr int kSlots = ROWS * 8 / NT;
  static constexpr int kChunks = ROWS / 8;  // 16-byte chunks of a transposed row

  // not transposed: where each slot's row begins (chunk included)
  const T *ptr[TR ? 1 : kSlots];
  // transposed: base (column included) and stride; the rows of the next slice when they are gathered
  const T *base;
  int64_t ld;
  const int32_t *order;
  int top_k, width_left;
  int next[TR ? kSlots : 1];

  static __device__ int k_row(int it) { return (it * NT + (int)threadIdx.x) / kChunks; }
  static __device__ int chunk() {
    const int t = threadIdx.x;
    if (!TR) return (t & 7) ^ ((t >> 3) & 7);
    // (NT / kChunks is a multiple of 16: the permutation is the same for every slot of a thread)
    const int pos = t % kChunks, r = t / kChunks;
    return (((pos >> 1) ^ unit_swizzle<ROWS>(r)) << 1) | (pos & 1);
  }

  // row_of(r): first element of the tile's row r
  template <typename RowOf>
  __device__ void begin_rows(RowOf row_of) {
    static_assert(!TR, "");
    const int c = chunk() * 8;
#pragma unroll
    for (int it = 0; it < kSlots; ++it) ptr[it] = row_of((it * NT + (int)threadIdx.x) >> 3) + c;
  }

  // columns: width columns from p on belong to the operand (at least one)
  __device__ void begin_columns(const T *p, int64_t stride, int width, const int32_t *order_, int top_k_) {
    static_assert(TR, "");
    static_assert(NT / kChunks % 16 == 0, "");
    const int c = chunk() * 8;
    if (ALIGNED) {
      base = p + (c < width ? c : 0);
      width_left = 8;
    } else {
      base = p + c;
      width_left = width - c;
    }
    ld = stride;
    order = order_;
    top_k = top_k_;
  }

  // The source rows of the slice that starts at k (gathered operands), asked for a step ahead.
  __device__ void ask_rows(int k, int k_end) {
    if (order == nullptr) return;
#pragma unroll
    for (int it = 0; it < kSlots; ++it) next[it] = order[min(k + k_row(it), k_end - 1)];
  }

  // The slice of k, k + 1, .. k + 63; what lies at or past k_end is zero.
  template <bool TAIL>
  __device__ void load(char *lds, int k, int k_end) {
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
    for (int it = 0; it < kSlots; ++it) {
      const T *src;
      bool there;
      int n;  // elements of the chunk that exist (not ALIGNED)
      if (TR) {
        const int r = k + k_row(it);
        there = !TAIL || r < k_end;
        const int64_t row = order ? (int64_t)(next[it] / top_k) : (int64_t)r;
        src = base + row * ld;
        n = width_left;
      } else {
        const int c = k + chunk() * 8;
        there = !TAIL || c < k_end;
        src = ptr[it] + k;
        n = k_end - c;
      }
      if (ALIGNED) {
        if (TAIL) src = there ? src : reinterpret_cast<const T *>(&kZeros);
        load_lds16(src, lds + (it * NT + wave * kWave) * 16);
      } else {
        s16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        const short *p = reinterpret_cast<const short *>(src);
        if (there) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < n) v[j] = p[j];
        }
        *reinterpret_cast<s16x8 *>(lds + (it * NT + (int)threadIdx.x) * 16) = v;
      }
    }
  }
};

// 16 result rows from `first` on, 32 of the slice's 64 summed elements (ks = 0, 1): lane l holds row
// l % 16, elements 8 (l / 16) .. + 7.
template <int ROWS, bool TR>
__device__ __forceinline__ s16x8 fragment(const char *lds, int first, int ks, int lane) {
  if (!TR) {
    const int row = first + (lane & 15);
    return *reinterpret_cast<const s16x8 *>(lds + row * (kStep * 2) + (((ks * 4 + (lane >> 4)) ^ (lane & 7)) << 4));
  }
  // a group of 16 lanes reads 4 rows of 16 columns and gets them transposed
  const int r = ks * 32 + (lane >> 4) * 8 + ((lane & 15) >> 2);
  const int at = r * (ROWS * 2) + (((first >> 4) ^ unit_swizzle<ROWS>(r)) << 5) + (lane & 3) * 8;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds + at));
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds + at + 4 * ROWS * 2));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// The t-th tile of BM rows over all groups, and how many there are.
struct GroupTile {
  int e, first, end;
};

__device__ __forceinline__ int group_tiles(const int32_t *offsets, int n_experts, int BM) {
  const int lane = threadIdx.x & 63;
  int sum = 0;
  for (int e = lane; e < n_experts; e += kWave) sum += (offsets[e + 1] - offsets[e] + BM - 1) / BM;
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) sum += __shfl_xor(sum, off, kWave);
  return __builtin_amdgcn_readfirstlane(sum);
}

__device__ __forceinline__ GroupTile find_group_tile(const int32_t *offsets, int n_experts, int BM, int t) {
  const int lane = threadIdx.x & 63;
  GroupTile g = {-1, 0, 0};
  int before = 0;
  for (int e0 = 0; e0 < n_experts; e0 += kWave) {
    const int e = e0 + lane;
    const int lo = e < n_experts ? offsets[e] : 0, hi = e < n_experts ? offsets[e + 1] : 0;
    const int tiles = (hi - lo + BM - 1) / BM;
    const int incl = before + wave_inclusive_scan(tiles, lane);
    const unsigned long long past = __ballot(incl > t);
    if (past != 0ull) {
      const int who = __ffsll((long long)past) - 1;
      const int start = __shfl(incl - tiles, who, kWave);
      g.e = e0 + who;
      g.first = __shfl(lo, who, kWave) + (t - start) * BM;
      g.end = __shfl(hi, who, kWave);
      break;
    }
    before = __shfl(incl, kWave - 1, kWave);
  }
  g.e = __builtin_amdgcn_readfirstlane(g.e);
  g.first = __builtin_amdgcn_readfirstlane(g.first);
  g.end = __builtin_amdgcn_readfirstlane(g.end);
  return g;
}

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

__device__ __forceinline__ float sigmoid_fast(float v) { return 1.0f / (1.0f + __expf(-v)); }

template <typename T>
__device__ __forceinline__ void store4(T *p, const f4 v, int n, bool vec) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  if (vec && n >= 4) {
    T4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (T)v[i];
    *reinterpret_cast<T4 *>(p) = o;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = (T)v[i];
  }
}

template <typename T>
__device__ __forceinline__ f4 load4(const T *p, int n, bool vec) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  f4 v = {0.f, 0.f, 0.f, 0.f};
  if (vec && n >= 4) {
    const T4 o = *reinterpret_cast<const T4 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)o[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) v[i] = (float)p[i];
  }
  return v;
}

// Four neighbouring results of place q, column j on (j < width): through the activation and out.
template <typename T, int MODE, int ACT>
__device__ __forceinline__ void finish(const ProductArgs &a, int64_t q, int j, const f4 v, const f4 up) {
  if (MODE == kForward) {
    const int n = a.d_out - j;
    T *o = static_cast<T *>(a.out) + q * a.ldo + j;
    f4 r = v;
    if (ACT == AA_ACT_RELU) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = v[i] < 0.f ? 0.f : v[i];
    }
    if (ACT == AA_ACT_GATED) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = v[i] * sigmoid_fast(v[i]) * up[i];
      if (a.pre) {
        T *h = static_cast<T *>(a.pre) + q * a.ldpre + j;
        store4(h, v, n, a.out_vec);
        store4(h + a.d_out, up, n, a.out_vec);
      }
    }
    store4(o, r, n, a.out_vec);
  } else {
    const int n = a.d_in - j;
    T *o = static_cast<T *>(a.out) + q * a.ldo + j;
    if (ACT == AA_ACT_NONE) {
      store4(o, v, n, a.out_vec);
    } else if (ACT == AA_ACT_RELU) {
      const f4 s = load4(static_cast<const T *>(a.saved) + q * a.lds + j, n, a.out_vec);
      f4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i) r[i] = s[i] > 0.f ? v[i] : 0.f;
      store4(o, r, n, a.out_vec);
    } else {
      const T *s = static_cast<const T *>(a.saved) + q * a.lds + j;
      const f4 g = load4(s, n, a.out_vec), u = load4(s + a.d_in, n, a.out_vec);
      f4 dg, du;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float z = sigmoid_fast(g[i]);
        dg[i] = v[i] * u[i] * (z + g[i] * z * (1.0f - z));
        du[i] = v[i] * g[i] * z;
      }
      store4(o, dg, n, a.out_vec);
      store4(o + a.d_in, du, n, a.out_vec);
    }
  }
}

// A block of WI x WJ waves, each FI x FJ fragments of 16 x 16 results: BM = 16 FI WI result rows
// (places of a group; grad_weight: rows of dw), BN = 16 FJ WJ columns.  With AA_ACT_GATED half of a wave's
// columns are the gate's, half the same columns of up.
template <typename T, int MODE, int ACT, int WI, int WJ, int FI, int FJ, bool ALIGNED>
__global__ __launch_bounds__(WI *WJ *kWave) void k_product(const ProductArgs a) {
  constexpr int NT = WI * WJ * kWave, BM = 16 * FI * WI, BN = 16 * FJ * WJ;
  constexpr bool TRP = MODE == kGradWeight, TRQ = MODE != kForward;
  constexpr bool GATED = MODE == kForward && ACT == AA_ACT_GATED;
  constexpr int OUT_N = GATED ? BN / 2 : BN;
  constexpr int kBytesP = BM * kStep * 2, kBytesQ = BN * kStep * 2;
  __shared__ __attribute__((aligned(256))) char smem[2][kBytesP + kBytesQ];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wi = wave / WJ, wj = wave % WJ;

  // which tile: each XCD (blocks go round the eight of them) takes a run of neighbouring tiles
  const int columns = MODE == kForward ? a.d_out : a.d_in;
  const int nj = (columns + OUT_N - 1) / OUT_N;
  int e, i0, i_end, j0, k, k_end;
  if (MODE == kGradWeight) {
    const int ni = (a.d_out + BM - 1) / BM;
    const int total = a.n_experts * ni * nj, chunk = (total + 7) / 8;
    const int t = ((int)blockIdx.x & 7) * chunk + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= chunk || t >= total) return;
    e = t / (ni * nj);
    i0 = (t % (ni * nj)) / nj * BM;
    j0 = t % nj * OUT_N;
    i_end = a.d_out;
    k = a.offsets[e];
    k_end = a.offsets[e + 1];
  } else {
    const int mi = group_tiles(a.offsets, a.n_experts, BM);
    const int total = mi * nj, chunk = (total + 7) / 8;
    const int t = ((int)blockIdx.x & 7) * chunk + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= chunk || t >= total) return;
    // runs of four row tiles by all column tiles: what an XCD works on at once shares rows and matrices
    constexpr int kRun = 4;
    const int run = t / (kRun * nj), in_run = t % (kRun * nj);
    const int rows_of_run = min(kRun, mi - run * kRun);
    const GroupTile g = find_group_tile(a.offsets, a.n_experts, BM, run * kRun + in_run % rows_of_run);
    e = g.e;
    i0 = g.first;
    i_end = g.end;
    j0 = in_run / rows_of_run * OUT_N;
    k = 0;
    k_end = MODE == kForward ? a.d_in : a.d_out;
  }

  Stage<T, BM, NT, TRP, ALIGNED> P;
  Stage<T, BN, NT, TRQ, ALIGNED> Q;
  if constexpr (MODE == kGradWeight) {
    P.begin_columns(static_cast<const T *>(a.rows) + i0, a.ld_rows, a.d_out - i0, nullptr, 1);
    Q.begin_columns(static_cast<const T *>(a.mat) + j0, a.ld_mat, a.d_in - j0, a.order, a.top_k);
  } else {
    const T *rows = static_cast<const T *>(a.rows);
    P.begin_rows([&](int r) {
      const int q = min(i0 + r, i_end - 1);
      const int64_t row = MODE == kForward && a.order ? a.order[q] / a.top_k : q;
      return rows + row * a.ld_rows;
    });
    const T *w = static_cast<const T *>(a.mat) + (size_t)e * a.d_out * a.d_in * (GATED ? 2 : 1);
    if constexpr (MODE == kForward) {
      Q.begin_rows([&](int r) {
        int n;
        if (GATED) {  // a wave's first FJ / 2 fragments are gate columns, the others the same of up
          constexpr int half = FJ * 8;
          const int c = r % (2 * half);
          n = min(j0 + r / (2 * half) * half + c % half, a.d_out - 1) + (c >= half ? a.d_out : 0);
        } else {
          n = min(j0 + r, a.d_out - 1);
        }
        return w + (size_t)n * a.d_in;
      });
    } else {
      Q.begin_columns(w + j0, a.d_in, a.d_in - j0, nullptr, 1);
    }
  }

  auto load = [&](int buf, int at) {
    if (at + kStep <= k_end) {
      P.template load<false>(smem[buf], at, k_end);
      Q.template load<false>(smem[buf] + kBytesP, at, k_end);
    } else {
      P.template load<true>(smem[buf], at, k_end);
      Q.template load<true>(smem[buf] + kBytesP, at, k_end);
    }
    if constexpr (TRQ) Q.ask_rows(at + kStep, k_end);
  };

  f4 acc[FI][FJ];
#pragma unroll
  for (int i = 0; i < FI; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

  if (k < k_end) {
    if constexpr (TRQ) Q.ask_rows(k, k_end);
    load(0, k);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int buf = 0;
    for (; k < k_end; k += kStep) {
      if (k + kStep < k_end) load(buf ^ 1, k + kStep);
      const char *p = smem[buf], *q = smem[buf] + kBytesP;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        s16x8 fp[FI], fq[FJ];
#pragma unroll
        for (int i = 0; i < FI; ++i) fp[i] = fragment<BM, TRP>(p, wi * FI * 16 + i * 16, ks, lane);
#pragma unroll
        for (int j = 0; j < FJ; ++j) fq[j] = fragment<BN, TRQ>(q, wj * FJ * 16 + j * 16, ks, lane);
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
          for (int j = 0; j < FJ; ++j) acc[i][j] = mfma16(fq[j], fp[i], acc[i][j], T());
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      buf ^= 1;
    }
  }

  const int ti = wi * FI * 16 + (lane & 15), tj = (lane >> 4) * 4;
  if constexpr (MODE == kGradWeight) {
    const size_t base = (size_t)e * a.d_out * a.d_in;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const int n = i0 + ti + i * 16;
      if (n >= i_end) continue;
#pragma unroll
      for (int j = 0; j < FJ; ++j) {
        const int c = j0 + wj * FJ * 16 + j * 16 + tj;
        if (c >= a.d_in) continue;
        const size_t at = base + (size_t)n * a.d_in + c;
        f4 v = acc[i][j];
        if (a.out_f32) {
          float *o = static_cast<float *>(a.out) + at;
          if (a.accumulate) v += load4(o, a.d_in - c, a.out_vec);
          store4(o, v, a.d_in - c, a.out_vec);
        } else {
          T *o = static_cast<T *>(a.out) + at;
          if (a.accumulate) v += load4(o, a.d_in - c, a.out_vec);
          store4(o, v, a.d_in - c, a.out_vec);
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const int q = i0 + ti + i * 16;
      if (q >= i_end) continue;
      constexpr int kOut = GATED ? FJ / 2 : FJ;
#pragma unroll
      for (int j = 0; j < kOut; ++j) {
        const int c = j0 + wj * kOut * 16 + j * 16 + tj;
        if (c < columns) finish<T, MODE, ACT>(a, q, c, acc[i][j], acc[i][GATED ? j + kOut : j]);
      }
    }
  }
}

template <typename T, int MODE, int ACT, int WI, int WJ, int FI, int FJ, bool ALIGNED>
hipError_t launch_tiles(const ProductArgs &a, hipStream_t st) {
  constexpr int BM = 16 * FI * WI, BN = 16 * FJ * WJ;
  constexpr int OUT_N = MODE == kForward && ACT == AA_ACT_GATED ? BN / 2 : BN;
  const int64_t nj = ((MODE == kForward ? a.d_out : a.d_in) + OUT_N - 1) / OUT_N;
  int64_t ni;
  if (MODE == kGradWeight)
    ni = (int64_t)a.n_experts * ((a.d_out + BM - 1) / BM);
  else  // every group may end inside a tile; there are no more groups with rows than rows
    ni = a.rows_max / BM + (a.rows_max < a.n_experts ? a.rows_max : a.n_experts);
  const int64_t blocks = (ni * nj + 7) / 8 * 8;
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL((k_product<T, MODE, ACT, WI, WJ, FI, FJ, ALIGNED>), dim3((uint32_t)blocks), dim3(WI * WJ * kWave), 0,
                     st, a);
  return hipGetLastError();
}

template <typename T, int MODE, int ACT>
hipError_t launch_product(const ProductArgs &a, hipStream_t st) {
  if (!a.aligned) return launch_tiles<T, MODE, ACT, 2, 2, 4, 4, false>(a, st);
  return launch_tiles<T, MODE, ACT, 2, 4, 8, 4, true>(a, st);
}

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

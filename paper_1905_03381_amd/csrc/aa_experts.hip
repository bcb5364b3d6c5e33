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

#include "aa_route.hpp"

#include <type_traits>

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

// A value the compiler shall not keep derived values of over the turns of a loop (it would run out of registers): for
// all it knows this one changes with k.
__device__ __forceinline__ uint32_t fresh(uint32_t v, int k) {
  asm("" : "+v"(v) : "s"(k));
  return v;
}
__device__ __forceinline__ int fresh_thread(int k) { return (int)fresh(threadIdx.x, k); }

// Permutation of the 32-byte units of a transposed operand's row r: the rows that one half of a wave
// reads at once (r % 4 and r / 8 % 2 vary) fall into different banks.
template <int ROWS>
__device__ __forceinline__ int unit_swizzle(int r) {
  return ROWS >= 128 ? (r & 3) | ((r >> 1) & 4) : ((r >> 1) & 1) | ((r >> 2) & 2);
}

// Permutation of the 16-byte chunks of row r (kStep elements) of an operand that is not transposed: the rows that
// neighbouring lanes read fall into different banks.
__device__ __forceinline__ int row_swizzle(int r) { return r & 7; }

// Moves one operand's slices into LDS.  ROWS: of the result that the tile covers; TR: the operand's
// rows run along the result.  Addresses are a base that is the same for the whole block and offsets of 32 bits a lane
// (registers are what the big tiles are short of); ALIGNED: 16-byte chunks exist whole or not at all and lie on 16-byte boundaries.
template <typename T, int ROWS, int NT, bool TR, bool GATHER, bool ALIGNED>
struct Stage {
  static constexpr int kSlots = ROWS * kStep / 8 / NT;
  static constexpr int kChunks = (TR ? ROWS : kStep) / 8;  // 16-byte chunks of a stored row
  static constexpr int kRowsASlot = NT / kChunks;

  const T *base;
  int64_t ld;
  // not transposed: where each slot's row begins, in units of 16 bytes (not ALIGNED: the row's number)
  uint32_t row_at[TR ? 1 : kSlots];
  // transposed: a thread's place in a slot's rows, in bytes (slots of odd number may permute differently), and the
  // columns left from there on; the rows of the next slice when they are gathered
  uint32_t at[2];
  int left[2];
  const int32_t *order;
  int top_k, next[TR && GATHER ? kSlots : 1];

  static __device__ int k_row(int it, int t) { return it * kRowsASlot + t / kChunks; }
  static __device__ int chunk(int it, int t) {
    if (!TR) return (t % kChunks) ^ row_swizzle(t / kChunks);
    // (kRowsASlot is a multiple of 8: bits 0 to 2 of the row are the same for every slot, bit 3 for every other)
    const int pos = t % kChunks;
    return (((pos >> 1) ^ unit_swizzle<ROWS>(k_row(it & 1, t))) << 1) | (pos & 1);
  }

  // row_of(r): number of the tile's row r among rows of `stride` elements from p on
  template <typename RowOf>
  __device__ void begin_rows(const T *p, int64_t stride, int t, RowOf row_of) {
    static_assert(!TR, "");
    base = p;
    ld = stride;
#pragma unroll
    for (int it = 0; it < kSlots; ++it) {
      const uint32_t row = row_of((it * NT + t) / kChunks);
      row_at[it] = ALIGNED ? (uint32_t)((uint64_t)row * (uint64_t)(ld / 8)) + (uint32_t)chunk(0, t) : row;
    }
  }

  // columns: width columns from p on belong to the operand (at least one)
  __device__ void begin_columns(const T *p, int64_t stride, int width, int t, const int32_t *order_, int top_k_) {
    static_assert(TR && kRowsASlot % 8 == 0, "");
    base = p;
    ld = stride;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = chunk(h, t) * 8, from = ALIGNED && c >= width ? 0 : c;
      at[h] = (uint32_t)(from + (GATHER ? 0 : t / kChunks * (int)ld)) * (uint32_t)sizeof(T);
      left[h] = width - c;
    }
    order = order_;
    top_k = top_k_;
  }

  // The source rows of the slice that starts at k (gathered operands), asked for a step ahead.
  __device__ void ask_rows(int k, int k_end) {
    if constexpr (TR && GATHER) {
      const int t = fresh_thread(k);
#pragma unroll
      for (int it = 0; it < kSlots; ++it) next[it] = order[min(k + k_row(it, t), k_end - 1)];
    }
  }

  // First element of a slot's chunk in the slice that starts at k.
  __device__ const T *source(int it, int k, int t) const {
    const char *b;
    if constexpr (!TR) {
      b = reinterpret_cast<const char *>(base + k);
      if constexpr (ALIGNED) return reinterpret_cast<const T *>(b + (uint64_t)fresh(row_at[it], k) * 16);
      else return base + (int64_t)row_at[it] * ld + k + chunk(0, t) * 8;
    } else if constexpr (GATHER) {
      b = reinterpret_cast<const char *>(base + (int64_t)(next[it] / top_k) * ld);
      return reinterpret_cast<const T *>(b + fresh(at[it & 1], k));
    } else {
      b = reinterpret_cast<const char *>(base + (int64_t)(k + it * kRowsASlot) * ld);
      return reinterpret_cast<const T *>(b + fresh(at[it & 1], k));
    }
  }

  // The slice of k, k + 1, .. k + kStep - 1; what lies at or past k_end is zero.
  template <bool TAIL>
  __device__ void load(char *lds, int k, int k_end) {
    const int t = fresh_thread(k), wave = __builtin_amdgcn_readfirstlane(t >> 6);
#pragma unroll
    for (int it = 0; it < kSlots; ++it) {
      const T *src = source(it, k, t);
      const int n = TR ? left[it & 1] : k_end - (k + chunk(0, t) * 8);  // elements of the chunk that exist (not ALIGNED)
      const bool there = !TAIL || (TR ? k + k_row(it, t) : k + chunk(0, t) * 8) < k_end;
      if (ALIGNED) {
        if (TAIL) src = there ? src : reinterpret_cast<const T *>(&kZeros);
        load_lds16(src, lds + (it * NT + wave * kWave) * 16);
      } else {
        s16x8 v;
        const short *p = reinterpret_cast<const short *>(src), *zero = reinterpret_cast<const short *>(&kZeros);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = *(there && j < n ? p + j : zero);  // (no branch: all are asked for at once)
        *reinterpret_cast<s16x8 *>(lds + (it * NT + t) * 16) = v;
      }
    }
  }
};

// All that this wave has asked for is there, but for the newest N transfers, and every wave of the block
// has come this far.
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Fragments of 16 result rows and 32 summed elements (the ks-th 32 of a slice): lane l holds row l % 16, elements
// 8 (l / 16) .. + 7.  fragment_at: a lane's place for the fragments from result row `first` (a multiple of 64) on;
// fragment: the i-th of them.
template <int ROWS, bool TR>
__device__ __forceinline__ uint32_t fragment_at(int first, int lane) {
  if (!TR) return (first + (lane & 15)) * (kStep * 2) + (((lane >> 4) ^ row_swizzle(lane & 15)) << 4);
  // a group of 16 lanes reads 4 rows of 16 columns and gets them transposed
  const int r = (lane >> 4) * 8 + ((lane & 15) >> 2);
  return r * (ROWS * 2) + (((first >> 4) ^ unit_swizzle<ROWS>(r)) << 5) + (lane & 3) * 8;
}

template <int ROWS, bool TR>
__device__ __forceinline__ s16x8 fragment(const char *lds, uint32_t at, int i, int ks) {
  if (!TR) return *reinterpret_cast<const s16x8 *>(lds + (at ^ (ks * 64)) + i * (16 * kStep * 2));
  const char *p = lds + (at ^ (i << 5)) + ks * (32 * ROWS * 2);
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)p);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + 4 * ROWS * 2));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Asks the scheduler to spread READS LDS reads and TRANSFERS transfers to LDS evenly over ALL matrix instructions: a
// burst of either would hold the wave at its issue while the matrix unit waits.
template <int READS, int TRANSFERS, int ALL, int M = 0>
__device__ __forceinline__ void interleave() {
  if constexpr (M < ALL) {
    constexpr int kRead = (M + 1) * READS / ALL - M * READS / ALL;
    constexpr int kMove = (M + 1) * TRANSFERS / ALL - M * TRANSFERS / ALL;
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // matrix instruction
    if constexpr (kRead > 0) __builtin_amdgcn_sched_group_barrier(0x100, kRead, 0);
    if constexpr (kMove > 0) __builtin_amdgcn_sched_group_barrier(0x010, kMove, 0);
    interleave<READS, TRANSFERS, ALL, M + 1>();
  }
}

// One tile of the result: its group, rows, first column, and the summed range.
struct Tile {
  int e, i0, i_end, j0, k0, k_end;
};

// before[e]: tiles of BM rows in the groups before e (e = 0 .. n_experts), by the first wave.
__device__ __forceinline__ void count_group_tiles(const int32_t *offsets, int n_experts, int BM, int *before) {
  const int lane = threadIdx.x & 63;
  if (threadIdx.x >= kWave) return;
  int sum = 0;
  for (int e0 = 0; e0 < n_experts; e0 += kWave) {
    const int e = e0 + lane;
    const int tiles = e < n_experts ? (offsets[e + 1] - offsets[e] + BM - 1) / BM : 0;
    const int incl = wave_inclusive_scan(tiles, lane);
    if (e < n_experts) before[e + 1] = sum + incl;
    sum += __shfl(incl, kWave - 1, kWave);
  }
  if (lane == 0) before[0] = 0;
}

// The group that holds row tile t.
__device__ __forceinline__ int group_of_tile(const int *before, int n_experts, int t) {
  const int lane = threadIdx.x & 63;
  for (int e0 = 0; e0 < n_experts; e0 += kWave) {
    const unsigned long long past = __ballot(e0 + lane < n_experts && before[min(e0 + lane, n_experts - 1) + 1] > t);
    if (past != 0ull) return __builtin_amdgcn_readfirstlane(e0 + __ffsll((long long)past) - 1);
  }
  return n_experts - 1;  // (not reached: t is below before[n_experts])
}

__device__ __forceinline__ float sigmoid_fast(float v) { return 1.0f / (1.0f + __expf(-v)); }

// Eight neighbouring results of a lane; the first n of them exist, vec: and can be moved 16 bytes at a time.
struct Eight {
  float v[8];
};

template <typename T>
__device__ __forceinline__ void store8(T *p, const Eight &x, int n, bool vec) {
  typedef T Line __attribute__((ext_vector_type(16 / sizeof(T))));
  constexpr int kPer = 16 / sizeof(T);
  if (vec && n >= 8) {
#pragma unroll
    for (int h = 0; h < 8 / kPer; ++h) {
      Line o;
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[i] = (T)x.v[h * kPer + i];
      reinterpret_cast<Line *>(p)[h] = o;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)x.v[i];
  }
}

template <typename T>
__device__ __forceinline__ Eight load8(const T *p, int n, bool vec) {
  typedef T Line __attribute__((ext_vector_type(16 / sizeof(T))));
  constexpr int kPer = 16 / sizeof(T);
  Eight x;
  if (vec && n >= 8) {
#pragma unroll
    for (int h = 0; h < 8 / kPer; ++h) {
      const Line o = reinterpret_cast<const Line *>(p)[h];
#pragma unroll
      for (int i = 0; i < kPer; ++i) x.v[h * kPer + i] = (float)o[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = i < n ? (float)p[i] : 0.f;
  }
  return x;
}

// What lane groups 0 .. 3 of 16 hold of fragments a and b (columns 4 g .. 4 g + 3 of each): group g gets columns
// 8 (g / 2) .. + 7 of fragment g % 2.
__device__ __forceinline__ Eight eight_columns(const f4 a, const f4 b) {
  Eight x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[i]), __float_as_uint(b[i]), false, false);
    x.v[i] = __uint_as_float(both[0]);
    x.v[4 + i] = __uint_as_float(both[1]);
  }
  return x;
}

// Eight neighbouring results of place q, column j on (j < width): through the activation and out.
template <typename T, int MODE, int ACT>
__device__ __forceinline__ void finish(const ProductArgs &a, int64_t q, int j, const Eight &v, const Eight &up) {
  T *o = static_cast<T *>(a.out) + q * a.ldo + j;
  const int n = (MODE == kForward ? a.d_out : a.d_in) - j;
  const bool vec = a.out_vec;
  Eight r = v;
  if (MODE == kForward) {
    if (ACT == AA_ACT_RELU) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r.v[i] = v.v[i] < 0.f ? 0.f : v.v[i];
    }
    if (ACT == AA_ACT_GATED) {
#pragma unroll
      for (int i = 0; i < 8; ++i) r.v[i] = v.v[i] * sigmoid_fast(v.v[i]) * up.v[i];
      if (a.pre) {
        T *h = static_cast<T *>(a.pre) + q * a.ldpre + j;
        store8(h, v, n, vec);
        store8(h + a.d_out, up, n, vec);
      }
    }
  } else if (ACT == AA_ACT_RELU) {
    const Eight s = load8(static_cast<const T *>(a.saved) + q * a.lds + j, n, vec);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = s.v[i] > 0.f ? v.v[i] : 0.f;
  } else if (ACT == AA_ACT_GATED) {
    const T *s = static_cast<const T *>(a.saved) + q * a.lds + j;
    const Eight g = load8(s, n, vec), u = load8(s + a.d_in, n, vec);
    Eight du;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float z = sigmoid_fast(g.v[i]);
      r.v[i] = v.v[i] * u.v[i] * (z + g.v[i] * z * (1.0f - z));
      du.v[i] = v.v[i] * g.v[i] * z;
    }
    store8(o + a.d_in, du, n, vec);
  }
  store8(o, r, n, vec);
}

template <typename T>
__device__ __forceinline__ void finish_weight(T *o, const Eight &v, int n, bool accumulate, bool vec) {
  Eight r = v;
  if (accumulate) {
    const Eight old = load8(o, n, vec);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] += old.v[i];
  }
  store8(o, r, n, vec);
}

// A block of WI x WJ waves, each FI x FJ fragments of 16 x 16 results: BM = 16 FI WI result rows
// (places of a group; grad_weight: rows of dw), BN = 16 FJ WJ columns.  With AA_ACT_GATED half of a wave's
// columns are the gate's, half the same columns of up.
template <typename T, int MODE, int ACT, int WI, int WJ, int FI, int FJ, bool GATHER, bool ALIGNED>
__global__ __launch_bounds__(WI *WJ *kWave, 2) void k_product(const ProductArgs a) {
  constexpr int NT = WI * WJ * kWave, BM = 16 * FI * WI, BN = 16 * FJ * WJ;
  constexpr bool TRP = MODE == kGradWeight, TRQ = MODE != kForward;
  constexpr bool GATED = MODE == kForward && ACT == AA_ACT_GATED;
  constexpr int OUT_N = GATED ? BN / 2 : BN, kOut = GATED ? FJ / 2 : FJ;
  constexpr int kBytesP = BM * kStep * 2, kBytesQ = BN * kStep * 2;
  constexpr int kBuffer = kBytesP + kBytesQ;
  __shared__ __attribute__((aligned(256))) char smem[2 * kBuffer];
  __shared__ int before[MODE == kGradWeight ? 1 : kMaxExperts + 1];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  const int columns = MODE == kForward ? a.d_out : a.d_in;
  const int nj = (columns + OUT_N - 1) / OUT_N;

  // Tiles: each XCD (blocks go round the eight of them) takes a run of neighbouring ones, its blocks in turns.
  int ni;
  if (MODE == kGradWeight) {
    ni = a.n_experts * ((a.d_out + BM - 1) / BM);
  } else {
    count_group_tiles(a.offsets, a.n_experts, BM, before);
    __syncthreads();
    ni = __builtin_amdgcn_readfirstlane(before[a.n_experts]);
  }
  const int64_t total = (int64_t)ni * nj, chunk = (total + 7) / 8;
  const int64_t t_end = min(total, ((int)(blockIdx.x & 7) + 1) * chunk);
  int64_t t = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
  if (t >= t_end) return;
  auto find = [&](int64_t at) __attribute__((always_inline)) {
    // runs of four row tiles by all column tiles: what an XCD works on at once shares rows and matrices
    constexpr int kRun = 4;
    const int run = (int)(at / (kRun * nj)), in_run = (int)(at % (kRun * nj));
    const int rows_of_run = min(kRun, ni - run * kRun);
    const int it = run * kRun + in_run % rows_of_run;
    Tile g;
    g.j0 = in_run / rows_of_run * OUT_N;
    if (MODE == kGradWeight) {
      const int per = (a.d_out + BM - 1) / BM;
      g.e = it / per;
      g.i0 = it % per * BM;
      g.i_end = a.d_out;
      g.k0 = __builtin_amdgcn_readfirstlane(a.offsets[g.e]);
      g.k_end = __builtin_amdgcn_readfirstlane(a.offsets[g.e + 1]);
    } else {
      g.e = group_of_tile(before, a.n_experts, it);
      g.i0 = __builtin_amdgcn_readfirstlane(a.offsets[g.e] + (it - before[g.e]) * BM);
      g.i_end = __builtin_amdgcn_readfirstlane(a.offsets[g.e + 1]);
      g.k0 = 0;
      g.k_end = MODE == kForward ? a.d_in : a.d_out;
    }
    return g;
  };

  Stage<T, BM, NT, TRP, false, ALIGNED> P;
  Stage<T, BN, NT, TRQ, GATHER && MODE == kGradWeight, ALIGNED> Q;
  constexpr int kReads = FI * (TRP ? 2 : 1) + FJ * (TRQ ? 2 : 1);
  constexpr int kLoads = decltype(P)::kSlots + decltype(Q)::kSlots;
  auto load = [&](char *to, int at, int k_end) __attribute__((always_inline)) {
    if (at + kStep <= k_end) {
      P.template load<false>(to, at, k_end);
      Q.template load<false>(to + kBytesP, at, k_end);
    } else {
      P.template load<true>(to, at, k_end);
      Q.template load<true>(to + kBytesP, at, k_end);
    }
    if constexpr (TRQ) Q.ask_rows(at + kStep, k_end);
  };
  // Takes up a tile: its addresses, and its first two slices on their way.
  auto begin = [&](const Tile &g) __attribute__((always_inline)) {
    const int tid = fresh_thread((int)t);
    if constexpr (MODE == kGradWeight) {
      P.begin_columns(static_cast<const T *>(a.rows) + g.i0, a.ld_rows, a.d_out - g.i0, tid, nullptr, 1);
      Q.begin_columns(static_cast<const T *>(a.mat) + g.j0, a.ld_mat, a.d_in - g.j0, tid, a.order, a.top_k);
    } else {
      P.begin_rows(static_cast<const T *>(a.rows), a.ld_rows, tid, [&](int r) {
        const int q = min(g.i0 + r, g.i_end - 1);
        return (uint32_t)(GATHER ? a.order[q] / a.top_k : q);
      });
      const T *w = static_cast<const T *>(a.mat) + (size_t)g.e * a.d_out * a.d_in * (GATED ? 2 : 1);
      if constexpr (MODE == kForward) {
        Q.begin_rows(w, a.d_in, tid, [&](int r) {
          // (GATED: a wave's first FJ / 2 fragments are gate columns, the others the same of up)
          const int c = r % (16 * FJ);
          return (uint32_t)(min(g.j0 + r / (16 * FJ) * (16 * kOut) + c % (16 * kOut), a.d_out - 1) +
                            (c >= 16 * kOut ? a.d_out : 0));
        });
      } else {
        Q.begin_columns(w + g.j0, a.d_in, a.d_in - g.j0, tid, nullptr, 1);
      }
    }
    if (g.k0 < g.k_end) {
      if constexpr (TRQ) Q.ask_rows(g.k0, g.k_end);
      load(smem, g.k0, g.k_end);
      if (g.k0 + kStep < g.k_end) load(smem + kBuffer, g.k0 + kStep, g.k_end);
    }
  };

  Tile g = find(t);
  begin(g);
  while (true) {
    f4 acc[FI][FJ];
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    // Two buffers.  While 32 summed elements are multiplied the next 32 are read, a fragment of the rows into the place
    // of one that has been used.  Early in the second half of a step everybody has read its buffer and the next
    // one has arrived: the slice two steps on goes into the free buffer during the rest.
    if (g.k0 < g.k_end) {
      const int k_end = g.k_end;
      int k = g.k0;
      if (ALIGNED && k + kStep < k_end) wait_and_meet<kLoads>();
      else wait_and_meet<0>();
      if (g.i0 + wi * FI * 16 < g.i_end && g.j0 + wj * kOut * 16 < columns) {
        s16x8 fp[2][FI], fq[2][FJ];
        const int in_wave = fresh_thread((int)t) & 63;
        const uint32_t p_at = fragment_at<BM, TRP>(wi * FI * 16, in_wave);
        const uint32_t q_at = fragment_at<BN, TRQ>(wj * FJ * 16, in_wave);
        auto read = [&](int to, const char *lds, int ks) {
          const uint32_t pa = fresh(p_at, k), qa = fresh(q_at, k);
#pragma unroll
          for (int j = 0; j < FJ; ++j) fq[to][j] = fragment<BN, TRQ>(lds + kBytesP, qa, j, ks);
#pragma unroll
          for (int i = 0; i < FI; ++i) fp[to][i] = fragment<BM, TRP>(lds, pa, i, ks);
        };
        auto multiply = [&](int ks, int from, int to) {
#pragma unroll
          for (int i = from; i < to; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[i][j] = mfma16(fq[ks][j], fp[ks][i], acc[i][j], T());
        };
        constexpr int kAhead = FI / 4;  // rows of the second half before the meeting
        // (reads past the last step: what lies in LDS there, not used)
        auto step = [&](char *__restrict here, const char *__restrict other, auto whole) __attribute__((always_inline)) {
          read(1, here, 1);
          multiply(0, 0, FI);
          interleave<kReads, 0, FI * FJ>();
          multiply(1, 0, kAhead);
          wait_and_meet<0>();
          if constexpr (decltype(whole)::value) {  // the slice two steps on is there and is a whole one
            read(0, other, 0);
            P.template load<false>(here, k + 2 * kStep, k_end);
            Q.template load<false>(here + kBytesP, k + 2 * kStep, k_end);
            if constexpr (TRQ) Q.ask_rows(k + 3 * kStep, k_end);
            multiply(1, kAhead, FI);
            interleave<kReads, kLoads, (FI - kAhead) * FJ>();
          } else {
            if (k + 2 * kStep < k_end) load(here, k + 2 * kStep, k_end);
            read(0, other, 0);
            multiply(1, kAhead, FI);
            interleave<kReads, 0, (FI - kAhead) * FJ>();
          }
          k += kStep;
        };
        read(0, smem, 0);
        int buf = 0;
        if (ALIGNED) {
          for (; k + 3 * kStep <= k_end; buf ^= 1)
            step(smem + buf * kBuffer, smem + (buf ^ 1) * kBuffer, std::true_type());
        }
        for (; k < k_end; buf ^= 1) step(smem + buf * kBuffer, smem + (buf ^ 1) * kBuffer, std::false_type());
      } else {  // a wave whose part of the tile lies outside the result only moves data
        for (int odd = 0; k < k_end; k += kStep, odd ^= 1) {
          wait_and_meet<0>();
          if (k + 2 * kStep < k_end) load(smem + odd * kBuffer, k + 2 * kStep, k_end);
        }
      }
    }

    // The next tile's first slices are on their way while this one's results are written.  (After the last meeting
    // nobody reads what LDS holds.)
    const Tile done = g;
    t += gridDim.x >> 3;
    if (t < t_end) {
      g = find(t);
      begin(g);
    }
    // A lane has four neighbouring columns in each fragment; after an exchange with the lane 16 away it has eight in
    // every second one.
    const int in_wave = fresh_thread((int)t) & 63, group = in_wave >> 4;
    const int ti = done.i0 + wi * FI * 16 + (in_wave & 15);
    const int tj = done.j0 + wj * kOut * 16 + (group & 1) * 16 + (group >> 1) * 8;
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const int r = ti + i * 16;
#pragma unroll
      for (int p = 0; p < kOut / 2; ++p) {
        const int c = tj + p * 32;
        Eight v = eight_columns(acc[i][2 * p], acc[i][2 * p + 1]), up;
        if (GATED) up = eight_columns(acc[i][FJ / 2 + 2 * p], acc[i][FJ / 2 + 2 * p + 1]);
        if (r < done.i_end && c < columns) {
          if constexpr (MODE == kGradWeight) {
            const size_t at = ((size_t)done.e * a.d_out + r) * a.d_in + c;
            if (a.out_f32) finish_weight(static_cast<float *>(a.out) + at, v, a.d_in - c, a.accumulate, a.out_vec);
            else finish_weight(static_cast<T *>(a.out) + at, v, a.d_in - c, a.accumulate, a.out_vec);
          } else {
            finish<T, MODE, ACT>(a, r, c, v, up);
          }
        }
      }
    }
    if (t >= t_end) break;
  }
}

template <typename T, int MODE, int ACT, int WI, int WJ, int FI, int FJ, bool GATHER, bool ALIGNED>
hipError_t launch_tiles(const ProductArgs &a, hipStream_t st) {
  constexpr int BM = 16 * FI * WI, BN = 16 * FJ * WJ;
  constexpr int OUT_N = MODE == kForward && ACT == AA_ACT_GATED ? BN / 2 : BN;
  const int64_t nj = ((MODE == kForward ? a.d_out : a.d_in) + OUT_N - 1) / OUT_N;
  int64_t ni;
  if (MODE == kGradWeight)
    ni = (int64_t)a.n_experts * ((a.d_out + BM - 1) / BM);
  else  // every group may end inside a tile; there are no more groups with rows than rows
    ni = a.rows_max / BM + (a.rows_max < a.n_experts ? a.rows_max : a.n_experts);
  // blocks that fit the chip at once walk the tiles
  constexpr int64_t kFit = 256 * (WI * WJ <= 4 ? 2 : 1);
  const int64_t blocks = min(kFit, (ni * nj + 7) / 8 * 8);
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL((k_product<T, MODE, ACT, WI, WJ, FI, FJ, GATHER, ALIGNED>), dim3((uint32_t)blocks), dim3(WI * WJ * kWave), 0,
                     st, a);
  return hipGetLastError();
}

template <typename T, int MODE, int ACT>
hipError_t launch_product(const ProductArgs &a, hipStream_t st) {
  // (grad_input's rows are never gathered)
  if (MODE != kGradInput && a.order) {
    if (!a.aligned) return launch_tiles<T, MODE, ACT, 2, 2, 4, 4, true, false>(a, st);
    return launch_tiles<T, MODE, ACT, 2, 4, 8, 4, true, true>(a, st);
  }
  if (!a.aligned) return launch_tiles<T, MODE, ACT, 2, 2, 4, 4, false, false>(a, st);
  return launch_tiles<T, MODE, ACT, 2, 4, 8, 4, false, true>(a, st);
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

// The experts' products: matrix products over ragged groups of rows, on the matrix cores.
//
// out = x w^T, dx = dout w and dw = dout^T x for each group of rows; sums in fp32, one rounding at the end.  Bound by the
// matrix units where a group's rows fill tiles, by reading the matrices where they do not.
//
// A block takes tiles of the result and walks the summed dimension in steps of 64.  Both
// operands' slices go from memory to LDS directly (16 bytes a lane, no registers between) while the step before
// is multiplied.  An operand whose rows run along the summed dimension is stored as rows of 128 bytes whose 16-byte
// chunks are permuted by the row (chunk ^ row % 8), so that the 16 rows a wave reads at once lie in different
// banks; one that runs along the result (the matrices in grad_input, both operands in grad_weight) is stored as it
// comes, in 32-byte units permuted by the row, and is transposed by the LDS read itself.  The matrix operand goes
// first into the matrix instruction, so that a lane ends with four neighbouring columns of one result row.
//
// What made the large tile fast, on bf16 products of 8192^3 (forward / grad_input / grad_weight in TFLOP/s): whole steps
// between two waits 830 at the cases' sizes; fragments read a half step ahead 1082 / 1020 / 964; reads and transfers
// spread over the matrix instructions, addresses of 32 bits a lane, one loop body (two of them moved the sums between registers
// and spilled) 1126 / 1295 / 1348; blocks that stay and ask for the next tile's slices before they write this one's results: 16,384 x 2048 x
// 2048 forward 1130 -> 1200.  Four waves of 128 x 128 (709) and tiles of 128 x 256 in steps of 32, two a compute unit
// (870 to 916), were slower.
//
// Operands off 16-byte boundaries or of widths that are no multiples of 8 are read into registers, sixteen bytes at a time at
// any address, while the slice before is multiplied, and written to LDS from there; a chunk in which a row ends is read from
// as much earlier and moved down.  (271 x 6 rows of 8 experts, 1893 x 2808, forward / grad_input: two bytes at a time, and waited
// for where they were asked for, 179 us; at once and ahead 56 / 139; ends without single elements 54 / 65.)
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
typedef s16x8 s16x8_any __attribute__((aligned(2)));  // (global memory is read at any address)

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

// Sixteen bytes at p, or zeros.  (Said to be global memory: a choice between two pointers would be read as memory of any
// kind, and what waits for LDS then waits for it.)
typedef const __attribute__((address_space(1))) s16x8_any global16;
__device__ __forceinline__ global16 *there_or_zeros(const void *p, bool there) {
  return there ? (global16 *)p : (global16 *)&kZeros;
}

__device__ __forceinline__ void load_lds16(const void *src, char *dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)src,
                                   (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
}

// A value the compiler shall not keep derived values of over the turns of a loop (it would run out of registers): for
// all it knows this one changes with k.
template <typename V>
__device__ __forceinline__ V fresh(V v, int k) {
  asm("" : "+v"(v) : "s"(k));
  return v;
}
__device__ __forceinline__ int fresh_thread(int k) { return (int)fresh((uint32_t)threadIdx.x, k); }

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
  // not transposed: where each slot's row begins, in units of 16 bytes (not ALIGNED: the row's number).  Gathered rows may lie
  // anywhere, also where there are few of them, and take 64 bits.
  typedef typename std::conditional<GATHER && ALIGNED, uint64_t, uint32_t>::type Place;
  Place row_at[TR ? 1 : kSlots];
  // transposed: a thread's place in a slot's rows, in bytes (slots of odd number may permute differently), and the
  // columns left from there on; the rows of the next slice when they are gathered
  uint32_t at[2];
  int left[2];
  const int32_t *order;
  int top_k, next[TR && GATHER ? kSlots : 1];
  // not ALIGNED: what waits for put(); elements by which a slot's chunk (even, odd) was read early, because the row ends
  // inside it; whether a whole row is shorter than a chunk
  s16x8 held[ALIGNED ? 1 : kSlots];
  int early[2];
  bool narrow;

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
      row_at[it] = ALIGNED ? (Place)((uint64_t)row * (uint64_t)(ld / 8)) + (uint32_t)chunk(0, t) : row;
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
      // (not ALIGNED: any stride, so that the thread's row is multiplied with it in 64 bits, where it is read)
      at[h] = (uint32_t)(from + (GATHER || !ALIGNED ? 0 : t / kChunks * (int)ld)) * (uint32_t)sizeof(T);
      left[h] = width - c;
    }
    order = order_;
    top_k = top_k_;
  }

  // The source rows of the slice that starts at k (gathered operands).  They are asked for before the transfers of the
  // slice before it: what waits for them then waits for no transfer.
  __device__ void ask_rows(int k, int k_end) {
    if constexpr (TR && GATHER) {
      const int t = fresh_thread(k);
#pragma unroll
      for (int it = 0; it < kSlots; ++it) next[it] = order[min(k + k_row(it, t), k_end - 1)];
    }
  }

  // First element of a slot's chunk in the slice that starts at k.
  __device__ const T *source(int it, int k, int t, int pair) const {
    const char *b;
    if constexpr (!TR) {
      b = reinterpret_cast<const char *>(base + k);
      if constexpr (ALIGNED) return reinterpret_cast<const T *>(b + (uint64_t)fresh(row_at[it], k) * 16);
      else return base + (int64_t)row_at[it] * ld + k + chunk(0, t) * 8;
    } else if constexpr (GATHER) {
      b = reinterpret_cast<const char *>(base + (int64_t)(pair / top_k) * ld);
      return reinterpret_cast<const T *>(b + fresh(at[it & 1], k));
    } else {
      b = reinterpret_cast<const char *>(base + (int64_t)(k + it * kRowsASlot + (ALIGNED ? 0 : t / kChunks)) * ld);
      return reinterpret_cast<const T *>(b + fresh(at[it & 1], k));
    }
  }

  // The slice of k, k + 1, .. k + kStep - 1; what lies at or past k_end is zero.  ALIGNED: its transfer to LDS.  Else
  // it is asked for here and waits in registers for put().
  template <bool TAIL>
  __device__ void load(char *lds, int k, int k_end) {
    const int t = fresh_thread(k), wave = __builtin_amdgcn_readfirstlane(t >> 6);
    int now[TR && GATHER ? kSlots : 1];
    if constexpr (TR && GATHER) {
#pragma unroll
      for (int it = 0; it < kSlots; ++it) now[it] = next[it];
      ask_rows(k + kStep, k_end);
    }
#pragma unroll
    for (int it = 0; it < kSlots; ++it) {
      const T *src = source(it, k, t, TR && GATHER ? now[TR && GATHER ? it : 0] : 0);
      const bool there = !TAIL || (TR ? k + k_row(it, t) : k + chunk(0, t) * 8) < k_end;
      if constexpr (ALIGNED) {
        if (TAIL) src = there ? src : reinterpret_cast<const T *>(&kZeros);
        load_lds16(src, lds + (it * NT + wave * kWave) * 16);
      } else {
        // elements of the chunk that exist
        const int n = TR ? left[it & 1] : k_end - (k + chunk(0, t) * 8);
        early[it & 1] = n > 0 && n < 8 && !narrow ? 8 - n : 0;
        held[it] = *there_or_zeros(src - early[it & 1], there && n > 0 && !narrow);
        if (narrow && there && n > 0) {
          const short *p = reinterpret_cast<const short *>(src);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const short v = p[j < n ? j : 0];
            held[it][j] = j < n ? v : (short)0;
          }
        }
      }
    }
  }

  __device__ void put(char *lds) {
#pragma unroll
    for (int it = 0; it < kSlots; ++it) {
      s16x8 v = held[it];
      const int n = early[it & 1];
      if (n != 0) {  // what was read early leaves at the front, zeros follow
        const s16x8 none = {0, 0, 0, 0, 0, 0, 0, 0};
        if (n & 4) v = __builtin_shufflevector(v, none, 4, 5, 6, 7, 8, 8, 8, 8);
        if (n & 2) v = __builtin_shufflevector(v, none, 2, 3, 4, 5, 6, 7, 8, 8);
        if (n & 1) v = __builtin_shufflevector(v, none, 1, 2, 3, 4, 5, 6, 7, 8);
      }
      *reinterpret_cast<s16x8 *>(lds + (it * NT + (int)threadIdx.x) * 16) = v;
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

// The same where nothing is transferred to LDS but written: what registers wait for may still be on its way.
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
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
  int64_t unit;  // grad_weight in parts: the part's number
};

constexpr int kSortMost = 256;  // experts that grad_weight sorts by their rows (more of them even out by themselves)

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

// N (4 or 8) neighbouring results of a lane, at any address; the first n of them exist.
template <int N>
struct Run {
  float v[N];
};

template <typename T, int N>
__device__ __forceinline__ void store_run(T *p, const Run<N> &x, int n) {
  constexpr int kPer = N * sizeof(T) < 16 ? N : 16 / sizeof(T);
  typedef T Line __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
  if (n >= N) {
#pragma unroll
    for (int h = 0; h < N / kPer; ++h) {
      Line o;
#pragma unroll
      for (int i = 0; i < kPer; ++i) o[i] = (T)x.v[h * kPer + i];
      reinterpret_cast<Line *>(p)[h] = o;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = (T)x.v[i];
  }
}

template <typename T, int N>
__device__ __forceinline__ Run<N> load_run(const T *p, int n) {
  constexpr int kPer = N * sizeof(T) < 16 ? N : 16 / sizeof(T);
  typedef T Line __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
  Run<N> x;
  if (n >= N) {
#pragma unroll
    for (int h = 0; h < N / kPer; ++h) {
      const Line o = reinterpret_cast<const Line *>(p)[h];
#pragma unroll
      for (int i = 0; i < kPer; ++i) x.v[h * kPer + i] = (float)o[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) x.v[i] = i < n ? (float)p[i] : 0.f;
  }
  return x;
}

// What lane groups 0 .. 3 of 16 hold of fragments a and b (columns 4 g .. 4 g + 3 of each): group g gets columns
// 8 (g / 2) .. + 7 of fragment g % 2.
__device__ __forceinline__ Run<8> eight_columns(const f4 a, const f4 b) {
  Run<8> x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[i]), __float_as_uint(b[i]), false, false);
    x.v[i] = __uint_as_float(both[0]);
    x.v[4 + i] = __uint_as_float(both[1]);
  }
  return x;
}

__device__ __forceinline__ Run<4> four_columns(const f4 a) { return {{a[0], a[1], a[2], a[3]}}; }

// Neighbouring results of place q, column j on (j < width): through the activation and out.
template <typename T, int MODE, int ACT, int N>
__device__ __forceinline__ void finish(const ProductArgs &a, int64_t q, int j, const Run<N> &v, const Run<N> &up) {
  T *o = static_cast<T *>(a.out) + q * a.ldo + j;
  const int n = (MODE == kForward ? a.d_out : a.d_in) - j;
  Run<N> r = v;
  if (MODE == kForward) {
    if (ACT == AA_ACT_RELU) {
#pragma unroll
      for (int i = 0; i < N; ++i) r.v[i] = v.v[i] < 0.f ? 0.f : v.v[i];
    }
    if (ACT == AA_ACT_GATED) {
#pragma unroll
      for (int i = 0; i < N; ++i) r.v[i] = v.v[i] * sigmoid_fast(v.v[i]) * up.v[i];
      if (a.pre) {
        T *h = static_cast<T *>(a.pre) + q * a.ldpre + j;
        store_run(h, v, n);
        store_run(h + a.d_out, up, n);
      }
    }
  } else if (ACT == AA_ACT_RELU) {
    const Run<N> s = load_run<T, N>(static_cast<const T *>(a.saved) + q * a.lds + j, n);
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] = s.v[i] > 0.f ? v.v[i] : 0.f;
  } else if (ACT == AA_ACT_GATED) {
    const T *s = static_cast<const T *>(a.saved) + q * a.lds + j;
    const Run<N> g = load_run<T, N>(s, n), u = load_run<T, N>(s + a.d_in, n);
    Run<N> du;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float z = sigmoid_fast(g.v[i]);
      r.v[i] = v.v[i] * u.v[i] * (z + g.v[i] * z * (1.0f - z));
      du.v[i] = v.v[i] * g.v[i] * z;
    }
    store_run(o + a.d_in, du, n);
  }
  store_run(o, r, n);
}

template <typename T, int N>
__device__ __forceinline__ void finish_weight(T *o, const Run<N> &v, int n, bool accumulate) {
  Run<N> r = v;
  if (accumulate) {
    const Run<N> old = load_run<T, N>(o, n);
#pragma unroll
    for (int i = 0; i < N; ++i) r.v[i] += old.v[i];
  }
  store_run(o, r, n);
}

// Where the parts of a sum over a long range of rows go: part s of tile t is [BM][BN] at (t parts + s) BM BN.
__device__ __forceinline__ int part_length(int rows, int parts) {
  return ((rows + kStep - 1) / kStep + parts - 1) / parts * kStep;
}

// A block of WI x WJ waves, each FI x FJ fragments of 16 x 16 results: BM = 16 FI WI result rows
// (places of a group; grad_weight: rows of dw), BN = 16 FJ WJ columns.  With AA_ACT_GATED half of a wave's
// columns are the gate's, half the same columns of up.
template <typename T, int MODE, int ACT, int WI, int WJ, int FI, int FJ, int NB, bool GATHER, bool ALIGNED>
__global__ __launch_bounds__(WI *WJ *kWave, 2) void k_product(const ProductArgs a) {
  constexpr int NT = WI * WJ * kWave, BM = 16 * FI * WI, BN = 16 * FJ * WJ;
  constexpr bool TRP = MODE == kGradWeight, TRQ = MODE != kForward;
  constexpr bool GATED = MODE == kForward && ACT == AA_ACT_GATED;
  constexpr int OUT_N = GATED ? BN / 2 : BN, kOut = GATED ? FJ / 2 : FJ;
  constexpr int kBytesP = BM * kStep * 2, kBytesQ = BN * kStep * 2;
  constexpr int kBuffer = kBytesP + kBytesQ;
  __shared__ __attribute__((aligned(256))) char smem[NB * kBuffer];
  __shared__ int before[MODE == kGradWeight ? kSortMost : kMaxExperts + 1];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int wi = wave / WJ, wj = wave % WJ;
  const int columns = MODE == kForward ? a.d_out : a.d_in;
  const int nj = (columns + OUT_N - 1) / OUT_N;

  // Units of work.  Result tiles are walked in runs of neighbouring ones for each XCD (blocks go round the eight of
  // them), its blocks in turns.  grad_weight: the blocks take the tiles of the experts in turns, those with most rows
  // first, every second turn in reverse, which evens out the rows a block gets; a.parts units a tile.
  const int per_e = (a.d_out + BM - 1) / BM;  // (grad_weight) tile rows of an expert
  const int blocks = gridDim.x, place = ((int)blockIdx.x & 7) * (blocks >> 3) + ((int)blockIdx.x >> 3);
  int ni;
  int64_t t, t_end;
  if (MODE == kGradWeight) {
    ni = a.n_experts * per_e;
    t = place;
    t_end = (int64_t)ni * nj * a.parts;
    if (a.n_experts <= kSortMost) {
      for (int e = threadIdx.x; e < a.n_experts; e += NT) {
        const int rows = a.offsets[e + 1] - a.offsets[e];
        int rank = 0;
        for (int o = 0; o < a.n_experts; ++o) {
          const int other = a.offsets[o + 1] - a.offsets[o];
          rank += other > rows || (other == rows && o < e) ? 1 : 0;
        }
        before[rank] = e;
      }
      __syncthreads();
    }
  } else {
    count_group_tiles(a.offsets, a.n_experts, BM, before);
    __syncthreads();
    ni = __builtin_amdgcn_readfirstlane(before[a.n_experts]);
    const int64_t total = (int64_t)ni * nj, chunk = (total + 7) / 8;
    t = (int)(blockIdx.x & 7) * chunk + (int)(blockIdx.x >> 3);
    t_end = min(total, ((int)(blockIdx.x & 7) + 1) * chunk);
  }
  if (t >= t_end) return;
  auto find = [&](int64_t at) __attribute__((always_inline)) {
    Tile g;
    if (MODE == kGradWeight) {
      const int64_t tile = at / a.parts;
      const int part = (int)(at - tile * a.parts), in_e = (int)(tile % (per_e * nj));
      g.e = (int)(tile / (per_e * nj));
      if (a.n_experts <= kSortMost) g.e = __builtin_amdgcn_readfirstlane(before[g.e]);
      g.i0 = in_e / nj * BM;
      g.j0 = in_e % nj * OUT_N;
      g.i_end = a.d_out;
      g.k0 = __builtin_amdgcn_readfirstlane(a.offsets[g.e]);
      g.k_end = __builtin_amdgcn_readfirstlane(a.offsets[g.e + 1]);
      g.unit = at;
      if (a.parts > 1) {
        const int length = part_length(g.k_end - g.k0, a.parts);
        g.k0 = min(g.k0 + part * length, g.k_end);
        g.k_end = min(g.k0 + length, g.k_end);
        g.unit = (((int64_t)g.e * per_e + in_e / nj) * nj + in_e % nj) * a.parts + part;
      }
    } else {
      // runs of four row tiles by all column tiles: what an XCD works on at once shares rows and matrices
      constexpr int kRun = 4;
      const int run = (int)(at / (kRun * nj)), in_run = (int)(at % (kRun * nj));
      const int rows_of_run = min(kRun, ni - run * kRun);
      const int it = run * kRun + in_run % rows_of_run;
      g.j0 = in_run / rows_of_run * OUT_N;
      g.e = group_of_tile(before, a.n_experts, it);
      g.i0 = __builtin_amdgcn_readfirstlane(a.offsets[g.e] + (it - before[g.e]) * BM);
      g.i_end = __builtin_amdgcn_readfirstlane(a.offsets[g.e + 1]);
      g.k0 = 0;
      g.k_end = MODE == kForward ? a.d_in : a.d_out;
    }
    return g;
  };
  auto following = [&](int64_t at) {
    if (MODE != kGradWeight) return at + (blocks >> 3);
    const int64_t turn = at / blocks + 1;  // (place in an odd turn: from the end)
    return turn * blocks + (turn & 1 ? blocks - 1 - place : place);
  };

  Stage<T, BM, NT, TRP, GATHER && MODE == kForward, ALIGNED> P;
  Stage<T, BN, NT, TRQ, GATHER && MODE == kGradWeight, ALIGNED> Q;
  P.narrow = (MODE == kForward ? a.d_in : a.d_out) < 8;
  Q.narrow = a.d_in < 8;
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
  };
  auto put = [&](char *to) __attribute__((always_inline)) {
    if constexpr (!ALIGNED) {
      P.put(to);
      Q.put(to + kBytesP);
    }
  };
  // The slice two steps on into the buffer that is free (not ALIGNED: it has come to the registers during the last
  // step, and the one after it is asked for).
  auto refill = [&](char *to, int at, int k_end) __attribute__((always_inline)) {
    if (at >= k_end) return;
    if constexpr (ALIGNED) {
      load(to, at, k_end);
    } else {
      put(to);
      if (at + kStep < k_end) load(nullptr, at + kStep, k_end);
    }
  };
  // Takes up a tile: its addresses, and its first slices on their way.
  constexpr int kFirst = NB == 2 ? 2 : NB - 1;
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
#pragma unroll
      for (int b = 0; b < kFirst; ++b)
        if (b == 0 || g.k0 + b * kStep < g.k_end) {
          load(smem + b * kBuffer, g.k0 + b * kStep, g.k_end);
          put(smem + b * kBuffer);
        }
      if (!ALIGNED && g.k0 + kFirst * kStep < g.k_end) load(nullptr, g.k0 + kFirst * kStep, g.k_end);
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

    const int in_wave = fresh_thread((int)t) & 63;
    const uint32_t p_at = fragment_at<BM, TRP>(wi * FI * 16, in_wave);
    const uint32_t q_at = fragment_at<BN, TRQ>(wj * FJ * 16, in_wave);
    // (a wave whose part of the tile lies outside the result only moves data)
    const bool live = g.i0 + wi * FI * 16 < g.i_end && g.j0 + wj * kOut * 16 < columns;
    const int k_end = g.k_end;
    int k = g.k0;
    // A ring of buffers, for tiles that are a small part of what has to be moved: NB - 1 slices on their way, one
    // meeting a step, after which the buffer read in the step before is free.
    if constexpr (NB > 2) {
      for (int buf = 0; k < k_end; k += kStep, buf = buf + 1 < NB ? buf + 1 : 0) {
        if (ALIGNED && k + (NB - 2) * kStep < k_end) wait_and_meet<(NB - 2) * kLoads>();
        else wait_and_meet<0>();
        if (k + (NB - 1) * kStep < k_end) load(smem + (buf > 0 ? buf - 1 : NB - 1) * kBuffer, k + (NB - 1) * kStep, k_end);
        if (!live) continue;
        const char *here = smem + buf * kBuffer;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
          s16x8 fp[FI], fq[FJ];
#pragma unroll
          for (int j = 0; j < FJ; ++j) fq[j] = fragment<BN, TRQ>(here + kBytesP, q_at, j, ks);
#pragma unroll
          for (int i = 0; i < FI; ++i) fp[i] = fragment<BM, TRP>(here, p_at, i, ks);
#pragma unroll
          for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[i][j] = mfma16(fq[j], fp[i], acc[i][j], T());
        }
      }
      __syncthreads();  // the buffers are the next tile's
    }
    // Two buffers.  While 32 summed elements are multiplied the next 32 are read, a fragment of the rows into the place
    // of one that has been used.  Early in the second half of a step everybody has read its buffer and the next
    // one has arrived: the slice two steps on goes into the free buffer during the rest.
    if (NB == 2 && k < k_end) {
      if (!ALIGNED) meet();
      else if (k + kStep < k_end) wait_and_meet<kLoads>();
      else wait_and_meet<0>();
      if (live) {
        s16x8 fp[2][FI], fq[2][FJ];
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
          if constexpr (ALIGNED) wait_and_meet<0>();
          else meet();
          if constexpr (decltype(whole)::value) {  // the slice two steps on is there and is a whole one
            read(0, other, 0);
            P.template load<false>(here, k + 2 * kStep, k_end);
            Q.template load<false>(here + kBytesP, k + 2 * kStep, k_end);
            multiply(1, kAhead, FI);
            interleave<kReads, kLoads, (FI - kAhead) * FJ>();
          } else {
            refill(here, k + 2 * kStep, k_end);
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
      } else {
        for (int odd = 0; k < k_end; k += kStep, odd ^= 1) {
          if constexpr (ALIGNED) wait_and_meet<0>();
          else meet();
          refill(smem + odd * kBuffer, k + 2 * kStep, k_end);
        }
      }
    }

    // The next tile's first slices are on their way while this one's results are written.  (After the last meeting
    // nobody reads what LDS holds.)
    const Tile done = g;
    t = following(t);
    if (t < t_end) {
      g = find(t);
      begin(g);
    }
    // A lane has four neighbouring columns in each fragment; after an exchange with the lane 16 away it has eight in
    // every second one.
    constexpr int kRuns = kOut >= 2 ? kOut / 2 : 1;
    const int lane = fresh_thread((int)t) & 63, group = lane >> 4;
    const int ti = done.i0 + wi * FI * 16 + (lane & 15);
    const int tj = done.j0 + wj * kOut * 16 + (kOut >= 2 ? (group & 1) * 16 + (group >> 1) * 8 : group * 4);
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const int r = ti + i * 16;
#pragma unroll
      for (int p = 0; p < kRuns; ++p) {
        const int c = tj + p * 32;
        const auto run = [&](int first) __attribute__((always_inline)) {
          if constexpr (kOut >= 2) return eight_columns(acc[i][first + 2 * p], acc[i][first + 2 * p + 1]);
          else return four_columns(acc[i][first]);
        };
        const auto v = run(0);
        auto up = v;
        if (GATED) up = run(GATED ? kOut : 0);
        if (r < done.i_end && c < columns) {
          if constexpr (MODE == kGradWeight) {
            const size_t at = ((size_t)done.e * a.d_out + r) * a.d_in + c;
            if (a.parts > 1)
              store_run(a.partial + (done.unit * BM + (r - done.i0)) * BN + (c - done.j0), v, 8);
            else if (a.out_f32)
              finish_weight(static_cast<float *>(a.out) + at, v, a.d_in - c, a.accumulate);
            else
              finish_weight(static_cast<T *>(a.out) + at, v, a.d_in - c, a.accumulate);
          } else {
            finish<T, MODE, ACT>(a, r, c, v, up);
          }
        }
      }
    }
    if (t >= t_end) break;
  }
}

// The product of a few rows: what is moved is the matrices, and there is no reuse to stage them for.  A block takes 16 NF
// result columns of one group (with AA_ACT_GATED half of them the gate's, half the same of up); its waves share the
// summed dimension out in chunks of 64, straight from memory into the matrix instructions' registers with kAhead
// chunks on their way and no meeting, and join their sums in LDS.  Rows go 16 MF at a time.
template <typename T, int ACT, int NF, int MF, bool GATHER>
__global__ __launch_bounds__(256) void k_product_few(const ProductArgs a) {
  constexpr bool GATED = ACT == AA_ACT_GATED;
  constexpr int kWaves = 4, kOut = GATED ? NF / 2 : NF, kAhead = 4;
  __shared__ f4 sums[kWaves - 1][NF][MF][kWave];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  // the blockIdx.y-th group that has rows
  int e = -1, lo = 0, hi = 0;
  for (int e0 = 0, seen = 0; e0 < a.n_experts && e < 0; e0 += kWave) {
    const int at = min(e0 + lane, a.n_experts - 1);
    const int from = a.offsets[at], to = a.offsets[at + 1];
    const bool some = e0 + lane < a.n_experts && to > from;
    const unsigned long long with = __ballot(some);
    const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(with >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)with, 0u));
    const unsigned long long mine = __ballot(some && seen + before == (int)blockIdx.y);
    if (mine != 0ull) {
      const int who = __ffsll((long long)mine) - 1;
      e = e0 + who;
      lo = __builtin_amdgcn_readlane(from, who);
      hi = __builtin_amdgcn_readlane(to, who);
    }
    seen += __popcll(with);
  }
  if (e < 0) return;
  e = __builtin_amdgcn_readfirstlane(e);
  // (rows at any address; what is left of a chunk of eight at the end comes last)
  const int j0 = blockIdx.x * (16 * kOut), K = a.d_in & ~7, rest = a.d_in & 7;
  const T *w = static_cast<const T *>(a.mat) + (size_t)e * a.d_out * a.d_in * (GATED ? 2 : 1);
  const T *wr[NF];  // a lane's matrix rows
#pragma unroll
  for (int f = 0; f < NF; ++f) {
    const int c = min(j0 + f % kOut * 16 + (lane & 15), a.d_out - 1) + (GATED && f >= kOut ? a.d_out : 0);
    wr[f] = w + (size_t)c * a.d_in + (lane >> 4) * 8;
  }
  for (int q0 = lo; q0 < hi; q0 += 16 * MF) {
    const T *xr[MF];
    f4 acc[NF][MF];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
      for (int m = 0; m < MF; ++m) acc[f][m] = f4{0.f, 0.f, 0.f, 0.f};
    s16x8 fw[kAhead][NF][2], fx[kAhead][MF][2];
    // (a chunk past the end reads zeros; one that ends inside reads zeros for what lies outside)
    auto ask_matrix = [&](int slot, int k) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = k + h * 32;
        const bool there = at + (lane >> 4) * 8 < K;
#pragma unroll
        for (int f = 0; f < NF; ++f)
          fw[slot][f][h] = __builtin_nontemporal_load(there_or_zeros(wr[f] + at, there));
      }
    };
    auto ask_rows = [&](int slot, int k) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = k + h * 32;
        const bool there = at + (lane >> 4) * 8 < K;
#pragma unroll
        for (int m = 0; m < MF; ++m)
          fx[slot][m][h] = *there_or_zeros(xr[m] + at, there);
      }
    };
    constexpr int kTurn = kWaves * kStep;
    int k = wave * kStep;
    // the matrix first: the rows' addresses wait for their numbers
#pragma unroll
    for (int s = 0; s < kAhead; ++s) ask_matrix(s, k + s * kTurn);
#pragma unroll
    for (int m = 0; m < MF; ++m) {
      const int q = min(q0 + m * 16 + (lane & 15), hi - 1);
      xr[m] = static_cast<const T *>(a.rows) + (int64_t)(GATHER ? a.order[q] / a.top_k : q) * a.ld_rows + (lane >> 4) * 8;
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) ask_rows(s, k + s * kTurn);
    while (k < K) {
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int m = 0; m < MF; ++m) acc[f][m] = mfma16(fw[s][f][h], fx[s][m][h], acc[f][m], T());
        ask_matrix(s, k + kAhead * kTurn);
        ask_rows(s, k + kAhead * kTurn);
        k += kTurn;
      }
    }
    if (rest != 0 && wave == kWaves - 1) {
      const auto ends = [&](const T *row) {  // (the first lanes of four hold it, the others zeros)
        s16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
        const short *p = reinterpret_cast<const short *>(row + K);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < rest && lane < 16) v[i] = p[i];
        return v;
      };
      s16x8 ew[NF], ex[MF];
#pragma unroll
      for (int f = 0; f < NF; ++f) ew[f] = ends(wr[f]);
#pragma unroll
      for (int m = 0; m < MF; ++m) ex[m] = ends(xr[m]);
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int m = 0; m < MF; ++m) acc[f][m] = mfma16(ew[f], ex[m], acc[f][m], T());
    }
    if (wave > 0) {
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int m = 0; m < MF; ++m) sums[wave - 1][f][m][lane] = acc[f][m];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int m = 0; m < MF; ++m)
#pragma unroll
          for (int o = 0; o < kWaves - 1; ++o) acc[f][m] += sums[o][f][m][lane];
#pragma unroll
      for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int f = 0; f < kOut; ++f) {
          const int q = q0 + m * 16 + (lane & 15), c = j0 + f * 16 + (lane >> 4) * 4;
          if (q < hi && c < a.d_out)
            finish<T, kForward, ACT>(a, q, c, four_columns(acc[f][m]), four_columns(acc[GATED ? f + kOut : f][m]));
        }
    }
    __syncthreads();  // (the sums are read)
  }
}

// Adds up the parts of grad_weight's tiles, in their order; four columns a thread.
template <typename T, int BM, int BN>
__global__ __launch_bounds__(256) void k_join_parts(const ProductArgs a) {
  const int per_i = (a.d_out + BM - 1) / BM, per_j = (a.d_in + BN - 1) / BN;
  const int tile = blockIdx.x / (BM * BN / 1024);
  const int in_tile = (blockIdx.x % (BM * BN / 1024) * 256 + threadIdx.x) * 4;
  const int e = tile / (per_i * per_j), in_e = tile % (per_i * per_j);
  const int r = in_e / per_j * BM + in_tile / BN, c = in_e % per_j * BN + in_tile % BN;
  if (r >= a.d_out || c >= a.d_in) return;
  const float *p = a.partial + (size_t)tile * a.parts * (BM * BN) + in_tile;
  f4 sum = *reinterpret_cast<const f4 *>(p);
#pragma unroll 4
  for (int s = 1; s < a.parts; ++s) sum += *reinterpret_cast<const f4 *>(p + (size_t)s * (BM * BN));
  const size_t at = ((size_t)e * a.d_out + r) * a.d_in + c;
  const Run<4> v = four_columns(sum);
  if (a.out_f32) finish_weight(static_cast<float *>(a.out) + at, v, a.d_in - c, a.accumulate);
  else finish_weight(static_cast<T *>(a.out) + at, v, a.d_in - c, a.accumulate);
}

constexpr int kUnits = 256;  // compute units

template <typename T, int MODE, int ACT, int WI, int WJ, int FI, int FJ, int NB, bool ALIGNED>
hipError_t launch_tiles(ProductArgs a, hipStream_t st) {
  constexpr int BM = 16 * FI * WI, BN = 16 * FJ * WJ;
  constexpr int OUT_N = MODE == kForward && ACT == AA_ACT_GATED ? BN / 2 : BN;
  constexpr int kLds = (BM + BN) * kStep * 2 * NB + 4200;
  constexpr int64_t kFit = kUnits * (WI * WJ > 4 ? 1 : kLds > 80 << 10 ? 1 : kLds > 53 << 10 ? 2 : 3);
  const int64_t nj = ((MODE == kForward ? a.d_out : a.d_in) + OUT_N - 1) / OUT_N;
  int64_t ni;
  a.parts = 1;
  if (MODE == kGradWeight) {
    ni = (int64_t)a.n_experts * ((a.d_out + BM - 1) / BM);
    // Few tiles: the rows in parts, so that every place on the chip has one, each part at least four steps long
    // on average, and as many as the workspace holds.
    const int64_t room = (int64_t)(a.partial_bytes / (sizeof(float) * BM * BN));
    const int64_t steps = a.rows_max / kStep / a.n_experts;
    const int64_t want = min(min(kFit / (ni * nj), room / (ni * nj)), steps / 4);
    if (want > 1) a.parts = (int32_t)want;
  } else {  // every group may end inside a tile; there are no more groups with rows than rows
    ni = a.rows_max / BM + (a.rows_max < a.n_experts ? a.rows_max : a.n_experts);
  }
  // blocks that fit the chip at once walk the tiles
  const int64_t blocks = min(kFit, (ni * nj * a.parts + 7) / 8 * 8);
  if (blocks == 0) return hipSuccess;
  const dim3 grid((uint32_t)blocks), block(WI * WJ * kWave);
  // (grad_input's rows are never gathered)
  if (MODE != kGradInput && a.order)
    hipLaunchKernelGGL((k_product<T, MODE, ACT, WI, WJ, FI, FJ, NB, MODE != kGradInput, ALIGNED>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_product<T, MODE, ACT, WI, WJ, FI, FJ, NB, false, ALIGNED>), grid, block, 0, st, a);
  if (a.parts > 1) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const dim3 join((uint32_t)(ni * nj * (BM * BN / 1024)));
    hipLaunchKernelGGL((k_join_parts<T, BM, BN>), join, dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

template <typename T, int ACT, int NF, int MF>
hipError_t launch_few(const ProductArgs &a, hipStream_t st) {
  const int out_n = 16 * (ACT == AA_ACT_GATED ? NF / 2 : NF);
  const dim3 grid((a.d_out + out_n - 1) / out_n, a.rows_max < a.n_experts ? a.rows_max : a.n_experts), block(256);
  if (a.order) hipLaunchKernelGGL((k_product_few<T, ACT, NF, MF, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_product_few<T, ACT, NF, MF, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

// Which tile, by what a pass takes at most (us; K / 64 steps; turns: tiles over the places for them on the chip), measured
// on bf16 products of 512 to 65,536 rows and widths of 128 to 4096:
//   256 x 256, one a compute unit    1.75 a step and 5 a tile     32 experts x 1024 rows, 1024 x 1024: 65 us (the next: 76)
//   128 x 128, two a compute unit    1.05 (0.6 where they are alone) and 3     8 x 512 rows, 2048 x 2048: 36 us (50, 149)
//   32 x 64, two, five slices ahead  0.42 and 3.5                 1 x 128 rows, 2048 x 2048: 15 us (31, 20)
// and, in forward, for rows that are a small part of what is read and too few of those tiles: k_product_few
//   8 experts of one row, 2048 x 1024: 12 us (32, 23, 21); 1 x 32 rows, 4096 x 4096: 22 us (58, 41, 39); but 32 x 25 rows,
//   1024 x 2048 (512 tiles of 128): 49 us (33, 29, 37).
template <typename T, int MODE, int ACT>
hipError_t launch_product(const ProductArgs &a, hipStream_t st) {
  if (MODE != kGradWeight && a.rows_max == 0) return hipSuccess;
  if (MODE == kGradWeight) {
    if (!a.aligned) return launch_tiles<T, MODE, ACT, 2, 2, 4, 4, 2, false>(a, st);
    // (parts make up for few tiles; 4 experts x 10,000 rows, 256 x 256: 30 us in tiles of 256, 27 of 128; 16 x 750 rows,
    // 1000 x 520: 30 and 43)
    if ((int64_t)a.d_in * a.d_out <= 256 * 256) return launch_tiles<T, MODE, ACT, 2, 2, 4, 4, 2, true>(a, st);
    return launch_tiles<T, MODE, ACT, 2, 4, 8, 4, 2, true>(a, st);
  } else {
    const int64_t groups = max(1, min(a.rows_max, a.n_experts)), rows = (a.rows_max + groups - 1) / groups;
    const int64_t wide = (int64_t)(MODE == kForward ? a.d_out : a.d_in) * (MODE == kForward && ACT == AA_ACT_GATED ? 2 : 1);
    const double steps = ((MODE == kForward ? a.d_in : a.d_out) + kStep - 1) / kStep;
    auto tiles = [&](int bm, int bn) { return groups * ((rows + bm - 1) / bm) * ((wide + bn - 1) / bn); };
    auto turns = [&](int64_t n, int64_t places) { return (double)((n + places - 1) / places); };
    const int64_t n256 = tiles(256, 256), n128 = tiles(128, 128), n32 = tiles(32, 64);
    const double t256 = turns(n256, kUnits) * (steps * 1.75 + 5.0);
    const double t128 = turns(n128, 2 * kUnits) * (steps * (n128 <= kUnits ? 0.6 : 1.05) + 3.0);
    const double t32 = turns(n32, 2 * kUnits) * (steps * 0.42 + 3.5);
    if constexpr (MODE == kForward) {
      if (rows <= 32 && n128 <= 320)
        return rows <= 16 ? launch_few<T, ACT, 2, 1>(a, st) : launch_few<T, ACT, 2, 2>(a, st);
    }
    // (what goes through registers: the one tile that has them)
    if (!a.aligned) return launch_tiles<T, MODE, ACT, 2, 2, 4, 4, 2, false>(a, st);
    if (t32 < t128 && t32 < t256) return launch_tiles<T, MODE, ACT, 2, 2, 1, 2, 6, true>(a, st);
    if (t128 < t256) return launch_tiles<T, MODE, ACT, 2, 2, 4, 4, 2, true>(a, st);
    return launch_tiles<T, MODE, ACT, 2, 4, 8, 4, 2, true>(a, st);
  }
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

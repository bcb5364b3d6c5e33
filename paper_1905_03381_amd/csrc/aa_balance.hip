// Balance loss of a router, the experts' choices and shares, and the gradient of its logits.
//
// With c_e the choices of expert e among the m K of the rows in use, p_te = s_te / sum_e s_te and q_t the softmax of a row:
//   loss = coef E / (m K) sum_e c_e P_e + z / m sum_t lse_t^2,   P_e = sum_t p_te / m,  lse_t = log sum_e exp x_te
//   d/dx_te = coef E / (m^2 K) p_te w_te (c_e - sum_e p_te c_e) + 2 z / m lse_t q_te,   w = 1 (softmax) or 1 - s_te (sigmoid).
// c_e may be counted from the mean of all: both c_e - sum p c then lose fewer digits.  The gradient of the routing weights (as
// k_route_grad has it) is worked out an expert at a time, too: the choices and what they are given go to their experts'
// lanes through LDS, so that no logit is asked for twice.
//
// A row is read once, by 16 lanes or a wave.  16,384 x 256 f32 of sigmoid scores: rows 10 us, join 5.  A wave has one turn of 664
// vector instructions, 34 of them exponentials, reciprocals and the like; they keep the units busy for 54 % of the rows' time, the
// rest is waited for: the count, then the logits, the sums over lanes, and the block's sums halved four times through LDS.  The
// gradient of 60,001 x 64 bf16, with a routing gradient: 9.4 us, vector instructions (4.2 M, 514 a wave) for 87 % of it.  Sums over
// rows: a block's in registers, the waves' in LDS, the blocks' by a second launch, each in a fixed order.
#include "aa_lines.hpp"
#include "aa_route_lanes.hpp"

namespace aa {

namespace {

// A row's EPL neighbouring logits of this lane, -inf past its end and for NaN; at any address.
template <typename T, int EPL>
__device__ __forceinline__ void load_experts(const T *row, int e0, int E, float (&x)[EPL]) {
  constexpr int kPer = EPL * sizeof(T) <= 16 ? EPL : 16 / sizeof(T);
  typedef T Part __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
#pragma unroll
  for (int i = 0; i < EPL; ++i) x[i] = kNegInf;
  if (e0 + EPL <= E) {
#pragma unroll
    for (int h = 0; h < EPL / kPer; ++h) {
      const Part v = *reinterpret_cast<const Part *>(row + e0 + h * kPer);
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[h * kPer + i] = (float)v[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e0 + i < E) x[i] = (float)row[e0 + i];
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) x[i] = x[i] > kNegInf ? x[i] : kNegInf;
}

template <int EPL>
__device__ __forceinline__ void load_experts(const void *logits, int dtype, int64_t at, int e0, int E, float (&x)[EPL]) {
  if (dtype == AA_BF16) load_experts<__bf16, EPL>(static_cast<const __bf16 *>(logits) + at, e0, E, x);
  else if (dtype == AA_F16) load_experts<_Float16, EPL>(static_cast<const _Float16 *>(logits) + at, e0, E, x);
  else load_experts<float, EPL>(static_cast<const float *>(logits) + at, e0, E, x);
}

template <typename T, int EPL>
__device__ __forceinline__ void store_experts(T *row, int e0, int E, const float (&x)[EPL]) {
  constexpr int kPer = EPL * sizeof(T) <= 16 ? EPL : 16 / sizeof(T);
  typedef T Part __attribute__((ext_vector_type(kPer), aligned(sizeof(T))));
  if (e0 + EPL <= E) {
#pragma unroll
    for (int h = 0; h < EPL / kPer; ++h) {
      Part v;
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] = (T)x[h * kPer + i];
      *reinterpret_cast<Part *>(row + e0 + h * kPer) = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e0 + i < E) row[e0 + i] = (T)x[i];
  }
}

// e^x of x <= 88 by the unit's 2^t, with what t = x log2 e loses of its digits made good (without, e^x is off by |x|
// roundings); 0 far below.  No branch: the compiler would make one for each logit.
__device__ __forceinline__ float exp_of(float x) {
  constexpr float kLog = 1.44269504f, kRest = 1.92596299e-8f;  // log2 e
  x = fmaxf(x, -150.f);
  const float t = x * kLog;
  const float rest = fmaf(x, kRest, fmaf(x, kLog, -t));
  const float y = __builtin_amdgcn_exp2f(t);
  return fmaf(y, rest * 0.693147181f, y);
}

// x - top for x <= top, also where top is infinite.
__device__ __forceinline__ float below(float x, float top) {
  const float v = x - top;
  return x == top ? 0.f : v;
}

// What a row's EPL logits a lane come to: the shares of the sum of scores (sigmoid: with the scores' complements), the
// softmax and log sum exp (0 where there is none that is finite).
template <bool SOFTMAX, int LPR, int EPL>
__device__ __forceinline__ void row_shares(const float (&x)[EPL], float (&p)[EPL], float (&rest)[EPL],
                                           float (&q)[EPL], float *lse) {
  float sum = 0.f, all = 0.f;
  if constexpr (!SOFTMAX) {
    // logits that e^x holds as they are: one exponential each
    bool far = false;
#pragma unroll
    for (int i = 0; i < EPL; ++i) far |= fabsf(x[i]) > 40.f && x[i] > kNegInf;
    if (__ballot(far) == 0ull) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        q[i] = exp_of(x[i]);  // (0 for -inf)
        rest[i] = __builtin_amdgcn_rcpf(1.f + q[i]);
        p[i] = q[i] * rest[i];
        sum += q[i];
        all += p[i];
      }
      sum = lanes_sum<LPR>(sum);
      all = lanes_sum<LPR>(all);
      const float inv = sum > 0.f ? __builtin_amdgcn_rcpf(sum) : 0.f, part = all > 0.f ? __builtin_amdgcn_rcpf(all) : 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        q[i] *= inv;
        p[i] *= part;
      }
      *lse = sum > 0.f ? __logf(sum) : 0.f;
      return;
    }
  }
  float top = kNegInf;
#pragma unroll
  for (int i = 0; i < EPL; ++i) top = fmaxf(top, x[i]);
  top = lanes_max<LPR>(top);
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const float e = exp_of(below(x[i], top));
    q[i] = x[i] > kNegInf ? e : 0.f;
    sum += q[i];
  }
  sum = lanes_sum<LPR>(sum);
  const float inv = sum > 0.f ? __builtin_amdgcn_rcpf(sum) : 0.f;
#pragma unroll
  for (int i = 0; i < EPL; ++i) q[i] *= inv;
  *lse = fabsf(top) < -kNegInf ? top + __logf(sum) : 0.f;
  if constexpr (SOFTMAX) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      p[i] = q[i];
      rest[i] = 1.f;
    }
    return;
  }
  // scores relative to the highest: in 32 bits those of low logits would all be 0
  const float low = fminf(top, 0.f);
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const float t = exp_of(-fabsf(x[i])), r = __builtin_amdgcn_rcpf(1.f + t), e = exp_of(fminf(x[i], 0.f) - low) * r;
    p[i] = x[i] > kNegInf ? e : 0.f;
    rest[i] = x[i] > 0.f ? t * r : r;
    all += p[i];
  }
  all = lanes_sum<LPR>(all);
  const float part = all > 0.f ? __builtin_amdgcn_rcpf(all) : 0.f;
#pragma unroll
  for (int i = 0; i < EPL; ++i) p[i] *= part;
}

// One block a compute unit, so that there are few parts to join (16,384 x 256 f32, both launches: 14 us; 512 blocks of half the
// threads 15).
constexpr int kRowsThreads = 1024, kRowsWaves = kRowsThreads / kWave;

// counts, shares and losses from the sums over all rows: E values of p and c, this thread's with number e; term and square:
// what goes into the losses.
__device__ __forceinline__ double finish_expert(const BalanceArgs &a, int rows, int e, float p, int c) {
  const double mean = rows > 0 ? (double)p / rows : 0.0;
  a.counts[e] = c;
  if (a.share) a.share[e] = (float)mean;
  return (double)c * mean;
}
__device__ __forceinline__ void finish_losses(const BalanceArgs &a, int rows, double term, double square) {
  if (!a.loss) return;
  a.loss[0] = rows > 0 ? (float)(term * a.coef * a.n_experts / ((double)rows * a.cfg.top_k)) : 0.f;
  a.loss[1] = rows > 0 ? (float)(square * a.z_coef / rows) : 0.f;
}

// Shares and choices of the rows that a block takes, a lane's experts in registers; what the block's waves have is added
// up in LDS, half of them at a time.  A block that is alone has them all.
template <bool SOFTMAX, int LPR, int EPL>
__global__ __launch_bounds__(kRowsThreads) void k_balance_rows(const BalanceArgs a) {
  constexpr int kRows = kWave / LPR;
  __shared__ float room[kRowsWaves / 2][EPL][kWave];
  __shared__ int hist[LPR * EPL];
  __shared__ float z_room[kRowsWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LPR, e0 = sub * EPL;
  const int rows = rows_in_use(a.count, a.n_max), E = a.n_experts, K = a.cfg.top_k;
  for (int e = threadIdx.x; e < LPR * EPL; e += kRowsThreads) hist[e] = 0;
  __syncthreads();
  float sums[EPL], z = 0.f;
#pragma unroll
  for (int i = 0; i < EPL; ++i) sums[i] = 0.f;
  const int64_t step = (int64_t)gridDim.x * kRowsWaves * kRows;
  for (int64_t base = ((int64_t)blockIdx.x * kRowsWaves + wave) * kRows; base < rows; base += step) {
    const int64_t row = base + lane / LPR;
    const bool live = row < rows;
    float x[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = kNegInf;
    int id = -1;
    if (live && sub < K) id = a.ids[row * K + sub];
    if (live) load_experts<EPL>(a.logits, a.dtype, row * a.ld, e0, E, x);
    if (id >= 0 && id < E) atomicAdd(&hist[id], 1);
    float p[EPL], rest[EPL], q[EPL], lse;
    row_shares<SOFTMAX, LPR, EPL>(x, p, rest, q, &lse);
#pragma unroll
    for (int i = 0; i < EPL; ++i) sums[i] += p[i];
    z += sub == 0 ? lse * lse : 0.f;
  }
  if constexpr (LPR == 16) {  // the wave's rows
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      float u, v;
      exchange<false>(sums[i], &u, &v);
      exchange<true>(u + v, &u, &v);
      sums[i] = u + v;
    }
  }
  z = lanes_sum<64>(z);
  if (lane == 0) z_room[wave] = z;
#pragma unroll
  for (int half = kRowsWaves / 2; half >= 1; half /= 2) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) room[wave - half][i][lane] = sums[i];
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int i = 0; i < EPL; ++i) sums[i] += room[wave][i][lane];
    }
    __syncthreads();
  }
  z = 0.f;
#pragma unroll
  for (int w = 0; w < kRowsWaves; ++w) z += z_room[w];
  if (gridDim.x == 1) {
    if (wave > 0) return;
    double term = 0.0;
    if (lane < LPR) {
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (e0 + i < E) term += finish_expert(a, rows, e0 + i, sums[i], hist[e0 + i]);
    }
    term = lanes_sum<64>(term);
    if (lane == 0) finish_losses(a, rows, term, (double)z);
    return;
  }
  const int wide = (E + 3) & ~3;
  float *part = a.part + (size_t)blockIdx.x * 2 * wide;
  int *choices = reinterpret_cast<int *>(part + wide);
  if (wave == 0 && lane < LPR) {
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (e0 + i < wide) part[e0 + i] = e0 + i < E ? sums[i] : 0.f;
  }
  for (int e = threadIdx.x; e < wide; e += kRowsThreads) choices[e] = e < LPR * EPL ? hist[e] : 0;
  if (threadIdx.x == 0) a.z_part[blockIdx.x] = z;
}

// The blocks' parts, added up in a fixed order: 16 experts a block, four a thread, 256 shares of the parts.  The last
// block to end has the losses (a block for all experts took twice as long).  256 experts of 256 parts: 4.9 us.
constexpr int kJoinThreads = 1024, kJoinExperts = 16;

__global__ __launch_bounds__(kJoinThreads) void k_balance_join(const BalanceArgs a, int parts) {
  typedef int i4 __attribute__((ext_vector_type(4)));
  constexpr int kWaves = kJoinThreads / kWave;
  __shared__ float room_p[kWaves][kJoinExperts];
  __shared__ int room_c[kWaves][kJoinExperts];
  __shared__ float room_z[kWaves];
  __shared__ int last;
  const int rows = rows_in_use(a.count, a.n_max), E = a.n_experts, wide = (E + 3) & ~3;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int first = blockIdx.x * kJoinExperts, e0 = first + (lane & 3) * 4;
  f4 p = {0.f, 0.f, 0.f, 0.f};
  i4 c = {0, 0, 0, 0};
  if (e0 < wide) {
    for (int b = threadIdx.x >> 2; b < parts; b += kJoinThreads / 4) {
      const float *at = a.part + (size_t)b * 2 * wide + e0;
      p += *reinterpret_cast<const f4 *>(at);
      c += *reinterpret_cast<const i4 *>(at + wide);
    }
  }
  float z = blockIdx.x == 0 && (int)threadIdx.x < parts ? a.z_part[threadIdx.x] : 0.f;
#pragma unroll
  for (int off = 4; off < kWave; off <<= 1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[i] += __shfl_xor(p[i], off, kWave);
      c[i] += __shfl_xor(c[i], off, kWave);
    }
  }
  z = lanes_sum<64>(z);
  if (lane < 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      room_p[wave][lane * 4 + i] = p[i];
      room_c[wave][lane * 4 + i] = c[i];
    }
  }
  if (lane == 0) room_z[wave] = z;
  __syncthreads();
  if (wave > 0) return;
  double term = 0.0;
  if (lane < kJoinExperts && first + lane < E) {
    float all = 0.f;
    int choices = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      all += room_p[w][lane];
      choices += room_c[w][lane];
    }
    term = finish_expert(a, rows, first + lane, all, choices);
  }
  term = lanes_sum<64>(term);
  double square = 0.0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) square += (double)room_z[w];
  if (gridDim.x == 1) {
    if (lane == 0) finish_losses(a, rows, term, square);
    return;
  }
  // the blocks' terms (and the first one's squares), past the caches that are not shared
  if (lane == 0) {
    __hip_atomic_store(a.terms + blockIdx.x, term, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (blockIdx.x == 0) __hip_atomic_store(a.terms + gridDim.x, square, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    stores_arrived();
    last = count_in(a.done, gridDim.x);
  }
  wave_sync();
  if (!last) return;
  term = lane < (int)gridDim.x ? __hip_atomic_load(a.terms + lane, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.0;
  term = lanes_sum<64>(term);
  square = __hip_atomic_load(a.terms + gridDim.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (lane == 0) finish_losses(a, rows, term, square);
}

// What an expert's place holds that no choice was given to (a NaN that arithmetic does not make).
constexpr uint32_t kNotChosen = 0x7FC0DEADu;

constexpr int kGradThreads = 256;

template <bool SOFTMAX, int LPR, int EPL>
__global__ __launch_bounds__(kGradThreads) void k_balance_grad(const RouteGradArgs a) {
  constexpr int kRows = kWave / LPR, kSlots = kGradThreads / LPR;
  constexpr int kPer = EPL < 4 ? EPL : 4;
  typedef uint32_t Words __attribute__((ext_vector_type(kPer)));
  __shared__ __attribute__((aligned(16))) uint32_t given[kSlots][LPR * EPL];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LPR, e0 = sub * EPL;
  const int rows = rows_in_use(a.count, a.n_max), E = a.n_experts, K = a.cfg.top_k;
  const bool renorm = a.cfg.renormalise != 0, route = a.dweights != nullptr;
  uint32_t *here = given[threadIdx.x / LPR];
  // the experts' choices, counted from their mean, and the factors of the two terms
  float counts[EPL], scale, z_scale;
  {
    float sum = 0.f;
    int c[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      c[i] = e0 + i < E ? a.counts[e0 + i] : 0;
      sum += (float)c[i];
    }
    // (any whole number near the mean does: what is added to all counts falls out)
    const int mean = (int)fminf(lanes_sum<LPR>(sum) / (float)E, 2147483520.f);
#pragma unroll
    for (int i = 0; i < EPL; ++i) counts[i] = (float)(c[i] - mean);
    const float part = (a.dloss ? *a.dloss : 1.f) / (float)rows;
    scale = part * a.coef * ((float)E / (float)K) / (float)rows;
    z_scale = part * 2.f * a.z_coef;
  }
  const int64_t step = (int64_t)gridDim.x * (kGradThreads / kWave) * kRows;
  for (int64_t base = ((int64_t)blockIdx.x * (kGradThreads / kWave) + wave) * kRows; base < rows; base += step) {
    const int64_t row = base + lane / LPR;
    const bool live = row < rows;
    float x[EPL], out[EPL];
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = kNegInf;
    int id = -1;
    float d = 0.f;
    if (route && live && sub < K) {
      id = a.ids[row * K + sub];
      d = a.dweights[row * K + sub] * a.cfg.scale;
    }
    if (live) load_experts<EPL>(a.logits, a.dtype, row * a.ld, e0, E, x);
    if (route) {
      Words none;
#pragma unroll
      for (int i = 0; i < kPer; ++i) none[i] = kNotChosen;
#pragma unroll
      for (int h = 0; h < EPL / kPer; ++h) *reinterpret_cast<Words *>(here + e0 + h * kPer) = none;
      wave_sync();
      if (id >= 0 && id < E) here[id] = __float_as_uint(d);
      wave_sync();
    }
    float p[EPL], rest[EPL], q[EPL], lse, dot = 0.f;
    row_shares<SOFTMAX, LPR, EPL>(x, p, rest, q, &lse);
#pragma unroll
    for (int i = 0; i < EPL; ++i) dot += p[i] * counts[i];
    dot = lanes_sum<LPR>(dot);
    lse *= z_scale;
#pragma unroll
    for (int i = 0; i < EPL; ++i) out[i] = scale * p[i] * rest[i] * (counts[i] - dot) + lse * q[i];
    if (route) {
      float g[EPL];  // what the chosen experts of this lane are given
      bool chosen[EPL];
#pragma unroll
      for (int h = 0; h < EPL / kPer; ++h) {
        const Words w = *reinterpret_cast<const Words *>(here + e0 + h * kPer);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          chosen[h * kPer + i] = w[i] != kNotChosen && x[h * kPer + i] > kNegInf;
          g[h * kPer + i] = chosen[h * kPer + i] ? __uint_as_float(w[i]) : 0.f;
        }
      }
      wave_sync();  // (read, before the next row's)
      // s: the scores, or (renormalised) the weights among the choices; with: their sum with what is given
      float s[EPL], sum = 0.f, with = 0.f;
      if (!renorm) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          if (SOFTMAX) s[i] = q[i];
          else s[i] = x[i] > 0.f ? 1.f - rest[i] : rest[i] * exp_of(x[i]);
          with += g[i] * s[i];
        }
        with = SOFTMAX ? lanes_sum<LPR>(with) : 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) out[i] += (SOFTMAX || chosen[i] ? s[i] * rest[i] : 0.f) * (g[i] - with);
      } else {
        float any = 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          s[i] = chosen[i] ? p[i] : 0.f;
          any = chosen[i] ? 1.f : any;
          sum += s[i];
        }
        sum = lanes_sum<LPR>(sum);
        bool there = sum > 0.f;
        if (__ballot(any > 0.f && sum < 0x1p-60f) != 0ull) {
          // Choices that are little beside the row's others, or nothing in 32 bits: relative to the highest of them.  (Where the
          // routing's 64 bits have 0, so have the weights, and there is no gradient.)
          float best = kNegInf, top = kNegInf;
#pragma unroll
          for (int i = 0; i < EPL; ++i) {
            s[i] = SOFTMAX ? x[i] : fminf(x[i], 0.f);
            best = fmaxf(best, chosen[i] ? s[i] : kNegInf);
            top = fmaxf(top, s[i]);
          }
          best = lanes_max<LPR>(best);
          if (SOFTMAX) top = lanes_max<LPR>(top);
          there = SOFTMAX ? best == top || best - top > kNoScore : best > kNoScore;
          sum = 0.f;
#pragma unroll
          for (int i = 0; i < EPL; ++i) {
            const float e = exp_of(fminf(below(s[i], best), 0.f));  // (what is above the highest choice is none)
            const float r = SOFTMAX ? 1.f : x[i] > 0.f ? 1.f - rest[i] : rest[i];
            s[i] = chosen[i] ? e * r : 0.f;
            sum += s[i];
          }
          sum = lanes_sum<LPR>(sum);
        }
        const float inv = there && sum > 0.f ? __builtin_amdgcn_rcpf(sum) : 0.f;
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          s[i] *= inv;
          with += g[i] * s[i];
        }
        with = lanes_sum<LPR>(with);
#pragma unroll
        for (int i = 0; i < EPL; ++i) out[i] += s[i] * rest[i] * (g[i] - with);
      }
    }
    if (!live) continue;
    const int64_t to = row * a.ld_out;
    if (a.dtype == AA_BF16) store_experts<__bf16, EPL>(static_cast<__bf16 *>(a.dlogits) + to, e0, E, out);
    else if (a.dtype == AA_F16) store_experts<_Float16, EPL>(static_cast<_Float16 *>(a.dlogits) + to, e0, E, out);
    else store_experts<float, EPL>(static_cast<float *>(a.dlogits) + to, e0, E, out);
  }
}

}  // namespace

hipError_t launch_balance(const BalanceArgs &a, hipStream_t st) {
  int blocks = 0;
  const hipError_t e = by_width(a.n_experts, a.cfg.top_k, 256, [&](auto lpr, auto epl) {
    constexpr int LPR = decltype(lpr)::value, EPL = decltype(epl)::value, kRows = kRowsThreads / LPR;
    const int64_t want = ((int64_t)a.n_max + kRows - 1) / kRows;
    // (a block that is alone takes a few turns in less than a second launch does: 256 rows of 64 experts in four turns 6.9 us, by
    // several blocks 9.6; 128 of 256 in two 11.1 and 12.7, 256 in four 17.0 and 12.8)
    blocks = (int)(want <= (EPL <= 4 ? 4 : 2) ? 1 : want < kBalanceBlocks ? want : kBalanceBlocks);
    if (a.cfg.score == AA_SCORE_SOFTMAX)
      hipLaunchKernelGGL((k_balance_rows<true, LPR, EPL>), dim3(blocks), dim3(kRowsThreads), 0, st, a);
    else
      hipLaunchKernelGGL((k_balance_rows<false, LPR, EPL>), dim3(blocks), dim3(kRowsThreads), 0, st, a);
    return hipGetLastError();
  });
  if (e != hipSuccess || blocks == 1) return e;
  hipLaunchKernelGGL(k_balance_join, dim3((a.n_experts + kJoinExperts - 1) / kJoinExperts), dim3(kJoinThreads), 0, st, a, blocks);
  return hipGetLastError();
}

hipError_t launch_balance_grad(const RouteGradArgs &a, hipStream_t st) {
  if (a.n_max == 0) return hipSuccess;
  return by_width(a.n_experts, a.cfg.top_k, 256, [&](auto lpr, auto epl) {
    constexpr int LPR = decltype(lpr)::value, EPL = decltype(epl)::value, kRows = kGradThreads / LPR;
    const int64_t want = ((int64_t)a.n_max + kRows - 1) / kRows, most = 2048;  // (what fits the chip; blocks take turns)
    const dim3 grid((uint32_t)(want < most ? want : most)), block(kGradThreads);
    if (a.cfg.score == AA_SCORE_SOFTMAX) hipLaunchKernelGGL((k_balance_grad<true, LPR, EPL>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_balance_grad<false, LPR, EPL>), grid, block, 0, st, a);
    return hipGetLastError();
  });
}

}  // namespace aa

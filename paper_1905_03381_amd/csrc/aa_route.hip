// Routing of rows to experts, its gradient, and the grouping of the (row, choice) pairs by expert.
#include "aa_route.hpp"

namespace aa {

namespace {

constexpr float kNegInf = -__builtin_inff();

// What the lanes of a wave wrote to LDS before is read by its other lanes after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ int rows_in_use(const int32_t *count, int n_max) {
  return count ? min(max(*count, 0), n_max) : n_max;
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, kWave));
  return v;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

__device__ __forceinline__ float wave_sum(float v) { return group_sum<kWave>(v); }

// One wave a row, expert e = lane + 64 i.  Scores and choice values are doubles: near scores are told apart
// as the formulas have them.
template <typename T, int EPL>
__global__ __launch_bounds__(256) void k_route(const RouteArgs a) {
  __shared__ double s_value[4][kMaxExperts];   // choice values, for the groups
  __shared__ double s_group[4][kMaxExperts];   // group values
  __shared__ uint8_t s_taken[4][kMaxExperts];  // groups to choose from
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * 4 + wave;
  if (row >= rows_in_use(a.count, a.n_max)) return;
  const int E = a.n_experts, K = a.cfg.top_k;
  const T *x_row = static_cast<const T *>(a.logits) + (int64_t)row * a.ld;
  float x[EPL];
  float top = kNegInf;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = lane + i * kWave;
    x[i] = e < E ? (float)x_row[e] : kNegInf;
    if (!(x[i] > kNegInf)) x[i] = kNegInf;  // (a NaN: not free)
    top = fmaxf(top, x[i]);
  }
  double s[EPL], c[EPL];
  if (a.cfg.score == AA_SCORE_SOFTMAX) {
    top = wave_max(top);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      // (+inf - +inf: those that are +inf share the whole)
      s[i] = !(x[i] > kNegInf) ? 0.0 : x[i] == top ? 1.0 : exp((double)x[i] - (double)top);
      sum += s[i];
    }
    sum = wave_sum(sum);
#pragma unroll
    for (int i = 0; i < EPL; ++i) s[i] = sum > 0.0 ? s[i] / sum : 0.0;
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) s[i] = x[i] > kNegInf ? 1.0 / (1.0 + exp(-(double)x[i])) : 0.0;
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = lane + i * kWave;
    // Without bias and groups the order is that of the logits, also where scores round to one value.
    c[i] = x[i] > kNegInf ? (a.bias ? s[i] + (double)a.bias[e] : a.cfg.n_groups > 1 ? s[i] : (double)x[i])
                          : (double)kNegInf;
    if (!(c[i] > (double)kNegInf)) c[i] = (double)kNegInf;
  }
  const int G = a.cfg.n_groups;
  if (G > 1) {
    const int size = E / G;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (lane + i * kWave < E) s_value[wave][lane + i * kWave] = c[i];
    wave_sync();
    for (int g = lane; g < G; g += kWave) {
      double first = kNegInf, second = kNegInf;
      for (int q = 0; q < size; ++q) {
        const double v = s_value[wave][g * size + q];
        if (v > first) {
          second = first;
          first = v;
        } else if (v > second) {
          second = v;
        }
      }
      s_group[wave][g] = a.cfg.group_best == 2 && second > (double)kNegInf ? first + second : first;
    }
    wave_sync();
    for (int g = lane; g < G; g += kWave) {
      const double v = s_group[wave][g];
      int rank = 0;
      for (int q = 0; q < G; ++q) {
        const double o = s_group[wave][q];
        rank += (o > v || (o == v && q < g)) ? 1 : 0;
      }
      s_taken[wave][g] = rank < a.cfg.top_groups && v > (double)kNegInf ? 1 : 0;
    }
    wave_sync();
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = lane + i * kWave;
      if (e < E && !s_taken[wave][e / size]) c[i] = (double)kNegInf;
    }
  }
  // lane k keeps choice k
  int my_id = -1;
  double my_score = 0.0;
  for (int k = 0; k < K; ++k) {
    double best = c[0], score = s[0];
    int at = lane;
#pragma unroll
    for (int i = 1; i < EPL; ++i)
      if (c[i] > best) {
        best = c[i];
        score = s[i];
        at = lane + i * kWave;
      }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) {
      const double ob = __shfl_xor(best, off, kWave), os = __shfl_xor(score, off, kWave);
      const int oa = __shfl_xor(at, off, kWave);
      if (ob > best || (ob == best && oa < at)) {
        best = ob;
        score = os;
        at = oa;
      }
    }
    if (!(best > (double)kNegInf)) break;
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (at == lane + i * kWave) c[i] = (double)kNegInf;
    if (lane == k) {
      my_id = at;
      my_score = score;
    }
  }
  if (a.cfg.renormalise) {
    const double sum = wave_sum(my_score);
    my_score = sum > 0.0 ? my_score / sum : 0.0;
  }
  if (lane < K) {
    const int64_t at = (int64_t)row * K + lane;
    a.ids[at] = my_id;
    a.weights[at] = my_id < 0 ? 0.0f : (float)(my_score * (double)a.cfg.scale);
  }
}

// One wave a row; lane k keeps choice k.  With v the score of the choices and a = scale dweights:
//   renormalised   ds_k = (a_k - sum a v / S) / S,  S = sum v
//   sigmoid        dlogit_k = ds_k v_k (1 - v_k), 0 elsewhere
//   softmax        dlogit_e = s_e (ds_e - sum ds v); renormalised: the softmax over the choices alone.
template <typename T, int EPL>
__global__ __launch_bounds__(256) void k_route_grad(const RouteGradArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = blockIdx.x * 4 + wave;
  if (row >= rows_in_use(a.count, a.n_max)) return;
  const int E = a.n_experts, K = a.cfg.top_k;
  const T *x_row = static_cast<const T *>(a.logits) + (int64_t)row * a.ld;
  int id = -1;
  float d = 0.f, xk = kNegInf;
  if (lane < K) {
    id = a.ids[(int64_t)row * K + lane];
    if (id < 0 || id >= E) id = -1;
    if (id >= 0) {
      d = a.dweights[(int64_t)row * K + lane] * a.cfg.scale;
      xk = (float)x_row[id];
      if (!(xk > kNegInf)) id = -1, xk = kNegInf, d = 0.f;
    }
  }
  const bool softmax = a.cfg.score == AA_SCORE_SOFTMAX, renorm = a.cfg.renormalise != 0;
  float base[EPL];  // what the experts that are not chosen get
  float v;          // this lane's choice
#pragma unroll
  for (int i = 0; i < EPL; ++i) base[i] = 0.f;
  if (softmax && !renorm) {
    float x[EPL], top = kNegInf, sum = 0.f;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      const int e = lane + i * kWave;
      x[i] = e < E ? (float)x_row[e] : kNegInf;
      if (!(x[i] > kNegInf)) x[i] = kNegInf;
      top = fmaxf(top, x[i]);
    }
    top = wave_max(top);
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      x[i] = !(x[i] > kNegInf) ? 0.f : x[i] == top ? 1.f : expf(x[i] - top);
      sum += x[i];
    }
    sum = wave_sum(sum);
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const float sk = id < 0 ? 0.f : xk == top ? inv : expf(xk - top) * inv;
    const float dot = wave_sum(d * sk);
#pragma unroll
    for (int i = 0; i < EPL; ++i) base[i] = -x[i] * inv * dot;
    v = sk * (d - dot);
  } else if (softmax) {
    const float top = wave_max(xk);
    const float ek = id < 0 ? 0.f : xk == top ? 1.f : expf(xk - top);
    const float sum = wave_sum(ek);
    const float wk = sum > 0.f ? ek / sum : 0.f;
    v = wk * (d - wave_sum(d * wk));
  } else {
    const float sk = id < 0 ? 0.f : 1.f / (1.f + expf(-xk));
    const float rest = id < 0 ? 0.f : 1.f / (1.f + expf(xk));  // 1 - sk, without the cancellation
    if (renorm) {
      const float sum = wave_sum(sk);
      const float wk = sum > 0.f ? sk / sum : 0.f;
      v = sum > 0.f ? wk * rest * (d - wave_sum(d * wk)) : 0.f;
    } else {
      v = d * sk * rest;
    }
  }
  T *out = static_cast<T *>(a.dlogits) + (int64_t)row * a.ld_out;
  for (int k = 0; k < K; ++k) {
    const int at = __builtin_amdgcn_readlane(id, k);
    const float vk = lane_read(v, k);
#pragma unroll
    for (int i = 0; i < EPL; ++i)
      if (at == lane + i * kWave) base[i] = vk;
  }
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (lane + i * kWave < E) out[lane + i * kWave] = (T)base[i];
}

// ---- grouping -------------------------------------------------------------------------------------------
// A stable counting sort: counts per tile, then every block adds up what lies before its tile and places
// its pairs.  Ranks inside a wave come from ballots over the bits of the expert's number.
constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanRounds = kPlanTile / kPlanThreads;

__global__ __launch_bounds__(kPlanThreads) void k_plan_counts(const PlanArgs a) {
  __shared__ int hist[kMaxExperts];
  const int E = a.n_experts;
  const int pairs = rows_in_use(a.count, a.n_max) * a.top_k;
  for (int e = threadIdx.x; e < E; e += kPlanThreads) hist[e] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kPlanRounds; ++r) {
    const int p = blockIdx.x * kPlanTile + r * kPlanThreads + threadIdx.x;
    const int e = p < pairs ? a.ids[p] : -1;
    if (e >= 0 && e < E) atomicAdd(&hist[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += kPlanThreads) a.table[(size_t)blockIdx.x * E + e] = hist[e];
}

__global__ __launch_bounds__(kPlanThreads) void k_plan_place(const PlanArgs a, int tiles) {
  __shared__ int place[kPlanWaves][kMaxExperts];  // first the waves' counts, then where their next pair goes
  __shared__ int scan[kPlanWaves + 1];
  const int E = a.n_experts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pairs = rows_in_use(a.count, a.n_max) * a.top_k;
  for (int i = threadIdx.x; i < kPlanWaves * E; i += kPlanThreads) place[i / E][i % E] = 0;
  const int first = blockIdx.x * kPlanTile + wave * (kPlanTile / kPlanWaves);
  int id[kPlanRounds];
#pragma unroll
  for (int r = 0; r < kPlanRounds; ++r) {
    const int p = first + r * kWave + lane;
    id[r] = p < pairs ? a.ids[p] : -1;
    if (id[r] >= E) id[r] = -1;
  }
  int before = 0, all = 0;  // of expert threadIdx.x
  if ((int)threadIdx.x < E)
    for (int t = 0; t < tiles; ++t) {
      const int c = a.table[(size_t)t * E + threadIdx.x];
      all += c;
      before += t < (int)blockIdx.x ? c : 0;
    }
  int total;
  const int start = block_exclusive_scan(all, scan, &total);  // (its barriers: `place` is cleared)
  if (blockIdx.x == 0) {
    if ((int)threadIdx.x < E) a.offsets[threadIdx.x] = start;
    if (threadIdx.x == 0) a.offsets[E] = total;
  }
#pragma unroll
  for (int r = 0; r < kPlanRounds; ++r)
    if (id[r] >= 0) atomicAdd(&place[wave][id[r]], 1);
  __syncthreads();
  if ((int)threadIdx.x < E) {
    int run = start + before;
    for (int w = 0; w < kPlanWaves; ++w) {
      const int c = place[w][threadIdx.x];
      place[w][threadIdx.x] = run;
      run += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kPlanRounds; ++r) {
    const int p = first + r * kWave + lane;
    unsigned long long same = __ballot(id[r] >= 0);
    for (int b = 1; b < E; b <<= 1) {
      const unsigned long long set = __ballot((id[r] & b) != 0);
      same &= (id[r] & b) ? set : ~set;
    }
    if (id[r] >= 0) {
      const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0u));
      const int at = place[wave][id[r]] + rank;
      wave_sync();
      if (rank == 0) place[wave][id[r]] = at + __popcll(same);
      wave_sync();
      a.order[at] = p;
      a.slot[p] = at;
    } else if (p < pairs) {
      a.slot[p] = -1;
    }
  }
}

template <typename T>
hipError_t route_by_width(const RouteArgs &a, hipStream_t st) {
  const dim3 grid((a.n_max + 3) / 4), block(256);
  const int E = a.n_experts;
  if (E <= 64) hipLaunchKernelGGL((k_route<T, 1>), grid, block, 0, st, a);
  else if (E <= 128) hipLaunchKernelGGL((k_route<T, 2>), grid, block, 0, st, a);
  else if (E <= 256) hipLaunchKernelGGL((k_route<T, 4>), grid, block, 0, st, a);
  else if (E <= 512) hipLaunchKernelGGL((k_route<T, 8>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_route<T, 16>), grid, block, 0, st, a);
  return hipGetLastError();
}

template <typename T>
hipError_t route_grad_by_width(const RouteGradArgs &a, hipStream_t st) {
  const dim3 grid((a.n_max + 3) / 4), block(256);
  const int E = a.n_experts;
  if (E <= 64) hipLaunchKernelGGL((k_route_grad<T, 1>), grid, block, 0, st, a);
  else if (E <= 128) hipLaunchKernelGGL((k_route_grad<T, 2>), grid, block, 0, st, a);
  else if (E <= 256) hipLaunchKernelGGL((k_route_grad<T, 4>), grid, block, 0, st, a);
  else if (E <= 512) hipLaunchKernelGGL((k_route_grad<T, 8>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_route_grad<T, 16>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_route(const RouteArgs &a, int32_t dtype, hipStream_t st) {
  if (a.n_max == 0) return hipSuccess;
  if (dtype == AA_BF16) return route_by_width<__bf16>(a, st);
  if (dtype == AA_F16) return route_by_width<_Float16>(a, st);
  return route_by_width<float>(a, st);
}

hipError_t launch_route_grad(const RouteGradArgs &a, int32_t dtype, hipStream_t st) {
  if (a.n_max == 0) return hipSuccess;
  if (dtype == AA_BF16) return route_grad_by_width<__bf16>(a, st);
  if (dtype == AA_F16) return route_grad_by_width<_Float16>(a, st);
  return route_grad_by_width<float>(a, st);
}

hipError_t launch_expert_plan(const PlanArgs &a, hipStream_t st) {
  const int tiles = (int)(((int64_t)a.n_max * a.top_k + kPlanTile - 1) / kPlanTile);
  if (tiles > 0) {
    hipLaunchKernelGGL(k_plan_counts, dim3(tiles), dim3(kPlanThreads), 0, st, a);
    if (hipGetLastError() != hipSuccess) return hipErrorLaunchFailure;
  }
  hipLaunchKernelGGL(k_plan_place, dim3(tiles > 0 ? tiles : 1), dim3(kPlanThreads), 0, st, a, tiles);
  return hipGetLastError();
}

}  // namespace aa

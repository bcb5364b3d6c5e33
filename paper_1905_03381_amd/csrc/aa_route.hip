// Routing of rows to experts, its gradient, and the grouping of the (row, choice) pairs by expert.
//
// A row's logits are held in registers, neighbouring experts in a lane, so that a tie's lowest index is the lowest lane's
// first.  What is exchanged between lanes goes over the vector units' own paths (LDS permutes took 124 us of a call that
// takes 36 now, 9 of it the plan: 16,384 rows, 256 experts in 8 groups, 8 choices).  Bound by instructions: a turn of
// the choice is a maximum over a lane's experts and over the lanes, scores are exponentials in 64 bits; reading the logits is
// a small part (of 65,536 rows of 128 experts 15 us, 2.3 TB/s, without a bias, 33 with one).
#include "aa_route_lanes.hpp"

#include <type_traits>

namespace aa {

namespace {

// exp(v) of v <= 0 in 64 bits, 0 far below: v = n ln 2 + r, |r| <= ln 2 / 2, and the power series of e^r to r^13 (the
// next term is below 2^-57).  Half the instructions of the library's, which serves all of the range.
__device__ __forceinline__ double exp_below(double v) {
  constexpr double kTerms[12] = {1.0 / 6227020800, 1.0 / 479001600, 1.0 / 39916800, 1.0 / 3628800, 1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720, 1.0 / 120, 1.0 / 24, 1.0 / 6, 1.0 / 2};
  v = v > -800.0 ? v : -800.0;
  const double n = rint(v * 1.4426950408889634);
  const double r = fma(-n, 2.3190468138462996e-17, fma(-n, 0.6931471805599453, v));
  double p = kTerms[0];
#pragma unroll
  for (int i = 1; i < 12; ++i) p = fma(p, r, kTerms[i]);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  return ldexp(p, (int)n);
}

// 1 / v for 1 <= v <= 2, by Newton's steps.
__device__ __forceinline__ double reciprocal(double v) {
  double r = __builtin_amdgcn_rcp(v);
  r = fma(fma(-v, r, 1.0), r, r);
  return fma(fma(-v, r, 1.0), r, r);
}

// 1 / (1 + e^-v), without overflow and without cancellation on either side.
__device__ __forceinline__ double sigmoid64(double v) {
  const double t = exp_below(v > 0.0 ? -v : v), r = reciprocal(1.0 + t);
  return v > 0.0 ? r : t * r;
}

// What the lanes of a row tell each other.
template <int LPR>
struct Choices {
  static constexpr int kMost = LPR == 16 ? 16 : kMaxChoices;
  int id[kWave / LPR][kMost];
};

// Takes the experts of groups that are not among the row's top_groups out of c.  A group's value is the sum of its
// group_best largest.  Groups of whole lanes, as many as a power of two.
template <int LPR, int EPL>
__device__ __forceinline__ void leave_groups(const RouteArgs &a, int sub, double *c) {
  const int G = a.cfg.n_groups;
  const double none = (double)kNegInf;
  const bool two = a.cfg.group_best == 2;
  const int lanes = a.n_experts / G / EPL;  // of a group
  double first = none, second = none;
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    second = fmax(second, fmin(first, c[i]));
    first = fmax(first, c[i]);
  }
  const auto join = [&](double f1, double s1, double f2, double s2) {
    second = fmax(fmax(s1, s2), fmin(f1, f2));
    first = fmax(f1, f2);
  };
  if (lanes > 1) join(first, second, lane_move<0xB1>(first), lane_move<0xB1>(second));
  if (lanes > 2) join(first, second, lane_move<0x4E>(first), lane_move<0x4E>(second));
  if (lanes > 4) join(first, second, lane_move<0x141>(first), lane_move<0x141>(second));
  if (lanes > 8) join(first, second, lane_move<0x140>(first), lane_move<0x140>(second));
  if constexpr (LPR == 64) {
    double f1, s1, f2, s2;
    if (lanes > 16) {
      exchange<false>(first, &f1, &f2);
      exchange<false>(second, &s1, &s2);
      join(f1, s1, f2, s2);
    }
    if (lanes > 32) {
      exchange<true>(first, &f1, &f2);
      exchange<true>(second, &s1, &s2);
      join(f1, s1, f2, s2);
    }
  }
  const double v = two && second > none ? first + second : first;
  const int g = sub / lanes;
  int rank = 0;
  for (int q = 0; q < G; ++q) {
    double o;
    if constexpr (LPR == 64)
      o = __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), q * lanes),
                           __builtin_amdgcn_readlane(__double2loint(v), q * lanes));
    else
      o = __shfl(v, q * lanes, LPR);
    rank += (o > v || (o == v && q < g)) ? 1 : 0;
  }
  if (rank >= a.cfg.top_groups) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) c[i] = none;
  }
}

// The same for groups of any size: a lane takes a group, through LDS.
template <int LPR, int EPL>
__device__ __forceinline__ void leave_any_groups(const RouteArgs &a, int sub, double *room, double *c) {
  const int E = a.n_experts, G = a.cfg.n_groups, size = E / G;
  const double none = (double)kNegInf;
  const bool two = a.cfg.group_best == 2;
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (sub * EPL + i < E) room[sub * EPL + i] = c[i];
  wave_sync();
  double v[EPL];  // of group sub + i LPR
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int g = sub + i * LPR;
    double first = none, second = none;
    if (g < G) {
      for (int q = 0; q < size; ++q) {
        const double o = room[g * size + q];
        second = fmax(second, fmin(first, o));
        first = fmax(first, o);
      }
    }
    v[i] = two && second > none ? first + second : first;
  }
  wave_sync();
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (sub + i * LPR < G) room[sub + i * LPR] = v[i];
  wave_sync();
  bool taken[EPL];
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int g = sub + i * LPR;
    int rank = 0;
    for (int q = 0; q < G; ++q) {
      const double o = room[q];
      rank += (o > v[i] || (o == v[i] && q < g)) ? 1 : 0;
    }
    taken[i] = rank < a.cfg.top_groups;
  }
  wave_sync();
#pragma unroll
  for (int i = 0; i < EPL; ++i)
    if (sub + i * LPR < G) room[sub + i * LPR] = taken[i] ? 1.0 : 0.0;
  wave_sync();
#pragma unroll
  for (int i = 0; i < EPL; ++i) {
    const int e = sub * EPL + i;
    if (e < E && room[e / size] == 0.0) c[i] = none;
  }
  wave_sync();  // (room is the next row's)
}

// What a choice goes by: the logits; scores, with a bias or groups of whole lanes; groups of any size.
enum By { kByLogit, kByScore, kByAnyGroups };

// One row, by LPR lanes of EPL neighbouring experts each (live: there is one).  Scores are doubles.  With a bias or
// groups so are the choice values: near scores are told apart as the formulas have them.  Without, the order is that
// of the logits, also where scores round to one value.  The turns of the choice go by 32 bits of each value, whose order is
// the same but for ties; experts that tie in them are computed again and compared in 64.
template <int LPR, int EPL, By BY>
__device__ __forceinline__ void route_row(const RouteArgs &a, int row, bool live, int lane, Choices<LPR> &ch, double *room) {
  const int sub = lane % LPR, in_wave = lane / LPR, e0 = sub * EPL;
  const int E = a.n_experts, K = a.cfg.top_k;
  const bool softmax = a.cfg.score == AA_SCORE_SOFTMAX, renorm = a.cfg.renormalise != 0;
  const int64_t from = (int64_t)row * a.ld;
  float x[EPL];
  if (live) {
    load_logits<EPL>(a.logits, a.dtype, from, e0, E, a.vec, x);
  } else {
#pragma unroll
    for (int i = 0; i < EPL; ++i) x[i] = kNegInf;
  }
  float top = kNegInf;
  if (softmax) {
#pragma unroll
    for (int i = 0; i < EPL; ++i) top = fmaxf(top, x[i]);
    top = lanes_max<LPR>(top);
  }
  // (+inf - +inf: those that are +inf share the whole)
  const auto raw = [&](float v) {
    if (!(v > kNegInf)) return 0.0;
    if (!softmax) return sigmoid64((double)v);
    return v == top ? 1.0 : exp_below((double)v - (double)top);
  };
  double inv = 1.0;
  const auto value = [&](float v, double score, int e) {
    const double c = score + (a.bias ? (double)a.bias[e] : 0.0);
    return v > kNegInf && c > (double)kNegInf ? c : (double)kNegInf;
  };
  float c[EPL];
  if constexpr (BY != kByLogit) {
    double s[EPL];
    double part = 0.0;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      s[i] = raw(x[i]);
      part += s[i];
    }
    if (softmax) {
      part = lanes_sum<LPR>(part);
      inv = part > 0.0 ? 1.0 / part : 0.0;
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) s[i] = value(x[i], s[i] * inv, min(e0 + i, E - 1));
    if constexpr (BY == kByAnyGroups) leave_any_groups<LPR, EPL>(a, sub, room, s);
    else if (a.cfg.n_groups > 1) leave_groups<LPR, EPL>(a, sub, s);
#pragma unroll
    for (int i = 0; i < EPL; ++i) c[i] = (float)s[i];
  } else {
    if (softmax && !renorm) {
      double part = 0.0;
#pragma unroll
      for (int i = 0; i < EPL; ++i) part += raw(x[i]);
      part = lanes_sum<LPR>(part);
      inv = part > 0.0 ? 1.0 / part : 0.0;
    }
#pragma unroll
    for (int i = 0; i < EPL; ++i) c[i] = x[i];
  }
  const auto of_row = [&](unsigned long long wave) {
    return LPR < kWave ? (wave >> (in_wave * LPR)) & ((1ull << (LPR & 63)) - 1ull) : wave;
  };
  int got = 0;
  for (int k = 0; k < K; ++k) {
    float all = c[0];
#pragma unroll
    for (int i = 1; i < EPL; ++i) all = larger(all, c[i]);
    all = lanes_max<LPR>(all);
    uint32_t held = 0;  // bit i: this lane's expert i has the largest value
#pragma unroll
    for (int i = 0; i < EPL; ++i) held |= c[i] == all ? 1u << i : 0u;
    if (!(all > kNegInf)) held = 0;
    unsigned long long wave = __ballot(held != 0);
    if (wave == 0ull) break;
    if constexpr (BY != kByLogit) {
      if (__any(__popcll(of_row(wave)) > 1 || (held & (held - 1)) != 0)) {
        double best = (double)kNegInf;
        int at = 0;
        for (uint32_t left = held; left != 0; left &= left - 1) {
          const int i = __ffs((int)left) - 1;
          float v;
          load_logits<1>(a.logits, a.dtype, from, e0 + i, E, false, &v);
          const double exact = value(v, raw(v) * inv, e0 + i);
          if (exact > best) best = exact, at = i;
        }
        const double most = lanes_max<LPR>(best);
        held = held != 0 && best == most ? 1u << at : 0u;
        wave = __ballot(held != 0);
      }
    }
    const unsigned long long who = of_row(wave);
    got += who != 0ull ? 1 : 0;
    if (sub != __ffsll((long long)who) - 1) held = 0;
    const int at = __ffs((int)held) - 1;  // (-1: the lowest lane that holds it is another)
    if (at >= 0) ch.id[in_wave][k] = e0 + at;
#pragma unroll
    for (int i = 0; i < EPL; ++i) c[i] = i == at ? kNegInf : c[i];
  }
  wave_sync();
  double score = 0.0;
  int id = -1;
  if (sub < got) {
    id = ch.id[in_wave][sub];
    float v;
    load_logits<1>(a.logits, a.dtype, from, id, E, false, &v);
    score = raw(v) * inv;
  }
  wave_sync();  // (the room is the next row's)
  if (renorm) {
    const double all = lanes_sum<LPR>(score);
    score = all > 0.0 ? score / all : 0.0;
  }
  if (live && sub < K) {
    const int64_t to = (int64_t)row * K + sub;
    a.ids[to] = id;
    a.weights[to] = id < 0 ? 0.0f : (float)(score * (double)a.cfg.scale);
  }
}

template <int LPR, int EPL, By BY>
__global__ __launch_bounds__(256) void k_route(const RouteArgs a) {
  constexpr int kRows = kWave / LPR;  // a wave at once
  extern __shared__ double room[];   // [rows of the block][E] (kByAnyGroups)
  __shared__ Choices<LPR> choices[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rows = rows_in_use(a.count, a.n_max);
  for (int64_t base = ((int64_t)blockIdx.x * 4 + wave) * kRows; base < rows; base += (int64_t)gridDim.x * 4 * kRows) {
    const int64_t row = base + lane / LPR;
    route_row<LPR, EPL, BY>(a, (int)row, row < rows, lane, choices[wave],
                            BY == kByAnyGroups ? room + (wave * kRows + lane / LPR) * a.n_experts : nullptr);
  }
}

// LPR lanes a row, EPL neighbouring experts each; lane k keeps choice k.  With v the score of the choices and
// a = scale dweights:
//   renormalised   ds_k = (a_k - sum a v / S) / S,  S = sum v
//   sigmoid        dlogit_k = ds_k v_k (1 - v_k), 0 elsewhere
//   softmax        dlogit_e = s_e (ds_e - sum ds v); renormalised: the softmax over the choices alone.
template <int LPR, int EPL>
__global__ __launch_bounds__(256) void k_route_grad(const RouteGradArgs a) {
  constexpr int kRows = kWave / LPR;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % LPR, e0 = sub * EPL;
  const int rows = rows_in_use(a.count, a.n_max);
  const int E = a.n_experts, K = a.cfg.top_k;
  const bool softmax = a.cfg.score == AA_SCORE_SOFTMAX, renorm = a.cfg.renormalise != 0;
  for (int64_t base = ((int64_t)blockIdx.x * 4 + wave) * kRows; base < rows; base += (int64_t)gridDim.x * 4 * kRows) {
    const int64_t row = base + lane / LPR;
    const bool live = row < rows;
    float x[EPL];
    if (live && softmax) load_logits<EPL>(a.logits, a.dtype, row * a.ld, e0, E, a.vec, x);
    int id = -1;
    float d = 0.f, xk = kNegInf;
    if (live && sub < K) {
      id = a.ids[row * K + sub];
      d = a.dweights[row * K + sub] * a.cfg.scale;
      if (id < 0 || id >= E) id = -1;
      if (id >= 0) load_logits<1>(a.logits, a.dtype, row * a.ld, id, E, false, &xk);
      if (!(xk > kNegInf)) id = -1, d = 0.f;
    }
    float base_[EPL];  // what the experts that are not chosen get
    float v;           // this lane's choice
#pragma unroll
    for (int i = 0; i < EPL; ++i) base_[i] = 0.f;
    float top = kNegInf;  // of the row
    if (softmax) {
      if (!live) {
#pragma unroll
        for (int i = 0; i < EPL; ++i) x[i] = kNegInf;
      }
#pragma unroll
      for (int i = 0; i < EPL; ++i) top = fmaxf(top, x[i]);
      top = lanes_max<LPR>(top);
    }
    if (softmax && !renorm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        x[i] = !(x[i] > kNegInf) ? 0.f : x[i] == top ? 1.f : expf(x[i] - top);
        sum += x[i];
      }
      sum = lanes_sum<LPR>(sum);
      const float inv = sum > 0.f ? 1.f / sum : 0.f;
      const float sk = id < 0 ? 0.f : xk == top ? inv : expf(xk - top) * inv;
      const float dot = lanes_sum<LPR>(d * sk);
#pragma unroll
      for (int i = 0; i < EPL; ++i) base_[i] = -x[i] * inv * dot;
      v = sk * (d - dot);
    } else if (softmax) {
      // Choices whose scores are 0 beside the row's others (a bias may choose masked experts alone) have no weights, and so no
      // gradient.  The row is read for that (65,536 rows of 64 experts, 8 choices 9.5 -> 10.7 us, 60,001 of 128 12.6 -> 16.0).
      const float best = lanes_max<LPR>(xk);
      const float ek = id < 0 ? 0.f : xk == best ? 1.f : expf(xk - best);
      const float sum = lanes_sum<LPR>(ek);
      const float wk = sum > 0.f && (best == top || best - top > kNoScore) ? ek / sum : 0.f;
      v = wk * (d - lanes_sum<LPR>(d * wk));
    } else {
      // With t = e^-|x| the score is e^min(x, 0) / (1 + t) and 1 - score, without the cancellation, t / (1 + t) or 1 / (1 + t).
      const float low = fminf(xk, 0.f), t = expf(-fabsf(xk)), r = 1.f / (1.f + t);
      const float rest = xk > 0.f ? t * r : r;
      if (renorm) {
        // Scores relative to the highest choice's e^min(x, 0): in 32 bits those of logits below -88 would all be 0.  (Where
        // they are 0 in k_route's 64 bits, so are the weights.)
        const float top = lanes_max<LPR>(low);
        const float sk = id < 0 ? 0.f : expf(low - top) * r;
        const float sum = lanes_sum<LPR>(sk);
        const float wk = top > kNoScore ? sk / sum : 0.f;
        v = wk * rest * (d - lanes_sum<LPR>(d * wk));
      } else {
        v = id < 0 ? 0.f : d * (xk > 0.f ? r : t * r) * rest;
      }
    }
    for (int k = 0; k < K; ++k) {
      const int at = __shfl(id, k, LPR) - e0;
      const float vk = __shfl(v, k, LPR);
#pragma unroll
      for (int i = 0; i < EPL; ++i)
        if (at == i) base_[i] = vk;
    }
    if (live) {
      const int64_t to = row * a.ld_out;
      if (a.dtype == AA_BF16) store_logits<__bf16, EPL>(static_cast<__bf16 *>(a.dlogits) + to, e0, E, a.vec, base_);
      else if (a.dtype == AA_F16) store_logits<_Float16, EPL>(static_cast<_Float16 *>(a.dlogits) + to, e0, E, a.vec, base_);
      else store_logits<float, EPL>(static_cast<float *>(a.dlogits) + to, e0, E, a.vec, base_);
    }
  }
}

// ---- grouping -------------------------------------------------------------------------------------------
// A stable counting sort: counts per tile, then every block adds up what lies before its tile and places
// its pairs.  Ranks inside a wave come from ballots over the bits of the expert's number.  A single tile counts for itself.
// What every block adds up grows with the square of the tiles: from tiles^2 E = kScanFrom on a launch between does it once.
// (8 choices; with and without: 64 experts 512 tiles 16.5 and 16.4 us, 2048 tiles 41 and 83; 256 experts 256 tiles 15.4 and
// 14.4, 2048 tiles 48 and 245; 1024 experts 64 tiles 13.5 and 13.3, 2048 tiles 67 and 883.)
constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / kWave;
constexpr int kPlanRounds = kPlanTile / kPlanThreads;
constexpr int64_t kScanFrom = 1 << 24;

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

// Turns the tiles' counts into those of all tiles before each, the totals behind the last: kScanExperts experts a block, its
// threads a share of the tiles each.
constexpr int kScanExperts = 16;
constexpr int kScanShares = kPlanThreads / kScanExperts;

__global__ __launch_bounds__(kPlanThreads) void k_plan_scan(const PlanArgs a, int tiles) {
  __shared__ int sums[kScanShares][kScanExperts];
  const int E = a.n_experts, in_block = threadIdx.x % kScanExperts, share = threadIdx.x / kScanExperts;
  const int e = blockIdx.x * kScanExperts + in_block, each = (tiles + kScanShares - 1) / kScanShares;
  const int from = min(share * each, tiles), to = e < E ? min(from + each, tiles) : from;
  int *column = a.table + e;
  int sum = 0;
#pragma unroll 8
  for (int t = from; t < to; ++t) sum += column[(size_t)t * E];
  sums[share][in_block] = sum;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int s = 0; s < kScanShares; ++s) {
    const int v = sums[s][in_block];
    all += v;
    before += s < share ? v : 0;
  }
  for (int t0 = from; t0 < to; t0 += 8) {  // (eight counts are asked for before the first is used)
    int c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = column[(size_t)min(t0 + i, to - 1) * E];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (t0 + i < to) column[(size_t)(t0 + i) * E] = before;
      before += c[i];
    }
  }
  if (share == 0 && e < E) column[(size_t)tiles * E] = all;
}

// The pairs of tile `tile` of `tiles`, by a block of kPlanThreads; MOST: experts there is room for; SCANNED: the table holds
// what k_plan_scan made of it.
template <int MOST, bool SCANNED>
__device__ __forceinline__ void place_tile(const PlanArgs &a, int tile, int tiles) {
  __shared__ int place[kPlanWaves][MOST];  // first the waves' counts, then where their next pair goes
  __shared__ int totals[2][MOST];          // of all tiles, of those before this one
  __shared__ int scan[kPlanWaves + 1];
  const int E = a.n_experts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pairs = rows_in_use(a.count, a.n_max) * a.top_k;
  for (int e = lane; e < E; e += kWave) place[wave][e] = 0;
  if ((int)threadIdx.x < E) totals[0][threadIdx.x] = totals[1][threadIdx.x] = 0;
  const int first = tile * kPlanTile + wave * (kPlanTile / kPlanWaves);
  int id[kPlanRounds];
#pragma unroll
  for (int r = 0; r < kPlanRounds; ++r) {
    const int p = first + r * kWave + lane;
    id[r] = p < pairs ? a.ids[p] : -1;
    if (id[r] >= E) id[r] = -1;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kPlanRounds; ++r)
    if (id[r] >= 0) atomicAdd(&place[wave][id[r]], 1);
  if constexpr (SCANNED) {
    if ((int)threadIdx.x < E) {
      totals[0][threadIdx.x] = a.table[(size_t)tiles * E + threadIdx.x];
      totals[1][threadIdx.x] = a.table[(size_t)tile * E + threadIdx.x];
    }
  } else if (tiles > 1) {
    // kPlanThreads / E threads an expert, each a share of the tiles
    const int shares = kPlanThreads / E, e = threadIdx.x % E, share = threadIdx.x / E;
    if (share < shares) {
      int before = 0, all = 0;
#pragma unroll 8
      for (int t = share; t < tiles; t += shares) {
        const int c = a.table[(size_t)t * E + e];
        all += c;
        before += t < tile ? c : 0;
      }
      atomicAdd(&totals[0][e], all);
      atomicAdd(&totals[1][e], before);
    }
  }
  __syncthreads();
  int all = 0;
  if ((int)threadIdx.x < E) {
    all = totals[0][threadIdx.x];
    if (tiles <= 1) {
#pragma unroll
      for (int w = 0; w < kPlanWaves; ++w) all += place[w][threadIdx.x];
    }
  }
  int total;
  const int start = block_exclusive_scan(all, scan, &total);
  if (tile == 0) {
    if ((int)threadIdx.x < E) a.offsets[threadIdx.x] = start;
    if (threadIdx.x == 0) a.offsets[E] = total;
  }
  if ((int)threadIdx.x < E) {
    int run = start + totals[1][threadIdx.x];
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

template <bool SCANNED>
__global__ __launch_bounds__(kPlanThreads) void k_plan_place(const PlanArgs a, int tiles) {
  place_tile<kMaxExperts, SCANNED>(a, blockIdx.x, tiles);
}

// Routing and plan of a few rows by one block: a launch instead of two.
template <int LPR, int EPL, By BY>
__global__ __launch_bounds__(kPlanThreads) void k_route_few(const RouteArgs a, const PlanArgs p) {
  constexpr int kRows = kWave / LPR;
  __shared__ Choices<LPR> choices[kPlanWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rows = rows_in_use(a.count, a.n_max);
  for (int base = wave * kRows; base < rows; base += kPlanWaves * kRows) {
    const int row = base + lane / LPR;
    route_row<LPR, EPL, BY>(a, row, row < rows, lane, choices[wave], nullptr);
  }
  __syncthreads();  // (the ids are written)
  place_tile<LPR * EPL, false>(p, 0, 1);
}

// No groups, or each of whole lanes, as many as a power of two.
bool groups_of_lanes(const RouteArgs &a, int epl) {
  const int size = a.n_experts / a.cfg.n_groups, lanes = size / epl;
  return a.cfg.n_groups == 1 || (size % epl == 0 && (lanes & (lanes - 1)) == 0);
}

}  // namespace

hipError_t launch_route(const RouteArgs &args, const PlanArgs *plan, hipStream_t st) {
  RouteArgs a = args;
  if (a.n_max == 0) return plan ? launch_expert_plan(*plan, st) : hipSuccess;
  bool planned = false;
  const bool by_score = a.bias || a.cfg.n_groups > 1;
  // Beyond 128 experts 16 lanes hold 16 each.  By logits that is better at any size (16,384 rows, 256 experts, 4 choices
  // 7.7 us, a wave a row 11.5); by scores it takes many registers, and rows that fill the chip (8 groups, 8 choices:
  // 16,384 rows 25.9 and 30.5 us, 4096 rows 12.1 and 11.0); groups of any size are worse (65,536 rows of 200 311 and 160).
  const bool many = !by_score || (a.n_max >= 8192 && groups_of_lanes(a, 16));
  const hipError_t e = by_width(a.n_experts, a.cfg.top_k, many ? 256 : 128, [&](auto lpr, auto epl) {
    constexpr int LPR = decltype(lpr)::value, EPL = decltype(epl)::value, kRows = kWave / LPR;
    a.vec = whole_lanes(a.logits, a.ld, a.n_experts, EPL, a.dtype);
    const bool any_groups = !groups_of_lanes(a, EPL);
    if constexpr (LPR * EPL <= 256 && EPL <= 8) {
      // Rows that its waves take at once: 1 to 64 rows, 64 experts, 6 choices 7.9 to 8.2 us, as two launches 10.5; 128
      // rows 11.0 and 10.5.  A wave a row: half as many (256 experts in groups with a bias, 5 rows 9.9 and 11.4 us, 16
      // rows 12.6 and 11.6).
      if (plan && !any_groups && (int64_t)a.n_max * a.cfg.top_k <= kPlanTile && a.n_max <= (LPR == 16 ? 64 : 8)) {
        planned = true;
        if (by_score)
          hipLaunchKernelGGL((k_route_few<LPR, EPL, kByScore>), dim3(1), dim3(kPlanThreads), 0, st, a, *plan);
        else
          hipLaunchKernelGGL((k_route_few<LPR, EPL, kByLogit>), dim3(1), dim3(kPlanThreads), 0, st, a, *plan);
        return hipGetLastError();
      }
    }
    const dim3 grid = blocks_for(a.n_max, 4 * kRows), block(256);
    const size_t room = (size_t)4 * kRows * a.n_experts * sizeof(double);
    if (any_groups) {
      if constexpr (LPR * EPL < 256 || LPR == 64) hipLaunchKernelGGL((k_route<LPR, EPL, kByAnyGroups>), grid, block, room, st, a);
    } else if (by_score) hipLaunchKernelGGL((k_route<LPR, EPL, kByScore>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_route<LPR, EPL, kByLogit>), grid, block, 0, st, a);
    return hipGetLastError();
  });
  if (e != hipSuccess || !plan || planned) return e;
  return launch_expert_plan(*plan, st);
}

hipError_t launch_route_grad(const RouteGradArgs &args, hipStream_t st) {
  RouteGradArgs a = args;
  if (a.n_max == 0) return hipSuccess;
  return by_width(a.n_experts, a.cfg.top_k, 128, [&](auto lpr, auto epl) {
    constexpr int LPR = decltype(lpr)::value, EPL = decltype(epl)::value;
    a.vec = whole_lanes(a.logits, a.ld, a.n_experts, EPL, a.dtype) &&
            whole_lanes(a.dlogits, a.ld_out, a.n_experts, EPL, a.dtype);
    hipLaunchKernelGGL((k_route_grad<LPR, EPL>), blocks_for(a.n_max, 4 * (kWave / LPR)), dim3(256), 0, st, a);
    return hipGetLastError();
  });
}

hipError_t launch_expert_plan(const PlanArgs &a, hipStream_t st) {
  const int tiles = (int)(((int64_t)a.n_max * a.top_k + kPlanTile - 1) / kPlanTile);
  const dim3 block(kPlanThreads);
  if (tiles > 1) {
    hipLaunchKernelGGL(k_plan_counts, dim3(tiles), block, 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if ((int64_t)tiles * tiles * a.n_experts > kScanFrom) {
    hipLaunchKernelGGL(k_plan_scan, dim3((a.n_experts + kScanExperts - 1) / kScanExperts), block, 0, st, a, tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k_plan_place<true>, dim3(tiles), block, 0, st, a, tiles);
  } else {
    hipLaunchKernelGGL(k_plan_place<false>, dim3(tiles > 0 ? tiles : 1), block, 0, st, a, tiles);
  }
  return hipGetLastError();
}

}  // namespace aa

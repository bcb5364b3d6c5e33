// One AdamW update of many tensors, and the norm of all their gradients.
//
// The tensors are cut into chunks of 2048 elements, listed once in a table on the device; a launch walks all of them, each block a
// run of neighbouring chunks, eight neighbouring elements a thread.  Bound by memory: 28 to 30 bytes an element with
// states in 32 bits, 16 to 18 with states in 8 (25.2 M elements, 32-bit states and gradients, 16-bit copies: 155 us, 4.9 TB/s; 46 M,
// 8-bit states, 16-bit gradients: 165 to 171, where the draws and the conversions also count: 38 M vector instructions).
//
// States in 8 bits: 256 neighbours share a power of two that brings their largest into [128, 256), and each is held
// as an e4m3 number (steps of an eighth to a sixteenth of it, down to 2^-17 of the largest).  v is held as its root, so
// that its range is twice that, and never as 0 where it is above: the denominator then errs to the safe side.  A
// state moves by 1 - beta a step, for v a thousandth, far less than half a step of the format: rounded to the nearest it would
// stay where it is for good.  So it is rounded at random, up as often as the fraction says, with 16-bit draws of the generator
// the keep draws use; its mean is then right.  m and v of an element share a draw.
#include "aa_adamw.hpp"

#include "aa_lines.hpp"

#include <type_traits>

namespace aa {

namespace {

constexpr int kBatch = 32;   // entries that travel as arguments of one launch

struct EntryBatch {
  TensorEntry e[kBatch];
};

// Entries [first, first + gridDim.x) of the table and the chunks that belong to them.
__global__ __launch_bounds__(256) void k_adamw_table(char *table, int64_t map, int64_t n_chunks, int32_t n, int32_t first,
                                                     const EntryBatch batch) {
  const TensorEntry e = batch.e[blockIdx.x];
  const int32_t tensor = first + (int32_t)blockIdx.x;
  if (threadIdx.x == 0) reinterpret_cast<TensorEntry *>(table + kTableEntries)[tensor] = e;
  if (tensor == 0)
    for (int w = threadIdx.x; w < kControlWords; w += 256) reinterpret_cast<int32_t *>(table)[w] = w == 0 ? (int32_t)n_chunks : w == 1 ? n : 0;
  int32_t *of = reinterpret_cast<int32_t *>(table + map) + e.first_chunk;
  const int64_t chunks = (e.n + kChunk - 1) / kChunk;
  for (int64_t c = threadIdx.x; c < chunks; c += 256) of[c] = tensor;
}

// Global memory, which a pointer that was itself read from memory does not say (memory of any kind is slower to ask for,
// and what waits for LDS then waits for it).
template <typename T>
using Global = __attribute__((address_space(1))) T *;

// Eight elements at p of which n (at least one) exist, the others 0.  PASSING: past the caches, where the tensors are more
// than they hold (25 M elements, states in 32 and gradients in 32 bits, with the norm 183 -> 178 us; 46 M, 8 and 16: 206 -> 189).
template <bool PASSING, typename T>
__device__ __forceinline__ Eight load_some(const T *p, int n) {
  const Global<const T> g = (Global<const T>)p;
  Eight o;
  if (n >= 8) {
    Line<T> t;
    if constexpr (PASSING) t = __builtin_nontemporal_load((Global<const Line<T>>)p);
    else t = *(Global<const Line<T>>)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = (float)t[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = i < n ? (float)g[i] : 0.f;
  }
  return o;
}

template <bool PASSING, typename T>
__device__ __forceinline__ void store_some(T *p, const Eight &o, int n) {
  const Global<T> g = (Global<T>)p;
  if (n >= 8) {
    Line<T> t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)o.v[i];
    if constexpr (PASSING) __builtin_nontemporal_store(t, (Global<Line<T>>)p);
    else *(Global<Line<T>>)p = t;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) g[i] = (T)o.v[i];
  }
}

// Gradients i .. i + 7 of a tensor, of which n (at least one) exist.
template <bool PASSING>
__device__ __forceinline__ Eight load_grad(const TensorEntry &e, int64_t i, int n) {
  if (e.grad_dtype == AA_BF16) return load_some<PASSING>(static_cast<const __bf16 *>(e.grad) + i, n);
  if (e.grad_dtype == AA_F16) return load_some<PASSING>(static_cast<const _Float16 *>(e.grad) + i, n);
  return load_some<PASSING>(static_cast<const float *>(e.grad) + i, n);
}

// Whether the call's numbers are the table's.
__device__ __forceinline__ bool is_table(const AdamWArgs &a) {
  const int32_t *numbers = reinterpret_cast<const int32_t *>(a.table);
  return numbers[0] == (int32_t)a.n_chunks && numbers[1] == a.n_tensors;
}

// Calls work(tensor's number, its entry, first and last element) for the parts of tensors in this block's chunks, a run of
// neighbouring ones: what is known of a tensor is asked for once a part.  ours: is_table().
template <typename Work>
__device__ __forceinline__ void walk(const AdamWArgs &a, bool ours, Work work) {
  const uint32_t all = (uint32_t)a.n_chunks, each = all / gridDim.x, more = all % gridDim.x;
  const int64_t begin = (int64_t)each * blockIdx.x + min(blockIdx.x, more);
  const int64_t end = begin + each + (blockIdx.x < more ? 1 : 0);
  for (int64_t c = begin; c < end;) {
    const int of_chunk = reinterpret_cast<const int32_t *>(a.table + a.map)[c];
    if (!ours) return;  // (nothing is walked; known only after the first tensor has been asked for)
    const int tensor = __builtin_amdgcn_readfirstlane(of_chunk);
    const TensorEntry &e = reinterpret_cast<const TensorEntry *>(a.table + kTableEntries)[tensor];
    const int64_t next = e.first_chunk + (e.n + kChunk - 1) / kChunk, to = next < end ? next : end;
    const int64_t last = (to - e.first_chunk) * kChunk;
    work(tensor, e, (c - e.first_chunk) * kChunk, last < e.n ? last : e.n);
    c = to;
  }
}

// Whether this block is the last of the grid to come here (its thread 0 only).  Additions to one word run one after the
// other (13 ns each), so that 32 blocks count together, and their last for them.  (The norm of 25 M elements: a release and an
// acquire a block 70 us, all blocks at one word 37.)
__device__ __forceinline__ bool last_block(int32_t *words) {
  stores_arrived();
  const int group = blockIdx.x / kGroupBlocks, groups = (gridDim.x + kGroupBlocks - 1) / kGroupBlocks;
  const int here = min((int)gridDim.x - group * kGroupBlocks, kGroupBlocks);
  return count_in(words + (1 + group) * kWordApart, here) && (groups == 1 || count_in(words, groups));
}

// The words of a call: 0 the norm, 1 the update.
__device__ __forceinline__ int32_t *done_words(const AdamWArgs &a, int call) {
  return reinterpret_cast<int32_t *>(a.table) + kWordApart + call * kDoneWords;
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  return v;
}

// The squares of gradients [from, to) of a tensor, 128 bytes a thread at once.
template <typename T>
__device__ __forceinline__ double squares(const T *g, int64_t from, int64_t to) {
  constexpr int kLines = 16 / sizeof(T), kTurn = 256 * 8;
  double sum = 0.0;
  for (int64_t i = from + threadIdx.x * 8; i < to; i += kLines * kTurn) {
    Line<T> x[kLines];
#pragma unroll
    for (int l = 0; l < kLines; ++l) {
      x[l] = Line<T>{};
      if (i + l * kTurn + 8 <= to) x[l] = *(Global<const Line<T>>)(g + i + l * kTurn);
    }
#pragma unroll
    for (int l = 0; l < kLines; ++l)
#pragma unroll
      for (int k = 0; k < 8; ++k) sum = fma((double)(float)x[l][k], (double)(float)x[l][k], sum);
  }
  // the line that the tensor ends in
  const int64_t rest = to - (to - from) % 8;
  if (rest + threadIdx.x < to) {
    const double x = (double)(float)((Global<const T>)g)[rest + threadIdx.x];
    sum = fma(x, x, sum);
  }
  return sum;
}

// Sum of squares in 64 bits (32 would end at gradients of 1.8e19).  Each block's part, and the last block adds them
// up in their order.  25.2 M elements in 32 bits 22 us, 4.6 TB/s.
__global__ __launch_bounds__(256) void k_grad_norm(const AdamWArgs a) {
  __shared__ double room[4];
  __shared__ int last;
  double *parts = reinterpret_cast<double *>(a.table + kTableParts);
  double sum = 0.0;
  const bool ours = is_table(a);
  walk(a, ours, [&](int, const TensorEntry &e, int64_t from, int64_t to) {
    if (e.grad_dtype == AA_BF16) sum += squares(static_cast<const __bf16 *>(e.grad), from, to);
    else if (e.grad_dtype == AA_F16) sum += squares(static_cast<const _Float16 *>(e.grad), from, to);
    else sum += squares(static_cast<const float *>(e.grad), from, to);
  });
  sum = wave_sum(sum);
  const int wave = threadIdx.x / kWave;
  if ((threadIdx.x & 63) == 0) room[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    __hip_atomic_store(parts + blockIdx.x, room[0] + room[1] + room[2] + room[3], __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
    last = last_block(done_words(a, 0));
  }
  __syncthreads();
  if (!last) return;
  sum = 0.0;
#pragma unroll
  for (int k = 0; k < kNormBlocks / 256; ++k) {
    const int b = k * 256 + (int)threadIdx.x;
    if (b < (int)gridDim.x) sum += __hip_atomic_load(parts + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  sum = wave_sum(sum);
  if ((threadIdx.x & 63) == 0) room[wave] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  const float scale = a.scale ? *a.scale : 1.f;
  // (the factor of a norm that is not finite, or of another table's gradients, leaves the update out)
  const float norm = (float)(sqrt(room[0] + room[1] + room[2] + room[3]) * fabs((double)scale));
  a.out[0] = norm;
  a.out[1] = !ours || !(norm < __builtin_inff()) ? __builtin_nanf("") : norm > a.max_norm ? scale * (a.max_norm / norm) : scale;
}

// What all elements of an update have in common (decay: lr weight_decay).
struct Step {
  float beta1, beta2, eps, factor, rate, root, decay;
  uint32_t k0, k1, t;
};

// Root of v >= 0 by the unit's instruction (one unit of the last place), which takes numbers below the normal ones for 0.
__device__ __forceinline__ float root_of(float v) {
  const bool low = v < 0x1p-96f;
  return __builtin_amdgcn_sqrtf(low ? v * 0x1p64f : v) * (low ? 0x1p-32f : 1.f);
}

// The new m and v (its root in r) of eight elements, and their parameters.  The decay is a product of its own, so that what it
// takes is rounded once, with the parameter: a factor 1 - lr weight_decay lies on a grid of 2^-24 (1e-7 became 1.2e-7, and what is
// below 3e-8 nothing, at every update alike).
__device__ __forceinline__ void update8(const Step &s, const Eight &g, Eight &m, Eight &v, Eight &r, Eight &p, float decay) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float d = g.v[k] * s.factor;
    m.v[k] = s.beta1 * m.v[k] + (1.f - s.beta1) * d;
    v.v[k] = s.beta2 * v.v[k] + (1.f - s.beta2) * (d * d);
    r.v[k] = root_of(v.v[k]);
    p.v[k] -= fmaf(decay, p.v[k], s.rate * m.v[k] * __builtin_amdgcn_rcpf(r.v[k] * s.root + s.eps));
  }
}

template <bool PASSING>
__device__ __forceinline__ void store_param(const TensorEntry &e, int64_t i, int n, const Eight &p) {
  store_some<PASSING>(e.param + i, p, n);
  if (!e.copy) return;
  if (e.copy_dtype == AA_BF16) store_some<PASSING>(static_cast<__bf16 *>(e.copy) + i, p, n);
  else store_some<PASSING>(static_cast<_Float16 *>(e.copy) + i, p, n);
}

struct Codes {
  uint32_t w[2];
};
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));

__device__ __forceinline__ Codes load_codes(const uint8_t *p, int n) {
  Codes c = {{0u, 0u}};
  if (n >= 8) {
    const u32x2_any v = *(Global<const u32x2_any>)p;
    c.w[0] = v[0];
    c.w[1] = v[1];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) c.w[k / 4] |= (uint32_t)((Global<const uint8_t>)p)[k] << (k % 4 * 8);
  }
  return c;
}

__device__ __forceinline__ void store_codes(uint8_t *p, int n, const Codes &c) {
  if (n >= 8) {
    u32x2_any v;
    v[0] = c.w[0];
    v[1] = c.w[1];
    *(Global<u32x2_any>)p = v;
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < n) ((Global<uint8_t>)p)[k] = (uint8_t)(c.w[k / 4] >> (k % 4 * 8));
  }
}

__device__ __forceinline__ Eight decode(const Codes &c, float scale) {
  Eight o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[h], false);
    const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[h], true);
    o.v[h * 4 + 0] = lo[0] * scale;
    o.v[h * 4 + 1] = lo[1] * scale;
    o.v[h * 4 + 2] = hi[0] * scale;
    o.v[h * 4 + 3] = hi[1] * scale;
  }
  return o;
}

// Largest value of 32 neighbouring lanes.
__device__ __forceinline__ float block_max(float v) {
  const auto move = [](float x, auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  v = fmaxf(v, move(v, std::integral_constant<int, 0xB1>()));
  v = fmaxf(v, move(v, std::integral_constant<int, 0x4E>()));
  v = fmaxf(v, move(v, std::integral_constant<int, 0x141>()));
  v = fmaxf(v, move(v, std::integral_constant<int, 0x140>()));
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Codes and scale of the block's states, by the unit's own conversion with a rounding by draw: it adds the upper bits of
// the word to what it cuts off, at numbers below the format's normal ones, too.  What is not finite becomes NaN and takes no part
// in the scale.  POSITIVE: no value is below 0, and what is above it is at least a step.
template <bool POSITIVE>
__device__ __forceinline__ Codes encode(const Eight &x, const uint4 &draws, float *scale) {
  const auto larger = [](float a, float b, float c) { return fmaxf(fmaxf(a, b), c); };
  float most = larger(fabsf(x.v[0]), fabsf(x.v[1]), fabsf(x.v[2]));
  most = larger(most, fabsf(x.v[3]), fabsf(x.v[4]));
  most = larger(most, fabsf(x.v[5]), fabsf(x.v[6]));
  most = block_max(fmaxf(most, fabsf(x.v[7])));
  if (__builtin_expect(__ballot(!(most < __builtin_inff())) != 0ull, 0)) {  // (a wave that holds an infinity)
    most = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) most = fmaxf(most, fabsf(x.v[k]) < __builtin_inff() ? fabsf(x.v[k]) : 0.f);
    most = block_max(most);
  }
  const int e = max((int)(__float_as_uint(most) >> 23) - 126 - 8, -126);
  *scale = most > 0.f ? __int_as_float((e + 127) << 23) : 0.f;
  const float inv = __int_as_float((127 - e) << 23);
  const uint32_t words[4] = {draws.x, draws.y, draws.z, draws.w};
  float y[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    y[k] = x.v[k] * inv;
    if (POSITIVE && x.v[k] > 0.f) y[k] = fmaxf(y[k], 0x1p-9f);
  }
  Codes c;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int w = 0;
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y[h * 4 + 0], (int)(words[h * 2] << 16), w, 0);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y[h * 4 + 1], (int)(words[h * 2] & 0xFFFF0000u), w, 1);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y[h * 4 + 2], (int)(words[h * 2 + 1] << 16), w, 2);
    w = __builtin_amdgcn_cvt_sr_fp8_f32(y[h * 4 + 3], (int)(words[h * 2 + 1] & 0xFFFF0000u), w, 3);
    c.w[h] = (uint32_t)w;
  }
  return c;
}

template <bool PASSING>
__global__ __launch_bounds__(256) void k_adamw_step(const AdamWArgs a) {
  const int32_t before = *a.t;
  const float factor = a.grad_factor ? *a.grad_factor : 1.f;
  // an empty batch, gradients that are not finite, or another table's numbers: nothing changes
  const bool ours = is_table(a);  // (asked for with the others)
  const bool skip = (a.count && *a.count <= 0) || !(fabsf(factor) < __builtin_inff()) || !ours;
  // The counter's new value is stored by the last block to come here: all waves of all have read the old one then.
  asm volatile("" ::"s"(before));
  __syncthreads();
  if (threadIdx.x == 0 && last_block(done_words(a, 1)) && !skip) *a.t = before + 1;
  if (skip) return;
  const float lr = a.cfg.lr * (a.lr_factor ? *a.lr_factor : 1.f);
  const float t = (float)before + 1.f;
  Step s;
  s.beta1 = a.cfg.beta1;
  s.beta2 = a.cfg.beta2;
  s.eps = a.cfg.eps;
  s.factor = factor;
  s.rate = lr / -expm1f(t * a.log_beta1);
  s.root = 1.f / sqrtf(-expm1f(t * a.log_beta2));
  s.decay = lr * a.cfg.weight_decay;
  s.k0 = (uint32_t)a.cfg.seed;
  s.k1 = (uint32_t)(a.cfg.seed >> 32);
  s.t = (uint32_t)before + 1u;
  walk(a, true, [&](int tensor, const TensorEntry &e, int64_t from, int64_t to) {
    const float decay = s.decay * e.decay;
    if (e.bits == 32) {
      for (int64_t i = from + threadIdx.x * 8; i < to; i += 256 * 8) {
        const int n = to - i < 8 ? (int)(to - i) : 8;
        float *pm = static_cast<float *>(e.m) + i, *pv = static_cast<float *>(e.v) + i;
        const Eight g = load_grad<PASSING>(e, i, n);
        Eight p = load_some<PASSING>(e.param + i, n), m = load_some<PASSING>(pm, n), v = load_some<PASSING>(pv, n), r;
        update8(s, g, m, v, r, p, decay);
        store_param<PASSING>(e, i, n, p);
        store_some<PASSING>(pm, m, n);
        store_some<PASSING>(pv, v, n);
      }
      return;
    }
    // (whole waves take part where one lane does: they share the scales)
    for (int64_t base = from; base < to; base += 256 * 8) {
      const int64_t i = base + threadIdx.x * 8;
      const int n = to - i < 8 ? (int)(to - i) : 8;
      uint8_t *pm = static_cast<uint8_t *>(e.m) + i, *pv = static_cast<uint8_t *>(e.v) + i;
      const Global<float> ms = (Global<float>)(e.m_scale + i / kStateBlock), vs = (Global<float>)(e.v_scale + i / kStateBlock);
      Eight m, v, r, p;
#pragma unroll
      for (int k = 0; k < 8; ++k) m.v[k] = r.v[k] = 0.f;
      if (n > 0) {
        const Eight g = load_grad<PASSING>(e, i, n);
        p = load_some<PASSING>(e.param + i, n);
        m = decode(load_codes(pm, n), *ms);
        v = decode(load_codes(pv, n), *vs);
#pragma unroll
        for (int k = 0; k < 8; ++k) v.v[k] *= v.v[k];
        update8(s, g, m, v, r, p, decay);
        store_param<PASSING>(e, i, n, p);
        if (n < 8) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (k >= n) m.v[k] = r.v[k] = 0.f;
        }
      }
      const uint4 draws = philox_words((uint32_t)(i / 8), 0x80000000u | (uint32_t)tensor, s.t, 0u, s.k0, s.k1);
      float m_scale, v_scale;
      const Codes cm = encode<false>(m, draws, &m_scale), cv = encode<true>(r, draws, &v_scale);
      if (n > 0) {
        store_codes(pm, n, cm);
        store_codes(pv, n, cv);
        if (threadIdx.x % (kStateBlock / 8) == 0) {
          *ms = m_scale;
          *vs = v_scale;
        }
      }
    }
  });
}

}  // namespace

hipError_t launch_adamw_table(const aa_adamw_tensor *tensors, int32_t n, char *table, hipStream_t st) {
  const int64_t map = (int64_t)table_map(n);
  int64_t n_chunks = 0;
  for (int32_t k = 0; k < n; ++k) n_chunks += (tensors[k].n + kChunk - 1) / kChunk;
  int64_t chunk = 0;
  for (int32_t first = 0; first < n; first += kBatch) {
    EntryBatch batch = {};
    const int here = n - first < kBatch ? n - first : kBatch;
    for (int k = 0; k < here; ++k) {
      const aa_adamw_tensor &t = tensors[first + k];
      batch.e[k] = {t.param, t.grad,       t.copy,       t.m,          t.v,     t.m_scale, t.v_scale,
                    t.n,     chunk,        t.grad_dtype, t.copy_dtype, t.state_bits, t.decay};
      chunk += (t.n + kChunk - 1) / kChunk;
    }
    hipLaunchKernelGGL(k_adamw_table, dim3(here), dim3(256), 0, st, table, map, n_chunks, n, first, batch);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_grad_norm(const AdamWArgs &a, hipStream_t st) {
  const int64_t blocks = a.n_chunks < 1 ? 1 : a.n_chunks < kNormBlocks ? a.n_chunks : kNormBlocks;
  hipLaunchKernelGGL(k_grad_norm, dim3((uint32_t)blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_adamw_step(const AdamWArgs &a, hipStream_t st) {
  const int64_t most = kMostBlocks, blocks = a.n_chunks < 1 ? 1 : a.n_chunks < most ? a.n_chunks : most;
  // (of 256 MB or more that a step moves, little is left in the caches for the next)
  if (a.n_chunks >= 8192) hipLaunchKernelGGL(k_adamw_step<true>, dim3((uint32_t)blocks), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_adamw_step<false>, dim3((uint32_t)blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace aa

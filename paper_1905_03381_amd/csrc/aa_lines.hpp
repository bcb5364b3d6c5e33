// Device helpers of the operators whose threads hold eight neighbouring columns of a row: 16-byte accesses at any
// address, the generator's words, sums over lanes.
#pragma once

#include "aa_common.hpp"

namespace aa {

// All four words of Philox4x32-10 (Salmon et al., SC'11).
__device__ __forceinline__ uint4 philox_words(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0,
                                              uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    const uint32_t n0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0, n2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
    c0 = n0;
    c1 = (uint32_t)p1;
    c2 = n2;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

struct Eight {
  float v[8];
};

template <typename T>
using Line = T __attribute__((ext_vector_type(8), aligned(sizeof(T))));  // (memory is read and written at any address)

// Columns of which n (at least one) exist, the others 0.
template <typename T>
__device__ __forceinline__ Line<T> load_line(const T *p, int n) {
  Line<T> o;
  if (n >= 8) {
    o = *reinterpret_cast<const Line<T> *>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const T v = p[i < n ? i : 0];  // (no branch: all are asked for at once)
      o[i] = i < n ? v : (T)0.f;
    }
  }
  return o;
}

// Eight columns at any address, for rows of odd widths: what begins inside a word of four bytes is moved by whole words and
// the ends (4422 rows of 1024 -> 8019 with residual and `pre`: 152 us by misaligned loads and stores, 127; where little else
// is moved, as in a norm, it is no gain).
template <typename T>
__device__ __forceinline__ Line<T> load_words(const T *p) {
  if constexpr (sizeof(T) == 2) {
    if (reinterpret_cast<uintptr_t>(p) & 2) {
      typedef T Words __attribute__((ext_vector_type(8), aligned(4)));
      const Words w = *reinterpret_cast<const Words *>(p - 1);  // (the half before p lies in p's own word)
      const Words end = p[7];
      return __builtin_shufflevector(w, end, 1, 2, 3, 4, 5, 6, 7, 8);
    }
  }
  return *reinterpret_cast<const Line<T> *>(p);
}

template <typename T>
__device__ __forceinline__ void store_words(T *p, const Line<T> &t) {
  if constexpr (sizeof(T) == 2) {
    if (reinterpret_cast<uintptr_t>(p) & 2) {
      typedef T Six __attribute__((ext_vector_type(6), aligned(4)));
      p[0] = t[0];
      *reinterpret_cast<Six *>(p + 1) = __builtin_shufflevector(t, t, 1, 2, 3, 4, 5, 6);
      p[7] = t[7];
      return;
    }
  }
  *reinterpret_cast<Line<T> *>(p) = t;
}

// load_line for a row that holds eight columns or more: what ends inside the eight is read from as much earlier and moved
// down, so that there is one address and one load (element by element took twice the registers).
template <typename T>
__device__ __forceinline__ Line<T> load_line_early(const T *p, int n) {
  const int early = n >= 8 ? 0 : 8 - n;
  Line<T> v = *reinterpret_cast<const Line<T> *>(p - early);
  const Line<T> none = {};
  if (early & 4) v = __builtin_shufflevector(v, none, 4, 5, 6, 7, 8, 8, 8, 8);
  if (early & 2) v = __builtin_shufflevector(v, none, 2, 3, 4, 5, 6, 7, 8, 8);
  if (early & 1) v = __builtin_shufflevector(v, none, 1, 2, 3, 4, 5, 6, 7, 8);
  return v;
}

template <typename T>
__device__ __forceinline__ Eight to_eight(const Line<T> &t) {
  Eight o;
#pragma unroll
  for (int i = 0; i < 8; ++i) o.v[i] = (float)t[i];
  return o;
}

template <typename T>
__device__ __forceinline__ Eight load8(const T *p, int n) {
  return to_eight<T>(load_line(p, n));
}

template <typename T>
__device__ __forceinline__ void store8(T *p, const Eight &o, int n) {
  if (n >= 8) {
    Line<T> t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)o.v[i];
    *reinterpret_cast<Line<T> *>(p) = t;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) p[i] = (T)o.v[i];
  }
}

// Sum over aligned groups of W (8 to 64) lanes; every lane gets it.
template <int W>
__device__ __forceinline__ float lanes_sum(float v, int lane) {
  if constexpr (W >= 16) {
    return row_group_sum<W>(v, lane);
  } else {
    v = dpp_add<0xB1>(v);     // quad_perm [1,0,3,2]
    v = dpp_add<0x4E>(v);     // quad_perm [2,3,0,1]
    return dpp_add<0x141>(v);  // row_half_mirror
  }
}

// What this thread has stored for the whole device has arrived there.  Such stores, and the loads behind count_in, go past
// the caches that are not shared, so that nothing has to be written back or thrown away.
__device__ __forceinline__ void stores_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// Counts one of `all` that come to `word`; true for the last of them, and the word is 0 again then.
__device__ __forceinline__ bool count_in(int32_t *word, int all) {
  if (__hip_atomic_fetch_add(word, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) != all - 1) return false;
  __hip_atomic_store(word, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return true;
}

}  // namespace aa

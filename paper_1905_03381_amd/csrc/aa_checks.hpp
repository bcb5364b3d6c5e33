// Argument checks of the C entries of the Boss's operators.
#pragma once

#include "aa_common.hpp"

#include <math.h>

namespace aa {

constexpr int32_t kMaxWidth = 1 << 24;             // row widths
constexpr int64_t kMaxPairs = (1ll << 31) - 4096;  // n_max * top_k

inline int32_t hip_status(hipError_t e) { return e == hipSuccess ? AA_OK : AA_ERR_HIP; }

inline hipStream_t as_stream(void *s) { return static_cast<hipStream_t>(s); }

inline bool on(const void *p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// 0 for an unknown type
inline int type_bytes(int32_t dtype) { return dtype == AA_F32 ? 4 : dtype == AA_BF16 || dtype == AA_F16 ? 2 : 0; }

// A matrix of `rows` rows: present (unless it has none), of a legal stride, on its type's alignment.
inline int32_t check_rows(const void *p, int64_t rows, int64_t ld, int64_t width, int bytes) {
  if (ld < width || ld > (1ll << 40)) return AA_ERR_SHAPE;
  if (rows > 0 && !p) return AA_ERR_NULL;
  return on(p, (size_t)bytes) ? AA_OK : AA_ERR_ALIGN;
}

// int32 / float arrays
inline int32_t check_words(const void *p, bool needed) {
  if (needed && !p) return AA_ERR_NULL;
  return on(p, 4) ? AA_OK : AA_ERR_ALIGN;
}

#define AA_TRY(expr)                    \
  do {                                  \
    const int32_t rc_ = (expr);         \
    if (rc_ != AA_OK) return rc_;       \
  } while (0)

// Rows of `width` elements can be moved 16 bytes at a time, but for a shorter end.
inline bool rows_on_16(const void *p, int64_t ld, int bytes) { return on(p, 16) && ld * bytes % 16 == 0; }

// What the kernels that move 16 bytes at a time address with 32 bits a lane: rows by their place in units of 16
// bytes (gathered ones, of which there may be more than rows_max, by 64 bits); rows that run along the result by their place
// among 31.
inline bool in_reach(const void *p, int64_t rows, int64_t ld) {
  return rows_on_16(p, ld, 2) && (rows == 0 || ld / 8 < (1ll << 32) / rows);
}
inline bool columns_in_reach(const void *p, int64_t ld) { return rows_on_16(p, ld, 2) && ld < (1ll << 25); }

inline int32_t check_ws(const void *ws, size_t ws_bytes, size_t need) {
  return !ws || !on(ws, 256) || ws_bytes < need ? AA_ERR_WORKSPACE : AA_OK;
}

inline int32_t check_pairs(int32_t n_max, int32_t top_k, int32_t n_experts) {
  if (n_max < 0 || top_k < 1 || top_k > AA_MAX_CHOICES || n_experts < 1 || n_experts > AA_MAX_EXPERTS)
    return AA_ERR_SHAPE;
  return (int64_t)n_max * top_k <= kMaxPairs ? AA_OK : AA_ERR_SHAPE;
}

inline int32_t check_route_config(const aa_route_config *c, int32_t n_max, int32_t n_experts) {
  if (!c) return AA_ERR_NULL;
  AA_TRY(check_pairs(n_max, c->top_k, n_experts));
  if (c->score != AA_SCORE_SOFTMAX && c->score != AA_SCORE_SIGMOID) return AA_ERR_SHAPE;
  if (c->n_groups < 1 || n_experts % c->n_groups != 0) return AA_ERR_SHAPE;
  if (c->top_groups < 1 || c->top_groups > c->n_groups) return AA_ERR_SHAPE;
  if (c->top_k > c->top_groups * (n_experts / c->n_groups)) return AA_ERR_SHAPE;
  if (c->group_best != 1 && c->group_best != 2) return AA_ERR_SHAPE;
  return isfinite(c->scale) ? AA_OK : AA_ERR_SHAPE;
}

}  // namespace aa

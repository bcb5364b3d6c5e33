// Host-side launch interface of the optimizer over many tensors (aa_adamw.hip).
#pragma once

#include "aa_common.hpp"

namespace aa {

constexpr int kStateBlock = AA_STATE_BLOCK;  // elements that share a scale
constexpr int kChunk = 2048;                 // elements a block takes at once
constexpr int kNormBlocks = 1024;

// What the kernels know of a tensor.
struct TensorEntry {
  float *param;
  const void *grad;
  void *copy, *m, *v;
  float *m_scale, *v_scale;
  int64_t n, first_chunk;
  int32_t grad_dtype, copy_dtype, bits;
  float decay;
};

// The table: control words (the numbers of chunks and of tensors, then for the norm and for the update the blocks that are done with the call),
// the norm's parts, the entries, and the tensor of each chunk.
constexpr int kMostBlocks = 2048, kGroupBlocks = 32;  // of a launch; that count themselves together
constexpr int kWordApart = 16;                        // int32 words between two that are counted in
constexpr int kDoneWords = (1 + kMostBlocks / kGroupBlocks) * kWordApart;
constexpr int kControlWords = kWordApart + 2 * kDoneWords;
constexpr size_t kTableParts = (kControlWords * sizeof(int32_t) + 255) / 256 * 256;
constexpr size_t kTableEntries = kTableParts + kNormBlocks * sizeof(double);
inline size_t table_map(int64_t n_tensors) { return align_up(kTableEntries + n_tensors * sizeof(TensorEntry), 256); }
inline size_t table_bytes(int64_t n_tensors, int64_t n_chunks) {
  return align_up(table_map(n_tensors) + n_chunks * sizeof(int32_t), 256);
}

struct AdamWArgs {
  char *table;
  int64_t map;  // byte offset of the chunks' tensors
  int32_t n_tensors;
  int64_t n_chunks;
  aa_adamw_config cfg;
  float log_beta1, log_beta2;
  const float *lr_factor, *grad_factor;
  const int32_t *count;
  int32_t *t;
  // norm
  float max_norm;
  const float *scale;
  float *out;
};

hipError_t launch_adamw_table(const aa_adamw_tensor *tensors, int32_t n, char *table, hipStream_t st);
hipError_t launch_grad_norm(const AdamWArgs &a, hipStream_t st);
hipError_t launch_adamw_step(const AdamWArgs &a, hipStream_t st);

}  // namespace aa

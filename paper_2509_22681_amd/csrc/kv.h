// The operators on a paged key/value cache (include/flame_kv.h): what the C entries hand to the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/flame_kv.h"
#include "kv_index.h"

namespace flame {

// rows of heads, strides in bytes
struct KvRows {
  char *p;
  int64_t row, head;
};

constexpr int kMaxRotationPairs = 64;
struct KvRotation {
  int32_t pairs, interleaved;
  uint64_t turns[kMaxRotationPairs];  // revolutions per position, modulo 1, times 2^64
};

// sequences of a batch: rows at offsets[b]..offsets[b+1] (NULL: row b), n_rows of them in the arrays
struct KvBatch {
  const int32_t *offsets, *kv_lens;
  int32_t n_seqs;
  int64_t n_rows;
  int32_t *faults;
};

struct KvAttention {
  KvBatch batch;
  KvRows q, out;
  KvRows k, v;                // packed keys (paged: unused)
  const int32_t *k_offsets;
  int64_t n_keys;
  KvPages pages;              // paged keys: table != NULL
  int32_t n_q_heads, n_kv_heads, head_dim, dtype;
  float scale;
  int32_t splits;             // flash kernel over pages: parts of a row tile's keys
  float *parts;
};

// How a call runs (kv_api.cpp): split kernel, or flash kernel with so many wavefronts per 32 rows and parts of the keys.
struct KvRoute {
  bool split;
  int32_t wavefronts, splits;
  int64_t workspace;          // bytes
};
KvRoute kv_route(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows, bool paged, bool decode, int64_t capacity);

hipError_t launch_kv_append(const KvBatch &batch, const KvPages &pages, const KvRows &k, const KvRows &v, const KvRows *q, const KvRows *q_out,
                            const KvRotation &rotation, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, hipStream_t stream);
hipError_t launch_kv_attention(const KvAttention &a, int wavefronts, hipStream_t stream);
// few query rows: split over the keys (kv_split.hip)
hipError_t launch_kv_split(const KvAttention &a, void *workspace, hipStream_t stream);
int64_t kv_split_workspace_bytes(int32_t head_dim, int64_t rows);   // rows times heads

}  // namespace flame

// The operators on a paged key/value cache (include/flame_kv.h): what the C entries hand to the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/flame_kv.h"
#include "../../include/flame_kvq.h"
#include "kv_index.h"

namespace flame {

// rows of heads, strides in bytes
struct KvRows {
  char *p;
  int64_t row, head;
};

// of a quantised cache: where the scale bytes lie, and its flame_kvq_form
struct KvScales {
  char *k, *v;
  int32_t form;
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
  int32_t form;               // of the pages: 0 as the element type, or a flame_kvq_form
  const char *k_scales, *v_scales;
  const int32_t *group_offsets, *prefix_lens;   // shared histories (else NULL); splits is 0 where their parts are of equal length
  int32_t n_groups;
  int32_t budget;             // workgroups of row tiles over the histories that there is room for, a key head
  int32_t split_blocks;       // workgroups of split attention over the sequences' own keys, in the same launch
  int64_t part_rows;
  int2 *cuts;                 // of up to 64 groups: where its parts begin, and how many a row tile has
  float *own;
};

// How a call runs (kv_api.cpp): split kernel, or flash kernel with so many wavefronts per 32 rows and parts of the keys.
struct KvRoute {
  bool split;
  int32_t wavefronts, splits;
  int64_t workspace;          // bytes
};
KvRoute kv_route(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows, bool paged, bool decode, int64_t capacity);
KvRoute kvq_route(const flame_kv_config &c, int32_t n_seqs, int64_t n_rows, bool decode, int64_t capacity);   // over a quantised cache

// The same for groups that share histories, and where the split part's workspace begins.
struct KvSharedRoute {
  int32_t wavefronts, splits, budget;
  int64_t slots, part_rows;                // row tiles (times parts) that there are at most, a key head; rows of parts
  int64_t cuts_at, own_at, split_at, workspace;
};
KvSharedRoute kv_shared_route(const flame_kv_config &c, int32_t n_groups, int64_t n_rows, int64_t capacity);

hipError_t launch_kv_append(const KvBatch &batch, const KvPages &pages, const KvRows &k, const KvRows &v, const KvRows *q, const KvRows *q_out,
                            const KvRotation &rotation, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, hipStream_t stream);
// quantised caches: as above, and rows back out of one
hipError_t launch_kvq_append(const KvBatch &batch, const KvPages &pages, const KvScales &scales, const KvRows &k, const KvRows &v, const KvRows *q, const KvRows *q_out,
                             const KvRotation &rotation, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype, hipStream_t stream);
hipError_t launch_kvq_read(const KvBatch &batch, const KvPages &pages, const KvScales &scales, const KvRows &k, const KvRows &v, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                           hipStream_t stream);
hipError_t launch_kvq_attention_f8(const KvAttention &a, int wavefronts, hipStream_t stream);
hipError_t launch_kvq_attention_f4(const KvAttention &a, int wavefronts, hipStream_t stream);
// shared histories (kv_shared.h)
hipError_t launch_kv_shared_plain(const KvAttention &a, const KvSharedRoute &route, void *split_workspace, hipStream_t stream);
hipError_t launch_kv_shared_f8(const KvAttention &a, const KvSharedRoute &route, void *split_workspace, hipStream_t stream);
hipError_t launch_kv_shared_f4(const KvAttention &a, const KvSharedRoute &route, void *split_workspace, hipStream_t stream);
hipError_t launch_kv_attention(const KvAttention &a, int wavefronts, hipStream_t stream);
// few query rows: split over the keys (kv_split.h)
hipError_t launch_kv_split(const KvAttention &a, void *workspace, hipStream_t stream);
hipError_t launch_kvq_split(const KvAttention &a, void *workspace, hipStream_t stream);
int64_t kv_split_workspace_bytes(int32_t head_dim, int64_t rows);   // rows times heads

}  // namespace flame

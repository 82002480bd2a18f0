// Split attention (kv_split.h) over a cache of the element type.
#include "kv_split.h"

namespace flame {

int64_t kv_split_workspace_bytes(int32_t head_dim, int64_t rows) {
  return split_parts_floats(head_dim) * 4 + (rows + 1) / 2 * 16;
}

hipError_t launch_kv_split(const KvAttention &a, void *workspace, hipStream_t stream) { return launch_split<kPlain>(a, workspace, stream); }

}  // namespace flame

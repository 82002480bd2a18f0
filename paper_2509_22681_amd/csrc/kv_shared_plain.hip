// Shared histories (kv_shared.h) in a cache of the element type.
#include "kv_shared.h"

namespace flame {

hipError_t launch_kv_shared_plain(const KvAttention &a, const KvSharedRoute &route, void *split_workspace, hipStream_t stream) { return launch_shared<kPlain>(a, route, split_workspace, stream); }

}  // namespace flame

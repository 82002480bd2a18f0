// Shared histories (kv_shared.h) in a cache of 8 bits.
#include "kv_shared.h"

namespace flame {

hipError_t launch_kv_shared_f8(const KvAttention &a, const KvSharedRoute &route, void *split_workspace, hipStream_t stream) { return launch_shared<kF8>(a, route, split_workspace, stream); }

}  // namespace flame

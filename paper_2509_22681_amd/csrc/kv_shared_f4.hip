// Shared histories (kv_shared.h) in a cache of 4 bits.
#include "kv_shared.h"

namespace flame {

hipError_t launch_kv_shared_f4(const KvAttention &a, const KvSharedRoute &route, void *split_workspace, hipStream_t stream) { return launch_shared<kF4>(a, route, split_workspace, stream); }

}  // namespace flame

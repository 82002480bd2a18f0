// Split attention (kv_split.h) over caches of 8 and 4 bits.
#include "kv_split.h"

namespace flame {

hipError_t launch_kvq_split(const KvAttention &a, void *workspace, hipStream_t stream) {
  return a.form == kF8 ? launch_split<kF8>(a, workspace, stream) : launch_split<kF4>(a, workspace, stream);
}

}  // namespace flame

// Row tiles (kv_flash.h) over caches of 4 bits.
#include "kv_flash.h"

namespace flame {

hipError_t launch_kvq_attention_f4(const KvAttention &a, int wavefronts, hipStream_t stream) {
  hipError_t e = hipErrorInvalidValue;
  flash_with_shape(a, wavefronts, [&](auto t, auto width, auto kp) { e = launch_flash<decltype(t), decltype(width)::value, true, decltype(kp)::value, kF4>(a, stream); });
  return e;
}

}  // namespace flame

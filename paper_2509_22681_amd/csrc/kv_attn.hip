// Row tiles (kv_flash.h) over packed keys and over a cache of the element type.
#include "kv_flash.h"

namespace flame {

hipError_t launch_kv_attention(const KvAttention &a, int wavefronts, hipStream_t stream) {
  hipError_t e = hipErrorInvalidValue;
  flash_with_shape(a, wavefronts, [&](auto t, auto width, auto kp) {
    using T = decltype(t);
    constexpr int DH = decltype(width)::value, KP = decltype(kp)::value;
    e = a.pages.table ? launch_flash<T, DH, true, KP, kPlain>(a, stream) : launch_flash<T, DH, false, KP, kPlain>(a, stream);
  });
  return e;
}

}  // namespace flame

// The angle of a rotated pair of features at a position.
//
// Revolutions per position are a 64-bit fraction, so position * turns modulo 2^64 is the fraction of a revolution up to that fraction's own error times the position.  It is
// three roundings of 64-bit mantissas and the cut to 64 bits, below 2^-61 of a revolution (times the revolutions per position, where there are more than one): 2^-30 at position 2^31.
// The top two bits after adding an eighth give the quadrant, the rest is an angle within +-1/8 revolution, for which fp32 has 2^-28.
#pragma once
#include "kv_device.h"

namespace flame {

__device__ __forceinline__ float2 cos_sin_of_turn(uint64_t turn) {
  const uint64_t shifted = turn + (1ull << 61);
  const int quadrant = (int)(shifted >> 62);
  const int64_t rest = (int64_t)(turn - ((uint64_t)quadrant << 62));      // within +-2^61
  const float half_turns = (float)(int32_t)(rest >> 32) * 0x1p-31f;       // a revolution is 2^64, so half ones are rest / 2^63
  float s, c;
  sincospif(half_turns, &s, &c);
  float2 r;
  r.x = quadrant == 0 ? c : quadrant == 1 ? -s : quadrant == 2 ? -c : s;
  r.y = quadrant == 0 ? s : quadrant == 1 ? c : quadrant == 2 ? -s : -c;
  return r;
}

}  // namespace flame

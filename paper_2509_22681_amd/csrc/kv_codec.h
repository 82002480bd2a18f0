// What a page holds of a head's row: values of the element type, or codes of 8 or 4 bits with a scale 2^e for each 32 features (include/flame_kvq.h).
#pragma once
#include "kv_device.h"

namespace flame {

enum : int { kPlain = 0, kF8 = FLAME_KVQ_F8, kF4 = FLAME_KVQ_F4 };

template <typename T, int FORM> constexpr int kv_row_bytes(int features) { return FORM == kPlain ? features * (int)sizeof(T) : FORM == kF8 ? features : features / 2; }
// A code at byte x has its scale at byte x >> kv_scale_shift.
template <int FORM> constexpr int kv_scale_shift() { return FORM == kF8 ? 5 : 4; }
__device__ __forceinline__ float kv_scale(uint32_t byte) { return __uint_as_float(byte << 23); }   // (2^-127 and NaN, bytes 0 and 255, are what the conversions take them for)

// The scale of block `i` of up to four, from a word of their bytes.
__device__ __forceinline__ float kv_scale_of(uint32_t bytes, int i) { return kv_scale(bytes >> (8 * i) & 0xff); }

// Form as a template argument of the launches.
template <typename F> inline void kv_with_form(int32_t form, F f) {
  if (form == kPlain) f(std::integral_constant<int, kPlain>{});
  else if (form == kF8) f(std::integral_constant<int, kF8>{});
  else f(std::integral_constant<int, kF4>{});
}

// Two features of a word of codes, times the scale: one instruction, exact (and NaN where the scale's byte is 255).  f8: the word's lower or upper half (I = 0, 1); f4: its byte I.
template <typename T> struct KvPair;
template <> struct KvPair<half_t> {
  typedef f16x2 vec;
  template <int FORM, int I> static __device__ __forceinline__ vec get(uint32_t w, float scale) {
    if constexpr (FORM == kF8) return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, I != 0);
    else return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, I);
  }
};
template <> struct KvPair<bf16_t> {
  typedef bf16x2 vec;
  template <int FORM, int I> static __device__ __forceinline__ vec get(uint32_t w, float scale) {
    if constexpr (FORM == kF8) return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, I != 0);
    else return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, I);
  }
};
template <> struct KvPair<float> {
  typedef float vec __attribute__((ext_vector_type(2)));
  template <int FORM, int I> static __device__ __forceinline__ vec get(uint32_t w, float scale) {
    if constexpr (FORM == kF8) return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, I != 0);
    else return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, I);
  }
};

// Eight features as they lie: 16 bytes of 16-bit values, 32 of fp32, from the words of their codes (two of f8, one of f4).
template <typename T, int FORM> __device__ __forceinline__ void kv_eight(const uint32_t *codes, float scale, typename KvPair<T>::vec (&x)[4]) {
  if constexpr (FORM == kF8) {
    x[0] = KvPair<T>::template get<FORM, 0>(codes[0], scale);
    x[1] = KvPair<T>::template get<FORM, 1>(codes[0], scale);
    x[2] = KvPair<T>::template get<FORM, 0>(codes[1], scale);
    x[3] = KvPair<T>::template get<FORM, 1>(codes[1], scale);
  } else {
    x[0] = KvPair<T>::template get<FORM, 0>(codes[0], scale);
    x[1] = KvPair<T>::template get<FORM, 1>(codes[0], scale);
    x[2] = KvPair<T>::template get<FORM, 2>(codes[0], scale);
    x[3] = KvPair<T>::template get<FORM, 3>(codes[0], scale);
  }
}

// The least exponent e of a block, and the largest size of a value in it (include/flame_kvq.h).
template <typename T, int FORM> constexpr int kv_least_exponent() { return FORM == kF8 ? (std::is_same<T, half_t>::value ? -15 : -117) : (std::is_same<T, half_t>::value ? -23 : -125); }
template <typename T, int FORM> constexpr float kv_largest() {
  return FORM == kF8 ? (std::is_same<T, half_t>::value ? 61440.f : 240.f * 0x1p120f) : (std::is_same<T, half_t>::value ? 49152.f : 1.5f * 0x1p127f);
}

}  // namespace flame

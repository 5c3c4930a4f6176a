// The 4-bit elements of a cache (include/otas_decode.h), eight of a head to a 32-bit word, the first in the lowest bits.
#pragma once
#include "common.h"
#include "window_kernels.h"

namespace otas {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kNoNumber = 255;   // the scale of a group with an element that is not finite

__device__ __forceinline__ float scale4(uint32_t byte) { return __uint_as_float(byte << 23); }   // 2^(byte - 127)

// Elements 2 I and 2 I + 1 of a word, times the scale: exact in either type.
template <int I> __device__ __forceinline__ uint32_t pair4_bf16(uint32_t word, float scale) {
  const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, I);
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  return u;
}
template <int I> __device__ __forceinline__ floatx2 pair4(uint32_t word, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, I);
}

// The scale of a group whose largest element has these bits without sign: 7 2^e = 1.75 2^(e + 2) is the largest that a scale
// of 2^e takes.
__device__ __forceinline__ uint32_t scale4_byte(uint32_t largest) {
  if (largest >= 0x7F800000u) return kNoNumber;
  const int e = (int)(largest >> 23) - 2 + ((largest & 0x7FFFFFu) > 0x600000u);
  return (uint32_t)min(max(e, 2), 252);
}

}  // namespace otas

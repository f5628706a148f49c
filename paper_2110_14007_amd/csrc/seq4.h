// Values of a 4-bit cache: codes of the magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6
// with a sign bit, two a byte (the low half first), and a byte b a block of 32
// for the scale 2^(b - 127); 255 stands for NaN.  gfx950 converts a byte's two
// codes times a power of two in one instruction, exact wherever the type has
// the value, infinite beyond it.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace tod {

// A float with the scale's exponent (the conversions read nothing else of it).
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// The two values of byte SEL of `codes`, as 16-bit elements.
template <typename ET, int SEL>
__device__ __forceinline__ uint32_t two_values(uint32_t codes, float scale) {
  if constexpr (std::is_same<ET, _Float16>::value)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL));
  else
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}

// The eight of all four bytes.
template <typename ET>
__device__ __forceinline__ auto eight_values(uint32_t codes, float scale) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  return u32x4{two_values<ET, 0>(codes, scale), two_values<ET, 1>(codes, scale),
               two_values<ET, 2>(codes, scale), two_values<ET, 3>(codes, scale)};
}

// Byte SEL of `codes` from two 16-bit elements over the scale: the nearest values, ties to the even
// code, beyond 6 to 6.
template <typename ET, int SEL>
__device__ __forceinline__ uint32_t two_codes(uint32_t codes, uint32_t pair, float scale) {
  typedef ET e2 __attribute__((ext_vector_type(2)));
  if constexpr (std::is_same<ET, _Float16>::value)
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(e2, pair), scale, SEL);
  else
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(e2, pair), scale,
                                                     SEL);
}

}  // namespace tod

// Numbers of 4 bits (e2m1) with a power of two for every 32 of them, as a paged cache holds them.
#pragma once
#include <algorithm>

#include "common.h"

namespace sif {

typedef __bf16 bf16x2_e2m1 __attribute__((ext_vector_type(2)));
// byte B of a word, two numbers, times a power of two, as bf16: exact but past the ends of that type
template <int B>
__device__ __forceinline__ uint32_t e2m1x2(uint32_t w, float power) {
  return __builtin_bit_cast(uint32_t, (bf16x2_e2m1)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, B));
}
// the power of two that a byte stands for; 255 is NaN
__device__ __forceinline__ float e2m1_power(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(std::max(byte << 23, 0x00400000u));
}

}  // namespace sif

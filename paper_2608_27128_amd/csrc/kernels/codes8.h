// 8-bit codes as matrix operands.
#pragma once
#include <hip/hip_runtime.h>

#include "rows.h"

namespace twinkv {

// Four codes as two pairs of bf16: whole numbers up to 127 are exact there, so the low half of the float is zero.
__device__ inline u32x2 codes4_bf16(unsigned w) {
  const unsigned a = __float_as_uint((float)(int8_t)w), b = __float_as_uint((float)(int8_t)(w >> 8));
  const unsigned c = __float_as_uint((float)(int8_t)(w >> 16)), d = __float_as_uint((float)(int8_t)(w >> 24));
  return u32x2{__builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x07060302u)};
}
__device__ inline bf16x8 codes8_bf16(unsigned lo, unsigned hi) {
  const u32x2 a = codes4_bf16(lo), b = codes4_bf16(hi);
  return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], b[0], b[1]});
}

}  // namespace twinkv

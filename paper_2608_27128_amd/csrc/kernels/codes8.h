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
__device__ inline f32x4 codes4_f32(unsigned w) {
  return f32x4{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)};
}

// x as a sum of N bf16, the largest first.
template <int N>
__device__ inline void split8(const float (&x)[8], bf16x8 (&p)[N]) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < N; ++n) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      p[n][e] = (bf16)r[e];
      r[e] -= (float)p[n][e];
    }
  }
}

}  // namespace twinkv

// Eight consecutive channels of a row in registers, for the kernels of the operators around the cache.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace twinkv {

typedef __bf16 bf16;
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

__device__ inline void load8(const float* p, float (&x)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(p);
  const f32x4 b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[e] = a[e];
    x[4 + e] = b[e];
  }
}

template <typename T>
struct Vec8;

template <>
struct Vec8<bf16> {
  bf16x8 x;
  __device__ static Vec8 load(const char* p) { return {*reinterpret_cast<const bf16x8*>(p)}; }
  __device__ static Vec8 from(const float (&f)[8]) {
    Vec8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r.x[e] = (bf16)f[e];  // to nearest, ties to even
    return r;
  }
  __device__ void store(char* p) const { *reinterpret_cast<bf16x8*>(p) = x; }
  __device__ void to(float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)x[e];
  }
};

template <>
struct Vec8<float> {
  f32x4 a, b;
  __device__ static Vec8 load(const char* p) {
    return {*reinterpret_cast<const f32x4*>(p), *reinterpret_cast<const f32x4*>(p + 16)};
  }
  __device__ static Vec8 from(const float (&f)[8]) {
    Vec8 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r.a[e] = f[e];
      r.b[e] = f[4 + e];
    }
    return r;
  }
  __device__ void store(char* p) const {
    *reinterpret_cast<f32x4*>(p) = a;
    *reinterpret_cast<f32x4*>(p + 16) = b;
  }
  __device__ void to(float (&f)[8]) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f[e] = a[e];
      f[4 + e] = b[e];
    }
  }
};

}  // namespace twinkv

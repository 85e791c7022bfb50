// K6: RMS norm of each head of the queries and keys, and the rotary embedding, in one pass.
//
// With y = x * weight / sqrt(mean(x^2) + eps), channels c and c + d/2 turn by the token's angle of the
// pair c.  HBM-bound: every element is read once and written once.
//  * A row (one head of one token) belongs to d/16 lanes.  A lane holds 8 channels of the first half
//    and the 8 they turn with, so the rotation needs no other lane and every access is 16 bytes wide;
//    the mean takes 2 or 3 exchanges between the row's lanes.
//  * A unit of lanes goes through several heads of its token with the token's cos and sin in registers:
//    they are fp32 and as long as the row, so reading them per row would double the traffic of bf16
//    rows.  Few tokens take one head a unit instead, so that there are units for the whole machine
//    (32 + 8 heads of 128, bf16, 1 head / 8 heads a unit: 64 tokens 3.7 / 6.4 us, 1024 7.2 / 8.7, 4096 17.2 / 15.7,
//    32k 182 / 131).
// 32k tokens, 40 heads of 128, bf16: 139 us a call, 4.9 TB/s where a large copy runs at 5.15.
#include <hip/hip_runtime.h>

#include "../cache_ops.h"
#include "rows.h"

namespace twinkv {
namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;  // heads in flight per lane

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(const NormRopeArgs a) {
  constexpr int kLanes = D / 16;             // lanes of a row
  constexpr int kTokens = kThreads / kLanes; // tokens of a workgroup
  constexpr int kHalf = D / 2 * (int)sizeof(T);
  const bool is_k = (int)blockIdx.y >= a.q.chunks;
  const NormRopeSide& s = is_k ? a.k : a.q;
  const int h0 = ((int)blockIdx.y - (is_k ? a.q.chunks : 0)) * a.per_unit;
  const int h1 = min(h0 + a.per_unit, s.heads);
  const int64_t t = (int64_t)blockIdx.x * kTokens + threadIdx.x / kLanes;
  const int c0 = (threadIdx.x % kLanes) * 8;  // first channel of this lane in either half
  if (t >= a.T) return;  // whole rows of lanes

  float cs[8] = {}, sn[8] = {}, w0[8] = {}, w1[8] = {};
  if (a.rope != nullptr) {
    const int64_t p = a.pos[t];
    const bool in = p >= 0 && p < a.n_pos;
    if (in) {
      load8(a.rope + p * D + c0, cs);
      load8(a.rope + p * D + D / 2 + c0, sn);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) cs[e] = sn[e] = __builtin_nanf("");
    }
  }
  if (s.weight != nullptr) {
    load8(s.weight + c0, w0);
    load8(s.weight + D / 2 + c0, w1);
  }
  const char* in = s.in + t * s.in_token + c0 * (int)sizeof(T);
  char* out = s.out + t * s.out_token + c0 * (int)sizeof(T);
  for (int h = h0; h < h1; h += kBatch) {
    Vec8<T> x0[kBatch], x1[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const char* p = in + (int64_t)min(h + b, h1 - 1) * s.in_head;
      x0[b] = Vec8<T>::load(p);
      x1[b] = Vec8<T>::load(p + kHalf);
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (h + b >= h1) break;
      float u[8], v[8];
      x0[b].to(u);
      x1[b].to(v);
      if (s.weight != nullptr) {
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += u[e] * u[e] + v[e] * v[e];
#pragma unroll
        for (int m = 1; m < kLanes; m <<= 1) sum += __shfl_xor(sum, m);
        const float r = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] *= r * w0[e];
          v[e] *= r * w1[e];
        }
      }
      if (a.rope != nullptr) {  // (not a turn by 0, which would make NaN of the partner of an infinity)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = u[e];
          u[e] = x * cs[e] - v[e] * sn[e];
          v[e] = v[e] * cs[e] + x * sn[e];
        }
      }
      char* p = out + (int64_t)(h + b) * s.out_head;
      Vec8<T>::from(u).store(p);
      Vec8<T>::from(v).store(p + kHalf);
    }
  }
}

template <typename T, int D>
int launch(const NormRopeArgs& a, hipStream_t stream) {
  constexpr int kTokens = kThreads / (D / 16);
  const int64_t bx = (a.T + kTokens - 1) / kTokens;
  const int by = a.q.chunks + a.k.chunks;
  if (bx == 0 || by == 0) return hipSuccess;
  hipLaunchKernelGGL((norm_rope_kernel<T, D>), dim3((unsigned)bx, (unsigned)by), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

int launch_norm_rope(const NormRopeArgs& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 0) return d == 128 ? launch<bf16, 128>(a, s) : launch<bf16, 64>(a, s);
  return d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}

}  // namespace twinkv

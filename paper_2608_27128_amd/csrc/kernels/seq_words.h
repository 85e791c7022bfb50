// A call's per-sequence words, read on the device: from the kernel arguments or from the workspace.
#pragma once
#include <hip/hip_runtime.h>

#include "../cache_ops.h"

namespace twinkv {

__device__ inline int32_t seq_word_of_lane(const SeqWords& t, int i) {
  return t.far != nullptr ? t.far[i] : t.near[i];
}
// i is the same in all lanes, and the word scalar from here on.
__device__ inline int32_t seq_word(const SeqWords& t, int i) {
  return __builtin_amdgcn_readfirstlane(seq_word_of_lane(t, i));
}

// The sequence whose range of the non-decreasing words w(s) = word[s * stride + at], s in [0, n], holds
// x: w(s) <= x < w(s + 1).  x lies in [w(0), w(n)).
__device__ inline int find_seq(const SeqWords& t, int n, int stride, int at, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (seq_word(t, mid * stride + at) <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

}  // namespace twinkv

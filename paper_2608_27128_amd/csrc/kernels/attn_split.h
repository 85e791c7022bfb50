// What the two attention kernels that split a problem's keys share (over rows of keys and values, and
// over the 4-bit cache).
//
// A row is one query of one query head; 16 rows make a tile.  Scores come as K q^T, so a lane holds one
// row (lane % 16) and, of a tile of 32 keys, the 8 that its lane group g = lane / 16 owns; the product
// with the values takes those 8 as its own 8 contraction places, so the weights never leave their lane.
// The output accumulators hold rows 4g .. 4g + 3 and one channel a lane.
//
// Softmax statistics: m (in units of log2) and l per row, fp32.  m is the maximum of some earlier tile,
// not the running one: weights stay right for any m, and as long as no score passes m by more than
// kSlack their sum cannot leave the range of fp32 (2^8 times a sum of at most 2^31 ones), nor the weights lose
// precision (bf16 and fp32 keep their relative precision at any size).  So the exchange between lanes and the
// rescaling of the accumulators run only in tiles where the maximum grows by more than that: the first
// few of a call.
#pragma once
#include <hip/hip_runtime.h>

#include "../cache_ops.h"
#include "rows.h"
#include "seq_words.h"

namespace twinkv {

constexpr float kSlack = 8.0f;
constexpr int kAttnWaves = 4;
constexpr float kNegInf = -__builtin_huge_valf();

__device__ inline void to_lds(const char* from, char* to) {  // 16 bytes a lane, `to` the wave's first
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from,
                                   (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
constexpr int kNoLoads = 0x0f70;  // s_waitcnt: vmcnt 0, the other counters at their largest

__device__ inline float group_max(float x) {  // over the 4 lane groups
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float group_sum(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The row statistics of a lane (its row is lane % 16), and one tile's weights from its scores.
struct RowStats {
  float m = kNegInf;   // what weights are relative to
  float l = 0.0f;      // this lane's share of the sum
  __device__ float base() const { return m == kNegInf ? 0.0f : m; }
  // s: this lane's 8 scores in log2 units, -inf where masked; become weights.  acc: O accumulators.
  template <int N>
  __device__ void update(float (&s)[8], f32x4 (&acc)[N]) {
    float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    if (__any(top > m + kSlack)) {
      const float next = fmaxf(m, group_max(top));
      // nothing seen before (m = -inf): the factor is 0, and so are the accumulators
      const float f = next == m ? 1.0f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
      const int g4 = ((int)threadIdx.x & 48) >> 2;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float fr = __shfl(f, g4 + r);  // of row 4g + r, from a lane that holds it
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n][r] *= fr;
      }
    }
    const float b = base();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] = __builtin_amdgcn_exp2f(s[e] - b);
      l += s[e];
    }
  }
};

// Where an item of the call stands.
struct AttnItem {
  int h, s;            // KV head, sequence
  int rt, split;       // row tile, split of its keys
  int nq;              // query tokens of the sequence
  int q0, k0, nk;      // its first query token, first key (or cache row), keys (rows)
  int splits, tiles;   // splits of its keys, and key tiles of each
  int64_t part;        // among the parts of all heads, where splits > 1
};
__device__ inline AttnItem attn_item(const AttnArgs& a, int item, int h) {
  AttnItem p;
  p.h = h;
  p.s = find_seq(a.seq, a.n_seqs, kAttnSeqWords, 2, item);
  const int w = p.s * kAttnSeqWords;
  p.q0 = seq_word(a.seq, w);
  p.k0 = seq_word(a.seq, w + 1);
  const int i = item - seq_word(a.seq, w + 2);
  p.splits = seq_word(a.seq, w + 3);
  p.tiles = seq_word(a.seq, w + 4);
  p.part = (int64_t)h * a.parts + seq_word(a.seq, w + 5) + i;
  p.rt = i / p.splits;
  p.split = i - p.rt * p.splits;
  p.nq = seq_word(a.seq, w + kAttnSeqWords) - p.q0;
  p.nk = seq_word(a.seq, w + kAttnSeqWords + 1) - p.k0;
  return p;
}

// Writes a tile's results: 16 rows whose sums are o[row][channel] (LDS, kStride floats a row), maxima m
// and sums l; direct, or as the item's part for the join.
template <typename T, int D, int kStride>
__device__ inline void write_rows(const AttnArgs& a, const AttnItem& p, int row0, const float* o, const float* m,
                                  const float* l, int tid, int threads) {
  const int n_rows = p.nq * a.group;
  const int64_t part = p.part * a.rows + (row0 - p.rt * a.rows);
  constexpr int kPieces = D / 8;
  for (int x = tid; x < kAttnRows * kPieces; x += threads) {
    const int r = x / kPieces, c = x % kPieces * 8;
    if (row0 + r >= n_rows) continue;
    float f[8];
    if (p.splits > 1) {
      float* to = a.part_o + (part + r) * D + c;
#pragma unroll
      for (int e = 0; e < 8; ++e) to[e] = o[r * kStride + c + e];
      if (c == 0) {
        float* ml = a.part_ml + (part + r) * 2;
        ml[0] = m[r];
        ml[1] = l[r];
      }
    } else {
      const float inv = l[r] > 0.0f ? 1.0f / l[r] : (l[r] == 0.0f ? 0.0f : l[r]);  // a NaN stays one
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = o[r * kStride + c + e] * inv;
      const int i = (row0 + r) / a.group, g = (row0 + r) - i * a.group;
      const int64_t head = (int64_t)p.h * a.group + g;
      Vec8<T>::from(f).store(a.out + head * a.o_head + (int64_t)(p.q0 + i) * a.o_token + c * (int)sizeof(T));
      if (a.lse != nullptr && c == 0)
        a.lse[head * a.Tq + p.q0 + i] = l[r] == 0.0f ? kNegInf : m[r] * 0.69314718055994530942f + logf(l[r]);
    }
  }
}

// Joins the four waves' tiles of the same 16 rows (each wave's statistics and accumulators over its own
// keys) and writes them.  channel(n, i): the channel of accumulator n of lane i.
template <typename T, int D, typename Channel>
__device__ inline void join_waves(const AttnArgs& a, const AttnItem& p, int row0, RowStats st,
                                  f32x4 (&acc)[D / 16], float* lds, const Channel& channel) {
  constexpr int kStride = D + 4;
  float* s_ml = lds;                       // [4 waves][2][16]
  float* s_o = lds + kAttnWaves * 2 * kAttnRows;  // [16][kStride] of one pair of waves, then of both
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
  const float l = group_sum(st.l);
  if (g == 0) {
    s_ml[(wave * 2) * kAttnRows + i] = st.m;
    s_ml[(wave * 2 + 1) * kAttnRows + i] = l;
  }
  __syncthreads();
  // factors of this wave's rows
  float fr[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int row = 4 * g + r;
    float top = kNegInf;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) top = fmaxf(top, s_ml[(w * 2) * kAttnRows + row]);
    const float own = s_ml[(wave * 2) * kAttnRows + row];
    fr[r] = own == top ? 1.0f : __builtin_amdgcn_exp2f(own - top);
  }
  for (int w = 0; w < kAttnWaves; ++w) {
    if (wave == w) {
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float* at = s_o + (4 * g + r) * kStride + channel(n, i);
          *at = (w == 0 ? 0.0f : *at) + acc[n][r] * fr[r];
        }
      }
    }
    __syncthreads();
  }
  // the rows' joint statistics
  if (threadIdx.x < kAttnRows) {
    float top = kNegInf, sum = 0.0f;
    const int row = threadIdx.x;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) top = fmaxf(top, s_ml[(w * 2) * kAttnRows + row]);
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      const float own = s_ml[(w * 2) * kAttnRows + row];
      sum += s_ml[(w * 2 + 1) * kAttnRows + row] * (own == top ? 1.0f : __builtin_amdgcn_exp2f(own - top));
    }
    s_ml[row] = top;
    s_ml[kAttnRows + row] = sum;
  }
  __syncthreads();
  write_rows<T, D, kStride>(a, p, row0, s_o, s_ml, s_ml + kAttnRows, (int)threadIdx.x, 64 * kAttnWaves);
}
template <int D>
constexpr int join_floats() {
  return kAttnWaves * 2 * kAttnRows + kAttnRows * (D + 4);
}

// One wave's own 16 rows, complete, through its own LDS.
template <typename T, int D, typename Channel>
__device__ inline void write_own(const AttnArgs& a, const AttnItem& p, int row0, const RowStats& st,
                                 const f32x4 (&acc)[D / 16], float* lds, const Channel& channel) {
  constexpr int kStride = D + 4;
  float* s_ml = lds;               // [2][16]
  float* s_o = lds + 2 * kAttnRows;
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const float l = group_sum(st.l);
  if (g == 0) {
    s_ml[i] = st.m;
    s_ml[kAttnRows + i] = l;
  }
#pragma unroll
  for (int n = 0; n < D / 16; ++n)
#pragma unroll
    for (int r = 0; r < 4; ++r) s_o[(4 * g + r) * kStride + channel(n, i)] = acc[n][r];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  write_rows<T, D, kStride>(a, p, row0, s_o, s_ml, s_ml + kAttnRows, lane, 64);
}
template <int D>
constexpr int own_floats() {
  return 2 * kAttnRows + kAttnRows * (D + 4);
}

}  // namespace twinkv

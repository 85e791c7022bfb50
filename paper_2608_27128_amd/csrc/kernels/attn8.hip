// K13: attention over the 8-bit cache.
//
// As over the 4-bit cache (attn4.hip): four waves share a tile of 16 rows (queries times the query heads of a KV
// head) and take 32 cached rows at a time each, the keys split over workgroups where there are too few problems.
// The tile of 32 rows is the cache's own block: one scale for its keys, which multiplies the scores, and one for
// its values, which multiplies the weights; both are powers of two, so neither rounds.  The codes themselves go into
// the products as whole numbers, exact in bf16: three instructions for two of them.
//  * scores: K q^T on v_mfma_f32_16x16x32_bf16, the channels dealt to the lane groups in runs of d/4, so that a
//    lane's codes of a row are 32 (16) consecutive bytes; the order of a contraction is free as long as q has the same.
//  * values: 8 rows of a channel lie side by side, a lane's 8 contraction places; a lane has the channels 2i and
//    2i + 1 of every 32, 16 bytes.
//  * fp32 queries: q and the scaled weights as sums of three bf16 (24 bits), three products each.
// The cache's bytes bound it: 4 queries over 128k rows of 8 heads of 128 take 45 us, 6.0 TB/s, and the join of their
// splits 6; turning the codes to bf16 keeps the vector units 44% busy meanwhile.
#include <hip/hip_runtime.h>

#include "attn_split.h"
#include "codes8.h"

namespace twinkv {
namespace {

template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 1;

// One wave's 32 rows of the cache on their way through registers.  A lane's addresses of one tile lie at fixed
// distances, and move by whole tiles.
template <int D>
struct Tile8 {
  static constexpr int kPieces = D / 64;  // 16-byte pieces of a lane's part of a key
  const uint8_t *kp, *vp, *ksp, *vsp;
  u32x4 k[2][kPieces];
  u32x4 v[D / 32];     // channels 32n + 2i, 32n + 2i + 1: 8 rows each
  unsigned ks, vs;
  __device__ Tile8(const Cache8& c, int h, int64_t row, int i, int g) {  // row: in the head, a multiple of 32
    row += (int64_t)h * c.C;
    kp = c.k_codes + (row + 8 * (i >> 2) + (i & 3)) * D + g * (D / 4);
    vp = c.v_codes + (row + 8 * g) * D + i * 16;
    ksp = c.k_scales + row / kCache8Block;
    vsp = c.v_scales + row / kCache8Block;
  }
  __device__ void load_keys() {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int n = 0; n < kPieces; ++n) k[m][n] = *reinterpret_cast<const u32x4*>(kp + m * 4 * D + n * 16);
    ks = *ksp;
  }
  __device__ void load_values() {
#pragma unroll
    for (int n = 0; n < D / 32; ++n) v[n] = *reinterpret_cast<const u32x4*>(vp + n * 256);
    vs = *vsp;
  }
  __device__ void next_keys(int rows) {
    kp += rows * D;
    ksp += rows / kCache8Block;
    load_keys();
  }
  __device__ void next_values(int rows) {
    vp += rows * D;
    vsp += rows / kCache8Block;
    load_values();
  }
};

// R: row tiles of 16 that a wave takes at once; what it unpacks serves them all.  kScores: the scores are
// kept in LDS (one row tile a problem).  The accumulated weights follow from there where an item has all of the
// problem's keys; otherwise the scores go out, and the weights follow in the join.  (A step of 64 sequences of 1024 to
// 4096 rows, 8 heads of 4 queries, from the append to the read: 97 us of kernels; with K14 after the attention, which
// reads the keys again, 166.)
template <typename T, int D, int R, bool kScores>
__global__ __launch_bounds__(64 * kAttnWaves, sizeof(T) == 2 && R == 1 ? 4 : 2) void attn8_kernel(const AttnArgs a) {
  constexpr int kSteps = D / 32;
  constexpr int N = kParts<T>;
  __shared__ float s_join[join_floats<D>()];
  extern __shared__ __attribute__((aligned(16))) float s_score[];  // [rows][keys of the item]
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const AttnItem p = attn_item(a, (int)blockIdx.x, (int)blockIdx.y);
  const int len = min(max(a.len[(int64_t)p.h * a.n_seqs + p.s], 0), p.nk);
  const int n_rows = p.nq * a.group, row0 = p.rt * R * kAttnRows;
  const int last = min(row0 + R * kAttnRows, n_rows) - 1;
  const int lim_all = len - (p.nq - 1 - row0 / a.group);      // every row sees so many
  const int lim_any = len - (p.nq - 1 - last / a.group);      // no row sees more
  const int t0 = p.split * p.tiles * kAttnTile;
  const int t1 = min(lim_any, t0 + p.tiles * kAttnTile);

  int lim[R];
  bf16x8 q[R][N][kSteps];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    // rows past the problem's repeat its last, and are not written
    const int row = min(row0 + r * kAttnRows + i, n_rows - 1);
    const int query = row / a.group;
    lim[r] = len - (p.nq - 1 - query);
    const int64_t head = (int64_t)p.h * a.group + (row - query * a.group);
    const char* src = a.q + head * a.q_head + (int64_t)(p.q0 + query) * a.q_token;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      float x[8];
      Vec8<T>::load(src + (g * (D / 4) + j * 8) * (int)sizeof(T)).to(x);
      bf16x8 parts[N];
      split8<N>(x, parts);
#pragma unroll
      for (int n = 0; n < N; ++n) q[r][n][j] = parts[n];
    }
  }

  RowStats st[R];
  f32x4 acc[R][D / 16];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < D / 16; ++n) acc[r][n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int kStep = kAttnTile * kAttnWaves;
  const int first = t0 + wave * kAttnTile;
  const int keys = min(p.tiles * kAttnTile, p.nk - t0);  // of the item, seen or not
  Tile8<D> now(a.cache, p.h, (int64_t)p.k0 + first, i, g);
  if (first < t1) {
    now.load_keys();
    now.load_values();
  }
  for (int t = first; t < t1; t += kStep) {
    float s[R][8];
    const float scale_k = a.scale_log2 * __uint_as_float(now.ks << 23);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      f32x4 d[R];
#pragma unroll
      for (int r = 0; r < R; ++r) d[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const bf16x8 k = codes8_bf16(now.k[m][j >> 1][2 * (j & 1)], now.k[m][j >> 1][2 * (j & 1) + 1]);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int n = N - 1; n >= 0; --n) d[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[r][n][j], d[r], 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[r][4 * m + e] = d[r][e] * scale_k;
    }
    // the next tile, or this one once more: a load on one path only would make the waits of both longer
    const int ahead = t + kStep < t1 ? kStep : 0;
    now.next_keys(ahead);
    if (t + kAttnTile > lim_all) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (t + 8 * g + e >= lim[r]) s[r][e] = kNegInf;
    }
    if constexpr (kScores) {
      // (lanes past the last row have its scores and write the same)
      float* to = s_score + min(i, n_rows - 1) * keys + (t - t0) + 8 * g;
      *reinterpret_cast<f32x4*>(to) = f32x4{s[0][0], s[0][1], s[0][2], s[0][3]};
      *reinterpret_cast<f32x4*>(to + 4) = f32x4{s[0][4], s[0][5], s[0][6], s[0][7]};
    }
    const float scale_v = __uint_as_float(now.vs << 23);
    bf16x8 w[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      st[r].update(s[r], acc[r]);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = s[r][e] * scale_v;
      split8<N>(x, w[r]);
    }
#pragma unroll
    for (int b = 0; b < D / 16; ++b) {
      const u32x4 c = now.v[b >> 1];
      const bf16x8 v = codes8_bf16(c[2 * (b & 1)], c[2 * (b & 1) + 1]);
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int n = N - 1; n >= 0; --n) acc[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[r][n], v, acc[r][b], 0, 0, 0);
    }
    now.next_values(ahead);
    asm volatile("" ::: "memory");  // here, and not where the next tile begins: the scores cover the way
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r > 0) {
      if (row0 + r * kAttnRows >= n_rows) break;  // the same for the workgroup
      __syncthreads();                            // the tile before has been written
    }
    join_waves<T, D>(a, p, row0 + r * kAttnRows, st[r], acc[r], s_join,
                     [](int n, int lane16) { return (n >> 1) * 32 + 2 * lane16 + (n & 1); });
  }
  if constexpr (kScores) {
    if (p.splits > 1) {  // the join knows the rows' sums
      float* to = score_rows_of(a, p) + t0;
      for (int j = 4 * (int)threadIdx.x; j < t1 - t0; j += 4 * 64 * kAttnWaves)
        for (int r = 0; r < n_rows; ++r)
          *reinterpret_cast<f32x4*>(to + (int64_t)r * a.cache.C + j) = *reinterpret_cast<const f32x4*>(s_score + r * keys + j);
      return;
    }
    __shared__ RowLse s_lse;
    // (the tile's maxima and sums lie first in the join's place)
    if (threadIdx.x < kAttnRows) s_lse.put((int)threadIdx.x, s_join[threadIdx.x], s_join[kAttnRows + threadIdx.x]);
    __syncthreads();
    add_weights(a, p, s_lse, (int)threadIdx.x, 64 * kAttnWaves,
                [&](int row, int j) { return *reinterpret_cast<const f32x4*>(s_score + row * keys + j); });
  }
}

template <typename T, int D, int R, bool kScores>
int run8(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((attn8_kernel<T, D, R, kScores>), dim3((unsigned)a.items, (unsigned)a.n_heads), dim3(64 * kAttnWaves),
                     4 * (unsigned)a.score_lds, s, a);
  return hipGetLastError();
}
template <typename T, int D>
int run8(const AttnArgs& a, hipStream_t s) {
  return a.mass_out != nullptr ? run8<T, D, 1, true>(a, s) : run8<T, D, 1, false>(a, s);
}

}  // namespace

int launch_attn8(const AttnArgs& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype != 0) return d == 128 ? run8<float, 128>(a, s) : run8<float, 64>(a, s);
  if (a.rows == kAttnPairRows && a.mass_out != nullptr) return hipErrorInvalidValue;  // (no such kernel)
  if (a.rows == kAttnPairRows) return d == 128 ? run8<bf16, 128, 2, false>(a, s) : run8<bf16, 64, 2, false>(a, s);
  return d == 128 ? run8<bf16, 128>(a, s) : run8<bf16, 64>(a, s);
}

}  // namespace twinkv

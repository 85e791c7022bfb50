// K8: attention over the 4-bit cache, and the join of split rows (for K9 too).
//
// Few rows (the query heads of a KV head, times the new tokens) meet all cached rows, so the cache is
// what has to be read: HBM-bound, as long as the unpacking stays cheap.  Four waves share a tile of 16 rows and
// take 32 cached rows at a time each:
//  * scores: K q^T on v_mfma_f32_16x16x32_bf16.  A lane converts 8 codes in 4 instructions, with their
//    scale (v_cvt_scalef32_pk_bf16_fp4; a code times a power of two is exact in bf16).  The channels are
//    dealt to the lane groups in runs of d/4, so that a lane's codes of a row are one 16-byte load and
//    share one scale; the order of a contraction is free as long as q has the same.
//  * the product with the values: the scale of a value belongs to its row, a contraction place, so it
//    multiplies the weights instead (one product of 16 rows x 32 keys per group of 32 channels; a power
//    of two, so the weight's rounding to bf16 is the only one: error against 64 bits 0.0023 of the result's norm, 0.0017 of
//    it the output's own; with weights of two bf16 parts 0.0017, and 4 queries over 128k rows take 44 us instead of 39).
//  * fp32 queries: q and the scaled weights as sums of three bf16 (24 bits), three products each.
// The keys are split over workgroups when there are too few problems for the machine (attn_split.h).
// A tile costs about 260 vector instructions a wave, 16 of them matrix products, which keep the vector units busy 41%
// of the time its bytes take: 256 sequences of 2k rows, 8 heads of 4, d 128 120 us (4.8 TB/s; copy rate 111 us), 64 of 1k to 4k 42 us, one of
// 128k rows 32 us and 6.5 us for its join, one of 512 rows 8 us (launch and latency).  More rows than 16 a problem
// (8 heads of 8, 7 tokens: 56) unpack the cache once per tile, or pair of tiles: 282 us for the first of these.
#include <hip/hip_runtime.h>

#include "attn_split.h"

namespace twinkv {
namespace {

template <typename T>
constexpr int kParts = sizeof(T) == 4 ? 3 : 1;

__device__ inline bf16x8 codes8(unsigned w, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One wave's 32 rows of the cache on their way through registers.  A lane's addresses of one tile lie at fixed
// distances, and move by whole tiles.
template <int D>
struct Tile4 {
  const uint8_t *kp, *ksp, *vp, *vsp;
  u32x4 k[2];          // d 64: words 0, 1
  unsigned ks[2];
  u32x4 v[D / 64];
  u32x4 vs[D / 64];    // [d/32] groups of 8 bytes
  __device__ Tile4(const Cache4& c, int h, int64_t row, int i, int g) {  // row: in the head, a multiple of 32
    row += (int64_t)h * c.C;
    const int64_t r = row + 8 * (i >> 2) + (i & 3), b = row / kCacheBlock + g;
    kp = c.k_codes + r * (D / 2) + g * (D / 8);
    ksp = c.k_scales + r * (D / 32) + g * (D / 4) / 32;
    vp = c.v_codes + b * (D * 4) + i * 16;
    vsp = c.v_scales + b * (D / 4);
  }
  __device__ void load_keys() {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      if constexpr (D == 128) {
        k[m] = *reinterpret_cast<const u32x4*>(kp + m * 4 * (D / 2));
      } else {
        const u32x2 w = *reinterpret_cast<const u32x2*>(kp + m * 4 * (D / 2));
        k[m] = u32x4{w[0], w[1], 0u, 0u};
      }
      ks[m] = ksp[m * 4 * (D / 32)];
    }
  }
  __device__ void load_values() {
#pragma unroll
    for (int a = 0; a < D / 64; ++a) {
      v[a] = *reinterpret_cast<const u32x4*>(vp + a * 256);
      vs[a] = *reinterpret_cast<const u32x4*>(vsp + a * 16);
    }
  }
  __device__ void next_keys(int rows) {
    kp += rows * (D / 2);
    ksp += rows * (D / 32);
    load_keys();
  }
  __device__ void next_values(int rows) {
    vp += rows * (D / 2);
    vsp += rows * (D / 32);
    load_values();
  }
};

// R: row tiles of 16 that a wave takes at once; what it unpacks serves them all.
template <typename T, int D, int R>
__global__ __launch_bounds__(64 * kAttnWaves, sizeof(T) == 2 && R == 1 ? 4 : 2) void attn4_kernel(const AttnArgs a) {
  constexpr int kSteps = D / 32;
  constexpr int N = kParts<T>;
  __shared__ float s_join[join_floats<D>()];
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
  Tile4<D> now(a.cache, p.h, (int64_t)p.k0 + first, i, g);
  if (first < t1) {
    now.load_keys();
    now.load_values();
  }
  for (int t = first; t < t1; t += kStep) {
    float s[R][8];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float scale = __uint_as_float(now.ks[m] << 23);
      f32x4 d[R];
#pragma unroll
      for (int r = 0; r < R; ++r) d[r] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < kSteps; ++j) {
        const bf16x8 k = codes8(now.k[m][j], scale);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int n = N - 1; n >= 0; --n) d[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[r][n][j], d[r], 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[r][4 * m + e] = d[r][e] * a.scale_log2;
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
      if (t + kAttnTile > len) {  // rows not in use: their scales may be anything
        const int use = min(max(len - (t + 8 * g), 0), 8);
        const unsigned lo = use >= 4 ? ~0u : (1u << (8 * use)) - 1u;
        const unsigned hi = use >= 8 ? ~0u : use <= 4 ? 0u : (1u << (8 * (use - 4))) - 1u;
#pragma unroll
        for (int x = 0; x < D / 64; ++x) now.vs[x] = u32x4{now.vs[x][0] & lo, now.vs[x][1] & hi, now.vs[x][2] & lo, now.vs[x][3] & hi};
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) st[r].update(s[r], acc[r]);
#pragma unroll
    for (int grp = 0; grp < D / 32; ++grp) {
      bf16x8 w[R][N];
      float scale[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const unsigned b = now.vs[grp >> 1][(grp & 1) * 2 + (e >> 2)];
        scale[e] = __uint_as_float(((b >> (8 * (e & 3))) & 255u) << 23);
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[r][e] * scale[e];
        split8<N>(x, w[r]);
      }
#pragma unroll
      for (int b = 2 * grp; b < 2 * grp + 2; ++b) {
        const bf16x8 v = codes8(now.v[b >> 2][b & 3], 1.0f);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int n = N - 1; n >= 0; --n) acc[r][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[r][n], v, acc[r][b], 0, 0, 0);
      }
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
    join_waves<T, D>(a, p, row0 + r * kAttnRows, st[r], acc[r], s_join, [](int n, int lane16) { return n * 16 + lane16; });
  }
}

// The join: a row tile's parts brought to one maximum.  The tile's items share its rows out among them (item
// `split` takes rows split, split + splits, ...).  Of a workgroup, D / 8 threads make a team that holds a row's
// channels; as many teams as there are parts (a power of two, at most all of them) work on one row and add up
// through LDS, the others on the next rows.
// Accumulated weights (8 bits) are a branch of the same kernel.  One without them has 48 registers instead of 79, and is no
// faster: 56 rows over 128k rows 6.9 us, with the branch 6.1; 64 queries over 32k keys 9.9 / 8.7; 4 over 128k 6.9 / 6.3; 16
// sequences of 5000 4.3 / 4.3.
constexpr int kJoinThreads = 256;
template <typename T, int D>
__global__ __launch_bounds__(kJoinThreads) void attn_join_kernel(const AttnArgs a) {
  constexpr int kPieces = D / 8, kTeams = kJoinThreads / kPieces;
  __shared__ float s_o[kTeams][D];
  __shared__ float s_ml[kTeams][2];
  const AttnItem p = attn_item(a, (int)blockIdx.x, (int)blockIdx.y);
  if (p.splits <= 1) return;
  const int c = threadIdx.x % kPieces * 8, team = threadIdx.x / kPieces;
  int per_row = 1;
  while (per_row < kTeams && per_row < p.splits) per_row *= 2;
  const int first = team & (per_row - 1), slot = team / per_row;  // part to begin with, row of those at hand
  const int rows = a.rows, n_rows = p.nq * a.group, at_once = kTeams / per_row;
  for (int r0 = p.split; r0 < rows && p.rt * rows + r0 < n_rows; r0 += at_once * p.splits) {
    const int r = r0 + slot * p.splits, row = p.rt * rows + r;
    const bool live = r < rows && row < n_rows;
    float top = kNegInf, sum = 0.0f, f[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](float m, float l, const float (&x)[8]) {
      const float next = fmaxf(top, m);
      const float u = next == top ? 1.0f : __builtin_amdgcn_exp2f(top - next);
      const float w = m == next ? 1.0f : __builtin_amdgcn_exp2f(m - next);
      top = next;
      sum = sum * u + l * w;
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = f[e] * u + x[e] * w;
    };
    if (live) {
      const int64_t part = (p.part - p.split) * rows + r;  // of split 0
      const float* ml = a.part_ml + part * 2;
      const float* o = a.part_o + part * D + c;
      for (int k = first; k < p.splits; k += per_row) {
        float x[8];
        load8(o + (int64_t)k * rows * D, x);
        add(ml[(int64_t)k * rows * 2], ml[(int64_t)k * rows * 2 + 1], x);
      }
    }
    if (per_row > 1) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s_o[team][c + e] = f[e];
      if (c == 0) {
        s_ml[team][0] = top;
        s_ml[team][1] = sum;
      }
      __syncthreads();
      if (first == 0) {
        for (int k = 1; k < per_row; ++k) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = s_o[team + k][c + e];
          add(s_ml[team + k][0], s_ml[team + k][1], x);
        }
      }
      __syncthreads();
    }
    if (!live || first != 0) continue;
    const float inv = sum > 0.0f ? 1.0f / sum : (sum == 0.0f ? 0.0f : sum);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] *= inv;
    const int i = row / a.group, g = row - i * a.group;
    const int64_t head = (int64_t)p.h * a.group + g;
    Vec8<T>::from(f).store(a.out + head * a.o_head + (int64_t)(p.q0 + i) * a.o_token + c * (int)sizeof(T));
    if (a.lse != nullptr && c == 0)
      a.lse[head * a.Tq + p.q0 + i] = sum == 0.0f ? kNegInf : top * 0.69314718055994530942f + logf(sum);
  }
  if (a.mass_out == nullptr) return;
  // The accumulated weights of the split's keys (one tile of 16 rows a problem): every row's maximum and sum again, 16
  // threads a row.
  __shared__ RowLse s_lse;
  static_assert(kJoinThreads == 16 * kAttnRows, "16 threads a row");
  const int r = threadIdx.x / 16;
  float top = kNegInf, sum = 0.0f;
  auto add = [&](float m, float l) {
    const float next = fmaxf(top, m);
    sum = sum * (next == top ? 1.0f : __builtin_amdgcn_exp2f(top - next)) + l * (m == next ? 1.0f : __builtin_amdgcn_exp2f(m - next));
    top = next;
  };
  const float* ml = a.part_ml + ((p.part - p.split) * rows + r) * 2;
  for (int k = threadIdx.x % 16; k < p.splits; k += 16) add(ml[(int64_t)k * rows * 2], ml[(int64_t)k * rows * 2 + 1]);
#pragma unroll
  for (int by = 1; by < 16; by *= 2) {
    const float m = __shfl_xor(top, by), l = __shfl_xor(sum, by);
    add(m, l);
  }
  if (threadIdx.x % 16 == 0) s_lse.put(r, top, sum);
  __syncthreads();
  const float* scores = score_rows_of(a, p);
  add_weights(a, p, s_lse, (int)threadIdx.x, kJoinThreads, [&](int row, int j) {
    return *reinterpret_cast<const f32x4*>(scores + (int64_t)row * a.cache.C + j);
  });
}

template <typename T, int D, int R>
int run4(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((attn4_kernel<T, D, R>), dim3((unsigned)a.items, (unsigned)a.n_heads), dim3(64 * kAttnWaves), 0, s, a);
  return hipGetLastError();
}
template <typename T, int D>
int run_join(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((attn_join_kernel<T, D>), dim3((unsigned)a.items, (unsigned)a.n_heads), dim3(kJoinThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int launch_attn4(const AttnArgs& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype != 0) return d == 128 ? run4<float, 128, 1>(a, s) : run4<float, 64, 1>(a, s);
  if (a.rows == kAttnPairRows) return d == 128 ? run4<bf16, 128, 2>(a, s) : run4<bf16, 64, 2>(a, s);
  return d == 128 ? run4<bf16, 128, 1>(a, s) : run4<bf16, 64, 1>(a, s);
}

int launch_attn_join(const AttnArgs& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 0) return d == 128 ? run_join<bf16, 128>(a, s) : run_join<bf16, 64>(a, s);
  return d == 128 ? run_join<float, 128>(a, s) : run_join<float, 64>(a, s);
}

}  // namespace twinkv

// K7: the 4-bit cache: compaction into it (the retained rows' positions, then the rows in 4 bits),
// appending new tokens, and reading rows back.
//
// An element x of a group of 32 channels with largest magnitude a is stored as the nearest of
// 0, .5, 1, 1.5, 2, 3, 4, 6 (with sign) to x / 2^e, e the smallest with a / 2^e < 7: below 7 the largest
// element still rounds to 6, and a coarser grid for all 32 would cost more than that one's error.
// The scale is a power of two, so x / 2^e is exact and the codes do not depend on how they are computed.
//
// Keys are read as rows by the attention (a contraction over channels) and stored as rows.  Values
// are contracted over tokens: 8 rows of a channel share a word, the matrix operand's 8 consecutive
// tokens.  So one wave makes 8 rows: each row belongs to d/8 lanes of 8 channels (16-byte loads of
// bf16), a group's maximum takes two quad exchanges, and the values' words are turned (8 rows x 8
// channels of nibbles) through 512 bytes of the wave's own LDS.  HBM-bound: 288 heads, 6553 of 16384 rows of 128
// each, bf16: the positions 13 us, the rows 260 us (1.22 GB, 4.7 TB/s), reading them back 249 us (4.9 TB/s).
#include <hip/hip_runtime.h>

#include "../cache_ops.h"
#include "rows.h"
#include "seq_words.h"

namespace twinkv {
namespace {

constexpr int kOk = 0, kMismatch = 1, kNonfinite = 2;  // TWINKV_PROBLEM_*
constexpr int kThreads = 256;                          // gather, read
constexpr int kPosThreads = 1024;
constexpr int kMaxWaves = 16;                          // append: blocks a workgroup takes at once

__device__ inline unsigned quad_xor1(unsigned x) {
  return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true);
}
__device__ inline unsigned quad_xor2(unsigned x) {
  return (unsigned)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true);
}

// 8 channels' codes; four neighbouring lanes hold a group of 32.
struct Coded {
  unsigned word;
  int byte;
  bool bad;
};
template <typename T>
__device__ inline Coded encode(const Vec8<T>& v) {
  float x[8];
  v.to(x);
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);  // NaN above infinity above numbers
  m = max(m, quad_xor1(m));
  m = max(m, quad_xor2(m));
  Coded c;
  c.bad = m >= 0x7f800000u;
  c.byte = c.bad ? 1 : min(max((int)((m + 0x200000u) >> 23) - 2, 1), 252);
  const float s = __uint_as_float((unsigned)c.byte << 23);
  unsigned w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  c.word = c.bad ? 0u : w;
  return c;
}

// What one wave needs of LDS to turn a block: the value words [8 rows][d/8].
template <int D>
struct TurnBuf {
  unsigned w[kCacheBlock * (D / 8)];
};

__device__ inline void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Channel of the value place p (see include/twinkv.h).
__device__ inline int channel_of_place(int p) {
  return (p & 64) + 16 * (p & 3) + ((p >> 2) & 15);
}

// One wave writes rows [lo, hi) of block `blk` of head h, row r from src(r) (its key and value rows,
// null outside); the block's other value rows stay (keep) or become zeros.  Returns whether an element
// was not finite.
template <typename T, int D, typename Src>
__device__ inline bool write_block(const Cache4& c, int h, int64_t blk, int lo, int hi, bool keep,
                                   TurnBuf<D>& buf, const Src& src) {
  constexpr int kLanes = D / 8;            // lanes of a row
  constexpr int kRows = 64 / kLanes;       // rows at a time
  constexpr int kPasses = kCacheBlock / kRows;
  constexpr int kGroups = D / 32;
  const int lane = threadIdx.x & 63;
  const int piece = lane % kLanes;
  Vec8<T> k[kPasses], v[kPasses];
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int r = u * kRows + lane / kLanes;
    // rows outside [lo, hi) load a row inside it and store nothing
    const int rr = min(max(r, lo), hi - 1);
    const char *kp, *vp;
    src(rr, kp, vp);
    k[u] = Vec8<T>::load(kp + piece * 8 * (int)sizeof(T));
    v[u] = Vec8<T>::load(vp + piece * 8 * (int)sizeof(T));
  }
  bool bad = false;
  const int64_t row0 = (int64_t)h * c.C + blk * kCacheBlock;
  const int64_t vblk = (int64_t)h * (c.C / kCacheBlock) + blk;
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int r = u * kRows + lane / kLanes;
    const Coded a = encode(k[u]), b = encode(v[u]);
    const bool mine = r >= lo && r < hi;
    if (mine) {
      bad |= a.bad | b.bad;
      *reinterpret_cast<unsigned*>(c.k_codes + (row0 + r) * (D / 2) + piece * 4) = a.word;
      if (piece % 4 == 0) {
        c.k_scales[(row0 + r) * kGroups + piece / 4] = (uint8_t)a.byte;
        c.v_scales[vblk * (kGroups * kCacheBlock) + (piece / 4) * kCacheBlock + r] = (uint8_t)b.byte;
      }
    }
    buf.w[r * kLanes + piece] = mine ? b.word : 0u;
  }
  wave_sync();
  constexpr int kPlaces = D / 64;          // value words a lane makes, side by side
  unsigned out[kPlaces];
#pragma unroll
  for (int n = 0; n < kPlaces; ++n) {
    const int ch = channel_of_place(lane * kPlaces + n);
    unsigned w = 0;
#pragma unroll
    for (int r = 0; r < kCacheBlock; ++r) w |= ((buf.w[r * kLanes + ch / 8] >> (4 * (ch % 8))) & 15u) << (4 * r);
    out[n] = w;
  }
  unsigned* to = reinterpret_cast<unsigned*>(c.v_codes) + vblk * D + lane * kPlaces;
  if (keep && (lo > 0 || hi < kCacheBlock)) {
    const unsigned upto = hi < kCacheBlock ? (1u << (4 * hi)) - 1u : ~0u;
    const unsigned mask = upto & ~((1u << (4 * lo)) - 1u);
#pragma unroll
    for (int n = 0; n < kPlaces; ++n) out[n] = (to[n] & ~mask) | out[n];
  }
#pragma unroll
  for (int n = 0; n < kPlaces; ++n) to[n] = out[n];
  wave_sync();                             // the buffer may be filled again
  return __any(bad);
}

// ---- compaction ----

// Exclusive ranks of the threads' counts in the workgroup, and their total.
__device__ inline int block_rank(int n, int& total, int* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = n;
  for (int off = 1; off < 64; off <<= 1) {
    const int up = __shfl_up(incl, off);
    if (lane >= off) incl += up;
  }
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPosThreads / 64; ++w) {
    before += w < wave ? s_wave[w] : 0;
    total += s_wave[w];
  }
  __syncthreads();
  return before + incl - n;
}

// K7a: one workgroup per problem lists its retained positions, 16 mask bytes a thread at a time.
__global__ __launch_bounds__(kPosThreads) void cache4_positions_kernel(const Cache4Args a) {
  __shared__ int s_wave[kPosThreads / 64];
  const int s = (int)blockIdx.x % a.n_seqs, h = (int)blockIdx.x / a.n_seqs;
  const int t0 = seq_word(a.seq, s * kCacheSeqWords), t1 = seq_word(a.seq, (s + 1) * kCacheSeqWords);
  const int r0 = seq_word(a.seq, s * kCacheSeqWords + 1), r1 = seq_word(a.seq, (s + 1) * kCacheSeqWords + 1);
  const int n = t1 - t0, cap = r1 - r0;
  const uint8_t* m = a.retained + (int64_t)h * a.T + t0;
  int32_t* pos = a.pos + (int64_t)h * a.cache.C + r0;
  int have = 0;
  for (int base = 0; base < n; base += kPosThreads * 16) {
    const int at = base + (int)threadIdx.x * 16;
    unsigned bits = 0;
    if (at + 16 <= n) {
      u32x4 w;
      __builtin_memcpy(&w, m + at, 16);
#pragma unroll
      for (int e = 0; e < 16; ++e) bits |= (((w[e >> 2] >> (8 * (e & 3))) & 255u) != 0 ? 1u : 0u) << e;
    } else {
      for (int e = 0; at + e < n; ++e) bits |= (m[at + e] != 0 ? 1u : 0u) << e;
    }
    int total;
    int row = have + block_rank(__popc(bits), total, s_wave);
    while (bits != 0) {
      const int e = __ffs(bits) - 1;
      bits &= bits - 1;
      if (row < cap) pos[row] = at + e;
      ++row;
    }
    have += total;
  }
  const bool over = have > cap;
  if (over) {
    __threadfence_block();
    __syncthreads();  // the rows listed above are taken back
  }
  for (int r = (over ? 0 : have) + (int)threadIdx.x; r < cap; r += kPosThreads) pos[r] = -1;
  if (threadIdx.x == 0) {
    const int64_t q = (int64_t)h * a.n_seqs + s;
    a.len_out[q] = over ? 0 : have;
    a.status[q] = over ? kMismatch : kOk;
  }
}

// K7b: a wave per block of 8 rows.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void cache4_gather_kernel(const Cache4Args a) {
  __shared__ TurnBuf<D> s_buf[kThreads / 64];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int b = (int)blockIdx.x * (kThreads / 64) + wave;
  const int h = (int)blockIdx.y;
  if (b >= a.n_blocks) return;
  const int s = find_seq(a.seq, a.n_seqs, kCacheSeqWords, 2, b);
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const int first = (b - seq_word(a.seq, s * kCacheSeqWords + 2)) * kCacheBlock;  // row of the problem
  const int hi = min(kCacheBlock, a.len_out[q] - first);
  if (hi <= 0) return;
  const int row0 = seq_word(a.seq, s * kCacheSeqWords + 1) + first;
  const int32_t* pos = a.pos + (int64_t)h * a.cache.C + row0;
  const int64_t t0 = seq_word(a.seq, s * kCacheSeqWords);
  const char* kb = a.keys + (int64_t)h * a.head_stride + t0 * a.token_stride;
  const char* vb = a.values + (int64_t)h * a.v_head_stride + t0 * a.v_token_stride;
  const bool bad = write_block<T, D>(a.cache, h, row0 / kCacheBlock, 0, hi, false, s_buf[wave],
                                     [&](int r, const char*& kp, const char*& vp) {
                                       const int64_t t = pos[r];
                                       kp = kb + t * a.token_stride;
                                       vp = vb + t * a.v_token_stride;
                                     });
  if (bad && (threadIdx.x & 63) == 0) a.status[q] = kNonfinite;
}

// ---- append ----

// One wave writes those of the problem's `n` new tokens (from t0) that belong to the j-th block from the
// one row `len` lies in.  Returns whether an element was not finite.
template <typename T, int D>
__device__ inline bool append_block(const Cache4Args& a, int h, int64_t r0, int len, int64_t t0, int n, int j,
                                    TurnBuf<D>& buf) {
  const int base = (len / kCacheBlock + j) * kCacheBlock;  // first row of the block, in the problem
  const int lo = max(len - base, 0), hi = min(len + n - base, kCacheBlock);
  if (hi <= lo) return false;
  const char* kb = a.keys + (int64_t)h * a.head_stride + (t0 + base - len) * a.token_stride;
  const char* vb = a.values + (int64_t)h * a.v_head_stride + (t0 + base - len) * a.v_token_stride;
  return write_block<T, D>(a.cache, h, (r0 + base) / kCacheBlock, lo, hi, true, buf,
                           [&](int r, const char*& kp, const char*& vp) {
                             kp = kb + (int64_t)r * a.token_stride;
                             vp = vb + (int64_t)r * a.v_token_stride;
                           });
}

struct AppendTo {
  int64_t r0, t0;
  int cap, n;
};
__device__ inline AppendTo append_to(const Cache4Args& a, int s) {
  AppendTo p;
  p.t0 = seq_word(a.seq, s * kCacheSeqWords);
  p.n = seq_word(a.seq, (s + 1) * kCacheSeqWords) - (int)p.t0;
  p.r0 = seq_word(a.seq, s * kCacheSeqWords + 1);
  p.cap = seq_word(a.seq, (s + 1) * kCacheSeqWords + 1) - (int)p.r0;
  return p;
}

// K7c: a workgroup takes one problem's new tokens, so that it alone reads len_in and writes len_out
// (which may be one array) and the status.  Up to 16 blocks; as two launches these take longer (8 heads, 4
// tokens 4.0 us here, 5.4 there; 64 sequences of 100 tokens 8.0 / 10.5).
template <typename T, int D>
__global__ __launch_bounds__(kMaxWaves * 64) void cache4_append_kernel(const Cache4Args a) {
  __shared__ TurnBuf<D> s_buf[kMaxWaves];
  __shared__ int s_bad;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int s = (int)blockIdx.x % a.n_seqs, h = (int)blockIdx.x / a.n_seqs;
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const AppendTo p = append_to(a, s);
  const int len = a.len_in[q];
  const bool fits = len >= 0 && len <= p.cap - p.n;
  if (threadIdx.x == 0) s_bad = 0;
  __syncthreads();
  if (fits && append_block<T, D>(a, h, p.r0, len, p.t0, p.n, wave, s_buf[wave]) && (threadIdx.x & 63) == 0)
    s_bad = 1;
  __syncthreads();
  if (threadIdx.x == 0) {
    a.len_out[q] = fits ? len + p.n : len;
    a.status[q] = !fits ? kMismatch : s_bad ? kNonfinite : kOk;
  }
}

// Many new tokens: the lengths and states first, then a wave per block of every problem.
__global__ __launch_bounds__(kThreads) void cache4_grow_kernel(const Cache4Args a) {
  const int q = (int)(blockIdx.x * kThreads + threadIdx.x);
  if (q >= a.n_heads * a.n_seqs) return;
  const int w = q % a.n_seqs * kCacheSeqWords;  // another sequence in each lane
  const int n = seq_word_of_lane(a.seq, w + kCacheSeqWords) - seq_word_of_lane(a.seq, w);
  const int cap = seq_word_of_lane(a.seq, w + kCacheSeqWords + 1) - seq_word_of_lane(a.seq, w + 1);
  const int len = a.len_in[q];
  const bool fits = len >= 0 && len <= cap - n;
  a.len_out[q] = fits ? len + n : len;
  a.status[q] = fits ? kOk : kMismatch;
}
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void cache4_append_many_kernel(const Cache4Args a) {
  __shared__ TurnBuf<D> s_buf[kThreads / 64];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int b = (int)blockIdx.x * (kThreads / 64) + wave;
  const int h = (int)blockIdx.y;
  if (b >= a.n_blocks) return;
  const int s = find_seq(a.seq, a.n_seqs, kCacheSeqWords, 2, b);
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const AppendTo p = append_to(a, s);
  // another wave may have made it NONFINITE already, which is as good as OK here
  if (__builtin_amdgcn_readfirstlane(a.status[q]) == kMismatch) return;
  const int len = a.len_out[q] - p.n;
  if (append_block<T, D>(a, h, p.r0, len, p.t0, p.n, b - seq_word(a.seq, s * kCacheSeqWords + 2), s_buf[wave]) &&
      (threadIdx.x & 63) == 0)
    a.status[q] = kNonfinite;
}

// ---- read ----

__device__ inline void decode(unsigned w, float scale, float (&x)[8]) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3);
  x[0] = (float)a[0] * scale, x[1] = (float)a[1] * scale, x[2] = (float)b[0] * scale, x[3] = (float)b[1] * scale;
  x[4] = (float)c[0] * scale, x[5] = (float)c[1] * scale, x[6] = (float)d[0] * scale, x[7] = (float)d[1] * scale;
}

// K7d: a wave per block of the cache that holds rows to read.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void cache4_read_kernel(const Cache4Args a) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes, kPasses = kCacheBlock / kRows, kGroups = D / 32;
  __shared__ TurnBuf<D> s_buf[kThreads / 64];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int b = (int)blockIdx.x * (kThreads / 64) + wave;
  const int h = (int)blockIdx.y;
  if (b >= a.n_blocks) return;
  const int s = find_seq(a.seq, a.n_seqs, kCacheSeqWords, 2, b);
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const int o0 = seq_word(a.seq, s * kCacheSeqWords), n = seq_word(a.seq, (s + 1) * kCacheSeqWords) - o0;
  const int64_t r0 = seq_word(a.seq, s * kCacheSeqWords + 1);
  const int cap = seq_word(a.seq, (s + 1) * kCacheSeqWords + 1) - (int)r0;
  const int len = min(a.len_in[q], cap);
  const int64_t first = a.first != nullptr ? a.first[q] : 0;
  const int64_t base = ((first >> 3) + (b - seq_word(a.seq, s * kCacheSeqWords + 2))) * kCacheBlock;  // cache row
  const int lane = threadIdx.x & 63, piece = lane % kLanes;
  const bool any = base >= 0 && base < len;  // else every row of the block is zero
  const int64_t row0 = (int64_t)h * a.cache.C + r0 + base;
  const int64_t vblk = (int64_t)h * (a.cache.C / kCacheBlock) + (r0 + base) / kCacheBlock;
  TurnBuf<D>& buf = s_buf[wave];
  if (any && a.values_out != nullptr) {
    constexpr int kPlaces = D / 64;
    const unsigned* from = reinterpret_cast<const unsigned*>(a.cache.v_codes) + vblk * D + lane * kPlaces;
#pragma unroll
    for (int p = 0; p < kPlaces; ++p) buf.w[channel_of_place(lane * kPlaces + p)] = from[p];
  }
  wave_sync();
#pragma unroll
  for (int u = 0; u < kPasses; ++u) {
    const int r = u * kRows + lane / kLanes;
    const int64_t o = base + r - first;  // output row of the problem
    if (o < 0 || o >= n) continue;
    const bool live = base + r >= 0 && base + r < len;
    const int64_t to = (((int64_t)h * a.C_out + o0 + o) * D + piece * 8) * (int64_t)sizeof(T);
    float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (a.keys_out != nullptr) {
      if (live) {
        const unsigned w = *reinterpret_cast<const unsigned*>(a.cache.k_codes + (row0 + r) * (D / 2) + piece * 4);
        decode(w, __uint_as_float((unsigned)a.cache.k_scales[(row0 + r) * kGroups + piece / 4] << 23), x);
      }
      Vec8<T>::from(x).store(a.keys_out + to);
    }
    if (a.values_out != nullptr) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = 0.0f;
      if (live) {
        unsigned w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= ((buf.w[piece * 8 + e] >> (4 * r)) & 15u) << (4 * e);
        const uint8_t byte = a.cache.v_scales[vblk * (kGroups * kCacheBlock) + (piece / 4) * kCacheBlock + r];
        decode(w, __uint_as_float((unsigned)byte << 23), x);
      }
      Vec8<T>::from(x).store(a.values_out + to);
    }
  }
}

template <typename T, int D>
int launch_gather(const Cache4Args& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n_blocks + kThreads / 64 - 1) / (kThreads / 64)), (unsigned)a.n_heads);
  hipLaunchKernelGGL((cache4_gather_kernel<T, D>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <typename T, int D>
int launch_append(const Cache4Args& a, int max_new, hipStream_t s) {
  const int blocks = (max_new + 2 * kCacheBlock - 2) / kCacheBlock;  // of one problem, at any len
  if (blocks <= kMaxWaves) {
    hipLaunchKernelGGL((cache4_append_kernel<T, D>), dim3((unsigned)a.n_heads * (unsigned)a.n_seqs),
                       dim3(64 * (unsigned)blocks), 0, s, a);
    return hipGetLastError();
  }
  const unsigned problems = (unsigned)a.n_heads * (unsigned)a.n_seqs;
  hipLaunchKernelGGL(cache4_grow_kernel, dim3((problems + kThreads - 1) / kThreads), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return (int)e;
  const dim3 grid((unsigned)((a.n_blocks + kThreads / 64 - 1) / (kThreads / 64)), (unsigned)a.n_heads);
  hipLaunchKernelGGL((cache4_append_many_kernel<T, D>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <typename T, int D>
int launch_read(const Cache4Args& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n_blocks + kThreads / 64 - 1) / (kThreads / 64)), (unsigned)a.n_heads);
  hipLaunchKernelGGL((cache4_read_kernel<T, D>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int launch_cache4_positions(const Cache4Args& a, void* stream) {
  hipLaunchKernelGGL(cache4_positions_kernel, dim3((unsigned)a.n_heads * (unsigned)a.n_seqs), dim3(kPosThreads), 0,
                     (hipStream_t)stream, a);
  return hipGetLastError();
}

int launch_cache4_gather(const Cache4Args& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (a.n_blocks == 0) return hipSuccess;
  if (dtype == 0) return d == 128 ? launch_gather<bf16, 128>(a, s) : launch_gather<bf16, 64>(a, s);
  return d == 128 ? launch_gather<float, 128>(a, s) : launch_gather<float, 64>(a, s);
}

int launch_cache4_append(const Cache4Args& a, int max_new, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 0) return d == 128 ? launch_append<bf16, 128>(a, max_new, s) : launch_append<bf16, 64>(a, max_new, s);
  return d == 128 ? launch_append<float, 128>(a, max_new, s) : launch_append<float, 64>(a, max_new, s);
}

int launch_cache4_read(const Cache4Args& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (a.n_blocks == 0) return hipSuccess;
  if (dtype == 0) return d == 128 ? launch_read<bf16, 128>(a, s) : launch_read<bf16, 64>(a, s);
  return d == 128 ? launch_read<float, 128>(a, s) : launch_read<float, 64>(a, s);
}

}  // namespace twinkv

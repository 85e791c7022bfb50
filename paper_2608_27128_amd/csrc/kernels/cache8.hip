// K11: the 8-bit cache: compaction into it, appending new tokens, reading rows back, and moving the rows that an
// eviction keeps into another cache.
//
// 32 rows of a head share a scale 2^e for their keys and one for their values, e the smallest with which the
// largest element x of them all has |x| / 2^e < 127.5; elements are the nearest whole numbers to x / 2^e, ties to
// the even one.  The scale is a power of two, so x / 2^e is exact, the codes do not depend on how they are
// computed, the values are exact in bf16, and rows that move to a block of the same scale keep their codes.  (The
// largest element over 127 as the scale would halve the step at best; but a block that grows row by row, as in
// decoding, would be rounded anew at almost every larger row.)
//
// Keys are stored as rows (the attention contracts over channels), values 8 rows of a channel side by side (it
// contracts over rows).  One wave makes the 32 rows of a scale: a lane has 8 rows of d/16 channels, so the turn
// from rows to channels stays in its registers (4 x 4 bytes in 8 v_perm), and the largest element takes six
// exchanges in the wave.
//
// HBM bounds all of it at size.  288 heads, 6553 of 16384 rows of 128 in bf16: gathered in 281 us (966 MB read, 483
// written: 5.2 TB/s), read back in 250 (5.8 TB/s).  64 sequences of 1024 to 4096 rows, three quarters moved: 135 us.
// Appended: 4096 rows to 288 heads 140 us (6.5 TB/s), 512 to 64 sequences of 8 heads 35 us (5.8 TB/s), 4096 to 8 heads 8.7 us,
// each after 2 to 4 us for the lengths; one row to each of 512 problems 6 us.
#include <hip/hip_runtime.h>

#include "../cache_ops.h"
#include "rows.h"
#include "seq_words.h"

namespace twinkv {
namespace {

constexpr int kOk = 0, kMismatch = 1, kNonfinite = 2;  // TWINKV_PROBLEM_*
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kByteMin = 1, kByteMax = 248;            // 127 * 2^121 is finite in fp32 and bf16
constexpr int kBlockBits = 5;
static_assert(1 << kBlockBits == kCache8Block, "rows of a block");
constexpr int kAppendBlocks = 4;                       // that one wave writes one after the other

// A lane's part of a block: rows 8 sub .. 8 sub + 7, channels at .. at + kCh.
template <int D>
struct Part {
  static constexpr int kCh = D / 16, kWords = kCh / 4;
  int sub, at;
  __device__ Part() : sub(((int)threadIdx.x & 63) >> 4), at(((int)threadIdx.x & 15) * kCh) {}
};

__device__ inline unsigned lane_xor(unsigned x, int by) { return (unsigned)__shfl_xor((int)x, by); }

__device__ inline float power_of(int byte) { return __uint_as_float((unsigned)byte << 23); }  // 2^(byte - 127)

// CH channels of a row.
template <typename T, int CH>
struct Piece;
template <>
struct Piece<bf16, 8> {
  u32x4 v;
  __device__ void load(const char* p) { v = *reinterpret_cast<const u32x4*>(p); }
  __device__ unsigned bits(int c) const { return c & 1 ? v[c >> 1] & 0xffff0000u : v[c >> 1] << 16; }
};
template <>
struct Piece<bf16, 4> {
  u32x2 v;
  __device__ void load(const char* p) { v = *reinterpret_cast<const u32x2*>(p); }
  __device__ unsigned bits(int c) const { return c & 1 ? v[c >> 1] & 0xffff0000u : v[c >> 1] << 16; }
};
template <>
struct Piece<float, 8> {
  u32x4 a, b;
  __device__ void load(const char* p) {
    a = *reinterpret_cast<const u32x4*>(p);
    b = *reinterpret_cast<const u32x4*>(p + 16);
  }
  __device__ unsigned bits(int c) const { return c < 4 ? a[c & 3] : b[c & 3]; }
};
template <>
struct Piece<float, 4> {
  u32x4 a;
  __device__ void load(const char* p) { a = *reinterpret_cast<const u32x4*>(p); }
  __device__ unsigned bits(int c) const { return a[c]; }
};

// The nearest whole number to y, |y| <= 127, in the low byte: 1.5 * 2^23 leaves a float no bits below 1.
__device__ inline unsigned nearest(float y) { return __float_as_uint(y + 12582912.0f); }
__device__ inline unsigned pack4(unsigned a, unsigned b, unsigned c, unsigned d) {
  const unsigned lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
  return lo | hi;
}
__device__ inline float code_of(unsigned word, int i) { return (float)(int8_t)(word >> (8 * i)); }

// 4 x 4 bytes: byte i of word j becomes byte j of word i.
__device__ inline void turn4(const unsigned (&w)[4], unsigned (&o)[4]) {
  const unsigned t0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), t1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
  const unsigned u0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), u1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
  o[0] = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
  o[1] = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}
// 8 rows of CH bytes as CH channels of 8 bytes, and back.
template <int CH>
__device__ inline void to_channels(const unsigned (&rows)[8][CH / 4], unsigned (&ch)[CH][2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int c = 0; c < CH / 4; ++c) {
      const unsigned w[4] = {rows[4 * h][c], rows[4 * h + 1][c], rows[4 * h + 2][c], rows[4 * h + 3][c]};
      unsigned o[4];
      turn4(w, o);
#pragma unroll
      for (int i = 0; i < 4; ++i) ch[4 * c + i][h] = o[i];
    }
}
template <int CH>
__device__ inline void to_rows(const unsigned (&ch)[CH][2], unsigned (&rows)[8][CH / 4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int c = 0; c < CH / 4; ++c) {
      const unsigned w[4] = {ch[4 * c][h], ch[4 * c + 1][h], ch[4 * c + 2][h], ch[4 * c + 3][h]};
      unsigned o[4];
      turn4(w, o);
#pragma unroll
      for (int i = 0; i < 4; ++i) rows[4 * h + i][c] = o[i];
    }
}

template <int W>
__device__ inline void load_words(const uint8_t* p, unsigned (&w)[W]) {
  if constexpr (W == 1) {
    w[0] = *reinterpret_cast<const unsigned*>(p);
  } else {
    const u32x2 x = *reinterpret_cast<const u32x2*>(p);
    w[0] = x[0];
    w[1] = x[1];
  }
}
template <int W>
__device__ inline void store_words(uint8_t* p, const unsigned (&w)[W]) {
  if constexpr (W == 1) *reinterpret_cast<unsigned*>(p) = w[0];
  else *reinterpret_cast<u32x2*>(p) = u32x2{w[0], w[1]};
}
template <int CH>
__device__ inline void load_channels(const uint8_t* p, unsigned (&ch)[CH][2]) {
#pragma unroll
  for (int c = 0; c < CH; c += 2) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(p + c * 8);
    ch[c][0] = x[0], ch[c][1] = x[1], ch[c + 1][0] = x[2], ch[c + 1][1] = x[3];
  }
}
template <int CH>
__device__ inline void store_channels(uint8_t* p, const unsigned (&ch)[CH][2]) {
#pragma unroll
  for (int c = 0; c < CH; c += 2)
    *reinterpret_cast<u32x4*>(p + c * 8) = u32x4{ch[c][0], ch[c][1], ch[c + 1][0], ch[c + 1][1]};
}

// The byte of the scale for a block whose largest magnitude has these bits: from 255/256 of a power of two on it
// rounds up to the next.
__device__ inline int byte_for(unsigned most) { return min(max((int)((most + 0x10000u) >> 23) - 6, kByteMin), kByteMax); }

// Codes of a lane's 8 rows (those whose bit is set in `rows`; the others' are zero) under the block's scale, whose
// byte is at least `least`.  A row with an element that is not finite is stored as zeros.  value(r, c): the
// element's bits.  All lanes of a wave call it.
template <int CH, typename Value>
__device__ inline int encode(unsigned rows, int least, unsigned (&w)[8][CH / 4], bool& bad, const Value& value) {
  unsigned top[8], odd = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    unsigned m = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) m = max(m, value(r, c) & 0x7fffffffu);  // NaN above infinity above numbers
    top[r] = (rows >> r) & 1u ? m : 0u;
    odd |= (top[r] >= 0x7f800000u ? 1u : 0u) << r;
  }
  if (__any(odd != 0)) {  // the whole row's, from the lanes that share it
    bad = true;
#pragma unroll
    for (int by = 1; by < 16; by *= 2) odd |= lane_xor(odd, by);
    rows &= ~odd;
  }
  unsigned most = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) most = max(most, (rows >> r) & 1u ? top[r] : 0u);
#pragma unroll
  for (int by = 1; by < 64; by *= 2) most = max(most, lane_xor(most, by));
  const int byte = max(byte_for(most), least);
  const float inv = power_of(254 - byte);
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    unsigned n[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c)  // (magnitudes past 127 are those of the largest scale)
      n[c] = nearest(fminf(fmaxf(__uint_as_float(value(r, c)) * inv, -127.0f), 127.0f));
#pragma unroll
    for (int c = 0; c < CH / 4; ++c)
      w[r][c] = (rows >> r) & 1u ? pack4(n[4 * c], n[4 * c + 1], n[4 * c + 2], n[4 * c + 3]) : 0u;
  }
  return byte;
}

// Where a block's codes lie.
template <int D>
struct Place {
  uint8_t *k, *v, *ks, *vs;
  __device__ Place(const Cache8& c, int h, int64_t row, const Part<D>& p) {  // row: in the head, a multiple of 32
    row += (int64_t)h * c.C;
    k = c.k_codes + (row + 8 * p.sub) * D + p.at;
    v = c.v_codes + (row + 8 * p.sub) * D + p.at * 8;
    ks = c.k_scales + row / kCache8Block;
    vs = c.v_scales + row / kCache8Block;
  }
};

__device__ inline unsigned rows_between(int sub, int lo, int hi) {  // bits of the 8 rows that lie in [lo, hi)
  const int a = min(max(lo - 8 * sub, 0), 8), b = min(max(hi - 8 * sub, 0), 8);
  return ((1u << b) - 1u) & ~((1u << a) - 1u);
}

// Writes rows [lo, hi) of a block, lo < hi, from the rows src(r) gives; with `keep`, the rows before lo are in use
// and stay, rounded again where the block's scale has to grow.
template <typename T, int D, typename Src>
__device__ inline bool write_block(const Cache8& c, int h, int64_t row, int lo, int hi, bool keep, const Src& src) {
  constexpr int CH = Part<D>::kCh, W = Part<D>::kWords;
  const Part<D> p;
  const Place<D> to(c, h, row, p);
  const unsigned mine = rows_between(p.sub, lo, hi);
  keep = keep && lo > 0;
  const int had_k = keep ? *to.ks : 0, had_v = keep ? *to.vs : 0;
  Piece<T, CH> k[8], v[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    // rows outside [lo, hi) load a row inside it and store nothing
    const char *kp, *vp;
    src(min(max(8 * p.sub + r, lo), hi - 1), kp, vp);
    k[r].load(kp + p.at * (int)sizeof(T));
    v[r].load(vp + p.at * (int)sizeof(T));
  }
  bool bad = false;
  unsigned w[8][W];
  const unsigned old = keep ? rows_between(p.sub, 0, lo) : 0u;
  {
    const int byte = encode<CH>(mine, had_k, w, bad, [&](int r, int ch) { return k[r].bits(ch); });
    const bool grew = keep && byte > had_k;
    const float f = power_of(max(127 + had_k - byte, 0));
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      if ((mine >> r) & 1u) store_words<W>(to.k + r * D, w[r]);
      if (grew && ((old >> r) & 1u)) {
        unsigned x[W];
        load_words<W>(to.k + r * D, x);
#pragma unroll
        for (int i = 0; i < W; ++i)
          x[i] = pack4(nearest(code_of(x[i], 0) * f), nearest(code_of(x[i], 1) * f), nearest(code_of(x[i], 2) * f),
                       nearest(code_of(x[i], 3) * f));
        store_words<W>(to.k + r * D, x);
      }
    }
    if ((threadIdx.x & 63) == 0) *to.ks = (uint8_t)byte;
  }
  {
    const int byte = encode<CH>(mine, had_v, w, bad, [&](int r, int ch) { return v[r].bits(ch); });
    const bool grew = keep && byte > had_v;
    const float f = power_of(max(127 + had_v - byte, 0));
    if (mine != 0 || (grew && old != 0)) {
      unsigned ch[CH][2];
      to_channels<CH>(w, ch);
      if (old != 0) {
        unsigned was[CH][2];
        load_channels<CH>(to.v, was);
        // the bytes of the rows in use: bit r of `old` as byte r
        const unsigned m0 = (old & 1u ? 0xffu : 0u) | (old & 2u ? 0xff00u : 0u) | (old & 4u ? 0xff0000u : 0u) | (old & 8u ? 0xff000000u : 0u);
        const unsigned o4 = old >> 4;
        const unsigned m1 = (o4 & 1u ? 0xffu : 0u) | (o4 & 2u ? 0xff00u : 0u) | (o4 & 4u ? 0xff0000u : 0u) | (o4 & 8u ? 0xff000000u : 0u);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
          if (grew) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
              was[i][e] = pack4(nearest(code_of(was[i][e], 0) * f), nearest(code_of(was[i][e], 1) * f),
                                nearest(code_of(was[i][e], 2) * f), nearest(code_of(was[i][e], 3) * f));
          }
          ch[i][0] |= was[i][0] & m0;
          ch[i][1] |= was[i][1] & m1;
        }
      }
      store_channels<CH>(to.v, ch);
    }
    if ((threadIdx.x & 63) == 0) *to.vs = (uint8_t)byte;
  }
  return bad;
}

// K11a: compaction, a wave per block of the cache, along the positions that K7a has listed.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void cache8_gather_kernel(const Cache8Args a) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = (int)blockIdx.x * kWaves + wave;
  const int h = (int)blockIdx.y;
  if (b >= a.n_blocks) return;
  const int s = find_seq(a.seq, a.n_seqs, kCacheSeqWords, 2, b);
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const int first = (b - seq_word(a.seq, s * kCacheSeqWords + 2)) * kCache8Block;  // row of the problem
  const int hi = min(kCache8Block, a.len_out[q] - first);
  const int row0 = seq_word(a.seq, s * kCacheSeqWords + 1) + first;
  const int64_t t0 = seq_word(a.seq, s * kCacheSeqWords);
  const int64_t at = (int64_t)h * a.cache.C + row0;
  const int at_lane = lane < kCache8Block ? a.pos[at + lane] : -1;  // (-1 on the rows past the last)
  if (a.mass_out != nullptr && lane < kCache8Block)
    a.mass_out[at + lane] = at_lane >= 0 && a.mass != nullptr ? a.mass[(int64_t)h * a.T + t0 + at_lane] : 0.0f;
  if (hi <= 0) return;
  const char* kb = a.keys + (int64_t)h * a.head_stride + t0 * a.token_stride;
  const char* vb = a.values + (int64_t)h * a.v_head_stride + t0 * a.v_token_stride;
  const bool bad = write_block<T, D>(a.cache, h, row0, 0, hi, false, [&](int r, const char*& kp, const char*& vp) {
    const int64_t t = __shfl(at_lane, r);
    kp = kb + t * a.token_stride;
    vp = vb + t * a.v_token_stride;
  });
  if (bad && lane == 0) a.status[q] = kNonfinite;
}

// ---- append ----

struct AppendTo {
  int64_t r0, t0;
  int cap, n;
};
__device__ inline AppendTo append_to(const Cache8Args& a, int s) {
  AppendTo p;
  p.t0 = seq_word(a.seq, s * kCacheSeqWords);
  p.n = seq_word(a.seq, (s + 1) * kCacheSeqWords) - (int)p.t0;
  p.r0 = seq_word(a.seq, s * kCacheSeqWords + 1);
  p.cap = seq_word(a.seq, (s + 1) * kCacheSeqWords + 1) - (int)p.r0;
  return p;
}

// One wave writes those of the problem's new tokens that belong to the j-th block from the one row `len` lies in.
template <typename T, int D>
__device__ inline bool append_block(const Cache8Args& a, int h, const AppendTo& p, int len, int j) {
  const int base = (len / kCache8Block + j) * kCache8Block;  // first row of the block, in the problem
  const int lo = max(len - base, 0), hi = min(len + p.n - base, kCache8Block);
  if (hi <= lo) return false;
  const char* kb = a.keys + (int64_t)h * a.head_stride + (p.t0 + base - len) * a.token_stride;
  const char* vb = a.values + (int64_t)h * a.v_head_stride + (p.t0 + base - len) * a.v_token_stride;
  return write_block<T, D>(a.cache, h, p.r0 + base, lo, hi, true, [&](int r, const char*& kp, const char*& vp) {
    kp = kb + (int64_t)r * a.token_stride;
    vp = vb + (int64_t)r * a.v_token_stride;
  });
}

// K11b: a wave takes one problem's new tokens, so that it alone reads len_in and writes len_out (which may be one
// array) and the status.
template <typename T, int D>
__global__ __launch_bounds__(64) void cache8_append_kernel(const Cache8Args a) {
  const int s = (int)blockIdx.x % a.n_seqs, h = (int)blockIdx.x / a.n_seqs;
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const AppendTo p = append_to(a, s);
  const int len = __builtin_amdgcn_readfirstlane(a.len_in[q]);
  const bool fits = len >= 0 && len <= p.cap - p.n;
  bool bad = false;
  if (fits)
    for (int j = 0; j <= kAppendBlocks; ++j) bad |= append_block<T, D>(a, h, p, len, j);
  if (threadIdx.x == 0) {
    a.len_out[q] = fits ? len + p.n : len;
    a.status[q] = !fits ? kMismatch : bad ? kNonfinite : kOk;
  }
}

// Many new tokens: the lengths and states first, then a wave per block of every problem.
__global__ __launch_bounds__(kThreads) void cache8_grow_kernel(const Cache8Args a) {
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
__global__ __launch_bounds__(kThreads) void cache8_append_many_kernel(const Cache8Args a) {
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int b = (int)blockIdx.x * kWaves + wave;
  const int h = (int)blockIdx.y;
  if (b >= a.n_blocks) return;
  const int s = find_seq(a.seq, a.n_seqs, kCacheSeqWords, 2, b);
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const AppendTo p = append_to(a, s);
  // another wave may have made it NONFINITE already, which is as good as OK here
  if (__builtin_amdgcn_readfirstlane(a.status[q]) == kMismatch) return;
  const int len = __builtin_amdgcn_readfirstlane(a.len_out[q]) - p.n;
  if (append_block<T, D>(a, h, p, len, b - seq_word(a.seq, s * kCacheSeqWords + 2)) && (threadIdx.x & 63) == 0)
    a.status[q] = kNonfinite;
}

// ---- read ----

template <typename T, int CH>
__device__ inline void store_values(char* to, const unsigned (&w)[CH / 4], float scale) {
  float x[CH];
#pragma unroll
  for (int c = 0; c < CH; ++c) x[c] = code_of(w[c / 4], c & 3) * scale;
  if constexpr (CH == 8) {
    Vec8<T>::from(x).store(to);
  } else if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<f32x4*>(to) = f32x4{x[0], x[1], x[2], x[3]};
  } else {
    typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4*>(to) = bf16x4{(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
  }
}

// K11c: a wave per block of the cache that holds rows to read.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void cache8_read_kernel(const Cache8Args a) {
  constexpr int CH = Part<D>::kCh, W = Part<D>::kWords;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int b = (int)blockIdx.x * kWaves + wave;
  const int h = (int)blockIdx.y;
  if (b >= a.n_blocks) return;
  const int s = find_seq(a.seq, a.n_seqs, kCacheSeqWords, 2, b);
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const int o0 = seq_word(a.seq, s * kCacheSeqWords), n = seq_word(a.seq, (s + 1) * kCacheSeqWords) - o0;
  const int64_t r0 = seq_word(a.seq, s * kCacheSeqWords + 1);
  const int cap = seq_word(a.seq, (s + 1) * kCacheSeqWords + 1) - (int)r0;
  const int len = min(__builtin_amdgcn_readfirstlane(a.len_in[q]), cap);
  const int64_t first = a.first != nullptr ? __builtin_amdgcn_readfirstlane(a.first[q]) : 0;
  // cache row of the block (first >> 5 rounds down, also below 0)
  const int64_t base = ((first >> 5) + (b - seq_word(a.seq, s * kCacheSeqWords + 2))) * kCache8Block;
  const bool any = base >= 0 && base < len;  // else every row of the block is zero
  const Part<D> p;
  const Place<D> from(a.cache, h, any ? r0 + base : 0, p);
  const unsigned live = any ? rows_between(p.sub, 0, (int)min((int64_t)kCache8Block, len - base)) : 0u;
  float scale_k = 0.0f, scale_v = 0.0f;
  unsigned ch[CH][2] = {}, kw[8][W] = {}, vw[8][W];
  if (live != 0) {
    if (a.values_out != nullptr) {
      load_channels<CH>(from.v, ch);
      scale_v = power_of(*from.vs);
    }
    if (a.keys_out != nullptr) {
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if ((live >> r) & 1u) load_words<W>(from.k + r * D, kw[r]);
      scale_k = power_of(*from.ks);
    }
  }
  to_rows<CH>(ch, vw);
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    const int64_t o = base + 8 * p.sub + r - first;  // output row of the problem
    if (o < 0 || o >= n) continue;
    const int64_t to = (((int64_t)h * a.C_out + o0 + o) * D + p.at) * (int64_t)sizeof(T);
    if (a.keys_out != nullptr) store_values<T, CH>(a.keys_out + to, kw[r], scale_k);
    if (a.values_out != nullptr) {
      if (((live >> r) & 1u) == 0)
#pragma unroll
        for (int i = 0; i < W; ++i) vw[r][i] = 0u;
      store_values<T, CH>(a.values_out + to, vw[r], scale_v);
    }
  }
}

// ---- the rows that an eviction keeps ----

// Codes of a lane's 8 rows (those whose bit is set in `rows`; the others' become zero) under their rows' scales, brought
// to the scale of the block they now share; returns its byte.  Where a row of the largest scale has a code over 64, that
// scale stays, and only rows of smaller ones change: no work for most blocks.
template <int CH>
__device__ inline int move_codes(unsigned rows, const int (&from)[8], unsigned (&w)[8][CH / 4]) {
  constexpr int W = CH / 4;
  int top = 0;
#pragma unroll
  for (int r = 0; r < 8; ++r) top = max(top, (rows >> r) & 1u ? from[r] : 0);
#pragma unroll
  for (int by = 16; by < 64; by *= 2) top = max(top, __shfl_xor(top, by));  // (16 lanes share a row)
  unsigned large = 0;  // a byte's upper bits differ: 64 .. 127 or -128 .. -65
#pragma unroll
  for (int r = 0; r < 8; ++r)
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if (((rows >> r) & 1u) == 0) w[r][i] = 0u;
      large |= from[r] == top ? (w[r][i] ^ (w[r][i] << 1)) & 0x80808080u : 0u;
    }
  int byte = top;
  if (!__any(large != 0)) {
    unsigned most = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      float m = 0.0f;
#pragma unroll
      for (int c = 0; c < CH; ++c) m = fmaxf(m, fabsf(code_of(w[r][c / 4], c & 3)));
      most = max(most, (rows >> r) & 1u ? __float_as_uint(m * power_of(from[r])) : 0u);
    }
#pragma unroll
    for (int by = 1; by < 64; by *= 2) most = max(most, lane_xor(most, by));
    byte = byte_for(most);
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) {
    if (from[r] == byte) continue;
    const float f = power_of(min(max(127 + from[r] - byte, 0), 254));  // (rows of zeros may come from far above)
#pragma unroll
    for (int i = 0; i < W; ++i)
      w[r][i] = pack4(nearest(code_of(w[r][i], 0) * f), nearest(code_of(w[r][i], 1) * f), nearest(code_of(w[r][i], 2) * f),
                      nearest(code_of(w[r][i], 3) * f));
  }
  return byte;
}

// K12b: a wave per block of the new cache.  Its rows come from rising rows of the old one: the keys straight, the
// values 32 rows of the old cache at a time, turned to rows in the wave's own LDS, from where each lane takes those
// that it needs.
template <int D>
__global__ __launch_bounds__(kThreads) void evict8_move_kernel(const Evict8Args a) {
  constexpr int CH = Part<D>::kCh, W = Part<D>::kWords;
  __shared__ unsigned s_rows[kWaves][kCache8Block][D / 4];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = (int)blockIdx.x * kWaves + wave;
  const int h = (int)blockIdx.y;
  if (b >= a.n_blocks) return;
  const int s = find_seq(a.seq, a.n_seqs, kEvict8SeqWords, 3, b);
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const int first = (b - seq_word(a.seq, s * kEvict8SeqWords + 3)) * kCache8Block;
  const int64_t from0 = seq_word(a.seq, s * kEvict8SeqWords), to0 = seq_word(a.seq, s * kEvict8SeqWords + 1) + first;
  const int hi = min(kCache8Block, __builtin_amdgcn_readfirstlane(a.len_out[q]) - first);
  // the rows' places in the old cache (-1 past the last), then their positions and weights
  const int64_t out = (int64_t)h * a.to.C + to0 + lane;
  int row = -1;
  if (lane < kCache8Block) {
    row = a.pos_out[out];
    const int64_t at = (int64_t)h * a.from.C + from0 + row;
    if (row >= 0 && a.pos != nullptr) a.pos_out[out] = a.pos[at];
    if (a.mass_out != nullptr) a.mass_out[out] = row >= 0 ? a.mass[at] : 0.0f;
  }
  if (hi <= 0) return;
  const Part<D> p;
  const unsigned mine = rows_between(p.sub, 0, hi);
  const int64_t head = (int64_t)h * a.from.C + from0;
  const Place<D> to(a.to, h, to0, p);
  int k_byte = 0, v_byte = 0;
  if (row >= 0) {
    k_byte = a.from.k_scales[(head + row) / kCache8Block];
    v_byte = a.from.v_scales[(head + row) / kCache8Block];
  }
  // (next, and what follows from it, is the same in all lanes)
  auto group_at = [&](int next) { return __builtin_amdgcn_readfirstlane(__shfl(row, next) / kCache8Block); };
  unsigned ch[CH][2];
  auto load_group = [&](int group) {
    load_channels<CH>(a.from.v_codes + (head + group * (int64_t)kCache8Block + 8 * p.sub) * D + p.at * 8, ch);
  };
  int group = group_at(0);
  int from[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) from[r] = __shfl(row, 8 * p.sub + r);  // (-1 past the last: in no group)
  unsigned w[8][W];
  int bytes[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) load_words<W>(a.from.k_codes + (head + max(from[r], 0)) * D + p.at, w[r]);
  load_group(group);
#pragma unroll
  for (int r = 0; r < 8; ++r) bytes[r] = __shfl(k_byte, 8 * p.sub + r);
  const int kb = move_codes<CH>(mine, bytes, w);
#pragma unroll
  for (int r = 0; r < 8; ++r)
    if ((mine >> r) & 1u) store_words<W>(to.k + r * D, w[r]);
  if (lane == 0) *to.ks = (uint8_t)kb;

#pragma unroll
  for (int r = 0; r < 8; ++r)
#pragma unroll
    for (int i = 0; i < W; ++i) w[r][i] = 0u;
  for (int next = 0; next < hi;) {
    next += (int)__popcll(__ballot(row >= 0 && row / kCache8Block == group));
    unsigned turned[8][W];
    to_rows<CH>(ch, turned);
    // the next group, or this one once more, on its way while this one goes through LDS
    const int ahead = next < hi ? group_at(next) : group;
    load_group(ahead);
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int i = 0; i < W; ++i) s_rows[wave][8 * p.sub + r][p.at / 4 + i] = turned[r][i];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int i = 0; i < W; ++i) turned[r][i] = s_rows[wave][from[r] & (kCache8Block - 1)][p.at / 4 + i];
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int i = 0; i < W; ++i) w[r][i] = from[r] >> kBlockBits == group ? turned[r][i] : w[r][i];
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    group = ahead;
  }
#pragma unroll
  for (int r = 0; r < 8; ++r) bytes[r] = __shfl(v_byte, 8 * p.sub + r);
  const int vb = move_codes<CH>(mine, bytes, w);
  if (mine != 0) {
    to_channels<CH>(w, ch);
    store_channels<CH>(to.v, ch);
  }
  if (lane == 0) *to.vs = (uint8_t)vb;
}

unsigned groups_of(int blocks) { return (unsigned)((blocks + kWaves - 1) / kWaves); }

template <typename T, int D>
int launch_append(const Cache8Args& a, int max_new, hipStream_t s) {
  const unsigned problems = (unsigned)a.n_heads * (unsigned)a.n_seqs;
  if (max_new <= kAppendBlocks * kCache8Block) {  // at any len: at most kAppendBlocks + 1 blocks
    hipLaunchKernelGGL((cache8_append_kernel<T, D>), dim3(problems), dim3(64), 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(cache8_grow_kernel, dim3((problems + kThreads - 1) / kThreads), dim3(kThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return (int)e;
  hipLaunchKernelGGL((cache8_append_many_kernel<T, D>), dim3(groups_of(a.n_blocks), (unsigned)a.n_heads), dim3(kThreads),
                     0, s, a);
  return hipGetLastError();
}
template <typename T, int D>
int launch_gather(const Cache8Args& a, hipStream_t s) {
  hipLaunchKernelGGL((cache8_gather_kernel<T, D>), dim3(groups_of(a.n_blocks), (unsigned)a.n_heads), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}
template <typename T, int D>
int launch_read(const Cache8Args& a, hipStream_t s) {
  hipLaunchKernelGGL((cache8_read_kernel<T, D>), dim3(groups_of(a.n_blocks), (unsigned)a.n_heads), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}
template <int D>
int launch_move(const Evict8Args& a, hipStream_t s) {
  hipLaunchKernelGGL((evict8_move_kernel<D>), dim3(groups_of(a.n_blocks), (unsigned)a.n_heads), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int launch_cache8_gather(const Cache8Args& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (a.n_blocks == 0) return hipSuccess;
  if (dtype == 0) return d == 128 ? launch_gather<bf16, 128>(a, s) : launch_gather<bf16, 64>(a, s);
  return d == 128 ? launch_gather<float, 128>(a, s) : launch_gather<float, 64>(a, s);
}

int launch_cache8_append(const Cache8Args& a, int max_new, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 0) return d == 128 ? launch_append<bf16, 128>(a, max_new, s) : launch_append<bf16, 64>(a, max_new, s);
  return d == 128 ? launch_append<float, 128>(a, max_new, s) : launch_append<float, 64>(a, max_new, s);
}

int launch_cache8_read(const Cache8Args& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (a.n_blocks == 0) return hipSuccess;
  if (dtype == 0) return d == 128 ? launch_read<bf16, 128>(a, s) : launch_read<bf16, 64>(a, s);
  return d == 128 ? launch_read<float, 128>(a, s) : launch_read<float, 64>(a, s);
}

int launch_evict8_move(const Evict8Args& a, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (a.n_blocks == 0) return hipSuccess;
  return d == 128 ? launch_move<128>(a, s) : launch_move<64>(a, s);
}

}  // namespace twinkv

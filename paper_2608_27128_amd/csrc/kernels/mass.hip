// K14: the attention weight that each key receives: sum over the queries that see it, and over the query heads that
// share it, of exp(scale q . k - lse).
//
// With the queries' log-sum-exp at hand a weight is final as it is computed, so this is one product Q K^T whose
// epilogue is a fused multiply-add, an exponential and an addition an element.  A workgroup owns a tile of keys, a
// part of them in each wave's registers for all of its work, and goes over the rows (row = query * group + query
// head) that see them; rows come to LDS 16 bytes a lane without registers, into one of two buffers while the other
// is read, and serve all four waves.  The products put a key in a lane and 16 rows in its registers, so a key's
// weights are added up inside the lane.
//  * bf16: v_mfma_f32_32x32x16_bf16, 64 keys a wave, 128 rows a step.
//  * fp32: a number is the sum of three bf16 (24 bits), a product the six of their products that reach 2^-24 of the
//    largest: 6 x 32 cycles for 16 channels, where v_mfma_f32_32x32x2_f32 takes 512.  Rows pass through registers and are
//    taken apart once for the four waves, 64 a step; 32 keys a wave.  A prompt of 4096 tokens (d 128, 8 heads of 4) 390 us,
//    with the fp32 instruction 665.
//  * keys in 8 bits: their codes become bf16, exactly, as they are loaded; the block's scale goes into the multiply-add.
// Which rows see a lane's key is one run of rows, so a mask is a subtraction and a comparison, and blocks that see all
// of the wave's keys, or none, have none.
//
// What bounds it at length is the matrix unit and the vector unit by turns: they hardly overlap from wave to wave, and a
// weight costs a multiply-add, an addition and an exponential of twice their price.  So, per block of 32 rows:
//  * kFused (bf16, d 128): one block's weights go between the next block's products, in the same wave.  A prompt of 32768
//    tokens (8 heads of 4): 4.1 ms, 1070 TFLOP/s; apart 4.5.  Two blocks' accumulators: 244 registers, 2 waves a SIMD.
//  * kApart (bf16 of d 64, fp32): products, then weights.  With half the products to hide behind, twice the waves count for
//    more: 8192 tokens of d 64 190 us, fused 217.
//  * kFew (bf16, at most kMassFew rows a key): the keys' way to the registers is the work, so one buffer of rows, and more
//    workgroups.  64 sequences of 1024 to 4096 keys, the last 32 queries: 88 us, 4.0 TB/s of keys; with 32 keys a wave 100, with
//    the keys of several tiles passing by one staged copy of the rows 106.
//
// Sums: 32 bits, in two levels, since one chain over 100000 rows loses 3 digits: a lane adds up to 16 steps'
// weights, then their sum to the total.  Rows are split over workgroups where there are too few keys, and a second kernel
// adds the parts in one order; nothing is added atomically.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attn_split.h"
#include "codes8.h"

namespace twinkv {
namespace {

constexpr int kThreads = 256;
constexpr int kFlush = 16;  // steps between additions to the total
constexpr int kAhead = 3;   // steps of the contraction whose rows are on their way from LDS

// A wave's keys, and the rows of a step.  P: bf16 parts of a key.
template <typename T, int D, int B, int P>
struct Keys;

template <int D, int B, int P>
struct Keys<bf16, D, B, P> {
  static constexpr int kBlocks = B, kRowBlocks = 4, kSteps = D / 16;  // of 32 keys, of 32 rows, of 16 channels
  bf16x8 k[kBlocks][kSteps];
  __device__ void load(int b, const char* row, int hi) {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) k[b][j] = *reinterpret_cast<const bf16x8*>(row + (2 * j + hi) * 16);
  }
  __device__ void load_codes(int b, const uint8_t* row, int hi) {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(row + (2 * j + hi) * 8);
      k[b][j] = codes8_bf16(w[0], w[1]);
    }
  }
  // The lane's 16 bytes of step j of its row.
  typedef bf16x8 Row;
  __device__ void product(int j, int b, const Row& q, f32x16& acc) const {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, k[b][j], acc, 0, 0, 0);
  }
  __device__ void product_each(int j, int b, const Row& q, f32x16& acc) const { product(j, b, q, acc); }
};

template <int D, int P>
struct Keys<float, D, 1, P> {
  static constexpr int kBlocks = 1, kRowBlocks = 2, kSteps = D / 16;
  bf16x8 k[kSteps][P];
  __device__ void load(int, const char* row, int hi) {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const f32x4* at = reinterpret_cast<const f32x4*>(row) + (2 * j + hi) * 2;
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = at[e / 4][e % 4];
      split8(x, k[j]);
    }
  }
  __device__ void load_codes(int, const uint8_t* row, int hi) {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const u32x2 w = *reinterpret_cast<const u32x2*>(row + (2 * j + hi) * 8);
      k[j][0] = codes8_bf16(w[0], w[1]);
    }
  }
  // The parts' products, the smallest first: of 24 bits those from 2^-24 of the largest on.
  struct Row {
    bf16x8 part[3];
  };
  __device__ void product(int j, int, const Row& q, f32x16& acc) const {
#pragma unroll
    for (int sum = 2; sum >= 0; --sum)
#pragma unroll
      for (int of_k = 0; of_k <= sum && of_k < P; ++of_k)
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q.part[sum - of_k], k[j][of_k], acc, 0, 0, 0);
  }
  // The products of the numbers that the parts are of, whose infinities keep their meaning: two channels at a time.
  static __device__ float number(float first, float rest) {  // (of an infinite number the rest is NaN)
    return __builtin_isfinite(first) ? first + rest : first;
  }
  __device__ void product_each(int j, int, const Row& q, f32x16& acc) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = number((float)q.part[0][e], (float)q.part[1][e] + (float)q.part[2][e]);
      float y = (float)k[j][0][e];
      if constexpr (P == 3) y = number(y, (float)k[j][1][e] + (float)k[j][2][e]);
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x, y, acc, 0, 0, 0);
    }
  }
};

// What an item is.  kByRows (mass_place): the items at work together are those of many tiles and the same rows, which one
// XCD's L2 then holds (a prompt of 32768 tokens reads 1.4 GB instead of 12.9; one of 4096 in fp32 takes 388 us for 421).
struct MassItem {
  int h, s, kt, split, splits;
  int q0, nq, k0, nk;
  int rows;       // of a split
  int64_t part;   // among the parts of all heads, where splits > 1
};
template <bool kByRows>
__device__ inline MassItem mass_item(const MassArgs& a, int item, int h) {
  MassItem p;
  p.h = h;
  p.s = find_seq(a.seq, a.n_seqs, kMassSeqWords, 2, item);
  const int w = p.s * kMassSeqWords;
  p.q0 = seq_word(a.seq, w);
  p.k0 = seq_word(a.seq, w + 1);
  const int item0 = seq_word(a.seq, w + 2), splits = seq_word(a.seq, w + 3);
  p.rows = seq_word(a.seq, w + 4);
  const int full = seq_word(a.seq, w + 5), shape = seq_word(a.seq, w + 6);
  p.nq = seq_word(a.seq, w + kMassSeqWords) - p.q0;
  p.nk = seq_word(a.seq, w + kMassSeqWords + 1) - p.k0;
  const MassPlace place = mass_place<kByRows>(item - item0, splits, full, shape, (p.nk + a.keys - 1) / a.keys);
  p.kt = place.tile;
  p.split = place.split;
  p.splits = place.splits;
  p.part = (int64_t)h * a.items + item0 + place.part;
  return p;
}

// kMode: how a block's products and weights go together (see above).
enum { kFused, kApart, kFew };
template <typename T, int D, int kMode>
constexpr int kMassWaves = kMode == kFused || (sizeof(T) == 4 && D == 128) ? 2 : (kMode == kFew && D == 128) || sizeof(T) == 4 ? 3 : 4;  // a SIMD
template <typename T, int D, int B, int kMode, bool kCodes>
__global__ __launch_bounds__(kThreads, (kMassWaves<T, D, kMode>)) void mass_kernel(const MassArgs a) {
  typedef Keys<T, D, B, kCodes || sizeof(T) == 2 ? 1 : 3> Own;
  typedef typename Own::Row Row;
  constexpr int kWaveKeys = 32 * Own::kBlocks, kTileKeys = 4 * kWaveKeys, kTileRows = 32 * Own::kRowBlocks;
  constexpr bool kSplit = sizeof(T) == 4;  // rows of fp32 lie in LDS as three tiles of bf16, their parts
  constexpr int kRowBytes = D * 2, kPieces = kRowBytes / 16, kAtOnce = kThreads / kPieces;
  constexpr int kCopies = kTileRows / kAtOnce;
  // Two objects, so that the compiler sees that reading one need not wait for the loads into the other.
  __shared__ __attribute__((aligned(16))) char s_even[(kSplit ? 3 : 1) * kTileRows * kRowBytes];
  __shared__ __attribute__((aligned(16))) char s_odd[kMode == kFew || kSplit ? 16 : kTileRows * kRowBytes];
  __shared__ __attribute__((aligned(16))) float s_lse[2][kTileRows];  // in log2 units
  __shared__ int s_odd_sum;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (8 heads at a time, one an XCD: of more at once an XCD's L2 would not hold the rows that its items share; 288 heads of
  // 8192 tokens 2460 us, all at once 2680)
  const unsigned eight = blockIdx.x / (8u * (unsigned)a.items), rest = blockIdx.x - eight * 8u * (unsigned)a.items;
  const unsigned heads = min(8u, (unsigned)a.n_heads - 8u * eight);
  const int h = (int)(8u * eight + rest % heads);
  const MassItem p = mass_item<true>(a, (int)(rest / heads), h);
  const int n = kCodes ? min(max(__builtin_amdgcn_readfirstlane(a.len[(int64_t)h * a.n_seqs + p.s]), 0), p.nk) : p.nk;
  const int offset = n - p.nq;                 // position of query 0
  const int key0 = p.kt * kTileKeys;
  // the rows that see a key of the tile: of the queries at positions key0 and after, up to the last key's window
  const int last_key = min(key0 + kTileKeys, n) - 1;
  const int n_rows = p.nq * a.group;
  auto query_at = [&](int64_t pos) { return (int)min(max(pos - offset, (int64_t)0), (int64_t)p.nq); };
  const int q_lo = query_at(key0);
  const int q_hi = key0 >= n ? q_lo : key0 < a.n_sink ? p.nq : max(query_at((int64_t)last_key + a.window), q_lo);
  const int64_t row_lo = (int64_t)q_lo * a.group + (int64_t)p.split * p.rows;
  const int row0 = (int)min(row_lo, (int64_t)n_rows);
  const int row1 = (int)min(row_lo + p.rows, (int64_t)q_hi * a.group);

  // this wave's keys (past the last: the last once more)
  const int wave_key = key0 + wave * kWaveKeys;
  Own own;
  float scale[Own::kBlocks];
#pragma unroll
  for (int b = 0; b < Own::kBlocks; ++b) scale[b] = a.scale_log2;
  if (row0 < row1) {
#pragma unroll
    for (int b = 0; b < Own::kBlocks; ++b) {
      const int64_t key = min(wave_key + 32 * b + col, n - 1);
      if constexpr (kCodes) {
        const int64_t at = (int64_t)h * a.cache.C + p.k0 + key;
        own.load_codes(b, a.cache.k_codes + at * D, hi);
        scale[b] *= __uint_as_float((unsigned)a.cache.k_scales[at / kCache8Block] << 23);
      } else {
        own.load(b, a.k + (int64_t)h * a.k_head + ((int64_t)p.k0 + key) * a.k_token, hi);
      }
    }
  }

  // These rows see all of the wave's keys; of each block of 32 keys some rows from some0 to some1 see a key.
  const int row_end = max(row0, row1);
  auto row_at = [&](int64_t pos) {
    const int64_t row = (int64_t)query_at(pos) * a.group;
    return __builtin_amdgcn_readfirstlane((int)min(max(row, (int64_t)row0), (int64_t)row_end));
  };
  const int far_key = wave_key + kWaveKeys - 1;
  const int all0 = far_key < n ? row_at(far_key) : row_end;
  const int all1 = far_key < a.n_sink ? row_end : row_at((int64_t)wave_key + a.window);
  int some0[Own::kBlocks], some1[Own::kBlocks];
#pragma unroll
  for (int b = 0; b < Own::kBlocks; ++b) {
    const int key = wave_key + 32 * b;
    some0[b] = row_at(key);
    some1[b] = key >= n ? row0 : key < a.n_sink ? row_end : row_at((int64_t)key + 31 + a.window);
  }
  auto all_see = [&](int row) { return row >= all0 && row + 32 <= all1; };           // of the 32 rows from `row` on
  auto some_see = [&](int row, int b) { return row < some1[b] && row + 32 > some0[b]; };

  // Rows to LDS.  Where whole runs of rows have the same query heads a thread's rows lie at fixed distances, and
  // move by a fixed one from step to step; otherwise, and in the last step, each row's place is worked out.
  const char* q_head0 = a.q + (int64_t)h * a.group * a.q_head + (int64_t)p.q0 * a.q_token;
  auto turn = [](int row) { return kRowBytes == 128 ? (row >> 1) & 7 : row & 15; };
  const unsigned inv_group = (unsigned)((0xffffffffull + (unsigned)a.group) / (unsigned)a.group);  // 2^32 / group, up
  auto query_of = [&](int r, int& sub) {  // r / group, r % group
    int q = a.group == 1 ? r : (int)__umulhi((unsigned)r, inv_group);
    sub = r - q * a.group;
    if (sub < 0) {
      sub += a.group;
      --q;
    }
    return q;
  };
  const bool even = kAtOnce % a.group == 0 && row0 % a.group == 0;
  const int64_t copy_bytes = even ? kAtOnce / a.group * a.q_token : 0, step_bytes = copy_bytes * kCopies;
  const int r_lane = tid / kPieces, piece = tid % kPieces;
  auto first_row = [&]() {
    int sub;
    const int query = query_of(row0 + r_lane, sub);
    return q_head0 + sub * a.q_head + (int64_t)query * a.q_token;
  };
  const char* from = first_row();
  float next_lse = 0.0f;
  auto bring_lse = [&](int r0) {
    if (tid < kTileRows) {
      next_lse = 0.0f;
      if (r0 + tid < row1) {
        int sub;
        const int query = query_of(r0 + tid, sub);
        next_lse = a.lse[((int64_t)h * a.group + sub) * a.Tq + p.q0 + query];
      }
    }
  };
  auto bring = [&](auto F, int r0) {
    char* to = (F == 0 ? s_even : s_odd) + wave * 1024;
    if (even && r0 + kTileRows <= n_rows) {
#pragma unroll
      for (int c = 0; c < kCopies; ++c)
        to_lds(from + c * copy_bytes + (piece ^ turn(c * kAtOnce + r_lane)) * 16, to + c * (kThreads * 16));
      from += step_bytes;
    } else {
#pragma unroll
      for (int c = 0; c < kCopies; ++c) {
        const int r = c * kAtOnce + r_lane;
        if (r0 + c * kAtOnce >= row1) break;
        int sub;
        const int query = query_of(min(r0 + r, n_rows - 1), sub);
        to_lds(q_head0 + sub * a.q_head + (int64_t)query * a.q_token + (piece ^ turn(r)) * 16, to + c * (kThreads * 16));
      }
    }
    bring_lse(r0);
  };
  // fp32: through registers, 8 channels a thread and row
  float next[kSplit ? kCopies : 1][8];
  auto fetch = [&](int r0) {
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      int sub;
      const int query = query_of(min(r0 + c * kAtOnce + r_lane, n_rows - 1), sub);
      const f32x4* row = reinterpret_cast<const f32x4*>(q_head0 + sub * a.q_head + (int64_t)query * a.q_token) + 2 * piece;
#pragma unroll
      for (int e = 0; e < 8; ++e) next[c][e] = row[e / 4][e % 4];
    }
    bring_lse(r0);
  };
  auto store = [&]() {
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      const int r = c * kAtOnce + r_lane;
      bf16x8 part[3];
      split8(next[c], part);
#pragma unroll
      for (int i = 0; i < 3; ++i)
        *reinterpret_cast<bf16x8*>(s_even + (i * kTileRows + r) * kRowBytes + (piece ^ turn(r)) * 16) = part[i];
    }
  };

  int r0 = row0;  // first row of the step
  float total[Own::kBlocks], run[Own::kBlocks];
#pragma unroll
  for (int b = 0; b < Own::kBlocks; ++b) total[b] = run[b] = 0.0f;
  f32x16 acc[kMode == kFused ? 2 : 1][Own::kBlocks];  // the block at hand, and the one before it
  f32x4 l[kMode == kFused ? 2 : 1][4];                // their rows' log-sum-exps
  bool before = false;                // there is one, whose rows see all of the wave's keys
  const int lane_row = col * kRowBytes;
  int place[Own::kSteps];
#pragma unroll
  for (int j = 0; j < Own::kSteps; ++j) place[j] = lane_row + ((2 * j + hi) ^ turn(col)) * 16;

  const std::integral_constant<int, 0> zero;
  const std::integral_constant<int, 1> one;
  enum { kAll, kSeen, kEach };  // whose weights
  const std::integral_constant<int, kAll> of_all;
  const std::integral_constant<int, kSeen> of_seen;
  // The rows of the item that see this lane's key of block b: from first[b] on, so many.
  int first[Own::kBlocks];
  unsigned many[Own::kBlocks];
#pragma unroll
  for (int b = 0; b < Own::kBlocks; ++b) {
    const int64_t pos = wave_key + 32 * b + col, lo = (pos - offset) * a.group;
    const int64_t end = pos >= n ? row0 : pos < a.n_sink ? row1 : min((int64_t)row1, lo + (int64_t)a.window * a.group);
    first[b] = (int)min(max(lo, (int64_t)row0), (int64_t)row1);
    many[b] = (unsigned)max(end - first[b], (int64_t)0);
  }
  auto seen = [&](int row, int b) { return (unsigned)(row - first[b]) < many[b]; };
  // The weights of the block of rows from `row` on, for key blocks B0 .. B1 - 1.  (kEach: of the rows that see a key and
  // whose log-sum-exp is not -inf, whatever their scores are.)
  auto weigh = [&](auto all, auto H, auto B0, auto B1, int row) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {  // rows 8x + 4hi .. + 3 of the block
#pragma unroll
      for (int b = B0; b < B1; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float arg = __builtin_fmaf(acc[H][b][4 * x + e], scale[b], -l[H][x][e]);
          if constexpr (all == kAll) run[b] += __builtin_amdgcn_exp2f(arg);
          else if constexpr (all == kSeen) run[b] += __builtin_amdgcn_exp2f(seen(row + 4 * hi + 8 * x + e, b) ? arg : kNegInf);
          else run[b] += seen(row + 4 * hi + 8 * x + e, b) && l[H][x][e] != kNegInf ? __builtin_amdgcn_exp2f(arg) : 0.0f;
        }
    }
  };
  auto row_piece = [&](const char* rows, int j) {
    if constexpr (kSplit) {
      Row q;
#pragma unroll
      for (int i = 0; i < 3; ++i) q.part[i] = *reinterpret_cast<const bf16x8*>(rows + i * kTileRows * kRowBytes + place[j]);
      return q;
    } else {
      return *reinterpret_cast<const Row*>(rows + place[j]);
    }
  };
  Row ahead[kAhead];               // the first pieces of the next block's rows
  auto look_ahead = [&](const char* rows) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) ahead[j] = row_piece(rows, j);
  };
  auto bring_stats = [&](auto H, int at, int rb) {
#pragma unroll
    for (int x = 0; x < 4; ++x) l[H][x] = *reinterpret_cast<const f32x4*>(&s_lse[at][32 * rb + 8 * x + 4 * hi]);
  };
  auto multiply = [&](auto H, auto B0, auto B1, const char* rows) {
#pragma unroll
    for (int b = B0; b < B1; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[H][b][e] = 0.0f;
    constexpr int kFirst = kMode == kFused || (D == 64 && !kSplit) ? Own::kSteps : 1;  // rows' pieces on their way before the products
    Row q[Own::kSteps];
#pragma unroll
    for (int j = 0; j < kFirst; ++j) q[j] = kMode == kFused && j < kAhead ? ahead[j] : row_piece(rows, j);
    if (kFirst > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < Own::kSteps; ++j) {
      if (j >= kFirst) q[j] = row_piece(rows, j);
#pragma unroll
      for (int b = B0; b < B1; ++b) own.product(j, b, q[j], acc[H][b]);
    }
  };
  const std::integral_constant<int, Own::kBlocks> blocks;
  // Block RB of the step in buffer F, where some rows do not see all: a block of keys after the other.
  auto block_masked = [&](auto H, auto F, auto RB) {
    const char* rows = (F == 0 ? s_even : s_odd) + RB * 32 * kRowBytes;
    const int row = r0 + 32 * RB;
    auto part = [&](auto B0, auto B1) {
      if (!some_see(row, B0)) return;
      multiply(H, B0, B1, rows);
      weigh(of_seen, H, B0, B1, row);
    };
    part(zero, one);
    if constexpr (Own::kBlocks == 2) part(one, blocks);
  };
  auto block_apart = [&](auto F, auto RB) {
    if (all_see(r0 + 32 * RB)) {
      multiply(zero, zero, blocks, (F == 0 ? s_even : s_odd) + RB * 32 * kRowBytes);
      bring_stats(zero, F, RB);
      weigh(of_all, zero, zero, blocks, 0);
    } else {
      bring_stats(zero, F, RB);
      block_masked(zero, F, RB);
    }
  };
  // Its products, and the weights of the block before.
  auto block_fused = [&](auto H, auto F, auto RB) {
    const bool all = all_see(r0 + 32 * RB);
    std::integral_constant<int, 1 - H> other;
    const char* rows = (F == 0 ? s_even : s_odd) + RB * 32 * kRowBytes;
    // The weights of the block before go between the products, two elements to each, their three steps on the elements of
    // three products at a time.
    if (all && before) {
      constexpr int kProducts = Own::kSteps * Own::kBlocks, kEach = 16 * Own::kBlocks / kProducts;
      Row q[Own::kSteps];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) q[j] = ahead[j];
#pragma unroll
      for (int b = 0; b < Own::kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[H][b][e] = 0.0f;
      float arg[2][kEach], w[2][kEach];
#pragma unroll
      for (int i = 0; i < kProducts + 2; ++i) {
        const int j = i / Own::kBlocks;
        __builtin_amdgcn_sched_barrier(0);
        if (i < kProducts) {
          if (i % Own::kBlocks == 0 && j + kAhead < Own::kSteps)
            q[j + kAhead] = row_piece(rows, j + kAhead);
          own.product(j, i % Own::kBlocks, q[j], acc[H][i % Own::kBlocks]);
        }
        if (i == kProducts - 3) bring_stats(H, F, RB);
        if (RB + 1 < Own::kRowBlocks && i == kProducts - 1) look_ahead(rows + 32 * kRowBytes);
#pragma unroll
        for (int x = 0; x < kEach; ++x) {
          const int e = (i * kEach + x) / Own::kBlocks, b = (i * kEach + x) % Own::kBlocks;  // element e of key block b
          if (i >= 2) run[x % Own::kBlocks] += w[i & 1][x];
          if (i >= 1 && i <= kProducts) w[(i - 1) & 1][x] = __builtin_amdgcn_exp2f(arg[(i - 1) & 1][x]);
          if (i < kProducts) arg[i & 1][x] = __builtin_fmaf(acc[1 - H][b][e], scale[b], -l[1 - H][e / 4][e % 4]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    } else {
      if (before) weigh(of_all, other, zero, blocks, 0);
      bring_stats(H, F, RB);
      if (all) multiply(H, zero, blocks, rows);
      else block_masked(H, F, RB);
      if constexpr (RB + 1 < Own::kRowBlocks) look_ahead(rows + 32 * kRowBytes);
    }
    before = all;
  };
  auto block = [&](auto H, auto F, auto RB) {
    if constexpr (kMode == kFused) block_fused(H, F, RB);
    else block_apart(F, RB);
  };
  int flush = 0;
  auto step = [&](auto F) {
    if (tid < kTileRows) {
      // a row that sees nothing has weight nowhere
      s_lse[F][tid] = next_lse == kNegInf ? -kNegInf : next_lse * 1.44269504088896340736f;
    }
    // this step's rows lie in LDS (the barrier alone does not wait for a wave's loads to LDS), and nobody reads the
    // other buffer
    if constexpr (kSplit) store();
    else __builtin_amdgcn_s_waitcnt(kNoLoads);
    __syncthreads();
    if constexpr (kSplit) {
      if (r0 + kTileRows < row1) fetch(r0 + kTileRows);
    } else {
      if (kMode != kFew && r0 + kTileRows < row1) bring(std::integral_constant<int, 1 - F>(), r0 + kTileRows);
    }
    if constexpr (kMode == kFused) look_ahead(F == 0 ? s_even : s_odd);
    block(zero, F, std::integral_constant<int, 0>());
    block(one, F, std::integral_constant<int, 1>());
    if constexpr (Own::kRowBlocks == 4) {
      block(zero, F, std::integral_constant<int, 2>());
      block(one, F, std::integral_constant<int, 3>());
    }
    r0 += kTileRows;
  };
  if (tid == 0) s_odd_sum = 0;
  if (row0 < row1) {
    if constexpr (kSplit) fetch(row0);
    else bring(zero, row0);
  }
  while (r0 < row1) {
    step(zero);
    if constexpr (kSplit) {
      __syncthreads();  // the rows have been read
    } else if constexpr (kMode == kFew) {
      __syncthreads();  // the rows have been read
      if (r0 < row1) bring(zero, r0);
    } else {
      if (r0 < row1) step(one);
    }
    if (++flush == kFlush / 2) {
      flush = 0;
#pragma unroll
      for (int b = 0; b < Own::kBlocks; ++b) {
        total[b] += run[b];
        run[b] = 0.0f;
      }
    }
  }
  if constexpr (kMode == kFused) {
    if (before) weigh(of_all, one, zero, blocks, 0);
  }
  float sum[Own::kBlocks];
  bool odd = false;  // a sum is NaN or infinite
#pragma unroll
  for (int b = 0; b < Own::kBlocks; ++b) {
    sum[b] = total[b] + run[b];
    sum[b] += __shfl_xor(sum[b], 32);
    odd |= !(sum[b] < -kNegInf);
  }
  // Such a sum is computed once more, where a row without weights counts for nothing whatever its scores are, and fp32
  // elements are multiplied as they are: an infinite one is not the sum of its parts.  (The same for the workgroup.  Where
  // there is none the check costs nothing measurable at length, 32768 tokens 3891 us / 3898, 8192 of d 64 185.0 / 185.4, and a
  // barrier in short items: 56 rows over 64 caches of 4096 75.8 / 76.7.  Where the last query of 4096 is NaN a call takes 146
  // us for 95, d 64 115 for 65, fp32 520 for 385.)
  if (row0 < row1) {
    if (__any(odd) && lane == 0) s_odd_sum = 1;
    __syncthreads();
    if (s_odd_sum != 0) {
      from = first_row();
      r0 = row0;
      flush = 0;
#pragma unroll
      for (int b = 0; b < Own::kBlocks; ++b) total[b] = run[b] = 0.0f;
      while (r0 < row1) {
        __syncthreads();  // the rows before have been read
        if constexpr (kSplit) {
          fetch(r0);
          store();
        } else {
          bring(zero, r0);
        }
        if (tid < kTileRows) s_lse[0][tid] = next_lse * 1.44269504088896340736f;
        if constexpr (!kSplit) __builtin_amdgcn_s_waitcnt(kNoLoads);
        __syncthreads();
#pragma unroll 1
        for (int rb = 0; rb < Own::kRowBlocks; ++rb) {
          bring_stats(zero, 0, rb);
          auto part = [&](auto B0, auto B1) {
            if (!some_see(r0 + 32 * rb, B0)) return;
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[0][B0][e] = 0.0f;
#pragma unroll
            for (int j = 0; j < Own::kSteps; ++j)
              own.product_each(j, B0, row_piece(s_even + rb * 32 * kRowBytes, j), acc[0][B0]);
            weigh(std::integral_constant<int, kEach>(), zero, B0, B1, r0 + 32 * rb);
          };
          part(zero, one);
          if constexpr (Own::kBlocks == 2) part(one, blocks);
        }
        r0 += kTileRows;
        if (++flush == kFlush) {
          flush = 0;
#pragma unroll
          for (int b = 0; b < Own::kBlocks; ++b) {
            total[b] += run[b];
            run[b] = 0.0f;
          }
        }
      }
#pragma unroll
      for (int b = 0; b < Own::kBlocks; ++b) {
        float again = total[b] + run[b];
        again += __shfl_xor(again, 32);
        if (!(sum[b] < -kNegInf)) sum[b] = again;  // the others stay as they are, bit for bit
      }
    }
  }
#pragma unroll
  for (int b = 0; b < Own::kBlocks; ++b) {
    const int j = wave_key + 32 * b + col;
    if (hi != 0 || j >= p.nk) continue;
    if (p.splits > 1) {
      a.part[p.part * kTileKeys + wave * kWaveKeys + 32 * b + col] = sum[b];
    } else {
      const int64_t at = (int64_t)h * a.Tk + p.k0 + j;
      a.mass_out[at] = j >= n ? 0.0f : a.mass != nullptr ? a.mass[at] + sum[b] : sum[b];
    }
  }
}

// The parts of a tile's keys: four keys a thread, several threads' sums of every so many splits, then those in their order.
// A workgroup looks for its tiles at `batch` items of a head: one each and most find none (a prompt of 32768 tokens, 17000
// items: 18 us, one item a workgroup 27; 8192 tokens of d 64: 6, 9).
template <int kTileKeys>
__global__ __launch_bounds__(kThreads) void mass_join_kernel(const MassArgs a, int batch) {
  constexpr int kLanes = kTileKeys / 4, kSums = kThreads / kLanes;
  __shared__ __attribute__((aligned(16))) float s_sum[kSums][kTileKeys];
  const int h = (int)(blockIdx.x % (unsigned)a.n_heads), first = (int)(blockIdx.x / (unsigned)a.n_heads) * batch;
  const int tid = (int)threadIdx.x, of = tid / kLanes, key = tid % kLanes * 4, end = min(first + batch, a.items);
  for (int item = first; item < end;) {
    const MassItem p = mass_item<false>(a, item, h);
    item += p.splits - p.split;
    if (p.splits <= 1 || p.split != 0) continue;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int k = of; k < p.splits; k += kSums) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(a.part + (p.part + k) * kTileKeys + key);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += x[e];
    }
    __syncthreads();  // the sums of the tile before have been read
    *reinterpret_cast<f32x4*>(&s_sum[of][key]) = sum;
    __syncthreads();
    const int j = p.kt * kTileKeys + tid;
    if (tid >= kTileKeys || j >= p.nk) continue;
    const int n = a.len != nullptr ? min(max(a.len[(int64_t)h * a.n_seqs + p.s], 0), p.nk) : p.nk;
    float all = 0.0f;
#pragma unroll
    for (int i = 0; i < kSums; ++i) all += s_sum[i][tid];
    const int64_t at = (int64_t)h * a.Tk + p.k0 + j;
    a.mass_out[at] = j >= n ? 0.0f : a.mass != nullptr ? a.mass[at] + all : all;
  }
}

template <typename T, int D, int B, int kMode>
int run(const MassArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.items * (unsigned)a.n_heads);
  if (a.k == nullptr) hipLaunchKernelGGL((mass_kernel<T, D, B, kMode, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((mass_kernel<T, D, B, kMode, false>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int launch_mass(const MassArgs& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype != 0) return d == 128 ? run<float, 128, 1, kApart>(a, s) : run<float, 64, 1, kApart>(a, s);
  if (a.few) return d == 128 ? run<bf16, 128, 2, kFew>(a, s) : run<bf16, 64, 2, kFew>(a, s);
  return d == 128 ? run<bf16, 128, 2, kFused>(a, s) : run<bf16, 64, 2, kApart>(a, s);
}

int launch_mass_join(const MassArgs& a, void* stream) {
  const int batch = std::min(std::max((int)((int64_t)a.items * a.n_heads / 1024), 1), 16);
  const dim3 grid((unsigned)((a.items + batch - 1) / batch) * (unsigned)a.n_heads);
  hipStream_t s = (hipStream_t)stream;
  if (a.keys == kMassKeys) hipLaunchKernelGGL(mass_join_kernel<kMassKeys>, grid, dim3(kThreads), 0, s, a, batch);
  else hipLaunchKernelGGL(mass_join_kernel<2 * kMassKeys>, grid, dim3(kThreads), 0, s, a, batch);
  return hipGetLastError();
}

}  // namespace twinkv

// K14: the attention weight that each key receives: sum over the queries that see it, and over the query heads that
// share it, of exp(scale q . k - lse).
//
// With the queries' log-sum-exp at hand a weight is final as it is computed, so this is one product Q K^T whose
// epilogue is a fused multiply-add, an exponential and an addition an element.  A workgroup owns a tile of keys, a
// part of them in each wave's registers for all of its work, and goes over the rows (row = query * group + query
// head) that see them; rows come to LDS 16 bytes a lane without registers, into one of two buffers while the other
// is read, and serve all four waves.  The products put a key in a lane and 16 rows in its registers, so a key's
// weights are added up inside the lane.
//  * bf16: v_mfma_f32_32x32x16_bf16, 64 keys a wave, 64 rows a step.
//  * fp32: v_mfma_f32_32x32x2_f32, 32 keys a wave, 32 rows a step.
//  * keys in 8 bits: their codes become bf16 (fp32 for fp32 queries) once, as they are loaded; the block's scale goes
//    into the multiply-add.
// Sums: 32 bits, in two levels, since one chain over 100000 rows loses 3 digits: a lane adds 16 steps' weights,
// then their sum to the total.  Rows are split over workgroups where there are too few keys, and a second kernel
// adds the parts in their order; nothing is added atomically.
#include <hip/hip_runtime.h>

#include "attn_split.h"
#include "codes8.h"

namespace twinkv {
namespace {

constexpr int kThreads = 256;
constexpr int kFlush = 16;  // steps between additions to the total

// A wave's keys, and the rows of a step.
template <typename T, int D>
struct Keys;

template <int D>
struct Keys<bf16, D> {
  static constexpr int kBlocks = 2, kRowBlocks = 2, kSteps = D / 16;  // of 32 keys, of 32 rows, of 16 channels
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
  // rows: the lane's row in LDS, its 16-byte pieces at place(piece)
  template <typename Place>
  __device__ void products(const char* row, int hi, const Place& place, f32x16 (&acc)[kBlocks]) const {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const bf16x8 q = *reinterpret_cast<const bf16x8*>(row + place(2 * j + hi));
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, k[b][j], acc[b], 0, 0, 0);
    }
  }
};

template <int D>
struct Keys<float, D> {
  static constexpr int kBlocks = 1, kRowBlocks = 1, kSteps = D / 8;
  f32x4 k[kBlocks][kSteps];
  __device__ void load(int b, const char* row, int hi) {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) k[b][j] = *reinterpret_cast<const f32x4*>(row + (2 * j + hi) * 16);
  }
  __device__ void load_codes(int b, const uint8_t* row, int hi) {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) k[b][j] = codes4_f32(*reinterpret_cast<const unsigned*>(row + (2 * j + hi) * 4));
  }
  template <typename Place>
  __device__ void products(const char* row, int hi, const Place& place, f32x16 (&acc)[kBlocks]) const {
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const f32x4 q = *reinterpret_cast<const f32x4*>(row + place(2 * j + hi));
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(q[e], k[0][j][e], acc[0], 0, 0, 0);
    }
  }
};

// What an item is.
struct MassItem {
  int h, s, kt, split, splits;
  int q0, nq, k0, nk;
  int rows;       // of a split
  int64_t part;   // among the parts of all heads, where splits > 1
};
__device__ inline MassItem mass_item(const MassArgs& a, int item, int h) {
  MassItem p;
  p.h = h;
  p.s = find_seq(a.seq, a.n_seqs, kMassSeqWords, 2, item);
  const int w = p.s * kMassSeqWords;
  p.q0 = seq_word(a.seq, w);
  p.k0 = seq_word(a.seq, w + 1);
  const int i = item - seq_word(a.seq, w + 2);
  p.splits = seq_word(a.seq, w + 3);
  p.rows = seq_word(a.seq, w + 4);
  p.part = (int64_t)h * a.parts + seq_word(a.seq, w + 5) + i;
  p.kt = i / p.splits;
  p.split = i - p.kt * p.splits;
  p.nq = seq_word(a.seq, w + kMassSeqWords) - p.q0;
  p.nk = seq_word(a.seq, w + kMassSeqWords + 1) - p.k0;
  return p;
}

template <typename T, int D, bool kCodes>
__global__ __launch_bounds__(kThreads, 2) void mass_kernel(const MassArgs a) {
  typedef Keys<T, D> Own;
  constexpr int kWaveKeys = 32 * Own::kBlocks, kTileKeys = 4 * kWaveKeys, kTileRows = 32 * Own::kRowBlocks;
  constexpr int kRowBytes = D * (int)sizeof(T), kPieces = kRowBytes / 16, kAtOnce = kThreads / kPieces;
  constexpr int kCopies = kTileRows / kAtOnce;
  static_assert(kTileKeys == mass_keys(sizeof(T) == 4), "the host's tiles");
  __shared__ __attribute__((aligned(16))) char s_q[2][kTileRows * kRowBytes];
  __shared__ __attribute__((aligned(16))) float s_lse[2][kTileRows];  // in log2 units
  __shared__ __attribute__((aligned(16))) int s_pos[2][kTileRows];    // of the rows' queries; below 0: no row
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = (int)(blockIdx.x % (unsigned)a.n_heads);
  const MassItem p = mass_item(a, (int)(blockIdx.x / (unsigned)a.n_heads), h);
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

  // Row r of a step for this thread's 16 bytes: query and query head move along by whole steps.
  const char* q_head0 = a.q + (int64_t)h * a.group * a.q_head + (int64_t)p.q0 * a.q_token;
  constexpr int kTurn = kRowBytes == 128 ? 1 : 0;
  auto turn = [](int row) { return kTurn ? (row >> 1) & 7 : row & 15; };
  const int step_q = kTileRows / a.group, step_g = kTileRows % a.group;
  int query[kCopies], sub[kCopies];
#pragma unroll
  for (int c = 0; c < kCopies; ++c) {
    const int r = row0 + c * kAtOnce + tid / kPieces;
    query[c] = r / a.group;
    sub[c] = r - query[c] * a.group;
  }
  int my_query = 0, my_sub = 0;  // of the row whose statistics this thread brings (the first wave)
  if (tid < kTileRows) {
    my_query = (row0 + tid) / a.group;
    my_sub = row0 + tid - my_query * a.group;
  }
  auto advance = [&](int& qu, int& su) {
    qu += step_q;
    su += step_g;
    if (su >= a.group) {
      su -= a.group;
      ++qu;
    }
  };
  float next_lse = 0.0f;
  int next_pos = -1;
  auto bring = [&](int buf) {
    char* to = s_q[buf] + wave * 1024;
#pragma unroll
    for (int c = 0; c < kCopies; ++c) {
      const int r = c * kAtOnce + tid / kPieces;
      const int piece = (tid % kPieces) ^ turn(r);
      const int64_t qu = min(query[c], p.nq - 1);  // rows past the last: any
      to_lds(q_head0 + sub[c] * a.q_head + qu * a.q_token + piece * 16, to + c * (kThreads * 16));
      advance(query[c], sub[c]);
    }
    if (tid < kTileRows) {
      next_pos = -1;
      next_lse = 0.0f;
      if (my_query * a.group + my_sub < row1) {
        next_pos = offset + my_query;
        next_lse = a.lse[((int64_t)h * a.group + my_sub) * a.Tq + p.q0 + my_query];
      }
      advance(my_query, my_sub);
    }
  };

  float total[Own::kBlocks], run[Own::kBlocks];
#pragma unroll
  for (int b = 0; b < Own::kBlocks; ++b) total[b] = run[b] = 0.0f;
  if (row0 < row1) bring(0);
  int buf = 0, flush = 0;
  for (int r0 = row0; r0 < row1; r0 += kTileRows, buf ^= 1) {
    if (tid < kTileRows) {
      // a row that sees nothing has weight nowhere
      s_lse[buf][tid] = next_lse == kNegInf ? -kNegInf : next_lse * 1.44269504088896340736f;
      s_pos[buf][tid] = next_pos;
    }
    // this step's rows lie in LDS (the barrier alone does not wait for a wave's loads to LDS), and nobody reads the
    // other buffer
    __builtin_amdgcn_s_waitcnt(kNoLoads);
    __syncthreads();
    if (r0 + kTileRows < row1) bring(buf ^ 1);
    const int last = min(r0 + kTileRows, row1) - 1;
    const int pos_lo = offset + r0 / a.group, pos_hi = offset + last / a.group;
    if (wave_key > pos_hi || (wave_key + kWaveKeys <= pos_lo - a.window + 1 && wave_key >= a.n_sink)) continue;
    const bool all = r0 + kTileRows <= row1 && wave_key + kWaveKeys <= n && wave_key + kWaveKeys - 1 <= pos_lo &&
                     (wave_key > pos_hi - a.window || wave_key + kWaveKeys <= a.n_sink);
#pragma unroll
    for (int rb = 0; rb < Own::kRowBlocks; ++rb) {
      f32x16 acc[Own::kBlocks];
#pragma unroll
      for (int b = 0; b < Own::kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[b][e] = 0.0f;
      const int row = 32 * rb + col;
      own.products(s_q[buf] + row * kRowBytes, hi, [&](int piece) { return (piece ^ turn(row)) * 16; }, acc);
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // rows 8x + 4hi .. + 3 of the block
        const f32x4 l = *reinterpret_cast<const f32x4*>(&s_lse[buf][32 * rb + 8 * x + 4 * hi]);
        if (all) {
#pragma unroll
          for (int b = 0; b < Own::kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) run[b] += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[b][4 * x + e], scale[b], -l[e]));
        } else {
          int at[4];
          __builtin_memcpy(at, &s_pos[buf][32 * rb + 8 * x + 4 * hi], 16);
#pragma unroll
          for (int b = 0; b < Own::kBlocks; ++b) {
            const int j = wave_key + 32 * b + col;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[b][4 * x + e], scale[b], -l[e]));
              const bool seen = (j < n) & (j <= at[e]) & ((at[e] - j < a.window) | (j < a.n_sink));
              run[b] += seen ? w : 0.0f;
            }
          }
        }
      }
    }
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
    float sum = total[b] + run[b];
    sum += __shfl_xor(sum, 32);
    const int j = wave_key + 32 * b + col;
    if (hi != 0 || j >= p.nk) continue;
    if (p.splits > 1) {
      a.part[p.part * kTileKeys + wave * kWaveKeys + 32 * b + col] = sum;
    } else {
      const int64_t at = (int64_t)h * a.Tk + p.k0 + j;
      a.mass_out[at] = j >= n ? 0.0f : a.mass != nullptr ? a.mass[at] + sum : sum;
    }
  }
}

// The parts of a tile's keys, in their order.
template <int kTileKeys>
__global__ __launch_bounds__(kTileKeys) void mass_join_kernel(const MassArgs a) {
  const int h = (int)(blockIdx.x % (unsigned)a.n_heads);
  const MassItem p = mass_item(a, (int)(blockIdx.x / (unsigned)a.n_heads), h);
  if (p.splits <= 1 || p.split != 0) return;
  const int j = p.kt * kTileKeys + (int)threadIdx.x;
  if (j >= p.nk) return;
  const int n = a.len != nullptr ? min(max(a.len[(int64_t)h * a.n_seqs + p.s], 0), p.nk) : p.nk;
  float sum = 0.0f;
  for (int k = 0; k < p.splits; ++k) sum += a.part[(p.part + k) * kTileKeys + threadIdx.x];
  const int64_t at = (int64_t)h * a.Tk + p.k0 + j;
  a.mass_out[at] = j >= n ? 0.0f : a.mass != nullptr ? a.mass[at] + sum : sum;
}

template <typename T, int D>
int run(const MassArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.items * (unsigned)a.n_heads);
  if (a.k == nullptr) hipLaunchKernelGGL((mass_kernel<T, D, true>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((mass_kernel<T, D, false>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int launch_mass(const MassArgs& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 0) return d == 128 ? run<bf16, 128>(a, s) : run<bf16, 64>(a, s);
  return d == 128 ? run<float, 128>(a, s) : run<float, 64>(a, s);
}

int launch_mass_join(const MassArgs& a, int dtype, void* stream) {
  const dim3 grid((unsigned)a.items * (unsigned)a.n_heads);
  if (dtype == 0) hipLaunchKernelGGL(mass_join_kernel<mass_keys(0)>, grid, dim3(mass_keys(0)), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(mass_join_kernel<mass_keys(1)>, grid, dim3(mass_keys(1)), 0, (hipStream_t)stream, a);
  return hipGetLastError();
}

}  // namespace twinkv

// K10: attention over the window and the sinks, bf16, many rows (prompts and chunks of prompts).
//
// A workgroup of 4 waves owns 128 rows (row = query * group + query head: the heads that share keys sit in one
// tile, so it spans few queries and little of its work is masked), 32 a wave, and goes over their keys in
// tiles of 64.
//  * K q^T on v_mfma_f32_32x32x16_bf16: a lane holds one row (lane % 32) and half of the tile's keys, so
//    maxima and sums need one exchange between two lanes, and that only when the maximum moves by more
//    than kSlack (attn_split.h).
//  * O^T = V^T P^T: the weights are the B operand as they lie; the contraction's order is chosen so that a
//    lane's keys are its own.  V^T comes from the row-major tile by ds_read_b64_tr_b16.  The accumulators
//    hold channels of the lane's own row, so rescaling and normalising them needs no exchange.
//  * Keys and values go from memory to LDS without registers, into one of two buffers while the other is
//    read; 16-byte pieces of the keys and 32-byte units of the values are turned by the row so that the
//    lanes of a read lie in different banks.  One barrier a tile.  (Through registers and LDS writes the 32k
//    prompt took 10% longer.)
//  * With too few row tiles for the machine a tile's keys are split over workgroups and joined (attn4.hip).
//  * Two workgroups fit a CU (64 KB of LDS each, 256 registers): one's softmax runs beside the other's
//    products.
// A prompt of 32k tokens, 32 heads of 128, window 4096: 2160 us, 956 TFLOP/s of the 1290 that a large bf16 product
// reaches; 8k tokens of d 64, causal, 322 us, 852 TFLOP/s.  In the profiled run the matrix units are busy 47% of
// the cycles and the vector units 39% (a third of that the exponentials), at a clock of 2.0 GHz; d 64 40% and 60%.  A
// form of the loop that took 12% more cycles took 5% more time.  Neither 256 rows a workgroup, which halves the memory
// traffic, nor opposite phases for a SIMD's two waves, nor the next tile's scores between this one's
// exponentials were faster.
// The weights are rounded to bf16 for the product.  With them as two bf16 parts, and two products, the error against
// 64 bits is that of the output's own rounding, 0.0016 of the result's norm instead of 0.0022, but the two prompts take
// 2860 and 444 us.
// Values that only some rows of a tile see: as in attn.hip.
#include <hip/hip_runtime.h>

#include "attn_split.h"

namespace twinkv {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kWaveRows = 32;
constexpr int kRows = kAttnBigRows;
constexpr int kKeys = kAttnBigTile;
static_assert(kRows == kThreads / 64 * kWaveRows, "a wave owns 32 rows");

template <int D>
struct Lds {
  char k[2][kKeys * D * 2];
  char v[2][kKeys * D * 2];
  int bad;  // the last tile that held a value which is not finite
};

// Where 16-byte piece `piece` of key row `row` lies in its tile, and where 32-byte unit `unit` of value row
// `row` does.
template <int D>
__device__ inline int k_place(int row, int piece) {
  return row * (D * 2) + ((piece ^ (D == 128 ? row & 15 : (row >> 1) & 7)) << 4);
}
template <int D>
__device__ inline int v_unit(int row, int unit) {
  return unit ^ (D == 128 ? 2 * (row & 3) : 2 * ((row >> 1) & 1));
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void attn_rows_kernel(const AttnArgs a) {
  constexpr int kSteps = D / 16;          // of the contraction over channels
  constexpr int kBlocks = D / 32;         // of 32 output channels
  constexpr int kRowBytes = D * 2;
  constexpr int kPieces = kRowBytes / 16;
  constexpr int kCopies = kKeys * kRowBytes / (kThreads * 16);  // 16-byte pieces a thread brings of each tile
  __shared__ __attribute__((aligned(16))) Lds<D> s;

  const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // heads side by side: with 8 of them each XCD's L2 keeps one head's keys; the last rows of a sequence,
  // which see most, first
  const int h = (int)(blockIdx.x % (unsigned)a.n_heads);
  const AttnItem p = attn_item(a, a.items - 1 - (int)(blockIdx.x / (unsigned)a.n_heads), h);
  const int n_rows = p.nq * a.group, row0 = p.rt * kRows;
  const int offset = p.nk - p.nq;         // position of query 0
  // what the workgroup's rows see
  const int pos_lo = offset + row0 / a.group;
  const int pos_hi = offset + (min(row0 + kRows, n_rows) - 1) / a.group;
  const int end = max(pos_hi + 1, 0);
  const int sinks = min(a.n_sink, end);
  int lo = min(max(pos_lo - a.window + 1, 0), end);
  int sink_tiles = (sinks + kKeys - 1) / kKeys;
  if (lo <= sink_tiles * kKeys) {         // the two meet
    if (sinks > 0) lo = 0;
    sink_tiles = 0;
  }
  // this item's tiles of them
  const int all_tiles = sink_tiles + (end - lo + kKeys - 1) / kKeys;
  const int first = p.split * p.tiles, tiles = min(all_tiles, first + p.tiles);
  // this lane's row; rows past the problem's repeat its last, and are not written
  const int row = min(row0 + wave * kWaveRows + r32, n_rows - 1);
  const int query = row / a.group;
  const int pos = offset + query;
  // and what the wave's rows see
  const int wave_lo = offset + min(row0 + wave * kWaveRows, n_rows - 1) / a.group;
  const int wave_hi = offset + min(row0 + wave * kWaveRows + kWaveRows - 1, n_rows - 1) / a.group;

  const char* kb = a.k + (int64_t)h * a.k_head + (int64_t)p.k0 * a.k_token;
  const char* vb = a.v + (int64_t)h * a.v_head + (int64_t)p.k0 * a.v_token;
  // Brings tile t into buffer t % 2: a wave instruction fills 1 KB of LDS in lane order, so it is the source
  // that is turned.  A lane's rows of the 4 (2) instructions lie kRowsAtOnce apart and turn alike: one offset
  // of the lane, the rest is the same for all (the host takes this kernel where 64 tokens' strides stay
  // within 32 bits).
  constexpr int kRowsAtOnce = kThreads / kPieces;
  const int r_lane = tid / kPieces, piece = tid % kPieces;
  const unsigned k_turned = ((k_place<D>(r_lane, piece) >> 4) & (kPieces - 1)) * 16;
  const unsigned v_turned = v_unit<D>(r_lane, piece >> 1) * 32 + (piece & 1) * 16;
  const unsigned k_lane = (unsigned)r_lane * (unsigned)a.k_token + k_turned;
  const unsigned v_lane = (unsigned)r_lane * (unsigned)a.v_token + v_turned;
  // Where the next tile to bring lies; what is the same for all lanes stays out of the loop, whose scalar
  // instructions are a good part of a wave's own time.
  const int64_t k_tile = (int64_t)kKeys * a.k_token, v_tile = (int64_t)kKeys * a.v_token;
  const int64_t k_step = (int64_t)kRowsAtOnce * a.k_token, v_step = (int64_t)kRowsAtOnce * a.v_token;
  auto base_of = [&](int t) { return t < sink_tiles ? t * kKeys : lo + (t - sink_tiles) * kKeys; };
  auto stop_of = [&](int t) { return t < sink_tiles ? sinks : end; };
  const char* k_from = kb + (int64_t)base_of(first) * a.k_token;
  const char* v_from = vb + (int64_t)base_of(first) * a.v_token;
  auto bring = [&](int t) {
    char* kl = s.k[t & 1] + wave * 1024;
    char* vl = s.v[t & 1] + wave * 1024;
    const bool sink_end = t == sink_tiles - 1;
    if (t != all_tiles - 1 && !sink_end) {
#pragma unroll
      for (int c = 0; c < kCopies; ++c) {
        to_lds(k_from + c * k_step + k_lane, kl + c * (kThreads * 16));
        to_lds(v_from + c * v_step + v_lane, vl + c * (kThreads * 16));
      }
    } else {  // the last key again past the end
      const int rows = (sink_end ? sinks - 1 : end - 1 - lo) % kKeys;
#pragma unroll
      for (int c = 0; c < kCopies; ++c) {
        const unsigned r = min(c * kRowsAtOnce + r_lane, rows);
        to_lds(k_from + (r * (unsigned)a.k_token + k_turned), kl + c * (kThreads * 16));
        to_lds(v_from + (r * (unsigned)a.v_token + v_turned), vl + c * (kThreads * 16));
      }
    }
    k_from = sink_end ? kb + (int64_t)lo * a.k_token : k_from + k_tile;
    v_from = sink_end ? vb + (int64_t)lo * a.v_token : v_from + v_tile;
  };
  // The window's tiles that rows at positions first .. last all see whole are a run, and so are the ones of
  // which some of them sees anything (from key 0 there may be sinks: no tile is left out before it).
  struct Run {
    int from, to;
  };
  auto whole_of = [&](int first, int last) {
    return Run{sink_tiles + max(last - a.window + 1 - lo + kKeys - 1, 0) / kKeys,
               sink_tiles + max(first + 1 - lo, 0) / kKeys};
  };
  const Run all_see = whole_of(pos_lo, pos_hi), all = whole_of(wave_lo, wave_hi);
  const Run some{lo == 0 ? 0 : sink_tiles + max(wave_lo - a.window + 1 - lo, 0) / kKeys,
                 sink_tiles + max(wave_hi - lo + kKeys, 0) / kKeys};

  // scale > 0 from here on: the sign goes to q.  0 (all weights alike) becomes as good as 0, so that masked
  // scores stay -inf.
  const float scale = fmaxf(fabsf(a.scale_log2), 1e-37f);
  bf16x8 q[kSteps];
  {
    const char* src = a.q + ((int64_t)h * a.group + (row - query * a.group)) * a.q_head +
                      (int64_t)(p.q0 + query) * a.q_token + hi * 16;
    const unsigned flip = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      u32x4 w = *reinterpret_cast<const u32x4*>(src + j * 32);
      w ^= flip;
      q[j] = __builtin_bit_cast(bf16x8, w);
    }
  }
  if (tid == 0) s.bad = -1;

  f32x16 acc[kBlocks];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[b][e] = 0.0f;
  float m = kNegInf, l = 0.0f;

  if (first < tiles) bring(first);
  for (int t = first; t < tiles; ++t) {
    // tile t lies in LDS (the barrier alone does not wait for a wave's loads to LDS), and nobody reads the
    // other buffer
    __builtin_amdgcn_s_waitcnt(kNoLoads);
    __syncthreads();
    if (t + 1 < tiles) bring(t + 1);
    const char* ks = s.k[t & 1];
    char* vs = s.v[t & 1];
    bool bad = false;
    if (t < all_see.from || t >= all_see.to) {
      // some row does not see some key: values that are past the range or not finite become zeros
      const int rows = stop_of(t) - base_of(t);
#pragma unroll
      for (int c = 0; c < kCopies; ++c) {
        const int at = c * kThreads + tid;
        s16x8 x = *reinterpret_cast<const s16x8*>(vs + at * 16);
        const bool out = at / kPieces >= rows;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool o = (x[e] & 0x7f80) == 0x7f80;
          odd |= o;
          if (o || out) x[e] = 0;
        }
        if (odd || out) *reinterpret_cast<s16x8*>(vs + at * 16) = x;
        if (odd && !out) s.bad = t;
      }
      __syncthreads();
      bad = s.bad == t;
    }
    if (t >= sink_tiles && (t < some.from || t >= some.to)) continue;  // nothing for this wave's rows

    // all of the tile's keys on their way before the first product waits for one of them
    bf16x8 k[kSteps][2];
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
#pragma unroll
      for (int b = 0; b < 2; ++b)
        k[j][b] = *reinterpret_cast<const bf16x8*>(ks + k_place<D>(b * 32 + r32, 2 * j + hi));
    __builtin_amdgcn_sched_barrier(0);
    f32x16 x[2];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) x[b][e] = 0.0f;
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
#pragma unroll
      for (int b = 0; b < 2; ++b) x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[j][b], q[j], x[b], 0, 0, 0);
    if (t < all.from || t >= all.to) {
      const int base = base_of(t), stop = stop_of(t);
      // the row sees [from, upto) of these keys, and those below n_sink
      const int upto = min(stop, pos + 1), from = pos - a.window + 1;
      const int j0 = base + 4 * hi;
      const unsigned seen = (unsigned)max(upto - from, 0);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int j = j0 + (b * 32 + 8 * (e >> 2) + (e & 3));
          if (!((unsigned)j - (unsigned)from < seen)) {
            if (base >= a.n_sink || !((j < upto) & (j < a.n_sink))) x[b][e] = kNegInf;
          }
        }
    }
    // (the maximum that a NaN passes through: v_maximum3_f32 takes the products' results as they are)
    float most = __builtin_elementwise_maximum(x[0][0], x[1][0]);
#pragma unroll
    for (int e = 1; e < 16; ++e) most = __builtin_elementwise_maximum(__builtin_elementwise_maximum(most, x[0][e]), x[1][e]);
    most *= scale;
    if (__any(most > m + kSlack)) {
      const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(most), __float_as_uint(most), false, false);
      const float next = fmaxf(m, fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1])));
      const float f = next == m ? 1.0f : __builtin_amdgcn_exp2f(m - next);
      m = next;
      l *= f;
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[b][e] *= f;
    }
    const float from = m == kNegInf ? 0.0f : m;
    bf16x8 w[4];                           // 16 keys each
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][e], scale, -from));
        sum[e & 1] += y;
        w[2 * b + (e >> 3)][e & 7] = (bf16)y;
      }
    l += sum[0] + sum[1];
    asm volatile("" : "+v"(l));  // added up here: put off, the sum would keep 32 registers
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        // lane i of 16 points at key row i / 4, 4 channels at i % 4; it gets channel i of the 4 keys
        s16x4 v[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int r = 16 * j + 8 * u + 4 * hi + ((lane & 15) >> 2);
          const int unit = v_unit<D>(r, 2 * b + ((lane >> 4) & 1));
          v[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) s16x4*)(vs + r * kRowBytes + unit * 32 + (lane & 3) * 8));
        }
        struct Two { s16x4 a, b; } two = {v[0], v[1]};
        acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, two), w[j], acc[b], 0, 0, 0);
      }
    if (bad) {
      // the values that are not finite, to the rows that see them
      const int base = base_of(t), stop = stop_of(t);
      for (int y = 0; y < kKeys; ++y) {
        const int j = base + y;
        if (j >= stop) break;
        const int e = 4 * ((y & 31) >> 3) + (y & 3);
        float mine = 0.0f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int z = 0; z < 16; ++z) mine = (y >> 5) == b && e == z ? (float)w[2 * b + (z >> 3)][z & 7] : mine;
        const float weight = __shfl(mine, r32 + 32 * ((y >> 2) & 1));
        if (!(j <= pos && (pos - j < a.window || j < a.n_sink))) continue;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int z = 0; z < 16; ++z) {
            const int ch = 32 * b + 8 * (z >> 2) + 4 * hi + (z & 3);
            const float v = (float)*reinterpret_cast<const bf16*>(vb + j * a.v_token + ch * 2);
            if ((__float_as_uint(v) & 0x7f800000u) == 0x7f800000u) acc[b][z] += weight * v;
          }
      }
    }
  }

  {
    const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(two[0]) + __uint_as_float(two[1]);
  }
  if (row0 + wave * kWaveRows + r32 >= n_rows) return;
  if (p.splits > 1) {
    const int64_t part = p.part * kRows + wave * kWaveRows + r32;
    float* to = a.part_o + part * D;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        *reinterpret_cast<f32x4*>(to + 32 * b + 8 * y + 4 * hi) =
            f32x4{acc[b][4 * y], acc[b][4 * y + 1], acc[b][4 * y + 2], acc[b][4 * y + 3]};
    if (hi == 0) {
      a.part_ml[part * 2] = m;
      a.part_ml[part * 2 + 1] = l;
    }
    return;
  }
  const float inv = l > 0.0f ? 1.0f / l : (l == 0.0f ? 0.0f : l);
  const int64_t head = (int64_t)h * a.group + (row - query * a.group);
  char* out = a.out + head * a.o_head + (int64_t)(p.q0 + query) * a.o_token;
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
      bf16x4 o;
#pragma unroll
      for (int z = 0; z < 4; ++z) o[z] = (bf16)(acc[b][4 * y + z] * inv);
      *reinterpret_cast<bf16x4*>(out + (32 * b + 8 * y + 4 * hi) * 2) = o;
    }
  if (a.lse != nullptr && hi == 0)
    a.lse[head * a.Tq + p.q0 + query] = l == 0.0f ? kNegInf : m * 0.69314718055994530942f + logf(l);
}

template <int D>
int run(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((attn_rows_kernel<D>), dim3((unsigned)a.items * (unsigned)a.n_heads), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int launch_attn_rows(const AttnArgs& a, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  return d == 128 ? run<128>(a, s) : run<64>(a, s);
}

}  // namespace twinkv

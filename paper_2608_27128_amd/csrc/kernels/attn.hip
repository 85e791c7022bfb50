// K9: attention over the window and the sinks, few rows or fp32.  Few rows: the keys split over waves and
// workgroups (attn_split.h).
//
// bf16: 32 keys a wave at a time.  K q^T takes the key rows as they lie in memory, 16 bytes a lane,
// without LDS.  The product with the values contracts over tokens, so the values' tile goes through the
// wave's own LDS and comes back transposed (ds_read_b64_tr_b16: 4 tokens of a channel to a lane); units of
// 32 bytes are rotated by the row so that the 4 rows such a read touches lie in different banks.
// Nothing of it is shared between waves, so there is no barrier in the loop.  HBM-bound: 64 sequences, 1028 keys of a
// window each, 8 heads of 4, d 128: 52 us, 5.1 TB/s.  (Fetching a tile's keys and values before the tile in
// front is done took 175 registers instead of 160 and 1-8% longer.)
// The weights are rounded to bf16 for the product with the values (error against 64 bits 0.0023 of the result's
// norm, 0.0017 of it the output's own rounding).  As two bf16 parts they would lose nothing, single tokens would take
// as long and 256 to 480 rows over 4k keys 4 to 10% longer; but the smaller part is often 0, and would make NaN of an
// infinite value that a row sees.
// fp32: v_mfma_f32_16x16x4_f32, whose operands are single values a lane: keys and values are read 16 bytes a lane, the
// contraction's and the channels' order chosen to fit.
//  * Few rows: straight from memory.
//  * Many: four row tiles share their keys through LDS (attn_wide_kernel), which reads a quarter as much: 2048 tokens,
//    32 heads of 128, causal, 326 us (443 in the kernel for few rows), 106 of the 153 TFLOP/s of a large product;
//    2048 tokens over 4k keys 865 (1117), 119 TFLOP/s.  Row tiles with the most keys go first: with the heads one
//    after the other the first of these took 461 us.  5 prompts of up to 1500 tokens, window 128, d 64 take 28 us
//    (31 with a row tile a wave and nothing shared), at most 7 key tiles one after the other.
// Values that no row of a tile sees are taken as zeros.  A tile that some rows see and others do not may
// hold a NaN or infinite value, which the product would spread (0 * inf) to the rows that do not: those
// elements are zeroed before the product and added one by one to the rows that see them.
#include <hip/hip_runtime.h>

#include "attn_split.h"

namespace twinkv {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Which keys a tile of rows sees.
struct Span {
  int pos_lo, pos_hi;  // positions of its first and last row
  int sinks;           // sink tiles cover [0, sinks)
  int sink_tiles;
  int lo, end;         // the other tiles cover [lo, end)
  int tiles;
};
__device__ inline Span span_of(const AttnArgs& a, const AttnItem& p, int row0, int last) {
  Span s;
  s.pos_lo = p.nk - p.nq + row0 / a.group;
  s.pos_hi = p.nk - p.nq + last / a.group;
  s.end = max(s.pos_hi + 1, 0);
  s.lo = min(max(s.pos_lo - a.window + 1, 0), s.end);
  s.sinks = min(a.n_sink, s.end);
  s.sink_tiles = (s.sinks + kAttnTile - 1) / kAttnTile;
  if (s.lo <= s.sink_tiles * kAttnTile) {  // the two meet
    if (s.sinks > 0) s.lo = 0;
    s.sink_tiles = 0;
  }
  s.tiles = s.sink_tiles + (s.end - s.lo + kAttnTile - 1) / kAttnTile;
  return s;
}

template <typename T>
__device__ inline bool not_finite(T x) {
  if constexpr (sizeof(T) == 4) return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u;
  else return (__builtin_bit_cast(uint16_t, x) & 0x7f80u) == 0x7f80u;
}

// One wave's tile.  channel(n, i) is the channel of accumulator n of lane i.
template <typename T, int D>
struct Tile;

template <int D>
struct Tile<bf16, D> {
  static constexpr int kLds = kAttnTile * D * 2;  // bytes a wave needs
  static constexpr int kSteps = D / 32, kPieces = D / 8, kLoads = kAttnTile * kPieces / 64;
  bf16x8 k[2][kSteps];
  bf16x8 v[kLoads];
  struct Query {
    bf16x8 x[kSteps];
    __device__ void load(const char* p, int g) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) x[j] = *reinterpret_cast<const bf16x8*>(p + j * 64 + g * 16);
    }
  };
  __device__ static int channel(int n, int i) { return n * 16 + i; }
  __device__ static int place(int row, int piece) {  // byte of a 16-byte piece in the tile
    const int turn = D == 128 ? row & 7 : (row >> 1) & 3;
    return row * (D * 2) + (((piece >> 1) ^ turn) * 32) + (piece & 1) * 16;
  }
  // keys base.. (clamped to end - 1, which is in the sequence)
  __device__ void load(const char* kb, int64_t k_token, const char* vb, int64_t v_token, int base, int end, int lane) {
    const int i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int t = min(base + 8 * (i >> 2) + 4 * m + (i & 3), end - 1);
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
        k[m][j] = *reinterpret_cast<const bf16x8*>(kb + t * k_token + j * 64 + g * 16);
    }
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int at = u * 64 + lane;
      const int t = min(base + at / kPieces, end - 1);
      v[u] = *reinterpret_cast<const bf16x8*>(vb + t * v_token + at % kPieces * 16);
    }
  }
  __device__ void scores(const Query& q, float (&s)[8]) const {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < kSteps; ++j) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[m][j], q.x[j], d, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[4 * m + r] = d[r];
    }
  }
  // Zeroes the values past the range and the ones that are not finite; returns whether there are such.
  __device__ bool clean(int base, int end, int lane) {
    bool bad = false;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const bool out = base + (u * 64 + lane) / kPieces >= end;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool odd = not_finite(v[u][e]);
        bad |= odd && !out;
        if (odd || out) v[u][e] = (bf16)0.0f;
      }
    }
    return __any(bad);
  }
  __device__ void stage(char* lds, int lane) const {
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      const int at = u * 64 + lane;
      *reinterpret_cast<bf16x8*>(lds + place(at / kPieces, at % kPieces)) = v[u];
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  __device__ static void product(const float (&s)[8], const Tile&, const char* lds, int lane, f32x4 (&acc)[D / 16]) {
    const int i = lane & 15, g = lane >> 4;
    bf16x8 w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = (bf16)s[e];
#pragma unroll
    for (int n = 0; n < D / 16; ++n) {
      // rows 8g .. 8g + 7 of channels 16n .. 16n + 15; lane i points at row i / 4, 4 channels at i % 4
      s16x4 h[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const char* at = lds + place(8 * g + 4 * u + (i >> 2), 2 * n) + (i & 3) * 8;
        h[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(uintptr_t)(__attribute__((address_space(3))) char*)at);
      }
      struct Two { s16x4 a, b; } two = {h[0], h[1]};
      acc[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, __builtin_bit_cast(bf16x8, two), acc[n], 0, 0, 0);
    }
    // the next tile's values are staged in the same place
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
};

template <int D>
struct Tile<float, D> {
  static constexpr int kLds = 16;
  static constexpr int kSteps = D / 16;
  f32x4 k[2][kSteps];
  f32x4 v[8][D / 64];
  struct Query {
    f32x4 x[kSteps];
    __device__ void load(const char* p, int g) {
#pragma unroll
      for (int j = 0; j < kSteps; ++j) x[j] = *reinterpret_cast<const f32x4*>(p + j * 64 + g * 16);
    }
  };
  __device__ static int channel(int n, int i) { return (n >> 2) * 64 + 4 * i + (n & 3); }
  __device__ void load(const char* kb, int64_t k_token, const char* vb, int64_t v_token, int base, int end, int lane) {
    const int i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int t = min(base + 8 * (i >> 2) + 4 * m + (i & 3), end - 1);
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
        k[m][j] = *reinterpret_cast<const f32x4*>(kb + t * k_token + j * 64 + g * 16);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = min(base + 8 * g + e, end - 1);
#pragma unroll
      for (int x = 0; x < D / 64; ++x) v[e][x] = *reinterpret_cast<const f32x4*>(vb + t * v_token + x * 256 + i * 16);
    }
  }
  // A tile in LDS: rows of D values, the 16-byte pieces of key row `row` turned by turn(row) so that the lanes of
  // a read lie in different banks.
  __device__ static int turn(int row) { return 4 * (row >> 3) + (row & 3); }
  __device__ void load(const char* kl, const char* vl, int lane) {
    const int i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int t = 8 * (i >> 2) + 4 * m + (i & 3);
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
        k[m][j] = *reinterpret_cast<const f32x4*>(kl + t * (D * 4) + ((4 * j + g) ^ turn(t)) * 16);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
        v[e][x] = *reinterpret_cast<const f32x4*>(vl + (8 * g + e) * (D * 4) + x * 256 + i * 16);
  }
  __device__ void scores(const Query& q, float (&s)[8]) const {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) d = __builtin_amdgcn_mfma_f32_16x16x4f32(k[m][j][e], q.x[j][e], d, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 4; ++r) s[4 * m + r] = d[r];
    }
  }
  __device__ bool clean(int base, int end, int lane) {
    const int g = lane >> 4;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const bool out = base + 8 * g + e >= end;
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const bool odd = not_finite(v[e][x][y]);
          bad |= odd && !out;
          if (odd || out) v[e][x][y] = 0.0f;
        }
    }
    return __any(bad);
  }
  __device__ void stage(char*, int) const {}
  __device__ static void product(const float (&s)[8], const Tile& t, const char*, int, f32x4 (&acc)[D / 16]) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
        acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(s[e], t.v[e][n >> 2][n & 3], acc[n], 0, 0, 0);
  }
};

// Adds a tile's values that are not finite to the rows that see them (accumulator rows 4g .. 4g + 3).
template <typename T, int D>
__device__ inline void add_odd(const AttnArgs& a, const char* vb, int base, int end, int pos, int window, int i, int g,
                               const float (&s)[8], f32x4 (&acc)[D / 16]) {
  int at[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) at[r] = __shfl(pos, 4 * g + r);
  for (int o = 0; o < 4; ++o) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int j = base + 8 * o + e;
      float w[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) w[r] = __shfl(s[e], 16 * o + 4 * g + r);
      if (j >= end) continue;
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        const T v = *reinterpret_cast<const T*>(vb + j * a.v_token + Tile<T, D>::channel(n, i) * (int)sizeof(T));
        if (!not_finite(v)) continue;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (j <= at[r] && (at[r] - j < window || j < a.n_sink)) acc[n][r] += w[r] * (float)v;
      }
    }
  }
}

// Few rows: a workgroup has 16, and its four waves share their keys.
template <typename T, int D>
__global__ __launch_bounds__(64 * kAttnWaves) void attn_kernel(const AttnArgs a) {
  typedef Tile<T, D> Keys;
  __shared__ __attribute__((aligned(16))) char s_values[kAttnWaves][Keys::kLds];
  __shared__ float s_join[join_floats<D>()];
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const AttnItem p = attn_item(a, (int)blockIdx.x, (int)blockIdx.y);
  const int n_rows = p.nq * a.group, row0 = p.rt * kAttnRows;
  const int last = min(row0 + kAttnRows, n_rows) - 1;
  const int row = min(row0 + i, n_rows - 1);  // rows past the problem's repeat its last, and are not written
  const int query = row / a.group;
  const int pos = p.nk - p.nq + query;
  const Span sp = span_of(a, p, row0, last);
  const int first = p.split * p.tiles + wave;
  const int stop = min(sp.tiles, (p.split + 1) * p.tiles);
  const int window = a.window;

  typename Keys::Query q;
  q.load(a.q + ((int64_t)p.h * a.group + (row - query * a.group)) * a.q_head + (int64_t)(p.q0 + query) * a.q_token, g);
  const char* kb = a.k + (int64_t)p.h * a.k_head + (int64_t)p.k0 * a.k_token;
  const char* vb = a.v + (int64_t)p.h * a.v_head + (int64_t)p.k0 * a.v_token;
  char* lds = s_values[wave];

  RowStats st;
  f32x4 acc[D / 16];
#pragma unroll
  for (int n = 0; n < D / 16; ++n) acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  Keys now;
  for (int x = first; x < stop; x += kAttnWaves) {
    const bool sink = x < sp.sink_tiles;
    const int base = sink ? x * kAttnTile : sp.lo + (x - sp.sink_tiles) * kAttnTile;
    const int end = sink ? sp.sinks : sp.end;
    now.load(kb, a.k_token, vb, a.v_token, base, end, lane);
    const bool all = base + kAttnTile <= end && base + kAttnTile - 1 <= sp.pos_lo &&
                     (base > sp.pos_hi - window || base + kAttnTile <= a.n_sink);
    bool bad = false;
    if (!all) bad = now.clean(base, end, lane);
    now.stage(lds, lane);
    float s[8];
    now.scores(q, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] *= a.scale_log2;
      if (!all) {
        const int j = base + 8 * g + e;
        if (!((j < end) & (j <= pos) & ((pos - j < window) | (j < a.n_sink)))) s[e] = kNegInf;
      }
    }
    st.update(s, acc);
    Keys::product(s, now, lds, lane, acc);
    if (bad) add_odd<T, D>(a, vb, base, end, pos, window, i, g, s, acc);
  }
  join_waves<T, D>(a, p, row0, st, acc, s_join, [](int n, int lane16) { return Keys::channel(n, lane16); });
}

// Many rows, fp32: a workgroup has 64, 16 a wave, and goes over their keys once.  A tile comes from memory to LDS
// without registers, into one of two buffers while the other is read, one barrier a tile.
template <int D>
__global__ __launch_bounds__(64 * kAttnWaves, 2) void attn_wide_kernel(const AttnArgs a) {
  typedef Tile<float, D> Keys;
  constexpr int kThreads = 64 * kAttnWaves, kRowBytes = D * 4, kPieces = kRowBytes / 16, kRowsAtOnce = kThreads / kPieces;
  struct Tiles {
    char k[2][kAttnTile * kRowBytes];
    char v[2][kAttnTile * kRowBytes];
  };
  union Lds {
    Tiles t;
    float own[kAttnWaves * own_floats<D>()];
  };
  __shared__ __attribute__((aligned(16))) Lds lds;
  const int tid = threadIdx.x, lane = tid & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // heads side by side, and the last rows of a sequence, which see most, first
  const int h = (int)(blockIdx.x % (unsigned)a.n_heads);
  const AttnItem p = attn_item(a, a.items - 1 - (int)(blockIdx.x / (unsigned)a.n_heads), h);
  const int n_rows = p.nq * a.group, offset = p.nk - p.nq;
  const Span sp = span_of(a, p, p.rt * kAttnWideRows, min((p.rt + 1) * kAttnWideRows, n_rows) - 1);
  // the wave's rows (there may be none), and this lane's; rows past the problem's repeat its last
  const int row0 = p.rt * kAttnWideRows + wave * kAttnRows;
  const int wave_lo = offset + min(row0, n_rows - 1) / a.group;
  const int wave_hi = offset + min(row0 + kAttnRows - 1, n_rows - 1) / a.group;
  const int row = min(row0 + i, n_rows - 1);
  const int query = row / a.group;
  const int pos = offset + query;
  const int window = a.window;

  typename Keys::Query q;
  q.load(a.q + ((int64_t)p.h * a.group + (row - query * a.group)) * a.q_head + (int64_t)(p.q0 + query) * a.q_token, g);
  const char* kb = a.k + (int64_t)p.h * a.k_head + (int64_t)p.k0 * a.k_token;
  const char* vb = a.v + (int64_t)p.h * a.v_head + (int64_t)p.k0 * a.v_token;

  auto base_of = [&](int x) { return x < sp.sink_tiles ? x * kAttnTile : sp.lo + (x - sp.sink_tiles) * kAttnTile; };
  auto end_of = [&](int x) { return x < sp.sink_tiles ? sp.sinks : sp.end; };
  // A wave instruction fills 1 KB of LDS in lane order, so it is the source that is turned.  Past the end the last
  // key comes again.
  auto bring = [&](int x) {
    const int base = base_of(x), end = end_of(x);
    char* kl = lds.t.k[x & 1] + wave * 1024;
    char* vl = lds.t.v[x & 1] + wave * 1024;
#pragma unroll
    for (int c = 0; c < kAttnTile / kRowsAtOnce; ++c) {
      const int r = c * kRowsAtOnce + tid / kPieces, piece = tid % kPieces;
      const int64_t t = min(base + r, end - 1);
      to_lds(kb + t * a.k_token + (piece ^ Keys::turn(r)) * 16, kl + c * (kThreads * 16));
      to_lds(vb + t * a.v_token + piece * 16, vl + c * (kThreads * 16));
    }
  };

  RowStats st;
  f32x4 acc[D / 16];
#pragma unroll
  for (int n = 0; n < D / 16; ++n) acc[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (sp.tiles > 0) bring(0);
  for (int x = 0; x < sp.tiles; ++x) {
    // tile x lies in LDS (the barrier alone does not wait for a wave's loads to LDS), and nobody reads the other
    // buffer
    __builtin_amdgcn_s_waitcnt(kNoLoads);
    __syncthreads();
    if (x + 1 < sp.tiles) bring(x + 1);
    const int base = base_of(x), end = end_of(x);
    if (row0 >= n_rows || base > wave_hi || (base + kAttnTile <= wave_lo - window + 1 && base >= a.n_sink))
      continue;  // nothing for this wave's rows
    Keys now;
    now.load(lds.t.k[x & 1], lds.t.v[x & 1], lane);
    const bool all = base + kAttnTile <= end && base + kAttnTile - 1 <= wave_lo &&
                     (base > wave_hi - window || base + kAttnTile <= a.n_sink);
    bool bad = false;
    if (!all) bad = now.clean(base, end, lane);
    float s[8];
    now.scores(q, s);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] *= a.scale_log2;
      if (!all) {
        const int j = base + 8 * g + e;
        if (!((j < end) & (j <= pos) & ((pos - j < window) | (j < a.n_sink)))) s[e] = kNegInf;
      }
    }
    st.update(s, acc);
    Keys::product(s, now, nullptr, lane, acc);
    if (bad) add_odd<float, D>(a, vb, base, end, pos, window, i, g, s, acc);
  }
  __syncthreads();  // the rows go out through the tiles' place
  write_own<float, D>(a, p, row0, st, acc, lds.own + wave * own_floats<D>(),
                      [](int n, int lane16) { return Keys::channel(n, lane16); });
}

template <typename T, int D>
int run(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((attn_kernel<T, D>), dim3((unsigned)a.items, (unsigned)a.n_heads), dim3(64 * kAttnWaves), 0, s, a);
  return hipGetLastError();
}
template <int D>
int run_wide(const AttnArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((attn_wide_kernel<D>), dim3((unsigned)a.items * (unsigned)a.n_heads), dim3(64 * kAttnWaves), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int launch_attn(const AttnArgs& a, int dtype, int d, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (dtype == 0) return d == 128 ? run<bf16, 128>(a, s) : run<bf16, 64>(a, s);
  if (a.rows == kAttnWideRows) return d == 128 ? run_wide<128>(a, s) : run_wide<64>(a, s);
  return d == 128 ? run<float, 128>(a, s) : run<float, 64>(a, s);
}

}  // namespace twinkv

// K12a: which rows of an 8-bit cache an eviction keeps: of `len` rows in use the `budget` first in the order sinks
// and last rows (by row), then more weight, equal weights by row, NaN after every number: the order of the policy
// selection (scorer.hip), on lengths that differ from head to head and are known on the device only.
//
// One workgroup per problem.  The budget-th smallest key (0 for protected rows, otherwise the weight's bits,
// order-reversing) comes from an MSB-first radix select; then the rows before the cut, and the first ones equal to
// it, are listed in rising order, 8 a thread, one scan of both counts.  Problems of up to CAP rows keep their keys
// in LDS, longer ones read their weights again in every pass.
//
// A chain of short steps that wait for each other bounds it (barriers, the scan of a histogram), not its 4 bytes a row.
// So few threads for few rows, whose barriers and histograms (2^8 bins, 4 passes) cost less, and for more rows more
// threads and 2^11 bins (3 passes).  8 problems of 300 / 2000 / 4001 / 9000 / 30000 rows: 7 / 10 / 12 / 19 / 32 us; 4608 of
// 107 rows 19, with 256 threads 28; 4001 rows with 256 threads 16; 30000 whose keys are read again 50.
#include <hip/hip_runtime.h>

#include "../cache_ops.h"
#include "block_select.h"
#include "rows.h"
#include "seq_words.h"

namespace twinkv {
namespace {

constexpr int kRun = 8;  // rows a thread lists

template <int NT, int CAP>
__global__ __launch_bounds__(NT) void evict8_select_kernel(const Evict8Args a) {
  constexpr int NW = NT / 64, DBITS = NT >= 512 ? 11 : 8;
  __shared__ __attribute__((aligned(16))) uint32_t s_key[CAP > 0 ? CAP : 4];
  __shared__ int s_hist[2][1 << DBITS];
  __shared__ uint32_t s_bits[NW][2];
  __shared__ int s_wave[NW], s_pick[3];
  const int s = (int)blockIdx.x % a.n_seqs, h = (int)blockIdx.x / a.n_seqs;
  const int64_t q = (int64_t)h * a.n_seqs + s;
  const int w = s * kEvict8SeqWords;
  const int from0 = seq_word(a.seq, w), to0 = seq_word(a.seq, w + 1), budget = seq_word(a.seq, w + 2);
  const int cap = seq_word(a.seq, w + kEvict8SeqWords) - from0, cap_to = seq_word(a.seq, w + kEvict8SeqWords + 1) - to0;
  const int len = min(max(__builtin_amdgcn_readfirstlane(a.len[q]), 0), cap);
  const int keep = min(len, budget);  // (<= cap_to, checked on the host)
  const float* mass = a.mass + (int64_t)h * a.from.C + from0;
  int32_t* out = a.pos_out + (int64_t)h * a.to.C + to0;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // (n_recent may be anything up to 2^31 - 1)
  auto key_in = [&](int t, float f) { return t < a.n_sink || t >= len - (int64_t)a.n_recent ? 0u : score_key(f); };
  auto key_of = [&](int t) {
    if constexpr (CAP > 0) return s_key[t];
    else return key_in(t, mass[t]);
  };

  uint32_t cut_key = 0u;
  int take_eq = 0, eq_total = 0;
  const bool cut = keep > 0 && keep < len;
  if (cut) {
    for (int i = tid; i < (1 << DBITS); i += NT) s_hist[0][i] = 0;
    uint32_t kand = ~0u, kor = 0u;
    auto see = [&](int t, float f) {
      const uint32_t k = key_in(t, f);
      if constexpr (CAP > 0) s_key[t] = k;
      kand &= k;
      kor |= k;
    };
    constexpr int kLoads = CAP > 0 ? CAP / NT : 8;  // in flight together
    for (int t0 = 0; t0 < len; t0 += kLoads * NT) {
      float f[kLoads];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) f[u] = mass[min(t0 + u * NT + tid, len - 1)];
#pragma unroll
      for (int u = 0; u < kLoads; ++u)
        if (t0 + u * NT + tid < len) see(t0 + u * NT + tid, f[u]);
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
      kand &= __shfl_xor(kand, off);
      kor |= __shfl_xor(kor, off);
    }
    if (lane == 0) {
      s_bits[wave][0] = kand;
      s_bits[wave][1] = kor;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      kand &= s_bits[i][0];
      kor |= s_bits[i][1];
    }
    cut_key = block_select_below<NT, DBITS>(
        len, keep, len, kand, kor,
        [&](int t, uint32_t& key) {
          key = key_of(t);
          return true;
        },
        s_hist, s_pick, take_eq, eq_total);
  }

  int below = 0, equal = 0;  // before this round
  for (int t0 = 0; t0 < len && keep > 0; t0 += NT * kRun) {
    const int t = t0 + tid * kRun;
    unsigned less = 0, same = 0;
#pragma unroll
    for (int e = 0; e < kRun; ++e) {
      if (t + e >= len) continue;
      const uint32_t k = cut ? key_of(t + e) : 0u;
      less |= (!cut || k < cut_key ? 1u : 0u) << e;
      same |= (cut && k == cut_key ? 1u : 0u) << e;
    }
    int total;
    const int before = sel_exclusive_scan<NT>((int)(__popc(less) | (__popc(same) << 16)), s_wave, total);
    int lt = below + (before & 0xffff), eq = equal + (before >> 16);
#pragma unroll
    for (int e = 0; e < kRun; ++e) {
      const bool is_less = (less >> e) & 1u, is_same = (same >> e) & 1u;
      if (is_less || (is_same && eq < take_eq)) out[lt + min(eq, take_eq)] = t + e;
      lt += is_less;
      eq += is_same;
    }
    below += total & 0xffff;
    equal += total >> 16;
  }
  for (int r = keep + tid; r < cap_to; r += NT) out[r] = -1;
  if (tid == 0) a.len_out[q] = keep;
}

template <int NT, int CAP>
int run(const Evict8Args& a, hipStream_t s) {
  hipLaunchKernelGGL((evict8_select_kernel<NT, CAP>), dim3((unsigned)a.n_heads * (unsigned)a.n_seqs), dim3(NT), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int launch_evict8_select(const Evict8Args& a, void* stream) {
  hipStream_t s = (hipStream_t)stream;
  if (a.max_rows <= 512) return run<128, 512>(a, s);
  if (a.max_rows <= 2048) return run<256, 2048>(a, s);
  if (a.max_rows <= 4096) return run<512, 4096>(a, s);
  // (more problems than CUs: 512 of 8000 rows 25 us, with 1024 threads 34; fewer, with 512 threads in brackets: 8 of 4224
  // rows 12.5 (14.1), of 6000 13.2 (14.8), of 8192 14.8 (16.6); 64 of 5000 14.6 (16.6); 256 of 4224 16.0 (17.9), of 8192 20.5
  // (22.3))
  if (a.max_rows <= 8192 && a.n_heads * (int64_t)a.n_seqs > 256) return run<512, 8192>(a, s);
  if (a.max_rows <= 16384) return run<1024, 16384>(a, s);
  if (a.max_rows <= 32768) return run<1024, 32768>(a, s);
  return run<1024, 0>(a, s);
}

}  // namespace twinkv

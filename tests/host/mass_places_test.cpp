// The places of the accumulated weights' items (csrc/cache_ops.h, mass_place) for the plans that the host layer makes
// (csrc/cache8_ops.cpp), on the CPU: in the order that the kernel runs them (by rows) every split of every tile of keys
// occurs once, in the place among the parts where the join looks for it, and the splits of a tile hold the rows that see
// one of its keys.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "cache_ops.h"
#include "twinkv.h"

#define CHECK(x)                                                        \
  do {                                                                  \
    if (!(x)) {                                                         \
      std::fprintf(stderr, "%s:%d: %s\n", __FILE__, __LINE__, #x);      \
      std::exit(1);                                                     \
    }                                                                   \
  } while (0)

namespace {
using namespace twinkv;
std::vector<int64_t> g_cu_q, g_cu_k;
int64_t g_items = 0, g_kinds[3] = {0, 0, 0};
int32_t word(const SeqWords& t, int64_t i) { return t.far ? t.far[i] : t.near[i]; }
}  // namespace

namespace twinkv {
int launch_upload(const void* src, size_t bytes, void* dst, void*) {
  std::memcpy(dst, src, bytes);
  return 0;
}
int launch_mass(const MassArgs& a, int, int, void*) {
  int64_t before = 0;
  for (int s = 0; s < a.n_seqs; ++s) {
    const int64_t w = (int64_t)s * kMassSeqWords, nq = g_cu_q[s + 1] - g_cu_q[s], nk = g_cu_k[s + 1] - g_cu_k[s];
    const int first = word(a.seq, w + 2), items = word(a.seq, w + kMassSeqWords + 2) - first;
    const int splits = word(a.seq, w + 3), rows = word(a.seq, w + 4), full = word(a.seq, w + 5), shape = word(a.seq, w + 6);
    const int tiles = (int)((nk + a.keys - 1) / a.keys);
    CHECK(first == before);
    before += items;
    std::vector<char> seen((size_t)items, 0);
    std::vector<int> of_tile((size_t)tiles, 0);
    for (int i = 0; i < items; ++i) {
      const MassPlace p = mass_place<true>(i, splits, full, shape, tiles);
      CHECK(p.tile >= 0 && p.tile < tiles && p.split >= 0 && p.split < p.splits);
      CHECK(p.part >= 0 && p.part < items && !seen[(size_t)p.part]);
      seen[(size_t)p.part] = 1;
      const MassPlace j = mass_place<false>(p.part, splits, full, shape, tiles);
      CHECK(j.tile == p.tile && j.split == p.split && j.splits == p.splits && j.part == p.part);
      ++of_tile[(size_t)p.tile];
      if (p.split == 0) {
        const int64_t k0 = (int64_t)p.tile * a.keys, k1 = std::min(nk, k0 + a.keys), offset = nk - nq;
        const int64_t lo = std::max<int64_t>(k0 - offset, 0);
        const int64_t hi = k0 < a.n_sink ? nq : std::min(nq, k1 - 1 + a.window - offset);
        CHECK((int64_t)p.splits * rows >= std::max<int64_t>(hi - lo, 0) * a.group);
      }
    }
    for (int t = 0; t < tiles; ++t) CHECK(of_tile[(size_t)t] >= 1);
    g_items += items;
    if (full < tiles) ++g_kinds[shape >> kMassShapeBits];
  }
  CHECK(a.items == before);
  return 0;
}
int launch_mass_join(const MassArgs&, void*) { return 0; }
int launch_attn8(const AttnArgs&, int, int, void*) { return 0; }
int launch_attn_join(const AttnArgs&, int, int, void*) { return 0; }
int launch_cache4_positions(const Cache4Args&, void*) { return 0; }
int launch_cache8_gather(const Cache8Args&, int, int, void*) { return 0; }
int launch_cache8_append(const Cache8Args&, int, int, int, void*) { return 0; }
int launch_cache8_read(const Cache8Args&, int, int, void*) { return 0; }
int launch_evict8_select(const Evict8Args&, void*) { return 0; }
int launch_evict8_move(const Evict8Args&, int, void*) { return 0; }
}  // namespace twinkv

int main() {
  std::mt19937_64 g(3);
  auto upto = [&](int64_t n) { return (int64_t)(g() % (uint64_t)(n + 1)); };
  auto log_upto = [&](int64_t n) {
    const double x = (double)(g() % 1000003) / 1000003.0;
    return (int64_t)std::exp(x * std::log((double)n + 1.0)) - 1;
  };
  void* fake = reinterpret_cast<void*>(0x100000);
  float* fakef = static_cast<float*>(fake);
  std::vector<char> ws(1 << 20);
  for (int round = 0; round < 1500; ++round) {
    const int S = round % 100 == 0 ? (int)(100 + upto(200)) : (int)(1 + upto(6));
    const int H = (int)(1 + upto(40)), G = (int)(1 + upto(round % 3 ? 8 : 40)), d = upto(1) ? 128 : 64;
    const int64_t long_q = log_upto(20000), long_k = log_upto(100000);
    const bool prompts = upto(2) > 0;
    g_cu_q.assign(1, 0);
    g_cu_k.assign(1, 0);
    for (int s = 0; s < S; ++s) {
      const int64_t n = upto(long_k);
      g_cu_k.push_back(g_cu_k.back() + n);
      g_cu_q.push_back(g_cu_q.back() + (prompts ? n - upto(n) * (upto(3) == 0) : upto(long_q)));
    }
    const int64_t window = upto(2) ? INT64_MAX : log_upto(100000), sink = upto(2) ? 0 : log_upto(3000);
    // (the workspace's parts are not touched here: its words alone lie at its beginning)
    CHECK(twinkv_attention_mass(fake, fake, (int)upto(1), d, H, G, S, g_cu_q.data(), g_cu_k.data(), 128, 128 * 64, 128,
                                128 * 64, window, sink, 0.1f, fakef, nullptr, fakef, ws.data(), (int64_t)1 << 50,
                                nullptr) == TWINKV_OK);
  }
  CHECK(g_items > 100000 && g_kinds[kMassRuns] > 100 && g_kinds[kMassDrops] > 50 && g_kinds[kMassRest] > 20);
  std::printf("mass places ok: %lld items, %lld batches of runs, %lld of drops, %lld with sinks\n", (long long)g_items,
              (long long)g_kinds[0], (long long)g_kinds[1], (long long)g_kinds[2]);
  return 0;
}

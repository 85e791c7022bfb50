// More of the host layer of the 8-bit cache (csrc/cache8_ops.cpp) on the CPU, under sanitizers, with stand-ins for the
// launchers:
//  * whatever queries a batch holds beside those of cached rows, the kernel that an attention starts is one that gives
//    the weights that were asked for;
//  * which batches take the kernel of two row tiles a wave, where a test on the GPU counts on it.
#include <algorithm>
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
int g_rows = 0, g_attn = 0, g_mass = 0, g_parts = 0;
bool g_scores = false;
}  // namespace

namespace twinkv {
int launch_upload(const void* src, size_t bytes, void* dst, void*) {
  std::memcpy(dst, src, bytes);
  return 0;
}
int launch_mass(const MassArgs&, int, int, void*) {
  ++g_mass;
  return 0;
}
int launch_mass_join(const MassArgs&, void*) { return 0; }
int launch_attn8(const AttnArgs& a, int, int, void*) {
  ++g_attn;
  g_rows = a.rows;
  g_parts = a.parts;
  g_scores = a.mass_out != nullptr;
  return 0;
}
int launch_attn_join(const AttnArgs& a, int, int, void*) {
  CHECK(a.parts > 0 && a.rows == g_rows);
  return 0;
}
int launch_cache4_positions(const Cache4Args&, void*) { return 0; }
int launch_cache8_gather(const Cache8Args&, int, int, void*) { return 0; }
int launch_cache8_append(const Cache8Args&, int, int, int, void*) { return 0; }
int launch_cache8_read(const Cache8Args&, int, int, void*) { return 0; }
int launch_evict8_select(const Evict8Args&, void*) { return 0; }
int launch_evict8_move(const Evict8Args&, int, void*) { return 0; }
}  // namespace twinkv

namespace {
void* const fake = reinterpret_cast<void*>(0x100000);

// An attention of these queries and rows a sequence.
void attend(int dtype, int d, int H, int G, const std::vector<int64_t>& nq, const std::vector<int64_t>& rows, bool want) {
  std::vector<int64_t> cu_q(1, 0), cu_k(1, 0);
  for (int64_t n : nq) cu_q.push_back(cu_q.back() + n);
  for (int64_t n : rows) cu_k.push_back(cu_k.back() + n);
  const int S = (int)nq.size();
  const int64_t need = twinkv_cache8_attention_workspace_bytes(dtype, d, H, G, S, cu_q.data(), cu_k.data(), want);
  CHECK(need >= 0);
  void* ws = std::malloc((size_t)need + 1);  // (its pages are not touched but for the words)
  twinkv_cache8 c{d, H, S, cu_k.data(), fake, fake, fake, fake};
  g_attn = g_mass = g_rows = 0;
  CHECK(twinkv_cache8_attention(fake, dtype, G, cu_q.data(), 128, 128 * 64, &c, static_cast<int32_t*>(fake), 0.1f, fake, 128,
                                128 * 64, nullptr, nullptr, want ? static_cast<float*>(fake) : nullptr, ws, need,
                                nullptr) == TWINKV_OK);
  std::free(ws);
  if (want && cu_k.back() > 0) {
    // from scores that the one kernel for them keeps, or afresh: one of the two
    CHECK(g_scores != (g_mass > 0));
    CHECK(!g_scores || g_rows == kAttnRows);
  }
}
}  // namespace

int main() {
  // few rows a problem beside an empty sequence with many queries, with enough work for two row tiles a wave
  for (int d : {64, 128}) {
    attend(TWINKV_BF16, d, 16, 8, {1, 40}, {131072, 0}, true);
    CHECK(g_scores && g_parts > 0);
    std::vector<int64_t> one(64, 1), rows(64, 4096);
    one.push_back(300), rows.push_back(0);
    attend(TWINKV_BF16, d, 8, 4, one, rows, true);
    CHECK(g_scores);
    one.back() = 512;
    attend(TWINKV_BF16, d, 8, 8, one, rows, true);
    CHECK(g_scores);
    attend(TWINKV_BF16, d, 8, 8, one, rows, false);  // no weights: as before
    CHECK(g_rows == kAttnPairRows);
  }
  std::mt19937_64 g(5);
  int pairs = 0, scores = 0;
  for (int round = 0; round < 2000; ++round) {
    const int S = 1 + (int)(g() % 80), H = 1 + (int)(g() % 32), G = 1 + (int)(g() % 16);
    std::vector<int64_t> nq, rows;
    const bool few = g() % 2 == 0;
    for (int s = 0; s < S; ++s) {
      const bool empty = g() % 4 == 0;
      rows.push_back(empty ? 0 : 32 * (1 + (int64_t)(g() % 400)));
      nq.push_back(few && !empty ? 1 + (int64_t)(g() % (uint64_t)std::max(1, 16 / G)) : (int64_t)(g() % 600));
    }
    const bool want = g() % 4 != 0;
    attend((int)(g() % 2), g() % 2 ? 64 : 128, H, G, nq, rows, want);
    pairs += g_rows == kAttnPairRows;
    scores += g_scores;
  }
  CHECK(pairs > 100 && scores > 100);
  // 28 rows a problem over 128k rows, and 17 to 40 over 64 sequences: two row tiles a wave, the weights afresh
  for (int d : {64, 128}) {
    attend(TWINKV_BF16, d, 8, 4, {7}, {131072}, true);
    CHECK(g_rows == kAttnPairRows && g_mass == 1 && g_parts > 0);
    std::vector<int64_t> nq, rows;
    for (int s = 0; s < 64; ++s) nq.push_back(17 + s % 24), rows.push_back(s == 5 ? 32 : 4096);
    attend(TWINKV_BF16, d, 4, 1, nq, rows, true);
    CHECK(g_rows == kAttnPairRows && g_mass == 1);
  }
  std::printf("cache8 plans ok: %d of two row tiles, %d with scores\n", pairs, scores);
  return 0;
}

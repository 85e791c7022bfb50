// The host layer of the accumulated attention weights and the 8-bit cache (csrc/cache8_ops.cpp) on the CPU, under
// sanitizers: stand-ins for the launchers read a call's per-sequence words as a kernel would and check that
//  * the weights' items are the splits of every key tile, each once, and cover the rows that see one of its keys
//    (written out again here, from the definition of the mask);
//  * the attention's splits cover the cache, and the scores of an item fit the LDS that it is given;
//  * the lists of blocks cover every row that a call may write, and an eviction's words are the two caches';
//  * parts, scores, words and their places lie inside the workspace the query asks for.
// "Device" buffers are host memory of exactly the size asked for.
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

int64_t g_mass = 0, g_joins = 0, g_far = 0, g_runs = 0, g_drops = 0, g_rest = 0, g_scores = 0, g_fresh = 0, g_split_scores = 0;
volatile unsigned char g_sink = 0;
std::vector<int64_t> g_cu_q, g_cu_k, g_cu_to, g_budget;
bool g_cached = false, g_want = false;
int g_d = 0, g_score_rows = 0;

int32_t word(const SeqWords& t, int64_t i) { return t.far ? t.far[i] : t.near[i]; }

void touch(const void* p, int64_t bytes) {
  if (bytes <= 0) return;
  unsigned char* c = static_cast<unsigned char*>(const_cast<void*>(p));
  c[0] = 1;
  c[bytes - 1] = 1;
  g_sink = g_sink ^ c[bytes / 2];
}

// Rows (query * group + head) that see a key of [k0, k1): first and one past the last.
void rows_seeing(const MassArgs& a, int64_t nq, int64_t nk, int64_t k0, int64_t k1, int64_t& lo, int64_t& hi) {
  lo = hi = 0;
  const int64_t offset = nk - nq;
  const int64_t first = std::max<int64_t>(k0 - offset, 0);
  const int64_t last = k0 < a.n_sink ? nq : std::min(nq, k1 - 1 + a.window - offset);
  if (first >= nq || last <= first) return;
  lo = first * a.group;
  hi = last * a.group;
}
}  // namespace

namespace twinkv {
int launch_upload(const void* src, size_t bytes, void* dst, void*) {
  std::memcpy(dst, src, bytes);
  return 0;
}
int launch_mass(const MassArgs& a, int dtype, int, void*) {
  ++g_mass;
  if (a.seq.far) ++g_far;
  CHECK(a.keys == (dtype == TWINKV_F32 ? kMassKeys : 2 * kMassKeys));
  CHECK((a.k == nullptr) == g_cached);
  CHECK((int64_t)a.items * a.n_heads * 256 <= (int64_t)UINT32_MAX);
  int64_t item = 0;
  bool split_any = false;
  for (int s = 0; s < a.n_seqs; ++s) {
    const int64_t w = (int64_t)s * kMassSeqWords;
    const int64_t nq = g_cu_q[s + 1] - g_cu_q[s], nk = g_cu_k[s + 1] - g_cu_k[s], tiles = (nk + a.keys - 1) / a.keys;
    CHECK(word(a.seq, w) == g_cu_q[s] && word(a.seq, w + 1) == g_cu_k[s] && word(a.seq, w + 2) == item);
    const int64_t most = word(a.seq, w + 3), rows = word(a.seq, w + 4), full = word(a.seq, w + 5);
    const int shape = word(a.seq, w + 6), kind = shape >> kMassShapeBits, by = shape & ((1 << kMassShapeBits) - 1);
    CHECK(most >= 1 && rows >= 1 && rows % kMassRowTile == 0 && by >= 1);
    split_any |= most > 1;
    if (full < tiles) ++(kind == kMassRuns ? g_runs : kind == kMassDrops ? g_drops : g_rest);
    const int64_t next = word(a.seq, w + kMassSeqWords + 2);
    // as the kernel takes an item apart
    int64_t tile = 0, split = 0;
    for (int64_t i = 0; item + i < next; ++i) {
      int64_t splits = most, tile0 = 0, left = i;
      if (left >= full * splits) {
        left -= full * splits;
        tile0 = full;
        if (kind == kMassRest) {
          splits = by;
        } else {
          const int64_t run = kind == kMassRuns ? by : 1, drop = kind == kMassRuns ? 1 : by;
          while (splits > drop && left >= run * splits) {
            left -= run * splits;
            tile0 += run;
            splits -= drop;
          }
        }
      }
      CHECK(tile0 + left / splits == tile && left % splits == split);
      if (split == 0) {
        int64_t lo = 0, hi = nq * a.group;
        if (!g_cached) rows_seeing(a, nq, nk, tile * a.keys, std::min(nk, (tile + 1) * a.keys), lo, hi);
        CHECK(splits * rows >= hi - lo);
      }
      if (++split == splits) split = 0, ++tile;
    }
    CHECK(split == 0 && tile == tiles);
    item = next;
  }
  CHECK(a.items == item && (a.part != nullptr) == split_any);
  if (split_any) touch(a.part, item * a.n_heads * a.keys * 4);
  if (g_cached) touch(a.lse, 4 * a.Tq * a.n_heads * a.group);
  return 0;
}
int launch_mass_join(const MassArgs& a, void*) {
  CHECK(a.part != nullptr);
  ++g_joins;
  return 0;
}
int launch_attn8(const AttnArgs& a, int, int d, void*) {
  CHECK(a.rows == kAttnRows || a.rows == kAttnPairRows);
  int64_t item = 0, part = 0, lds = 0;
  for (int s = 0; s < a.n_seqs; ++s) {
    const int64_t w = (int64_t)s * kAttnSeqWords;
    const int64_t nq = g_cu_q[s + 1] - g_cu_q[s], nk = g_cu_k[s + 1] - g_cu_k[s];
    CHECK(word(a.seq, w) == g_cu_q[s] && word(a.seq, w + 1) == g_cu_k[s] && word(a.seq, w + 2) == item);
    const int64_t splits = word(a.seq, w + 3), tiles = word(a.seq, w + 4), row_tiles = (nq * a.group + a.rows - 1) / a.rows;
    CHECK(splits >= 1 && tiles >= 1 && splits * tiles * kAttnTile >= nk);
    CHECK(splits == 1 || word(a.seq, w + 5) == part);
    if (a.mass_out != nullptr && nk > 0) {
      CHECK(row_tiles == 1 && nq * a.group <= a.score_rows);
      lds = std::max(lds, nq * a.group * std::min(nk, tiles * kAttnTile));
      if (splits > 1) ++g_split_scores;
    }
    item += row_tiles * splits;
    if (splits > 1) part += row_tiles * splits;
  }
  CHECK(a.items == item && a.parts == part);
  CHECK(lds <= a.score_lds && 4 * a.score_lds <= kAttnMostLds);
  touch(a.part_o, part * a.n_heads * a.rows * d * 4);
  touch(a.part_ml, part * a.n_heads * a.rows * 8);
  if (a.mass_out != nullptr) {
    ++g_scores;
    CHECK(g_want && a.rows == kAttnRows && a.score_rows >= 1 && a.score_rows <= kAttnRows);
    if (part > 0) touch(a.score, 4 * (int64_t)a.n_heads * a.score_rows * g_cu_k.back());
    if (part > 0) CHECK(reinterpret_cast<uintptr_t>(a.score) % 128 == 0);
  } else if (g_want && g_cu_k.back() > 0) {
    ++g_fresh;
    touch(a.lse, 4 * a.Tq * a.n_heads * a.group);
  }
  return 0;
}
int launch_attn_join(const AttnArgs& a, int, int, void*) {
  CHECK(a.parts > 0);
  return 0;
}
static void check_blocks(const Cache8Args& a, bool aligned) {
  int64_t at = 0;
  for (int s = 0; s <= a.n_seqs; ++s) {
    CHECK(word(a.seq, s * kCacheSeqWords) == g_cu_q[s] && word(a.seq, s * kCacheSeqWords + 1) == g_cu_k[s]);
    CHECK(word(a.seq, s * kCacheSeqWords + 2) == at);
    if (s == a.n_seqs) break;
    const int64_t n = aligned ? g_cu_k[s + 1] - g_cu_k[s] : g_cu_q[s + 1] - g_cu_q[s];
    const int64_t blocks = word(a.seq, (s + 1) * kCacheSeqWords + 2) - at;
    for (int first = 0; first < (aligned ? 1 : kCache8Block); ++first)  // rows first .. first + n - 1
      CHECK(n == 0 || (first + n - 1) / kCache8Block < blocks);
    at += blocks;
  }
  CHECK(a.n_blocks == at);
  if (a.seq.far) ++g_far;
}
int launch_cache4_positions(const Cache4Args&, void*) { return 0; }
int launch_cache8_gather(const Cache8Args& a, int, int, void*) {
  check_blocks(a, true);
  return 0;
}
int launch_cache8_append(const Cache8Args& a, int most, int, int, void*) {
  for (int s = 0; s < a.n_seqs; ++s) CHECK(g_cu_q[s + 1] - g_cu_q[s] <= most);
  check_blocks(a, false);
  return 0;
}
int launch_cache8_read(const Cache8Args& a, int, int, void*) {
  check_blocks(a, false);
  return 0;
}
static void check_evict(const Evict8Args& a) {
  int64_t longest = 0;
  for (int s = 0; s <= a.n_seqs; ++s) {
    const int64_t w = (int64_t)s * kEvict8SeqWords;
    CHECK(word(a.seq, w) == g_cu_k[s] && word(a.seq, w + 1) == g_cu_to[s] && word(a.seq, w + 3) == g_cu_to[s] / kCache8Block);
    if (s == a.n_seqs) break;
    CHECK(word(a.seq, w + 2) == g_budget[s]);
    longest = std::max(longest, g_cu_k[s + 1] - g_cu_k[s]);
  }
  CHECK(a.n_blocks == g_cu_to.back() / kCache8Block && a.max_rows == longest);
  if (a.seq.far) ++g_far;
}
int launch_evict8_select(const Evict8Args& a, void*) {
  check_evict(a);
  return 0;
}
int launch_evict8_move(const Evict8Args& a, int, void*) {
  check_evict(a);
  return 0;
}
}  // namespace twinkv

int main() {
  std::mt19937_64 g(11);
  auto upto = [&](int64_t n) { return (int64_t)(g() % (uint64_t)(n + 1)); };
  auto log_upto = [&](int64_t n) {
    const double x = (double)(g() % 1000003) / 1000003.0;
    return (int64_t)std::exp(x * std::log((double)n + 1.0)) - 1;
  };
  void* fake = reinterpret_cast<void*>(0x100000);
  float* fakef = static_cast<float*>(fake);
  for (int round = 0; round < 1500; ++round) {
    const int S = round % 50 == 0 ? (int)(1 + upto(400)) : (int)(1 + upto(8));
    const int H = (int)(1 + upto(15)), G = (int)(1 + upto(round % 3 ? 8 : 40)), d = upto(1) ? 128 : 64;
    const int dtype = (int)upto(1);
    g_cu_q.assign(1, 0);
    g_cu_k.assign(1, 0);
    const int64_t long_q = log_upto(20000), long_k = log_upto(200000);
    const bool prompts = upto(2) == 0, steps = !prompts && upto(1) == 0;
    for (int s = 0; s < S; ++s) {
      const int64_t n = upto(long_k);
      g_cu_k.push_back(g_cu_k.back() + n);
      g_cu_q.push_back(g_cu_q.back() + (prompts ? n : steps ? 1 + upto(std::max(0, 16 / G - 1)) : upto(3) * upto(long_q) / 3));
    }
    const int64_t window = upto(3) ? log_upto(300000) : INT64_MAX, sink = upto(1) ? 0 : log_upto(3000);
    g_cached = false;
    int64_t need = twinkv_mass_workspace_bytes(dtype, d, H, G, S, g_cu_q.data(), g_cu_k.data(), window, sink);
    CHECK(need >= 0 && need < (int64_t)1 << 31);
    {
      std::vector<char> ws((size_t)std::max<int64_t>(need, 1));
      CHECK(twinkv_attention_mass(fake, fake, dtype, d, H, G, S, g_cu_q.data(), g_cu_k.data(), 128, 128 * 64, 128, 128 * 64,
                                  window, sink, 0.1f, fakef, nullptr, fakef, need > 0 ? ws.data() : nullptr, need,
                                  nullptr) == TWINKV_OK);
    }
    // the cache's rows: multiples of 32
    for (auto& x : g_cu_k) x = x / 32 * 32;
    g_cached = true;
    twinkv_cache8 c{d, H, S, g_cu_k.data(), fake, fake, fake, fake};
    int32_t* len = static_cast<int32_t*>(fake);
    g_want = upto(2) > 0;
    need = twinkv_cache8_attention_workspace_bytes(dtype, d, H, G, S, g_cu_q.data(), g_cu_k.data(), g_want);
    CHECK(need >= 0);
    if (need < (int64_t)1 << 31) {
      std::vector<char> ws((size_t)std::max<int64_t>(need, 1));
      CHECK(twinkv_cache8_attention(fake, dtype, G, g_cu_q.data(), 128, 128 * 64, &c, len, 0.1f, fake, 128, 128 * 64, nullptr,
                                    nullptr, g_want ? fakef : nullptr, need > 0 ? ws.data() : nullptr, need,
                                    nullptr) == TWINKV_OK);
    }
    const int64_t nc = twinkv_cache8_workspace_bytes(S);
    std::vector<char> wsc((size_t)std::max<int64_t>(nc, 1));
    void* w = nc > 0 ? wsc.data() : nullptr;
    CHECK(twinkv_cache8_append(fake, fake, dtype, g_cu_q.data(), 128, 128, 128, 128, &c, len, len, len, w, nc, nullptr) ==
          TWINKV_OK);
    CHECK(twinkv_cache8_read(&c, len, nullptr, dtype, g_cu_q.data(), fake, fake, w, nc, nullptr) == TWINKV_OK);
    CHECK(twinkv_cache8_compact(fake, fake, dtype, g_cu_q.data(), 128, 128, 128, 128, static_cast<uint8_t*>(fake), &c, fakef,
                                len, fakef, len, len, w, nc, nullptr) == TWINKV_OK);
    g_cu_to.assign(1, 0);
    g_budget.clear();
    for (int s = 0; s < S; ++s) {
      const int64_t rows = 32 * upto(200);
      g_cu_to.push_back(g_cu_to.back() + rows);
      g_budget.push_back(upto(rows));
    }
    char* there = static_cast<char*>(fake) + 65536;
    twinkv_cache8 to{d, H, S, g_cu_to.data(), there, there + 16, there + 32, there + 48};
    CHECK(twinkv_cache8_evict(&c, len, fakef, nullptr, g_budget.data(), (int)upto(10), INT32_MAX, &to, len, fakef, len, w, nc,
                              nullptr) == TWINKV_OK);
  }
  CHECK(g_mass > 1200 && g_joins > 200 && g_far > 40 && g_runs > 40 && g_drops > 20 && g_rest > 8);
  CHECK(g_scores > 80 && g_fresh > 80 && g_split_scores > 40);
  std::printf("cache8 ops ok: %lld weights, %lld joined, %lld runs, %lld with scores\n", (long long)g_mass,
              (long long)g_joins, (long long)g_runs, (long long)g_scores);
  return 0;
}

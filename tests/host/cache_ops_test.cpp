// The host layer of the operators around the cache (csrc/cache_ops.cpp) on the CPU, under sanitizers: stand-ins
// for the launchers read a call's per-sequence words as a kernel would and check that
//  * every item of an attention belongs to one row tile and split, and that a tile's splits cover all the key
//    tiles that its rows see (the spans written out again here, from the definition of the mask);
//  * parts, words and their places lie inside the workspace the query asks for;
//  * the block lists of the 4-bit cache cover every row that a call may write.
// "Device" buffers are host memory of exactly the size asked for.
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
int64_t g_attn = 0, g_joins = 0, g_far = 0, g_splits = 0, g_big = 0, g_wide = 0;
volatile unsigned char g_sink = 0;
std::vector<int64_t> g_cu_q, g_cu_k;

int32_t word(const twinkv::SeqWords& t, int64_t i) { return t.far ? t.far[i] : t.near[i]; }

void touch(void* p, int64_t bytes) {
  if (bytes <= 0) return;
  unsigned char* c = static_cast<unsigned char*>(p);
  c[0] = 1;
  c[bytes - 1] = 1;
  g_sink = g_sink ^ c[bytes / 2];
}

// Key tiles that the rows [row0, row0 + rows) see in the kernels' numbering: sink tiles, then window tiles.
int64_t tiles_of(const twinkv::AttnArgs& a, int64_t nq, int64_t nk, int64_t row0, int64_t rows, int64_t keys) {
  const int64_t last = std::min(row0 + rows, nq * a.group) - 1;
  const int64_t pos_lo = nk - nq + row0 / a.group, pos_hi = nk - nq + last / a.group;
  const int64_t end = std::max<int64_t>(pos_hi + 1, 0), sinks = std::min<int64_t>(a.n_sink, end);
  int64_t lo = std::min(std::max<int64_t>(pos_lo - a.window + 1, 0), end), sink_tiles = (sinks + keys - 1) / keys;
  if (lo <= sink_tiles * keys) {
    if (sinks > 0) lo = 0;
    sink_tiles = 0;
  }
  return sink_tiles + (end - lo + keys - 1) / keys;
}

void check_items(const twinkv::AttnArgs& a, int d, int64_t keys, bool cached) {
  ++g_attn;
  if (a.seq.far) ++g_far;
  int64_t item = 0, part = 0;
  for (int s = 0; s < a.n_seqs; ++s) {
    const int64_t w = (int64_t)s * twinkv::kAttnSeqWords;
    const int64_t nq = g_cu_q[s + 1] - g_cu_q[s], nk = g_cu_k[s + 1] - g_cu_k[s];
    CHECK(word(a.seq, w) == g_cu_q[s] && word(a.seq, w + 1) == g_cu_k[s]);
    CHECK(word(a.seq, w + 2) == item);
    const int64_t splits = word(a.seq, w + 3), tiles = word(a.seq, w + 4);
    CHECK(splits >= 1 && tiles >= 1);
    CHECK(splits == 1 || word(a.seq, w + 5) == part);
    const int64_t row_tiles = (nq * a.group + a.rows - 1) / a.rows;
    const int64_t own = a.rows == twinkv::kAttnWideRows ? twinkv::kAttnRows : a.rows;  // rows of a wave's tile
    for (int64_t r = 0; r * own < nq * a.group; r += std::max<int64_t>(1, row_tiles / 7)) {
      const int64_t need = cached ? (nk + keys - 1) / keys : tiles_of(a, nq, nk, r * own, own, keys);
      CHECK(splits * tiles >= need);
      CHECK((splits * tiles + 1) * keys < INT32_MAX);
    }
    item += row_tiles * splits;
    if (splits > 1) part += row_tiles * splits, ++g_splits;
  }
  const int64_t w = (int64_t)a.n_seqs * twinkv::kAttnSeqWords;
  CHECK(word(a.seq, w) == g_cu_q.back() && word(a.seq, w + 1) == g_cu_k.back() && word(a.seq, w + 2) == item);
  CHECK(a.items == item && a.parts == part);
  const int64_t rows = part * a.n_heads * a.rows;
  touch(a.part_o, rows * d * 4);
  touch(a.part_ml, rows * 8);
}
}  // namespace

namespace twinkv {
int launch_upload(const void* src, size_t bytes, void* dst, void*) {
  std::memcpy(dst, src, bytes);
  return 0;
}
int launch_norm_rope(const NormRopeArgs& a, int, int, void*) {
  CHECK(a.per_unit >= 1 && a.q.chunks * a.per_unit >= a.q.heads && a.k.chunks * a.per_unit >= a.k.heads);
  CHECK(a.q.heads == 0 || (a.q.chunks - 1) * a.per_unit < a.q.heads);
  return 0;
}
int launch_attn(const AttnArgs& a, int dtype, int d, void*) {
  CHECK(a.rows == kAttnRows || (dtype == TWINKV_F32 && a.rows == kAttnWideRows && a.parts == 0));
  if (a.rows == kAttnWideRows) ++g_wide;
  check_items(a, d, kAttnTile, false);
  return 0;
}
int launch_attn_rows(const AttnArgs& a, int d, void*) {
  CHECK(a.rows == kAttnBigRows);
  ++g_big;
  check_items(a, d, kAttnBigTile, false);
  return 0;
}
int launch_attn4(const AttnArgs& a, int, int d, void*) {
  CHECK(a.rows == kAttnRows || a.rows == kAttnPairRows);
  check_items(a, d, kAttnTile, true);
  return 0;
}
int launch_attn_join(const AttnArgs& a, int, int, void*) {
  CHECK(a.parts > 0);
  ++g_joins;
  return 0;
}
static void check_blocks(const Cache4Args& a, bool aligned) {
  int64_t at = 0;
  for (int s = 0; s <= a.n_seqs; ++s) {
    CHECK(word(a.seq, s * kCacheSeqWords) == g_cu_q[s] && word(a.seq, s * kCacheSeqWords + 1) == g_cu_k[s]);
    CHECK(word(a.seq, s * kCacheSeqWords + 2) == at);
    if (s == a.n_seqs) break;
    const int64_t n = aligned ? g_cu_k[s + 1] - g_cu_k[s] : g_cu_q[s + 1] - g_cu_q[s];
    const int64_t blocks = word(a.seq, (s + 1) * kCacheSeqWords + 2) - at;
    // rows first .. first + n - 1, whatever first is
    for (int first = 0; first < (aligned ? 1 : kCacheBlock); ++first)
      CHECK(n == 0 || (first + n - 1) / kCacheBlock < blocks);
    at += blocks;
  }
  CHECK(a.n_blocks == at);
  if (a.seq.far) ++g_far;
}
int launch_cache4_positions(const Cache4Args&, void*) { return 0; }
int launch_cache4_gather(const Cache4Args& a, int, int, void*) {
  check_blocks(a, true);
  return 0;
}
int launch_cache4_append(const Cache4Args& a, int most, int, int, void*) {
  for (int s = 0; s < a.n_seqs; ++s) CHECK(g_cu_q[s + 1] - g_cu_q[s] <= most);
  check_blocks(a, false);
  return 0;
}
int launch_cache4_read(const Cache4Args& a, int, int, void*) {
  check_blocks(a, false);
  return 0;
}
}  // namespace twinkv

int main() {
  std::mt19937_64 g(7);
  auto upto = [&](int64_t n) { return (int64_t)(g() % (uint64_t)(n + 1)); };
  auto log_upto = [&](int64_t n) {
    const double x = (double)(g() % 1000003) / 1000003.0;
    return (int64_t)std::exp(x * std::log((double)n + 1.0)) - 1;
  };
  void* fake = reinterpret_cast<void*>(0x100000);
  for (int round = 0; round < 4000; ++round) {
    const int S = round % 50 == 0 ? (int)(1 + upto(400)) : (int)(1 + upto(8));
    const int H = (int)(1 + upto(15)), G = (int)(1 + upto(round % 3 ? 8 : 40)), d = upto(1) ? 128 : 64;
    const int dtype = (int)upto(1);
    g_cu_q.assign(1, 0);
    g_cu_k.assign(1, 0);
    const int64_t long_q = log_upto(4000), long_k = log_upto(round % 99 == 0 && S < 20 ? 40000000 : 200000);
    for (int s = 0; s < S; ++s) {
      g_cu_q.push_back(g_cu_q.back() + upto(3) * upto(long_q) / 3);
      g_cu_k.push_back(g_cu_k.back() + upto(long_k));
    }
    const int64_t window = upto(3) ? log_upto(300000) : INT64_MAX, sink = upto(1) ? 0 : log_upto(3000);
    const int64_t need = twinkv_attention_workspace_bytes(dtype, d, H, G, S, g_cu_q.data(), g_cu_k.data(), window, sink);
    if (need < 0 || need >= (int64_t)1 << 30) std::fprintf(stderr, "need %lld\n", (long long)need);
    CHECK(need >= 0 && need < (int64_t)1 << 30);
    std::vector<char> ws((size_t)std::max<int64_t>(need, 1));
    void* w = need > 0 ? ws.data() : nullptr;
    CHECK(twinkv_sink_attention(fake, fake, fake, dtype, d, H, G, S, g_cu_q.data(), g_cu_k.data(), 128, 128 * 64, 128,
                                128 * 64, 128, 128 * 64, window, sink, 0.1f, fake, 128, 128 * 64, nullptr, w, need,
                                nullptr) == TWINKV_OK);
    // the cache's rows: multiples of 32
    for (auto& x : g_cu_k) x = x / 32 * 32;
    twinkv_cache4 c{d, H, S, g_cu_k.data(), fake, fake, fake, fake};
    const int64_t need4 = twinkv_attention_workspace_bytes(dtype, d, H, G, S, g_cu_q.data(), g_cu_k.data(), INT64_MAX, 0);
    std::vector<char> ws4((size_t)std::max<int64_t>(need4, 1));
    w = need4 > 0 ? ws4.data() : nullptr;
    int32_t* len = static_cast<int32_t*>(fake);
    CHECK(twinkv_cache4_attention(fake, dtype, G, g_cu_q.data(), 128, 128 * 64, &c, len, 0.1f, fake, 128, 128 * 64, nullptr,
                                  w, need4, nullptr) == TWINKV_OK);
    const int64_t nc = twinkv_cache4_workspace_bytes(S);
    std::vector<char> wsc((size_t)std::max<int64_t>(nc, 1));
    w = nc > 0 ? wsc.data() : nullptr;
    CHECK(twinkv_cache4_append(fake, fake, dtype, g_cu_q.data(), 128, 128, 128, 128, &c, len, len, len, w, nc, nullptr) ==
          TWINKV_OK);
    CHECK(twinkv_cache4_read(&c, len, nullptr, dtype, g_cu_q.data(), fake, fake, w, nc, nullptr) == TWINKV_OK);
    CHECK(twinkv_cache4_compact(fake, fake, dtype, g_cu_q.data(), 128, 128, 128, 128, static_cast<uint8_t*>(fake), &c, len,
                                len, len, w, nc, nullptr) == TWINKV_OK);
    CHECK(twinkv_qk_norm_rope(fake, fake, dtype, d, H * G, H, g_cu_q.back(), 128, 128 * 64, 128, 128 * 64, nullptr, nullptr,
                              1e-6f, nullptr, 0, nullptr, fake, 128, 128 * 64, fake, 128, 128 * 64, nullptr) == TWINKV_OK);
  }
  // strides that the kernel for many rows cannot take go to the other
  g_cu_q = {0, 5000};
  g_cu_k = {0, 5000};
  const int64_t before = g_big;
  const int64_t need = twinkv_attention_workspace_bytes(0, 128, 2, 4, 1, g_cu_q.data(), g_cu_k.data(), 5000, 0);
  std::vector<char> ws((size_t)std::max<int64_t>(need, 1));
  CHECK(twinkv_sink_attention(fake, fake, fake, 0, 128, 2, 4, 1, g_cu_q.data(), g_cu_k.data(), 128, 1024, 128, 1 << 25, 128,
                              1024, 5000, 0, 0.1f, fake, 128, 1024, nullptr, ws.data(), need, nullptr) == TWINKV_OK);
  CHECK(g_big == before);
  CHECK(g_attn > 4000 && g_joins > 100 && g_far > 50 && g_splits > 100 && g_big > 100 && g_wide > 10);
  std::printf("cache ops ok: %lld attentions, %lld for many rows, %lld split sequences\n", (long long)g_attn,
              (long long)g_big, (long long)g_splits);
  return 0;
}

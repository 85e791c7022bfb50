// More of the host layer of the operators around the cache (csrc/cache_ops.cpp) on the CPU, under sanitizers, with
// stand-ins for the launchers: which outputs are refused because two of their rows share a place, and which kernel and
// splits the attention chooses where a test or a bound counts on them.
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
// The last attention: rows of an item, and each sequence's splits.
int g_rows = 0;
std::vector<int64_t> g_splits;
int planned(const twinkv::AttnArgs& a) {
  g_rows = a.rows;
  g_splits.clear();
  for (int s = 0; s < a.n_seqs; ++s) {
    const int64_t w = (int64_t)s * twinkv::kAttnSeqWords + 3;
    g_splits.push_back(a.seq.far ? a.seq.far[w] : a.seq.near[w]);
  }
  return 0;
}
}  // namespace

namespace twinkv {
int launch_upload(const void* src, size_t bytes, void* dst, void*) {
  std::memcpy(dst, src, bytes);
  return 0;
}
int launch_norm_rope(const NormRopeArgs&, int, int, void*) { return 0; }
int launch_attn(const AttnArgs& a, int, int, void*) { return planned(a); }
int launch_attn_rows(const AttnArgs& a, int, void*) { return planned(a); }
int launch_attn4(const AttnArgs& a, int, int, void*) { return planned(a); }
int launch_attn_join(const AttnArgs&, int, int, void*) { return 0; }
int launch_cache4_positions(const Cache4Args&, void*) { return 0; }
int launch_cache4_gather(const Cache4Args&, int, int, void*) { return 0; }
int launch_cache4_append(const Cache4Args&, int, int, int, void*) { return 0; }
int launch_cache4_read(const Cache4Args&, int, int, void*) { return 0; }
}  // namespace twinkv

namespace {
void* const fake = reinterpret_cast<void*>(0x100000);

bool overlap(int64_t heads, int64_t T, int64_t hs, int64_t ts, int64_t d) {
  std::vector<int64_t> at;
  for (int64_t h = 0; h < heads; ++h)
    for (int64_t t = 0; t < T; ++t) at.push_back(h * hs + t * ts);
  std::sort(at.begin(), at.end());
  for (size_t i = 1; i < at.size(); ++i)
    if (at[i] - at[i - 1] < d) return true;
  return false;
}

// What each call with an output says to rows at these strides (8 elements are 16 bytes or more of both types).
void check_output(int64_t heads, int64_t T, int64_t hs, int64_t ts, int d, int dtype, int code) {
  CHECK(twinkv_qk_norm_rope(fake, fake, dtype, d, (int)heads, 1, T, d * T, d, d * T, d, nullptr, nullptr, 1e-6f, nullptr, 0,
                            nullptr, fake, hs, ts, fake, d * T, d, nullptr) == code);
  CHECK(twinkv_qk_norm_rope(nullptr, fake, dtype, d, 0, (int)heads, T, 0, 0, d * T, d, nullptr, nullptr, 1e-6f, nullptr, 0,
                            nullptr, nullptr, 0, 0, fake, hs, ts, nullptr) == code);
  const int64_t cq[2] = {0, T}, ck[2] = {0, 64};
  CHECK(twinkv_sink_attention(fake, fake, fake, dtype, d, 1, (int)heads, 1, cq, ck, d * T, d, 64 * d, d, 64 * d, d, 64, 0,
                              0.1f, fake, hs, ts, nullptr, nullptr, 0, nullptr) == code);
  const twinkv_cache4 c{d, (int)heads, 1, ck, fake, fake, fake, fake};
  CHECK(twinkv_cache4_attention(fake, dtype, 1, cq, d * T, d, &c, static_cast<int32_t*>(fake), 0.1f, fake, hs, ts, nullptr,
                                nullptr, 0, nullptr) == code);
}

void outputs() {
  std::mt19937_64 g(11);
  auto from = [&](int64_t a, int64_t b) { return a + (int64_t)(g() % (uint64_t)(b - a + 1)); };
  int64_t refused = 0, odd = 0;
  for (int round = 0; round < 20000; ++round) {
    const int d = round % 2 ? 128 : 64;
    const int64_t heads = from(1, 9), T = from(1, 40);
    const int64_t ts = d + 8 * from(0, round % 3 ? 2 : 60);
    // heads apart by a few tokens and a bit, or by about all of them
    const int64_t hs = from(0, 1) ? ts * from(1, 6) + 8 * from(0, ts / 8) : ts * T + 8 * from(-ts / 8, 4);
    if (hs < ts) continue;
    const bool meet = overlap(heads, T, hs, ts, d);
    refused += meet;
    odd += !meet && heads > 1 && T > 1 && hs < (T - 1) * ts + d;  // heads between each other's tokens
    check_output(heads, T, hs, ts, d, (int)from(0, 1), meet ? TWINKV_E_ARG : TWINKV_OK);
  }
  for (const int d : {64, 128}) {
    check_output(4, 3, d, d, d, 0, TWINKV_E_ARG);
    check_output(2, 3, 2 * d, d, d, 0, TWINKV_E_ARG);
    check_output(2, 2, 2 * d, d, d, 0, TWINKV_OK);
    check_output(4, 1, d, d, d, 0, TWINKV_OK);          // one token: the heads side by side
    check_output(4, 3, d, 4 * d, d, 0, TWINKV_OK);      // token major
    check_output(3, 3, INT64_MAX / 16 * 8, INT64_MAX / 16 * 8, d, 0, TWINKV_E_ARG);
  }
  CHECK(refused > 1000 && odd > 100);
  std::printf("outputs: %lld refused, %lld interleaved\n", (long long)refused, (long long)odd);
}

typedef std::vector<int64_t> Lens;
void attend(int dtype, int d, int H, int G, const Lens& nq, const Lens& nk, int64_t window, int64_t sink) {
  Lens cq{0}, ck{0};
  for (size_t s = 0; s < nq.size(); ++s) {
    cq.push_back(cq.back() + nq[s]);
    ck.push_back(ck.back() + nk[s]);
  }
  const int S = (int)nq.size();
  const int64_t need = twinkv_attention_workspace_bytes(dtype, d, H, G, S, cq.data(), ck.data(), window, sink);
  CHECK(need >= 0 && need < (int64_t)1 << 31);
  std::vector<char> ws((size_t)std::max<int64_t>(need, 1));
  const int64_t t = (int64_t)d * H * G;
  CHECK(twinkv_sink_attention(fake, fake, fake, dtype, d, H, G, S, cq.data(), ck.data(), d, t, d, (int64_t)d * H, d,
                              (int64_t)d * H, window, sink, 0.1f, fake, d, t, nullptr, ws.data(), need, nullptr) == TWINKV_OK);
}

// The shapes of tests/test_gpu_cache_ops_edges.py that are there for split keys in the kernel for many bf16 rows.
void many_rows_split() {
  const int64_t all = (int64_t)1 << 40;
  auto split = [&](int d, int H, int G, const Lens& nq, const Lens& nk, int64_t window, int64_t sink) {
    attend(0, d, H, G, nq, nk, window, sink);
    CHECK(g_rows == twinkv::kAttnBigRows && *std::max_element(g_splits.begin(), g_splits.end()) > 1);
  };
  for (const int d : {64, 128}) {
    split(d, 4, 4, {200}, {5000}, 1 << 20, 4);
    split(d, 4, 8, {150}, {9000}, 6000, 70);
    split(d, 4, 4, {130, 60, 0, 301}, {7001, 90, 0, 5000}, all, 0);
    CHECK(g_splits[1] == 1);
    split(d, 2, 5, {513}, {6000}, 2500, 33);
    split(d, 4, 4, {200}, {6000}, 4000, 4);
  }
}

// One token over a long cache beside others: its run of key tiles does not grow with what the others have to do, and
// theirs are as without it.
void lone_sequences() {
  const int64_t all = (int64_t)1 << 40;
  for (const int d : {64, 128})
    for (const int64_t prompt : {2048, 8192, 32768}) {
      attend(0, d, 8, 4, {1, prompt}, {131072, prompt}, all, 0);
      CHECK(g_rows == twinkv::kAttnBigRows && g_splits[0] >= 32 && g_splits[1] == 1);
      attend(0, d, 8, 4, {prompt, 1}, {prompt, 131072}, all, 0);
      CHECK(g_rows == twinkv::kAttnBigRows && g_splits[0] == 1 && g_splits[1] >= 32);
    }
  attend(1, 128, 8, 4, {1, 8192}, {131072, 8192}, all, 0);
  CHECK(g_rows == twinkv::kAttnRows && g_splits[0] >= 8 && g_splits[1] == 1);
  // a chunk of few row tiles among single tokens
  Lens nq(65, 1), nk(65, 4096);
  nq[64] = 512, nk[64] = 32768;
  attend(0, 128, 8, 4, nq, nk, all, 0);
  CHECK(g_rows == twinkv::kAttnBigRows && g_splits[64] >= 4 && g_splits[0] == 1 && g_splits[63] == 1);
  // batches alike, or nearly, are as before
  attend(0, 128, 8, 4, Lens(16, 200), Lens(16, 8192), all, 0);
  CHECK(*std::max_element(g_splits.begin(), g_splits.end()) == 1);
  attend(0, 128, 8, 4, {8192}, {8192}, all, 0);
  CHECK(g_splits[0] == 1);
}

// fp32: where the kernel of four row tiles a workgroup is no faster than split keys it is not taken.
void wide_fp32() {
  auto rows = [&](int d, int H, int G, int64_t n, int64_t window) {
    attend(1, d, H, G, {n}, {n}, window, 0);
    return g_rows;
  };
  const int64_t all = (int64_t)1 << 40;
  CHECK(rows(64, 8, 1, 4096, all) == twinkv::kAttnRows && rows(64, 2, 4, 4096, all) == twinkv::kAttnRows);
  CHECK(rows(64, 8, 1, 5000, all) == twinkv::kAttnRows);
  CHECK(rows(64, 8, 1, 8192, all) == twinkv::kAttnWideRows && rows(64, 8, 2, 3000, all) == twinkv::kAttnWideRows);
  CHECK(rows(64, 8, 1, 4096, 1024) == twinkv::kAttnWideRows && rows(64, 8, 4, 2048, all) == twinkv::kAttnWideRows);
  CHECK(rows(128, 8, 1, 4096, all) == twinkv::kAttnWideRows && rows(128, 8, 1, 2048, all) == twinkv::kAttnRows);
  CHECK(rows(128, 8, 4, 512, all) == twinkv::kAttnWideRows && rows(64, 8, 1, 1500, 128) == twinkv::kAttnWideRows);
}
}  // namespace

int main() {
  outputs();
  many_rows_split();
  lone_sequences();
  wide_fp32();
  std::printf("cache plans ok\n");
  return 0;
}

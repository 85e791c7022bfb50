// Host layer of the operators around the cache (include/twinkv.h): argument validation, the
// per-sequence words, the split of the attention's keys, and the kernel launches (K6 norm and rotation,
// K7 4-bit cache, K8 / K9 attention).  Nothing here allocates.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "cache_ops.h"
#include "twinkv.h"
#include "twinkv_internal.h"

namespace twinkv {
namespace {

constexpr int64_t kMaxTokens = kAttnMaxKeys;  // of a batch: token indices are 32-bit inside the kernels
constexpr int kMaxHeads = 65535;              // a grid's second dimension
constexpr size_t kAlign = 256;

size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

char* aligned_base(void* ws) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(ws);
  return reinterpret_cast<char*>((p + kAlign - 1) / kAlign * kAlign);
}

int hip_status(int e) { return e == 0 ? TWINKV_OK : TWINKV_E_HIP; }

// A launch of `blocks` workgroups of `threads`: a grid dimension's threads are counted in 32 bits.
bool grid_ok(int64_t blocks, int threads) { return blocks * threads <= (int64_t)UINT32_MAX; }

int check_type(int dtype, int d) {
  return (dtype != TWINKV_BF16 && dtype != TWINKV_F32) || (d != 64 && d != 128) ? TWINKV_E_UNSUPPORTED : TWINKV_OK;
}

int check_cu(int n_seqs, const int64_t* cu) {
  if (cu == nullptr) return TWINKV_E_NULL;
  if (n_seqs < 1 || cu[0] != 0) return TWINKV_E_ARG;
  for (int s = 0; s < n_seqs; ++s)
    if (cu[s + 1] < cu[s]) return TWINKV_E_ARG;
  return cu[n_seqs] > kMaxTokens ? TWINKV_E_ARG : TWINKV_OK;
}

// Rows of d channels at strides (elements); a pointer may be null where there is nothing to address.
int check_rows(const void* p, int dtype, int d, int64_t head_stride, int64_t token_stride, bool empty) {
  if (p == nullptr) return empty ? TWINKV_OK : TWINKV_E_NULL;
  const int64_t esz = dtype == TWINKV_F32 ? 4 : 2;
  if (token_stride < d || head_stride < 0) return TWINKV_E_ARG;
  if (reinterpret_cast<uintptr_t>(p) % 16 != 0) return TWINKV_E_ARG;
  return token_stride * esz % 16 != 0 || head_stride * esz % 16 != 0 ? TWINKV_E_ARG : TWINKV_OK;
}

// Rows that are written: heads that share a place (a stride of 0, say) would overwrite each other.
int check_out(const void* p, int dtype, int d, int64_t head_stride, int64_t token_stride, int64_t heads, bool empty) {
  const int rc = check_rows(p, dtype, d, head_stride, token_stride, empty);
  return rc == TWINKV_OK && !empty && heads > 1 && head_stride < d ? TWINKV_E_ARG : rc;
}

// Whether rows (head, token) and (head', token') of an output with head_stride >= token_stride >= d share a place.
// Heads dh apart lie dh * head_stride apart, and the nearest that a token comes to that is one of two.
bool heads_overlap(int64_t head_stride, int64_t token_stride, int64_t heads, int64_t T, int d) {
  typedef __int128 Wide;
  if (T < 2 || head_stride < token_stride) return false;
  const Wide last = (Wide)(T - 1) * token_stride;
  for (int64_t dh = 1; dh < heads; ++dh) {
    const Wide at = (Wide)dh * head_stride;
    if (at >= last + d) break;
    const Wide token = std::min(at / token_stride, (Wide)(T - 1)), below = at - token * token_stride;
    if (below < d || (token < T - 1 && token_stride - below < d)) return true;
  }
  return false;
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Collects a call's per-sequence words: into the kernel arguments, or piece by piece into the workspace.
class WordWriter {
 public:
  WordWriter(SeqWords& to, int64_t n_words, void* far, void* stream)
      : to_(to), far_(n_words > kTabWords ? static_cast<int32_t*>(far) : nullptr), stream_(stream) {
    to_.far = far_;
  }
  void put(int32_t w) {
    if (n_ == kTabWords) flush();
    to_.near[n_++] = w;
  }
  int finish() {
    if (far_ != nullptr && n_ > 0) flush();
    return error_;
  }

 private:
  void flush() {
    if (error_ == 0) error_ = launch_upload(to_.near, 4 * (size_t)n_, far_ + done_, stream_);
    done_ += n_;
    n_ = 0;
  }
  SeqWords& to_;
  int32_t* far_;
  void* stream_;
  int n_ = 0, error_ = 0;
  int64_t done_ = 0;
};

size_t words_bytes(int n_seqs, int per_seq) {
  const int64_t n = ((int64_t)n_seqs + 1) * per_seq;
  return n > kTabWords ? align_up(4 * (size_t)n) : 0;
}

// ---- the 4-bit cache ----

int check_cache(const twinkv_cache4* c) {
  if (c == nullptr) return TWINKV_E_NULL;
  if (c->d != 64 && c->d != 128) return TWINKV_E_UNSUPPORTED;
  if (c->n_heads < 1 || c->n_heads > kMaxHeads) return TWINKV_E_ARG;
  const int rc = check_cu(c->n_seqs, c->cu_rows);
  if (rc != TWINKV_OK) return rc;
  if ((int64_t)c->n_heads * c->n_seqs > (int64_t)INT32_MAX / 4) return TWINKV_E_ARG;
  for (int s = 0; s < c->n_seqs; ++s)
    if (c->cu_rows[s + 1] % kCacheTile != 0) return TWINKV_E_ARG;
  if (c->cu_rows[c->n_seqs] > 0 && (c->k_codes == nullptr || c->k_scales == nullptr || c->v_codes == nullptr ||
                                    c->v_scales == nullptr))
    return TWINKV_E_NULL;
  if (!aligned16(c->k_codes) || !aligned16(c->k_scales) || !aligned16(c->v_codes) || !aligned16(c->v_scales))
    return TWINKV_E_ARG;
  return TWINKV_OK;
}

Cache4 device_cache(const twinkv_cache4* c) {
  return Cache4{static_cast<uint8_t*>(c->k_codes), static_cast<uint8_t*>(c->k_scales), static_cast<uint8_t*>(c->v_codes),
                static_cast<uint8_t*>(c->v_scales), c->cu_rows[c->n_seqs]};
}

// Blocks of 8 cache rows that n rows touch, at any first row.
int64_t blocks_of(int64_t n, bool aligned) {
  return n == 0 ? 0 : (n + (aligned ? kCacheBlock - 1 : 2 * kCacheBlock - 2)) / kCacheBlock;
}

enum class Blocks { kCache, kTokens };  // every row of the cache, or the rows the call's tokens take

// The words and the block list of a call whose token offsets are cu.
int cache_words(const twinkv_cache4* c, const int64_t* cu, Blocks which, Cache4Args& a, void* workspace,
                int64_t workspace_bytes, void* stream) {
  int64_t blocks = 0;
  for (int s = 0; s < c->n_seqs; ++s)
    blocks += which == Blocks::kCache ? blocks_of(c->cu_rows[s + 1] - c->cu_rows[s], true)
                                      : blocks_of(cu[s + 1] - cu[s], false);
  if (!grid_ok(blocks, 64) || !grid_ok((int64_t)c->n_heads * c->n_seqs, 1024)) return TWINKV_E_ARG;
  const size_t need = words_bytes(c->n_seqs, kCacheSeqWords);
  if (need > 0 && (workspace == nullptr || workspace_bytes < (int64_t)(need + kAlign))) return TWINKV_E_WORKSPACE;
  WordWriter w(a.seq, ((int64_t)c->n_seqs + 1) * kCacheSeqWords, need > 0 ? aligned_base(workspace) : nullptr, stream);
  int64_t at = 0;
  for (int s = 0; s <= c->n_seqs; ++s) {
    w.put((int32_t)cu[s]);
    w.put((int32_t)c->cu_rows[s]);
    w.put((int32_t)at);
    if (s < c->n_seqs)
      at += which == Blocks::kCache ? blocks_of(c->cu_rows[s + 1] - c->cu_rows[s], true)
                                    : blocks_of(cu[s + 1] - cu[s], false);
  }
  a.cache = device_cache(c);
  a.n_heads = c->n_heads;
  a.n_seqs = c->n_seqs;
  a.n_blocks = (int)blocks;
  return hip_status(w.finish());
}

void set_rows(Cache4Args& a, const void* keys, const void* values, int dtype, int64_t head_stride,
              int64_t token_stride, int64_t v_head_stride, int64_t v_token_stride) {
  const int64_t esz = dtype == TWINKV_F32 ? 4 : 2;
  a.keys = static_cast<const char*>(keys);
  a.values = static_cast<const char*>(values);
  a.head_stride = head_stride * esz;
  a.token_stride = token_stride * esz;
  a.v_head_stride = v_head_stride * esz;
  a.v_token_stride = v_token_stride * esz;
}

// ---- attention ----

// How a call's rows and keys are cut into items (attn.hip, attn4.hip, attn_rows.hip).
struct AttnPlan {
  int64_t window = 0, n_sink = 0;
  int rows = kAttnRows, keys = kAttnTile;  // of a tile
  int64_t split_tiles = 0;                 // the most key tiles of a split
  int64_t whole_tiles = 0;                 // up to so many are not split
  // a sequence with fewer row tiles than lone_rows (of all heads) and more key tiles than lone_run: its splits have
  // about lone_tiles at most
  int64_t lone_rows = 0, lone_run = 0, lone_tiles = 0;
  int64_t items = 0, parts = 0;            // per head
};

int64_t row_tiles(int64_t nq, int group, const AttnPlan& p) { return (nq * group + p.rows - 1) / p.rows; }

// The most key tiles a row tile of the sequence goes through.
int64_t key_tiles(int64_t nq, int64_t nk, int group, const AttnPlan& p) {
  const int64_t queries = std::min<int64_t>(nq, p.rows / group + 2);
  const int64_t near = std::min(nk, p.window + queries), sinks = std::min(nk, p.n_sink);
  const int64_t apart = (near + p.keys - 1) / p.keys + (sinks + p.keys - 1) / p.keys;
  return std::min(apart, (nk + p.keys - 1) / p.keys) + 1;
}

// A sequence's splits, of at most split_tiles tiles each, as equal as whole rounds of 4 tiles (the waves of
// the kernels for few rows) make them.
struct Splits {
  int64_t n, tiles;
};
Splits splits_of(int64_t tiles, int64_t rows, const AttnPlan& p) {
  int64_t most = p.split_tiles;
  if (rows < p.lone_rows && tiles > p.lone_run)
    most = std::min(most, std::max(p.lone_tiles, (rows * tiles + 2 * p.lone_rows - 1) / (2 * p.lone_rows)));
  const int64_t n = tiles <= p.whole_tiles ? 1 : (tiles + most - 1) / most;
  const int64_t each = ((tiles + n - 1) / n + 3) / 4 * 4;
  return Splits{std::max<int64_t>(1, (tiles + each - 1) / each), each};
}

// Row tiles of all heads, key tiles that they go through, and the most that one does.
struct AttnWork {
  int64_t rows = 0, tiles = 0, longest = 0;
};
AttnWork work_of(int n_heads, int group, int n_seqs, const int64_t* cu_q, const int64_t* cu_k, const AttnPlan& p) {
  AttnWork w;
  for (int s = 0; s < n_seqs; ++s) {
    const int64_t nq = cu_q[s + 1] - cu_q[s];
    if (nq == 0) continue;
    const int64_t rows = n_heads * row_tiles(nq, group, p), keys = key_tiles(nq, cu_k[s + 1] - cu_k[s], group, p);
    w.rows += rows;
    w.tiles += rows * keys;
    w.longest = std::max(w.longest, keys);
  }
  return w;
}

// The whole work is cut into about kItems workgroups, two a CU: decoding over 64 caches of 1k to 4k rows is at the
// copy rate so, and 20% slower with twice as many and their join.
constexpr int64_t kItems = 512;
// A split has at least two tiles a wave (8 heads of 4, one query over 4k keys 15.6 us, with twice that 18.5).  The
// 4-bit kernel takes a tile in less time than its join does: 4 a wave, and up to 8 a wave are not split
// (512 cached rows 8.1 us, split 10.3; 8k rows 13.3 / 14.7).  In the kernel for many rows, whose parts are larger, a
// split has 1024 keys (a prompt of 512 tokens: 18 us unsplit, 34 in splits of 512 keys), and there is one
// only where tiles of rows would leave CUs without work.
constexpr int64_t kLeast = 8, kLeastCached = 16, kWholeCached = 32, kLeastBig = 16, kCus = 256;
// What each workgroup has to do in the mean goes by the whole batch.  A sequence of few rows over far more keys than
// the others (one token over a long cache beside a prompt) would be one run about that long, and end the call alone.
// So a sequence with more than kLone times the mean run and too few row tiles to fill the machine is split whatever the
// others are: into runs of at most kLoneTiles (in the kernel for many rows kLoneBig) tiles, longer only where its own
// work fills the machine with them.  Without / with, us, 8 heads of 4, d 128: one token over 128k keys and a prompt of
// 8k tokens (alone 120 and 600) 2770 to 3200 by their order / 780, fp32 7900 to 8400 / 5900; 512 tokens over 32k and 64
// single ones over 4k each 1055 / 540; 8 tokens over 128k keys and 56 over 20k 1660 / 1530 (with kLoneTiles 256 1590,
// and fp32 a loss: 3155 / 3040, with 256 3270).
constexpr int64_t kLone = 2, kLoneTiles = 512, kLoneBig = 64;
// The kernel for many rows is taken for more rows than one tile of the other has, if it need not split the
// keys or there is enough work (in 16 rows x 32 keys).  Few rows / many, us, 8 heads, d 128: 64 rows over 4k keys 25 /
// 42, 256 38 / 56, 512 60 / 58, 2048 155 / 67; 64 over 32k 57 / 40, 2048 1145 / 298; 16 sequences of 32 rows over
// 4k keys 96 / 57; prompts of 512 tokens, 4 rows a token, 30 / 18, of 64 tokens 8.7 / 8.5.
constexpr int64_t kMuchWork = 20480;

// What a call's keys are: rows of any kind, rows that the kernel for many rows takes too, fp32 rows, a 4-bit
// cache under bf16 or fp32 queries.
enum class KeysAre { kRows, kRowsOfMany, kRowsFp32, kCached, kCachedFp32 };

int64_t live_of(int n_seqs, const int64_t* cu_q) {  // sequences with queries
  int64_t n = 0;
  for (int s = 0; s < n_seqs; ++s) n += cu_q[s + 1] > cu_q[s];
  return n;
}

// 4 bits, bf16: with so much work (as above) and more than a row tile in the mean a wave takes two row tiles at
// once.  One / two, us, 8 heads of 8, d 128: 3 queries over 32k rows 25 / 28, over 128k 58 / 50, over 64 caches of 4k 94 /
// 72; 7 queries over 32k 34 / 36, over 64 caches of 4k 182 / 143.
constexpr int64_t kPairWork = 49152;

// fp32: the kernel for many rows takes four row tiles a workgroup and does not split their keys, so it is taken where
// the most key tiles that a row tile has are no more than each of kItems such workgroups has in the mean, up to three
// times that where they are few, and at most half of it where they are many and d is 64 (whose tiles are half the work
// for the same waits).  Split / wide, us, 8 heads, that ratio in brackets: d 128, 4 rows a token, causal, 256 tokens (4)
// 22 / 27, 512 (2) 72 / 62, 1024 (1) 164 / 132, 2048 (0.5) 456 / 333; window 128, 256 tokens (4) 20 / 21, 512 (2) 39 / 23,
// 2048 (0.5) 144 / 69; a row a token, causal, 2048 tokens (2) 168 / 183, 4096 (1) 495 / 457.  d 64, a row a token, causal,
// 2048 tokens (2) 86 / 113, 4096 (1) 256 / 258 (2 heads of 4 rows a token 227 / 249), 5000 (0.82) 327 / 338, 8192 (0.5)
// 769 / 709; two rows a token, 2048 tokens (1) 136 / 136, 3000 (0.68) 240 / 224.
constexpr int64_t kWideTiles = 20, kLongTiles64 = 96;

int attn_plan(KeysAre keys, int d, int n_heads, int group, int n_seqs, const int64_t* cu_q, const int64_t* cu_k, int64_t window,
              int64_t n_sink, AttnPlan& p) {
  p.window = std::min<int64_t>(window, kAttnMaxKeys);
  p.n_sink = std::min<int64_t>(n_sink, kAttnMaxKeys);
  const bool cached = keys == KeysAre::kCached || keys == KeysAre::kCachedFp32;
  AttnWork few = work_of(n_heads, group, n_seqs, cu_q, cu_k, p);
  if (keys == KeysAre::kCached && few.tiles >= kPairWork && cu_q[n_seqs] * group > kAttnRows * live_of(n_seqs, cu_q)) {
    p.rows = kAttnPairRows;
    few = work_of(n_heads, group, n_seqs, cu_q, cu_k, p);
  }
  int64_t each = std::max(cached ? kLeastCached : kLeast, (few.tiles + kItems - 1) / kItems);
  p.whole_tiles = cached ? kWholeCached : kLeast;
  p.lone_rows = kItems;
  p.lone_run = kLone * few.tiles / std::max<int64_t>(few.rows, 1);
  p.lone_tiles = kLoneTiles;
  if (keys == KeysAre::kRowsOfMany) {
    AttnPlan big = p;
    big.rows = kAttnBigRows;
    big.keys = kAttnBigTile;
    const AttnWork w = work_of(n_heads, group, n_seqs, cu_q, cu_k, big);
    if (cu_q[n_seqs] * group > kAttnRows * live_of(n_seqs, cu_q) && (few.tiles >= kMuchWork || w.longest <= kLeastBig)) {
      p = big;
      p.whole_tiles = kLeastBig;
      each = w.rows >= kCus ? kAttnMaxKeys : std::max(kLeastBig, (w.tiles + kItems - 1) / kItems);
      p.lone_rows = kCus;
      p.lone_run = kLone * w.tiles / std::max<int64_t>(w.rows, 1);
      p.lone_tiles = kLoneBig;
    }
  }
  const int64_t halves = few.longest <= kWideTiles ? 6 : d == 64 && few.longest > kLongTiles64 ? 1 : 2;
  if (keys == KeysAre::kRowsFp32 && 2 * few.longest * (kAttnWideRows / kAttnRows) * kItems <= halves * few.tiles &&
      cu_q[n_seqs] * group > kAttnRows * live_of(n_seqs, cu_q)) {
    p.rows = kAttnWideRows;
    each = kAttnMaxKeys;
    p.whole_tiles = kAttnMaxKeys;  // (nor for one sequence among others)
  }
  p.split_tiles = (std::min<int64_t>(each, kAttnMaxKeys / 64) + 3) / 4 * 4;
  for (int s = 0; s < n_seqs; ++s) {
    const int64_t nq = cu_q[s + 1] - cu_q[s];
    const int64_t rows = row_tiles(nq, group, p);
    const int64_t splits = splits_of(key_tiles(nq, cu_k[s + 1] - cu_k[s], group, p), n_heads * rows, p).n;
    p.items += rows * splits;
    if (splits > 1) p.parts += rows * splits;
  }
  return grid_ok(p.items * (p.rows == kAttnBigRows || p.rows == kAttnWideRows ? n_heads : 1), 256) ? TWINKV_OK : TWINKV_E_ARG;
}

struct AttnLayout {
  size_t words = 0, part_o = 0, part_ml = 0, total = 0;
};
AttnLayout attn_layout(const AttnPlan& p, int d, int n_heads, int n_seqs) {
  AttnLayout L;
  size_t off = words_bytes(n_seqs, kAttnSeqWords);
  const size_t rows = (size_t)n_heads * (size_t)p.parts * (size_t)p.rows;
  L.part_o = off;
  off = align_up(off + 4 * rows * (size_t)d);
  L.part_ml = off;
  off = align_up(off + 8 * rows);
  L.total = off > 0 ? off + kAlign : 0;
  return L;
}

int check_heads(int n_heads, int group) {
  return n_heads < 1 || n_heads > kMaxHeads || group < 1 || (int64_t)n_heads * group > (int64_t)INT32_MAX / 4
             ? TWINKV_E_ARG : TWINKV_OK;
}

// Rows are numbered in 32 bits inside a sequence.
int check_queries(int n_seqs, const int64_t* cu_q, int group) {
  for (int s = 0; s < n_seqs; ++s)
    if ((cu_q[s + 1] - cu_q[s]) * group > kMaxTokens) return TWINKV_E_ARG;
  return TWINKV_OK;
}

// The queries' and outputs' side of a call, the plan, the words and the parts.
int attn_args(KeysAre keys, const void* q, int dtype, int d, int n_heads, int group, int n_seqs, const int64_t* cu_q,
              const int64_t* cu_k, int64_t q_head_stride, int64_t q_token_stride, int64_t window, int64_t n_sink,
              float scale, void* out, int64_t out_head_stride, int64_t out_token_stride, float* lse,
              void* workspace, int64_t workspace_bytes, void* stream, AttnArgs& a) {
  AttnPlan p;
  const int rc = attn_plan(keys, d, n_heads, group, n_seqs, cu_q, cu_k, window, n_sink, p);
  if (rc != TWINKV_OK) return rc;
  const AttnLayout L = attn_layout(p, d, n_heads, n_seqs);
  if (L.total > 0 && (workspace == nullptr || workspace_bytes < (int64_t)L.total)) return TWINKV_E_WORKSPACE;
  if (heads_overlap(out_head_stride, out_token_stride, (int64_t)n_heads * group, cu_q[n_seqs], d)) return TWINKV_E_ARG;
  char* ws = L.total > 0 ? aligned_base(workspace) : nullptr;
  const int64_t esz = dtype == TWINKV_F32 ? 4 : 2;
  a.q = static_cast<const char*>(q);
  a.k = nullptr;
  a.v = nullptr;
  a.out = static_cast<char*>(out);
  a.q_head = q_head_stride * esz;
  a.q_token = q_token_stride * esz;
  a.k_head = a.k_token = a.v_head = a.v_token = 0;
  a.o_head = out_head_stride * esz;
  a.o_token = out_token_stride * esz;
  a.cache = Cache4{nullptr, nullptr, nullptr, nullptr, 0};
  a.len = nullptr;
  a.lse = lse;
  a.Tq = cu_q[n_seqs];
  a.scale_log2 = (float)((double)scale * 1.4426950408889634074);
  a.window = (int)p.window;
  a.n_sink = (int)p.n_sink;
  a.n_heads = n_heads;
  a.group = group;
  a.n_seqs = n_seqs;
  a.items = (int)p.items;
  a.parts = (int)p.parts;
  a.rows = p.rows;
  a.part_o = reinterpret_cast<float*>(ws + L.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + L.part_ml);
  WordWriter w(a.seq, ((int64_t)n_seqs + 1) * kAttnSeqWords, ws, stream);
  int64_t item = 0, part = 0;
  for (int s = 0; s <= n_seqs; ++s) {
    Splits splits{1, 0};
    int64_t tiles = 0;
    if (s < n_seqs) {
      const int64_t nq = cu_q[s + 1] - cu_q[s];
      tiles = row_tiles(nq, group, p);
      splits = splits_of(key_tiles(nq, cu_k[s + 1] - cu_k[s], group, p), n_heads * tiles, p);
    }
    w.put((int32_t)cu_q[s]);
    w.put((int32_t)cu_k[s]);
    w.put((int32_t)item);
    w.put((int32_t)splits.n);
    w.put((int32_t)splits.tiles);
    w.put((int32_t)part);
    item += tiles * splits.n;
    if (splits.n > 1) part += tiles * splits.n;
  }
  return hip_status(w.finish());
}

}  // namespace
}  // namespace twinkv

using namespace twinkv;

extern "C" {

int twinkv_qk_norm_rope(const void* q, const void* k, int dtype, int d, int n_q_heads, int n_k_heads, int64_t T,
                        int64_t q_head_stride, int64_t q_token_stride, int64_t k_head_stride,
                        int64_t k_token_stride, const float* q_weight, const float* k_weight, float eps,
                        const float* rope, int64_t n_pos, const int32_t* positions, void* q_out,
                        int64_t qo_head_stride, int64_t qo_token_stride, void* k_out, int64_t ko_head_stride,
                        int64_t ko_token_stride, void* stream) {
  int rc = check_type(dtype, d);
  if (rc != TWINKV_OK) return rc;
  if (n_q_heads < 0 || n_k_heads < 0 || T < 0 || T > kMaxTokens) return TWINKV_E_ARG;
  if ((int64_t)n_q_heads + n_k_heads > kMaxHeads) return TWINKV_E_ARG;
  if (!std::isfinite(eps) || eps < 0.0f) return TWINKV_E_ARG;
  const bool no_q = n_q_heads == 0 || T == 0, no_k = n_k_heads == 0 || T == 0;
  if ((rc = check_rows(q, dtype, d, q_head_stride, q_token_stride, no_q)) != TWINKV_OK) return rc;
  if ((rc = check_out(q_out, dtype, d, qo_head_stride, qo_token_stride, n_q_heads, no_q)) != TWINKV_OK) return rc;
  if ((rc = check_rows(k, dtype, d, k_head_stride, k_token_stride, no_k)) != TWINKV_OK) return rc;
  if ((rc = check_out(k_out, dtype, d, ko_head_stride, ko_token_stride, n_k_heads, no_k)) != TWINKV_OK) return rc;
  if (!aligned16(q_weight) || !aligned16(k_weight) || !aligned16(rope)) return TWINKV_E_ARG;
  if (rope != nullptr) {
    if (n_pos < 0) return TWINKV_E_ARG;
    if (positions == nullptr && T > 0) return TWINKV_E_NULL;
  }
  if (heads_overlap(qo_head_stride, qo_token_stride, no_q ? 0 : n_q_heads, T, d) ||
      heads_overlap(ko_head_stride, ko_token_stride, no_k ? 0 : n_k_heads, T, d))
    return TWINKV_E_ARG;
  if (no_q && no_k) return TWINKV_OK;
  if (!grid_ok((T + 31) / 32, 256)) return TWINKV_E_ARG;
  const int64_t esz = dtype == TWINKV_F32 ? 4 : 2;
  NormRopeArgs a;
  // heads a unit of lanes goes through with its token's cos and sin: as many as leave units for every
  // SIMD of the machine (about 16000 rows of lanes; both ends measured in norm_rope.hip)
  const int64_t rows = T * ((int64_t)n_q_heads + n_k_heads);
  a.per_unit = (int)std::min<int64_t>(std::max<int64_t>(rows / 16384, 1), 8);
  auto side = [&](const void* in, void* out, int64_t ih, int64_t it, int64_t oh, int64_t ot, const float* weight,
                  int heads) {
    return NormRopeSide{static_cast<const char*>(in), static_cast<char*>(out), ih * esz, it * esz, oh * esz, ot * esz,
                        weight, heads, (heads + a.per_unit - 1) / a.per_unit};
  };
  a.q = side(q, q_out, q_head_stride, q_token_stride, qo_head_stride, qo_token_stride, q_weight, n_q_heads);
  a.k = side(k, k_out, k_head_stride, k_token_stride, ko_head_stride, ko_token_stride, k_weight, n_k_heads);
  a.T = T;
  a.n_pos = n_pos;
  a.rope = rope;
  a.pos = positions;
  a.eps = eps;
  return hip_status(launch_norm_rope(a, dtype, d, stream));
}

int64_t twinkv_attention_workspace_bytes(int dtype, int d, int n_heads, int group, int n_seqs, const int64_t* cu_q,
                                         const int64_t* cu_k, int64_t window, int64_t n_sink) {
  int rc = check_type(dtype, d);
  if (rc == TWINKV_OK) rc = check_heads(n_heads, group);
  if (rc == TWINKV_OK) rc = check_cu(n_seqs, cu_q);
  if (rc == TWINKV_OK) rc = check_cu(n_seqs, cu_k);
  if (rc == TWINKV_OK) rc = check_queries(n_seqs, cu_q, group);
  if (rc == TWINKV_OK && (window < 0 || n_sink < 0)) rc = TWINKV_E_ARG;
  if (rc != TWINKV_OK) return -rc;
  int64_t most = 0;  // of the plans that the two calls may make
  for (const KeysAre keys : {KeysAre::kRows, dtype == TWINKV_BF16 ? KeysAre::kCached : KeysAre::kCachedFp32,
                             dtype == TWINKV_BF16 ? KeysAre::kRowsOfMany : KeysAre::kRowsFp32}) {
    AttnPlan p;
    rc = attn_plan(keys, d, n_heads, group, n_seqs, cu_q, cu_k, window, n_sink, p);
    if (rc != TWINKV_OK) return -rc;
    most = std::max(most, (int64_t)attn_layout(p, d, n_heads, n_seqs).total);
  }
  return most;
}

int twinkv_sink_attention(const void* q, const void* k, const void* v, int dtype, int d, int n_heads, int group,
                          int n_seqs, const int64_t* cu_q, const int64_t* cu_k, int64_t q_head_stride,
                          int64_t q_token_stride, int64_t k_head_stride, int64_t k_token_stride,
                          int64_t v_head_stride, int64_t v_token_stride, int64_t window, int64_t n_sink, float scale,
                          void* out, int64_t out_head_stride, int64_t out_token_stride, float* lse, void* workspace,
                          int64_t workspace_bytes, void* stream) {
  int rc = check_type(dtype, d);
  if (rc != TWINKV_OK) return rc;
  if ((rc = check_heads(n_heads, group)) != TWINKV_OK) return rc;
  if ((rc = check_cu(n_seqs, cu_q)) != TWINKV_OK) return rc;
  if ((rc = check_cu(n_seqs, cu_k)) != TWINKV_OK) return rc;
  if ((rc = check_queries(n_seqs, cu_q, group)) != TWINKV_OK) return rc;
  if (window < 0 || n_sink < 0 || !std::isfinite(scale)) return TWINKV_E_ARG;
  const bool no_q = cu_q[n_seqs] == 0, no_k = cu_k[n_seqs] == 0;
  if ((rc = check_rows(q, dtype, d, q_head_stride, q_token_stride, no_q)) != TWINKV_OK) return rc;
  if ((rc = check_out(out, dtype, d, out_head_stride, out_token_stride, (int64_t)n_heads * group, no_q)) != TWINKV_OK)
    return rc;
  if ((rc = check_rows(k, dtype, d, k_head_stride, k_token_stride, no_k)) != TWINKV_OK) return rc;
  if ((rc = check_rows(v, dtype, d, v_head_stride, v_token_stride, no_k)) != TWINKV_OK) return rc;
  if (no_q) return TWINKV_OK;
  AttnArgs a;
  // the kernel for many rows: 64 tokens' strides within 32 bits (the other takes any)
  const KeysAre keys = dtype != TWINKV_BF16 ? KeysAre::kRowsFp32
                       : std::max(k_token_stride, v_token_stride) <= INT32_MAX / (2 * 64) ? KeysAre::kRowsOfMany
                                                                                         : KeysAre::kRows;
  rc = attn_args(keys, q, dtype, d, n_heads, group, n_seqs, cu_q, cu_k, q_head_stride, q_token_stride, window, n_sink,
                 scale, out, out_head_stride, out_token_stride, lse, workspace, workspace_bytes, stream, a);
  if (rc != TWINKV_OK) return rc;
  const int64_t esz = dtype == TWINKV_F32 ? 4 : 2;
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.k_head = k_head_stride * esz;
  a.k_token = k_token_stride * esz;
  a.v_head = v_head_stride * esz;
  a.v_token = v_token_stride * esz;
  const int e = a.rows == kAttnBigRows ? launch_attn_rows(a, d, stream) : launch_attn(a, dtype, d, stream);
  if (e != 0 || a.parts == 0) return hip_status(e);
  return hip_status(launch_attn_join(a, dtype, d, stream));
}

int64_t twinkv_cache4_workspace_bytes(int n_seqs) {
  if (n_seqs < 1) return -TWINKV_E_ARG;
  const size_t n = words_bytes(n_seqs, kCacheSeqWords);
  return n > 0 ? (int64_t)(n + kAlign) : 0;
}

int twinkv_cache4_compact(const void* keys, const void* values, int dtype, const int64_t* cu_seqlens,
                          int64_t head_stride, int64_t token_stride, int64_t v_head_stride, int64_t v_token_stride,
                          const uint8_t* retained, const twinkv_cache4* cache, int32_t* pos_out, int32_t* len_out,
                          int32_t* status, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc != TWINKV_OK) return rc;
  if ((rc = check_type(dtype, cache->d)) != TWINKV_OK) return rc;
  if ((rc = check_cu(cache->n_seqs, cu_seqlens)) != TWINKV_OK) return rc;
  const int64_t T = cu_seqlens[cache->n_seqs], C = cache->cu_rows[cache->n_seqs];
  if ((rc = check_rows(keys, dtype, cache->d, head_stride, token_stride, T == 0)) != TWINKV_OK) return rc;
  if ((rc = check_rows(values, dtype, cache->d, v_head_stride, v_token_stride, T == 0)) != TWINKV_OK) return rc;
  if ((retained == nullptr && T > 0) || (pos_out == nullptr && C > 0) || len_out == nullptr || status == nullptr)
    return TWINKV_E_NULL;
  Cache4Args a = {};
  rc = cache_words(cache, cu_seqlens, Blocks::kCache, a, workspace, workspace_bytes, stream);
  if (rc != TWINKV_OK) return rc;
  set_rows(a, keys, values, dtype, head_stride, token_stride, v_head_stride, v_token_stride);
  a.retained = retained;
  a.T = T;
  a.pos = pos_out;
  a.len_out = len_out;
  a.status = status;
  if (launch_cache4_positions(a, stream) != 0) return TWINKV_E_HIP;
  return hip_status(launch_cache4_gather(a, dtype, cache->d, stream));
}

int twinkv_cache4_append(const void* keys, const void* values, int dtype, const int64_t* cu_new, int64_t head_stride,
                         int64_t token_stride, int64_t v_head_stride, int64_t v_token_stride,
                         const twinkv_cache4* cache, const int32_t* len_in, int32_t* len_out, int32_t* status,
                         void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc != TWINKV_OK) return rc;
  if ((rc = check_type(dtype, cache->d)) != TWINKV_OK) return rc;
  if ((rc = check_cu(cache->n_seqs, cu_new)) != TWINKV_OK) return rc;
  const bool none = cu_new[cache->n_seqs] == 0;
  if ((rc = check_rows(keys, dtype, cache->d, head_stride, token_stride, none)) != TWINKV_OK) return rc;
  if ((rc = check_rows(values, dtype, cache->d, v_head_stride, v_token_stride, none)) != TWINKV_OK) return rc;
  if (len_in == nullptr || len_out == nullptr || status == nullptr) return TWINKV_E_NULL;
  Cache4Args a = {};
  rc = cache_words(cache, cu_new, Blocks::kTokens, a, workspace, workspace_bytes, stream);
  if (rc != TWINKV_OK) return rc;
  set_rows(a, keys, values, dtype, head_stride, token_stride, v_head_stride, v_token_stride);
  a.len_in = len_in;
  a.len_out = len_out;
  a.status = status;
  int64_t most = 0;
  for (int s = 0; s < cache->n_seqs; ++s) most = std::max(most, cu_new[s + 1] - cu_new[s]);
  return hip_status(launch_cache4_append(a, (int)std::max<int64_t>(most, 1), dtype, cache->d, stream));
}

int twinkv_cache4_read(const twinkv_cache4* cache, const int32_t* len, const int32_t* first, int dtype,
                       const int64_t* cu_out, void* keys_out, void* values_out, void* workspace,
                       int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc != TWINKV_OK) return rc;
  if ((rc = check_type(dtype, cache->d)) != TWINKV_OK) return rc;
  if ((rc = check_cu(cache->n_seqs, cu_out)) != TWINKV_OK) return rc;
  if (len == nullptr) return TWINKV_E_NULL;
  if (!aligned16(keys_out) || !aligned16(values_out)) return TWINKV_E_ARG;
  Cache4Args a = {};
  rc = cache_words(cache, cu_out, Blocks::kTokens, a, workspace, workspace_bytes, stream);
  if (rc != TWINKV_OK) return rc;
  a.len_in = len;
  a.first = first;
  a.keys_out = static_cast<char*>(keys_out);
  a.values_out = static_cast<char*>(values_out);
  a.C_out = cu_out[cache->n_seqs];
  return hip_status(launch_cache4_read(a, dtype, cache->d, stream));
}

int twinkv_cache4_attention(const void* q, int dtype, int group, const int64_t* cu_q, int64_t q_head_stride,
                            int64_t q_token_stride, const twinkv_cache4* cache, const int32_t* len, float scale,
                            void* out, int64_t out_head_stride, int64_t out_token_stride, float* lse, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc != TWINKV_OK) return rc;
  const int d = cache->d, n_seqs = cache->n_seqs;
  if ((rc = check_type(dtype, d)) != TWINKV_OK) return rc;
  if ((rc = check_heads(cache->n_heads, group)) != TWINKV_OK) return rc;
  if ((rc = check_cu(n_seqs, cu_q)) != TWINKV_OK) return rc;
  if ((rc = check_queries(n_seqs, cu_q, group)) != TWINKV_OK) return rc;
  if (!std::isfinite(scale)) return TWINKV_E_ARG;
  const bool no_q = cu_q[n_seqs] == 0;
  if ((rc = check_rows(q, dtype, d, q_head_stride, q_token_stride, no_q)) != TWINKV_OK) return rc;
  if ((rc = check_out(out, dtype, d, out_head_stride, out_token_stride, (int64_t)cache->n_heads * group, no_q)) != TWINKV_OK)
    return rc;
  if (len == nullptr) return TWINKV_E_NULL;
  if (no_q) return TWINKV_OK;
  AttnArgs a;
  rc = attn_args(dtype == TWINKV_BF16 ? KeysAre::kCached : KeysAre::kCachedFp32, q, dtype, d, cache->n_heads, group, n_seqs,
                 cu_q, cache->cu_rows, q_head_stride, q_token_stride, INT64_MAX, 0, scale, out, out_head_stride,
                 out_token_stride, lse, workspace, workspace_bytes, stream, a);
  if (rc != TWINKV_OK) return rc;
  a.cache = device_cache(cache);
  a.len = len;
  const int e = launch_attn4(a, dtype, d, stream);
  if (e != 0 || a.parts == 0) return hip_status(e);
  return hip_status(launch_attn_join(a, dtype, d, stream));
}

}  // extern "C"

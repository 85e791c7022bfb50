// Host layer of the accumulated attention weights (K14) and of the 8-bit cache (include/twinkv.h): writing and
// reading it (K11), attention over it (K13) and eviction from it (K12).  Argument checks and the attention's plan:
// cache_host.h.  Nothing here allocates.
#include "cache_host.h"

namespace twinkv {
namespace {

// ---- accumulated weights ----

// A sequence's key tiles, and the splits of the rows that see one (kMassSeqWords).
struct MassSeq {
  int64_t tiles = 0, splits = 1, rows = 0;
  int64_t full = 0;
  MassShape shape = kMassRest;
  int64_t by = 1;
  int64_t items = 0;
};
struct MassPlan {
  int64_t keys = 0;        // of a tile
  int64_t most_rows = 0;   // of a split
  int64_t items = 0;
  bool split = false, few = false;
};

// The most rows that see a key of one tile.  `cached`: how many keys there are is known on the device only.
int64_t rows_seeing(int64_t nq, int64_t nk, int group, int64_t window, int64_t n_sink, int64_t keys, bool cached) {
  if (cached) return nq * group;
  const int64_t seen = std::min(nq, nk);  // queries at positions from 0 on
  return (n_sink > 0 ? seen : std::min(seen, window + keys - 1)) * group;
}

// Items of equal work, many to a CU so that the last ones to end leave little of the machine idle (16384: a window of
// 9460 in 9828 tokens of d 64 282 us, with 2048 items 306), but of 1024 rows at least, whose products cover the way of
// the item's keys to the registers (a prompt of 8192 tokens, d 64: 190 us, with 256 rows 238, with 4096 200); of fewer
// where there would not be two for every CU.
constexpr int64_t kMassItems = 16384, kMassSlots = 2 * kCus, kMassLeast = 1024;
// Up to so many items for each CU, these are counted for splits of half to four times that size, and the split is taken
// whose fullest CU has least to do; an item's start takes as long as 0.7 of a step of kMassRowTile rows, and an item alone
// on its CU 1.5 times as long as one of many.  (Sequences of 244 and 2061 tokens, 8 query heads a head: 66 us, without the
// count 78.)
constexpr int64_t kMassCounted = 16;
constexpr double kMassStart = 0.7, kMassAlone = 1.5;
// Up to so many rows (bf16) the keys' way to the registers is what takes the time: one buffer of rows and no look-ahead,
// for more workgroups a CU.  (64 sequences of 1024 to 4096 keys, d 128: the last 32 queries of 4 heads 88 us for 103, the
// last one 74 for 90.)
constexpr int64_t kMassFew = 256;

MassSeq mass_seq(int64_t nq, int64_t nk, int group, int64_t window, int64_t n_sink, bool cached, const MassPlan& p) {
  MassSeq m;
  const int64_t rows = rows_seeing(nq, nk, group, window, n_sink, p.keys, cached), tile_rows = p.keys * group;
  m.tiles = (nk + p.keys - 1) / p.keys;
  if (!cached && window >= nk && nq > 0 && rows > p.most_rows) {
    // Causal: tile by tile the rows that see one get fewer by tile_rows, once the tile lies behind the first query.
    // Splits of a whole number of them, or whole parts of them, and tiles of ever fewer splits: no item is empty.
    m.full = std::min(m.tiles, std::max<int64_t>(nk - nq, 0) / p.keys + 1);
    int64_t run = 1, drop = 1;
    if (p.most_rows >= tile_rows) {
      run = p.most_rows / tile_rows;
      m.rows = run * tile_rows;
      m.shape = kMassRuns;
      m.by = run;
    } else {
      drop = tile_rows / p.most_rows;
      while (tile_rows % (drop * kMassRowTile) != 0) --drop;
      m.rows = tile_rows / drop;
      m.shape = kMassDrops;
      m.by = drop;
    }
    m.splits = (rows + m.rows - 1) / m.rows;
    m.items = m.full * m.splits;
    int64_t splits = m.splits;
    for (int64_t t = m.full; t < m.tiles; t += run, splits -= splits > drop ? drop : 0)
      m.items += std::min(run, m.tiles - t) * splits;
    return m;
  }
  m.splits = std::max<int64_t>(1, (rows + p.most_rows - 1) / p.most_rows);
  const int64_t each = (rows + m.splits - 1) / m.splits;
  m.rows = std::max<int64_t>(1, (each + kMassRowTile - 1) / kMassRowTile) * kMassRowTile;
  m.splits = std::max<int64_t>(1, (rows + m.rows - 1) / m.rows);
  // tiles with sinks are seen by all queries, the others by those of a window
  m.full = cached || n_sink == 0 ? m.tiles : std::min(m.tiles, (n_sink + p.keys - 1) / p.keys);
  const int64_t rest = std::max<int64_t>(1, (rows_seeing(nq, nk, group, window, 0, p.keys, cached) + m.rows - 1) / m.rows);
  m.by = rest;
  m.items = m.full * m.splits + (m.tiles - m.full) * rest;
  return m;
}

int mass_plan(int dtype, int n_heads, int group, int n_seqs, const int64_t* cu_q, const int64_t* cu_k, int64_t window,
              int64_t n_sink, bool cached, MassPlan& p) {
  p.keys = dtype == TWINKV_BF16 ? 2 * kMassKeys : kMassKeys;
  double work = 0;  // rows times tiles
  int64_t longest = 0;
  for (int s = 0; s < n_seqs; ++s) {
    const int64_t nq = cu_q[s + 1] - cu_q[s], nk = cu_k[s + 1] - cu_k[s];
    if (nk == 0) continue;
    const int64_t tiles = (nk + p.keys - 1) / p.keys, sinks = std::min(tiles, (n_sink + p.keys - 1) / p.keys);
    const int64_t most = rows_seeing(nq, nk, group, window, 1, p.keys, cached);
    const int64_t rest = rows_seeing(nq, nk, group, window, 0, p.keys, cached);
    // of a whole prompt the mean key is seen by half of the queries
    const double part = window >= nk && !cached ? 1.0 - 0.5 * std::min(1.0, (double)nq / (double)nk) : 1.0;
    longest = std::max(longest, sinks > 0 ? most : rest);
    work += (double)n_heads * part * ((double)sinks * (double)most + (double)(tiles - sinks) * (double)rest);
  }
  p.few = longest <= kMassFew;
  const int64_t even = (int64_t)(work / kMassSlots);
  const int64_t base = std::max((int64_t)(work / kMassItems), std::min(kMassLeast, std::max<int64_t>(even, kMassRowTile)));
  auto items_of = [&](int64_t most_rows, int64_t& rows) {
    p.most_rows = most_rows;
    p.items = rows = 0;
    p.split = false;
    for (int s = 0; s < n_seqs; ++s) {
      const MassSeq m = mass_seq(cu_q[s + 1] - cu_q[s], cu_k[s + 1] - cu_k[s], group, window, n_sink, cached, p);
      p.items += m.items;
      p.split |= m.splits > 1;
      rows = std::max(rows, m.rows);
    }
  };
  int64_t rows, best = base;
  items_of(base, rows);
  if (p.split && p.items * n_heads < kMassCounted * kCus) {
    double least = 0;
    for (const int64_t most_rows : {base, base / 2, 2 * base, 4 * base}) {
      if (most_rows < kMassRowTile) continue;
      items_of(most_rows, rows);
      const double fullest = std::max((double)((p.items * n_heads + kCus - 1) / kCus), kMassAlone);
      const double cost = fullest * ((double)rows / kMassRowTile + kMassStart);
      if (least == 0 || cost < 0.95 * least) {
        least = cost;
        best = most_rows;
      }
    }
    items_of(best, rows);
  }
  return grid_ok(p.items * n_heads, 256) && p.items <= INT32_MAX ? TWINKV_OK : TWINKV_E_ARG;
}

struct MassLayout {
  size_t part = 0, total = 0;
};
MassLayout mass_layout(const MassPlan& p, int n_heads, int n_seqs) {
  MassLayout L;
  L.part = words_bytes(n_seqs, kMassSeqWords);
  const size_t end = align_up(L.part + (p.split ? 4 * (size_t)n_heads * (size_t)p.items * (size_t)p.keys : 0));
  L.total = end > 0 ? end + kAlign : 0;
  return L;
}

// The rows' side of a call, the plan, the words and the parts.
int mass_args(int dtype, int d, const void* q, int n_heads, int group, int n_seqs, const int64_t* cu_q, const int64_t* cu_k,
              int64_t q_head_stride, int64_t q_token_stride, int64_t window, int64_t n_sink, float scale, bool cached,
              const float* lse, const float* mass, float* mass_out, void* workspace, int64_t workspace_bytes,
              void* stream, MassArgs& a) {
  MassPlan p;
  window = std::min<int64_t>(window, kAttnMaxKeys);
  n_sink = std::min<int64_t>(n_sink, kAttnMaxKeys);
  const int rc = mass_plan(dtype, n_heads, group, n_seqs, cu_q, cu_k, window, n_sink, cached, p);
  if (rc != TWINKV_OK) return rc;
  const MassLayout L = mass_layout(p, n_heads, n_seqs);
  if (L.total > 0 && (workspace == nullptr || workspace_bytes < (int64_t)L.total)) return TWINKV_E_WORKSPACE;
  char* ws = L.total > 0 ? aligned_base(workspace) : nullptr;
  const int64_t esz = dtype == TWINKV_F32 ? 4 : 2;
  a.q = static_cast<const char*>(q);
  a.k = nullptr;
  a.q_head = q_head_stride * esz;
  a.q_token = q_token_stride * esz;
  a.k_head = a.k_token = 0;
  a.cache = Cache8{nullptr, nullptr, nullptr, nullptr, 0};
  a.len = nullptr;
  a.lse = lse;
  a.mass = mass;
  a.mass_out = mass_out;
  a.Tq = cu_q[n_seqs];
  a.Tk = cu_k[n_seqs];
  a.scale_log2 = (float)((double)scale * 1.4426950408889634074);
  a.window = (int)window;
  a.n_sink = (int)n_sink;
  a.n_heads = n_heads;
  a.group = group;
  a.n_seqs = n_seqs;
  a.items = (int)p.items;
  a.keys = (int)p.keys;
  a.few = p.few;
  a.part = p.split ? reinterpret_cast<float*>(ws + L.part) : nullptr;
  WordWriter w(a.seq, ((int64_t)n_seqs + 1) * kMassSeqWords, ws, stream);
  int64_t item = 0;
  for (int s = 0; s <= n_seqs; ++s) {
    MassSeq m;
    if (s < n_seqs) m = mass_seq(cu_q[s + 1] - cu_q[s], cu_k[s + 1] - cu_k[s], group, window, n_sink, cached, p);
    w.put((int32_t)cu_q[s]);
    w.put((int32_t)cu_k[s]);
    w.put((int32_t)item);
    w.put((int32_t)m.splits);
    w.put((int32_t)std::min<int64_t>(m.rows, INT32_MAX));
    w.put((int32_t)m.full);
    w.put((int32_t)m.shape << kMassShapeBits | (int32_t)m.by);
    item += m.items;
  }
  return hip_status(w.finish());
}

int run_mass(const MassArgs& a, int dtype, int d, void* stream) {
  if (a.items == 0) return TWINKV_OK;
  const int e = launch_mass(a, dtype, d, stream);
  if (e != 0 || a.part == nullptr) return hip_status(e);
  return hip_status(launch_mass_join(a, stream));
}

KeysAre cached_keys(int dtype) { return dtype == TWINKV_BF16 ? KeysAre::kCached : KeysAre::kCachedFp32; }

// How the accumulated weights of an attention over the cache come about.  With at most one tile of rows a problem (and
// at least one row: an item) the attention keeps its scores, 4 bytes a row and key, and the weights follow in the same
// kernels; otherwise they are computed afresh from the queries' log-sum-exps.
bool keeps_scores(int group, int n_seqs, const int64_t* cu_q, const int64_t* cu_rows) {
  for (int s = 0; s < n_seqs; ++s) {
    const int64_t rows = (cu_q[s + 1] - cu_q[s]) * group;
    if (cu_rows[s + 1] > cu_rows[s] && (rows < 1 || rows > kAttnRows)) return false;
  }
  return true;
}

// An attention's plan, and its workspace: its own; with weights wanted the scores, or the log-sum-exps where the caller
// wants none and the weights' own.
struct Attn8Layout {
  AttnPlan plan;
  size_t attn = 0, lse = 0, mass = 0;
  bool scores = false;
  int score_rows = 0, score_lds = 0;
  int64_t total() const { return (int64_t)(attn + lse + mass); }
};
int attn8_layout(int dtype, int d, int n_heads, int group, int n_seqs, const int64_t* cu_q, const int64_t* cu_rows,
                 bool want_mass, Attn8Layout& L) {
  L.scores = want_mass && keeps_scores(group, n_seqs, cu_q, cu_rows);
  int64_t most_tiles = kAttnMaxKeys;  // of a split
  // Scores are kept for one tile of rows an item.  (Queries of sequences without rows count in the plan's mean, and
  // could ask for two.)
  const int most_rows = L.scores ? kAttnRows : kAttnPairRows;
  if (L.scores) {
    for (int s = 0; s < n_seqs; ++s)
      if (cu_rows[s + 1] > cu_rows[s]) L.score_rows = std::max(L.score_rows, (int)((cu_q[s + 1] - cu_q[s]) * group));
    most_tiles = kAttnMostLds / (4 * kAttnTile * std::max(L.score_rows, 1));
  }
  int rc = attn_plan(cached_keys(dtype), d, n_heads, group, n_seqs, cu_q, cu_rows, INT64_MAX, 0, L.plan, most_tiles,
                     most_rows);
  if (rc != TWINKV_OK) return rc;
  L.attn = attn_layout(L.plan, d, n_heads, n_seqs).total;
  if (!want_mass) return TWINKV_OK;
  if (L.scores) {
    for (int s = 0; s < n_seqs; ++s) {
      const int64_t nk = cu_rows[s + 1] - cu_rows[s], nq = cu_q[s + 1] - cu_q[s];
      if (nk == 0) continue;
      const Splits splits = splits_of(key_tiles(nq, nk, group, L.plan), n_heads * row_tiles(nq, group, L.plan), L.plan);
      L.score_lds = std::max(L.score_lds, (int)(nq * group * std::min(nk, splits.tiles * kAttnTile)));
    }
    if (L.plan.parts > 0)
      L.mass = align_up(4 * (size_t)n_heads * (size_t)L.score_rows * (size_t)cu_rows[n_seqs]) + kAlign;
    return TWINKV_OK;
  }
  MassPlan m;
  rc = mass_plan(dtype, n_heads, group, n_seqs, cu_q, cu_rows, kAttnMaxKeys, 0, true, m);
  if (rc != TWINKV_OK) return rc;
  L.lse = align_up(4 * (size_t)n_heads * (size_t)group * (size_t)cu_q[n_seqs]) + kAlign;
  L.mass = mass_layout(m, n_heads, n_seqs).total;
  return TWINKV_OK;
}

bool shares(const twinkv_cache8* a, const twinkv_cache8* b) {
  const void* x[] = {a->k_codes, a->k_scales, a->v_codes, a->v_scales};
  const void* y[] = {b->k_codes, b->k_scales, b->v_codes, b->v_scales};
  for (const void* p : x)
    for (const void* q : y)
      if (p != nullptr && p == q) return true;
  return false;
}

}  // namespace
}  // namespace twinkv

using namespace twinkv;

extern "C" {

int64_t twinkv_mass_workspace_bytes(int dtype, int d, int n_heads, int group, int n_seqs, const int64_t* cu_q,
                                    const int64_t* cu_k, int64_t window, int64_t n_sink) {
  int rc = check_type(dtype, d);
  if (rc == TWINKV_OK) rc = check_heads(n_heads, group);
  if (rc == TWINKV_OK) rc = check_cu(n_seqs, cu_q);
  if (rc == TWINKV_OK) rc = check_cu(n_seqs, cu_k);
  if (rc == TWINKV_OK) rc = check_queries(n_seqs, cu_q, group);
  if (rc == TWINKV_OK && (window < 0 || n_sink < 0)) rc = TWINKV_E_ARG;
  if (rc != TWINKV_OK) return -rc;
  MassPlan p;
  rc = mass_plan(dtype, n_heads, group, n_seqs, cu_q, cu_k, std::min<int64_t>(window, kAttnMaxKeys),
                 std::min<int64_t>(n_sink, kAttnMaxKeys), false, p);
  return rc != TWINKV_OK ? -rc : (int64_t)mass_layout(p, n_heads, n_seqs).total;
}

int twinkv_attention_mass(const void* q, const void* k, int dtype, int d, int n_heads, int group, int n_seqs,
                          const int64_t* cu_q, const int64_t* cu_k, int64_t q_head_stride, int64_t q_token_stride,
                          int64_t k_head_stride, int64_t k_token_stride, int64_t window, int64_t n_sink, float scale,
                          const float* lse, const float* mass, float* mass_out, void* workspace,
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
  if ((rc = check_rows(k, dtype, d, k_head_stride, k_token_stride, no_k)) != TWINKV_OK) return rc;
  if ((lse == nullptr && !no_q) || (mass_out == nullptr && !no_k)) return TWINKV_E_NULL;
  if (no_k) return TWINKV_OK;
  MassArgs a;
  rc = mass_args(dtype, d, q, n_heads, group, n_seqs, cu_q, cu_k, q_head_stride, q_token_stride, window, n_sink, scale, false,
                 lse, mass, mass_out, workspace, workspace_bytes, stream, a);
  if (rc != TWINKV_OK) return rc;
  const int64_t esz = dtype == TWINKV_F32 ? 4 : 2;
  a.k = static_cast<const char*>(k);
  a.k_head = k_head_stride * esz;
  a.k_token = k_token_stride * esz;
  return run_mass(a, dtype, d, stream);
}

int64_t twinkv_cache8_workspace_bytes(int n_seqs) {
  if (n_seqs < 1) return -TWINKV_E_ARG;
  const size_t n = words_bytes(n_seqs, std::max(kCacheSeqWords, kEvict8SeqWords));
  return n > 0 ? (int64_t)(n + kAlign) : 0;
}

int twinkv_cache8_compact(const void* keys, const void* values, int dtype, const int64_t* cu_seqlens,
                          int64_t head_stride, int64_t token_stride, int64_t v_head_stride, int64_t v_token_stride,
                          const uint8_t* retained, const twinkv_cache8* cache, const float* token_mass,
                          int32_t* pos_out, float* mass_out, int32_t* len_out, int32_t* status, void* workspace,
                          int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc != TWINKV_OK) return rc;
  if ((rc = check_type(dtype, cache->d)) != TWINKV_OK) return rc;
  if ((rc = check_cu(cache->n_seqs, cu_seqlens)) != TWINKV_OK) return rc;
  const int64_t T = cu_seqlens[cache->n_seqs], C = cache->cu_rows[cache->n_seqs];
  if ((rc = check_rows(keys, dtype, cache->d, head_stride, token_stride, T == 0)) != TWINKV_OK) return rc;
  if ((rc = check_rows(values, dtype, cache->d, v_head_stride, v_token_stride, T == 0)) != TWINKV_OK) return rc;
  if ((retained == nullptr && T > 0) || (pos_out == nullptr && C > 0) || len_out == nullptr || status == nullptr)
    return TWINKV_E_NULL;
  if (token_mass != nullptr && mass_out == nullptr && C > 0) return TWINKV_E_NULL;
  Cache8Args a = {};
  rc = cache_words(cache, cu_seqlens, Blocks::kCache, kCache8Block, a, workspace, workspace_bytes, stream);
  if (rc != TWINKV_OK) return rc;
  set_rows(a, keys, values, dtype, head_stride, token_stride, v_head_stride, v_token_stride);
  a.retained = retained;
  a.T = T;
  a.pos = pos_out;
  a.len_out = len_out;
  a.status = status;
  a.mass = token_mass;
  a.mass_out = mass_out;
  if (launch_cache4_positions(a, stream) != 0) return TWINKV_E_HIP;
  return hip_status(launch_cache8_gather(a, dtype, cache->d, stream));
}

int twinkv_cache8_append(const void* keys, const void* values, int dtype, const int64_t* cu_new, int64_t head_stride,
                         int64_t token_stride, int64_t v_head_stride, int64_t v_token_stride,
                         const twinkv_cache8* cache, const int32_t* len_in, int32_t* len_out, int32_t* status,
                         void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc != TWINKV_OK) return rc;
  if ((rc = check_type(dtype, cache->d)) != TWINKV_OK) return rc;
  if ((rc = check_cu(cache->n_seqs, cu_new)) != TWINKV_OK) return rc;
  const bool none = cu_new[cache->n_seqs] == 0;
  if ((rc = check_rows(keys, dtype, cache->d, head_stride, token_stride, none)) != TWINKV_OK) return rc;
  if ((rc = check_rows(values, dtype, cache->d, v_head_stride, v_token_stride, none)) != TWINKV_OK) return rc;
  if (len_in == nullptr || len_out == nullptr || status == nullptr) return TWINKV_E_NULL;
  Cache8Args a = {};
  rc = cache_words(cache, cu_new, Blocks::kTokens, kCache8Block, a, workspace, workspace_bytes, stream);
  if (rc != TWINKV_OK) return rc;
  set_rows(a, keys, values, dtype, head_stride, token_stride, v_head_stride, v_token_stride);
  a.len_in = len_in;
  a.len_out = len_out;
  a.status = status;
  int64_t most = 0;
  for (int s = 0; s < cache->n_seqs; ++s) most = std::max(most, cu_new[s + 1] - cu_new[s]);
  return hip_status(launch_cache8_append(a, (int)most, dtype, cache->d, stream));
}

int twinkv_cache8_read(const twinkv_cache8* cache, const int32_t* len, const int32_t* first, int dtype,
                       const int64_t* cu_out, void* keys_out, void* values_out, void* workspace,
                       int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc != TWINKV_OK) return rc;
  if ((rc = check_type(dtype, cache->d)) != TWINKV_OK) return rc;
  if ((rc = check_cu(cache->n_seqs, cu_out)) != TWINKV_OK) return rc;
  if (len == nullptr) return TWINKV_E_NULL;
  if (!aligned16(keys_out) || !aligned16(values_out)) return TWINKV_E_ARG;
  Cache8Args a = {};
  rc = cache_words(cache, cu_out, Blocks::kTokens, kCache8Block, a, workspace, workspace_bytes, stream);
  if (rc != TWINKV_OK) return rc;
  a.len_in = len;
  a.first = first;
  a.keys_out = static_cast<char*>(keys_out);
  a.values_out = static_cast<char*>(values_out);
  a.C_out = cu_out[cache->n_seqs];
  return hip_status(launch_cache8_read(a, dtype, cache->d, stream));
}

int64_t twinkv_cache8_attention_workspace_bytes(int dtype, int d, int n_heads, int group, int n_seqs,
                                                const int64_t* cu_q, const int64_t* cu_rows, int want_mass) {
  int rc = check_type(dtype, d);
  if (rc == TWINKV_OK) rc = check_heads(n_heads, group);
  if (rc == TWINKV_OK) rc = check_cu(n_seqs, cu_q);
  if (rc == TWINKV_OK) rc = check_cu(n_seqs, cu_rows);
  if (rc == TWINKV_OK) rc = check_queries(n_seqs, cu_q, group);
  Attn8Layout L;
  if (rc == TWINKV_OK) rc = attn8_layout(dtype, d, n_heads, group, n_seqs, cu_q, cu_rows, want_mass != 0, L);
  return rc != TWINKV_OK ? -rc : L.total();
}

int twinkv_cache8_attention(const void* q, int dtype, int group, const int64_t* cu_q, int64_t q_head_stride,
                            int64_t q_token_stride, const twinkv_cache8* cache, const int32_t* len, float scale,
                            void* out, int64_t out_head_stride, int64_t out_token_stride, float* lse, const float* mass,
                            float* mass_out, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(cache);
  if (rc != TWINKV_OK) return rc;
  const int d = cache->d, n_seqs = cache->n_seqs, n_heads = cache->n_heads;
  if ((rc = check_type(dtype, d)) != TWINKV_OK) return rc;
  if ((rc = check_heads(n_heads, group)) != TWINKV_OK) return rc;
  if ((rc = check_cu(n_seqs, cu_q)) != TWINKV_OK) return rc;
  if ((rc = check_queries(n_seqs, cu_q, group)) != TWINKV_OK) return rc;
  if (!std::isfinite(scale)) return TWINKV_E_ARG;
  const bool no_q = cu_q[n_seqs] == 0;
  if ((rc = check_rows(q, dtype, d, q_head_stride, q_token_stride, no_q)) != TWINKV_OK) return rc;
  if ((rc = check_out(out, dtype, d, out_head_stride, out_token_stride, (int64_t)n_heads * group, no_q)) != TWINKV_OK)
    return rc;
  if (len == nullptr || (mass != nullptr && mass_out == nullptr)) return TWINKV_E_NULL;
  if (!aligned16(mass) || !aligned16(mass_out)) return TWINKV_E_ARG;
  const bool want_mass = mass_out != nullptr && cache->cu_rows[n_seqs] > 0;
  if (no_q && !want_mass) return TWINKV_OK;
  Attn8Layout L;
  if ((rc = attn8_layout(dtype, d, n_heads, group, n_seqs, cu_q, cache->cu_rows, want_mass, L)) != TWINKV_OK) return rc;
  if (L.total() > 0 && (workspace == nullptr || workspace_bytes < L.total())) return TWINKV_E_WORKSPACE;
  char* ws = static_cast<char*>(workspace);
  if (want_mass && !L.scores && lse == nullptr) lse = reinterpret_cast<float*>(aligned_base(ws + L.attn));
  if (!no_q) {
    AttnArgs a;
    rc = attn_args(L.plan, q, dtype, d, n_heads, group, n_seqs, cu_q, cache->cu_rows, q_head_stride,
                   q_token_stride, scale, out, out_head_stride, out_token_stride, lse, ws, (int64_t)L.attn, stream,
                   a);
    if (rc != TWINKV_OK) return rc;
    a.cache = device_cache(cache);
    a.len = len;
    if (L.scores) {
      a.score = L.mass > 0 ? reinterpret_cast<float*>(aligned_base(ws + L.attn)) : nullptr;
      a.score_rows = L.score_rows;
      a.score_lds = L.score_lds;
      a.mass = mass;
      a.mass_out = mass_out;
    }
    int e = launch_attn8(a, dtype, d, stream);
    if (e == 0 && a.parts > 0) e = launch_attn_join(a, dtype, d, stream);
    if (e != 0) return TWINKV_E_HIP;
  }
  if (!want_mass || L.scores) return TWINKV_OK;
  MassArgs a;
  rc = mass_args(dtype, d, q, n_heads, group, n_seqs, cu_q, cache->cu_rows, q_head_stride, q_token_stride, INT64_MAX, 0, scale,
                 true, lse, mass, mass_out, ws + L.attn + L.lse, (int64_t)L.mass, stream, a);
  if (rc != TWINKV_OK) return rc;
  a.cache = device_cache(cache);
  a.len = len;
  return run_mass(a, dtype, d, stream);
}

int twinkv_cache8_evict(const twinkv_cache8* from, const int32_t* len, const float* mass, const int32_t* pos,
                        const int64_t* budget, int n_sink, int n_recent, const twinkv_cache8* to, int32_t* len_out,
                        float* mass_out, int32_t* pos_out, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_cache(from);
  if (rc != TWINKV_OK) return rc;
  if ((rc = check_cache(to)) != TWINKV_OK) return rc;
  if (from->d != to->d || from->n_heads != to->n_heads || from->n_seqs != to->n_seqs) return TWINKV_E_ARG;
  const int n_seqs = from->n_seqs;
  const int64_t C = from->cu_rows[n_seqs], C_to = to->cu_rows[n_seqs];
  if (budget == nullptr || len == nullptr || len_out == nullptr || (mass == nullptr && C > 0) ||
      (pos_out == nullptr && C_to > 0))
    return TWINKV_E_NULL;
  if (n_sink < 0 || n_recent < 0 || !aligned16(mass) || shares(from, to)) return TWINKV_E_ARG;
  int64_t blocks = 0, most = 0;
  for (int s = 0; s < n_seqs; ++s) {
    const int64_t rows = to->cu_rows[s + 1] - to->cu_rows[s];
    if (budget[s] < 0 || budget[s] > rows) return TWINKV_E_ARG;
    blocks += rows / kCache8Block;
    most = std::max(most, from->cu_rows[s + 1] - from->cu_rows[s]);
  }
  if (!grid_ok(blocks, 64) || !grid_ok((int64_t)from->n_heads * n_seqs, 1024)) return TWINKV_E_ARG;
  const size_t need = words_bytes(n_seqs, kEvict8SeqWords);
  if (need > 0 && (workspace == nullptr || workspace_bytes < (int64_t)(need + kAlign))) return TWINKV_E_WORKSPACE;
  Evict8Args a = {};
  WordWriter w(a.seq, ((int64_t)n_seqs + 1) * kEvict8SeqWords, need > 0 ? aligned_base(workspace) : nullptr, stream);
  for (int s = 0; s <= n_seqs; ++s) {
    w.put((int32_t)from->cu_rows[s]);
    w.put((int32_t)to->cu_rows[s]);
    w.put(s < n_seqs ? (int32_t)budget[s] : 0);
    w.put((int32_t)(to->cu_rows[s] / kCache8Block));
  }
  if ((rc = hip_status(w.finish())) != TWINKV_OK) return rc;
  a.from = device_cache(from);
  a.to = device_cache(to);
  a.len = len;
  a.mass = mass;
  a.pos = pos;
  a.len_out = len_out;
  a.mass_out = mass_out;
  a.pos_out = pos_out;
  a.n_heads = from->n_heads;
  a.n_seqs = n_seqs;
  a.n_sink = n_sink;
  a.n_recent = n_recent;
  a.n_blocks = (int)blocks;
  a.max_rows = (int)most;
  if (launch_evict8_select(a, stream) != 0) return TWINKV_E_HIP;
  return hip_status(launch_evict8_move(a, from->d, stream));
}

}  // extern "C"

// Host layer of the operators around the cache (include/twinkv.h): norm and rotation (K6), the 4-bit cache (K7)
// and attention (K8 / K9 / K10).  Argument checks, words and plans: cache_host.h.  Nothing here allocates.
#include "cache_host.h"

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
  AttnPlan p;
  rc = attn_plan(keys, d, n_heads, group, n_seqs, cu_q, cu_k, window, n_sink, p);
  if (rc != TWINKV_OK) return rc;
  rc = attn_args(p, q, dtype, d, n_heads, group, n_seqs, cu_q, cu_k, q_head_stride, q_token_stride, scale, out,
                 out_head_stride, out_token_stride, lse, workspace, workspace_bytes, stream, a);
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
  rc = cache_words(cache, cu_seqlens, Blocks::kCache, kCacheBlock, a, workspace, workspace_bytes, stream);
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
  rc = cache_words(cache, cu_new, Blocks::kTokens, kCacheBlock, a, workspace, workspace_bytes, stream);
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
  rc = cache_words(cache, cu_out, Blocks::kTokens, kCacheBlock, a, workspace, workspace_bytes, stream);
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
  AttnPlan p;
  rc = attn_plan(dtype == TWINKV_BF16 ? KeysAre::kCached : KeysAre::kCachedFp32, d, cache->n_heads, group, n_seqs, cu_q,
                 cache->cu_rows, INT64_MAX, 0, p);
  if (rc != TWINKV_OK) return rc;
  rc = attn_args(p, q, dtype, d, cache->n_heads, group, n_seqs, cu_q, cache->cu_rows, q_head_stride, q_token_stride, scale,
                 out, out_head_stride, out_token_stride, lse, workspace, workspace_bytes, stream, a);
  if (rc != TWINKV_OK) return rc;
  a.cache = device_cache(cache);
  a.len = len;
  const int e = launch_attn4(a, dtype, d, stream);
  if (e != 0 || a.parts == 0) return hip_status(e);
  return hip_status(launch_attn_join(a, dtype, d, stream));
}

}  // extern "C"

/*
 * twinkv.h -- C ABI of the TwinKV redundancy / repair library for AMD MI355X (gfx950).
 *
 * TwinKV (paper: "TwinKV: A Composable Repair Pass for KV Cache Eviction via Pairwise
 * Key Redundancy") works per (layer, KV head) on the keys of one sequence (Sec. 3.1):
 *   - Eq. 1: sim(i, j) = k_hat_i . k_hat_j with k_hat = k / ||k||_2 (Sec. 3.2);
 *   - twin rule: j is a twin of i iff sim(i, j) > tau and |i - j| > w (Sec. 3.2, Eq. 2);
 *   - Eq. 4: b_i(S0) = max over j in S0, |i - j| > w of sim(i, j), or -1 if no such j;
 *   - repair (Sec. 3.4): orphans (i not in S0, b_i < tau) and redundant donors (j in S0,
 *     outside the protected sink / recent regions, b_j >= tau) are ranked by severity
 *     (orphans by ascending b, donors by descending b) and the m = min(|O|, |D|) most severe
 *     pairs are swapped, so |S1| = |S0| = K exactly;
 *   - the standalone scorer (Sec. 3.2, Eq. 2-3): twin counts r_i, scores s_i = -r_i / n, and
 *     the retained set of the K highest scores with the sink / recent regions kept first;
 *   - the prevalence statistic of Sec. 2 (Fig. 1b): tokens with at least one twin;
 *   - a wrapped policy's retained set from its per-token scores (Sec. 3.1: K positions per
 *     head and layer; Sec. 3.2: the sink / recent regions at the maximum score), the S0 the
 *     repair takes;
 *   - KV compaction (Sec. 3.1): only the keys and values at the retained positions are kept
 *     for generation, gathered here into a dense cache.
 *
 * Problems.  A batch holds n_heads (layer, KV head) pairs times n_seqs sequences.  Sequence s
 * owns global token positions [cu_seqlens[s], cu_seqlens[s+1]) and T = cu_seqlens[n_seqs].
 * Problem q = h * n_seqs + s is (head h, sequence s); problems are independent (Sec. 3.1).
 * Indices reported by the library are 0-based positions inside the sequence.
 *
 * Memory.  Unless marked "(host)", pointers are DEVICE pointers owned by the caller.  The
 * library allocates nothing: scratch space is the caller's `workspace` (size from
 * twinkv_workspace_bytes).  Keys: element (h, t, c) is at keys[h*head_stride + t*token_stride
 * + c] (strides in elements, channels contiguous); the pointer and both strides (in bytes)
 * must be multiples of 16.  Per-token arrays (retained masks, scores, indices) are contiguous
 * [n_heads][T].  Every entry point enqueues work on `stream` (a hipStream_t passed as void*;
 * NULL = the default stream) and returns without waiting; results are valid once the stream
 * has reached that point.  The small per-sequence table built from the host arrays reaches
 * the workspace as the arguments of kernels, so the host arrays are consumed
 * before the call returns and no host memory is read later.  A call enqueues kernel launches
 * only (no memset, no host copy, no allocation), so it may be captured into a HIP graph; a
 * replay repeats the captured batch description (sequence lengths, budgets, tau, w) and
 * re-reads the device buffers it was given.  twinkv_profile_sim_events adds event records.
 *
 * Errors.  Argument errors are detected on the host before anything is enqueued and are
 * returned synchronously (TWINKV_E_*).  A HIP failure while enqueueing returns TWINKV_E_HIP.
 * Data-dependent conditions are reported per problem (TWINKV_PROBLEM_*), never by failing.
 * Concurrent calls are safe as long as they use different workspaces.
 */
#ifndef TWINKV_H
#define TWINKV_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Return codes. */
#define TWINKV_OK             0
#define TWINKV_E_NULL         1  /* a required pointer is NULL */
#define TWINKV_E_ARG          2  /* an argument value is out of range or inconsistent */
#define TWINKV_E_UNSUPPORTED  3  /* head dimension or dtype not supported */
#define TWINKV_E_WORKSPACE    4  /* workspace missing or smaller than required */
#define TWINKV_E_HIP          5  /* the HIP runtime reported an error */
#define TWINKV_E_CAPACITY     6  /* the batch needs more than the static scratch buffer holds */

/* Key element types. */
#define TWINKV_BF16 0
#define TWINKV_F32  1

/* Operations, for twinkv_workspace_bytes. */
#define TWINKV_OP_NN_SCORES          0
#define TWINKV_OP_REPAIR             1
#define TWINKV_OP_REPAIR_FROM_SCORES 2
#define TWINKV_OP_TWIN_COUNTS        3
#define TWINKV_OP_SCORE_EVICT        4
#define TWINKV_OP_COMPACT            5

/* Most thresholds twinkv_prevalence takes in one call. */
#define TWINKV_MAX_TAUS 32

/* Most nested retained sets twinkv_nn_scores_levels takes in one call. */
#define TWINKV_MAX_LEVELS 4

/* Per-problem status codes (stats[q][3] / status[q]). */
#define TWINKV_PROBLEM_OK              0
#define TWINKV_PROBLEM_BUDGET_MISMATCH 1  /* |S0| differs from the budget; S1 = S0 */
#define TWINKV_PROBLEM_NONFINITE       2  /* a key (or a given score) is NaN/Inf; S1 = S0 */

/*
 * Bytes of workspace `op` needs for this batch; negative (-TWINKV_E_*) on invalid arguments.
 * cu_seqlens (host, n_seqs + 1 entries, non-decreasing, cu_seqlens[0] = 0).
 * dtype and d are ignored for TWINKV_OP_REPAIR_FROM_SCORES and TWINKV_OP_COMPACT.
 */
int64_t twinkv_workspace_bytes(int op, int dtype, int d, int n_heads, int n_seqs,
                               const int64_t* cu_seqlens);

/*
 * Best twin of every token (Sec. 3.2 Eq. 1 + the twin rule's window; Sec. 3.4 Eq. 4).
 *
 *   keys       [n_heads][T][d] bf16 or fp32 (see Memory).  d must be 64 or 128.
 *   retained   [n_heads][T] uint8, nonzero = in S0; NULL skips the retained reduction.
 *   w          window half-width, >= 0: pairs with |i - j| <= w are never compared.
 *   best_all   [n_heads][T] fp32: max over j with |i-j| > w of sim(i, j); -1 if none.  Nullable.
 *   arg_all    [n_heads][T] int32: the maximising j (position in the sequence); -1 if none.
 *              On near-equal candidates the reported j is one whose similarity is within
 *              2^-15 (3.1e-5) of the maximum for bf16 keys with d = 128 and 2^-17 (7.6e-6)
 *              otherwise; on exact equality it is the smallest such j.  Nullable.
 *   best_ret   [n_heads][T] fp32: b_i(S0) of Eq. 4 (-1 if no retained j beyond the window).
 *              Nullable; must be NULL when retained is NULL.
 *   arg_ret    [n_heads][T] int32: the maximising retained j, -1 if none.  Nullable.
 *   status     [n_heads * n_seqs] int32 TWINKV_PROBLEM_* (only OK / NONFINITE).  Nullable.
 *              The scores of a problem with a non-finite key are unspecified (the similarity
 *              is undefined there); every other problem's are unaffected.
 *
 * Similarities are computed from the stored key values with fp32 accumulation; their error
 * against exact arithmetic is below 1e-4 for bf16 and fp32 keys (this includes the rounding
 * down of reported values by less than the tie bound above).  Every result is independent of
 * a key's length as Eq. 1 is: scaling a key by a power of two changes no output bit, as long
 * as its elements, their products with the other keys' elements and its norm stay in fp32's
 * normal range (below 2^120 and above 2^-126 in magnitude).
 */
int twinkv_nn_scores(const void* keys, int dtype, int d, int n_heads, int n_seqs,
                     const int64_t* cu_seqlens, int64_t head_stride, int64_t token_stride,
                     const uint8_t* retained, int w,
                     float* best_all, int32_t* arg_all, float* best_ret, int32_t* arg_ret,
                     int32_t* status,
                     void* workspace, int64_t workspace_bytes, void* stream);

/*
 * The full repair pass of Sec. 3.4 for every problem: Eq. 4 scores, orphan / donor
 * classification, severity ranking and the budget-preserving swap.
 *
 *   retained_in   [n_heads][T] uint8, the wrapped policy's S0 (nonzero = retained).
 *   retained_out  [n_heads][T] uint8, receives S1 as 0/1.  May alias retained_in.
 *   budget        (host) [n_seqs] int64: K = |S0| of every problem of sequence s.  A problem
 *                 whose |S0| differs gets TWINKV_PROBLEM_BUDGET_MISMATCH and S1 = S0.
 *   tau           duplicate threshold (finite).  Orphan: b < tau.  Donor: b >= tau.
 *   w             window half-width, >= 0.
 *   n_sink, n_recent  >= 0: positions [0, n_sink) and [len - n_recent, len) are protected
 *                 (never donors).
 *   stats         [n_heads * n_seqs][4] int32 = {|O|, |D|, m, status}.
 *   best_all, arg_all, best_ret, arg_ret   optional outputs as in twinkv_nn_scores (nullable).
 *                 When best_all and arg_all are both NULL, similarities against evicted keys
 *                 are skipped (only S0 columns are needed for b).
 *
 * Ranking ties resolve by ascending position (among equal b, the earlier orphan is admitted
 * and the earlier donor evicted first).
 */
int twinkv_repair(const void* keys, int dtype, int d, int n_heads, int n_seqs,
                  const int64_t* cu_seqlens, int64_t head_stride, int64_t token_stride,
                  const uint8_t* retained_in, uint8_t* retained_out,
                  const int64_t* budget, float tau, int w, int n_sink, int n_recent,
                  int32_t* stats,
                  float* best_all, int32_t* arg_all, float* best_ret, int32_t* arg_ret,
                  void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Classification, severity ranking and swap of Sec. 3.4 from given scores b = b_i(S0)
 * ([n_heads][T] fp32), e.g. produced by twinkv_nn_scores or by another scorer.  Arguments as
 * in twinkv_repair.  A NaN/Inf score gives TWINKV_PROBLEM_NONFINITE and S1 = S0.
 */
int twinkv_repair_from_scores(const float* b, const uint8_t* retained_in, uint8_t* retained_out,
                              int n_heads, int n_seqs, const int64_t* cu_seqlens,
                              const int64_t* budget, float tau, int n_sink, int n_recent,
                              int32_t* stats,
                              void* workspace, int64_t workspace_bytes, void* stream);

/*
 * twinkv_repair_from_scores for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): no workspace
 * argument.  The only scratch the call needs, the per-sequence table, lives in a static
 * device buffer of the library (64 KiB per GPU, held until the process ends), so at most
 * TWINKV_NOALLOC_MAX_SEQS sequences per call; a larger batch returns TWINKV_E_CAPACITY before
 * anything is enqueued.  The buffer of the current device is used (the stream must belong to
 * it).  Every call on one GPU shares that buffer: calls that overlap on one GPU (different
 * streams, or host threads enqueueing concurrently) race and must be serialised by the
 * caller.  Nothing in the buffer needs to start at zero (each call writes the whole table it
 * reads).  The call allocates nothing; results equal twinkv_repair_from_scores.
 */
#define TWINKV_NOALLOC_MAX_SEQS 2048
int twinkv_repair_from_scores_noalloc(const float* b, const uint8_t* retained_in,
                                      uint8_t* retained_out, int n_heads, int n_seqs,
                                      const int64_t* cu_seqlens, const int64_t* budget,
                                      float tau, int n_sink, int n_recent, int32_t* stats,
                                      void* stream);

/*
 * Twin counts of Sec. 3.2 Eq. 2 for every token:
 *   counts[h][t] = #{ j in t's sequence : |i - j| > w, sim(i, j) > tau },  i = t's position.
 *
 *   keys, dtype, d, n_heads, n_seqs, cu_seqlens, strides, w   as in twinkv_nn_scores.
 *   tau      twin threshold (finite).
 *   counts   [n_heads][T] int32 (required).
 *   status   [n_heads * n_seqs] int32 TWINKV_PROBLEM_* (only OK / NONFINITE).  Nullable.
 *            The counts of a problem with a non-finite key are unspecified.
 *   workspace  twinkv_workspace_bytes(TWINKV_OP_TWIN_COUNTS, ...) bytes.
 *
 * The decision sim > tau is taken on fp32 similarities (error below 1e-4, typically 1e-6):
 * pairs whose exact similarity is that close to tau may fall on either side.
 */
int twinkv_twin_counts(const void* keys, int dtype, int d, int n_heads, int n_seqs,
                       const int64_t* cu_seqlens, int64_t head_stride, int64_t token_stride,
                       float tau, int w, int32_t* counts, int32_t* status,
                       void* workspace, int64_t workspace_bytes, void* stream);

/*
 * b_i(S_k) of Sec. 3.4 Eq. 4 for nested retained sets S_1 within S_2 within ... within S_L
 * (for example the retained sets of one policy at increasing budgets), in one call.
 * The tokens of each level group G_k = S_k minus S_{k-1} are swept once as the retained
 * columns, so the similarity work is N * |S_L| per problem (plus N * (N - |S_L|) when the
 * all-keys result is asked for), instead of N * (|S_1| + ... + |S_L|) for L separate calls.
 *
 *   level     [n_heads][T] uint8: k in 1..n_levels = the smallest set that holds the token;
 *             0 = in none.  Values above n_levels count as 0.
 *   n_levels  1 <= L <= TWINKV_MAX_LEVELS.
 *   best_lvl  [n_levels][n_heads][T] fp32: b_i(S_k) (-1 if no j of S_k lies outside the
 *             window).  Required.
 *   arg_lvl   [n_levels][n_heads][T] int32: the maximising position, -1 if none.  Nullable.
 *   best_all, arg_all  as in twinkv_nn_scores.  Nullable; when both are NULL the tokens in
 *             no set are never swept as columns.
 *   workspace twinkv_levels_workspace_bytes(dtype, d, n_heads, n_seqs, cu_seqlens,
 *             n_levels, want_all) bytes, want_all = (best_all or arg_all given).
 * Other arguments as in twinkv_nn_scores.  Results equal those of separate
 * twinkv_nn_scores calls with retained = S_k, bit for bit: every value is the same
 * computation, and equal values go to the smaller position in both.
 */
int twinkv_nn_scores_levels(const void* keys, int dtype, int d, int n_heads, int n_seqs,
                            const int64_t* cu_seqlens, int64_t head_stride, int64_t token_stride,
                            const uint8_t* level, int n_levels, int w, float* best_all,
                            int32_t* arg_all, float* best_lvl, int32_t* arg_lvl, int32_t* status,
                            void* workspace, int64_t workspace_bytes, void* stream);

/* Workspace bytes of twinkv_nn_scores_levels; negative (-TWINKV_E_*) on invalid arguments. */
int64_t twinkv_levels_workspace_bytes(int dtype, int d, int n_heads, int n_seqs,
                                      const int64_t* cu_seqlens, int n_levels, int want_all);

/*
 * The standalone TwinKV scorer of Sec. 3.2: Eq. 2 twin counts, Eq. 3 scores
 * s_i = -r_i / n (n = the sequence length), and the retained set of the `budget` highest
 * scores.  The sink region [0, n_sink) and recent region [len - n_recent, len) take the
 * maximum score, so they are kept first; among equal scores the later position is kept
 * first (recency).  With budget >= len every token is kept; with budget 0 none.
 *
 *   budget        (host) [n_seqs] int64 in [0, 2^31 - 1]: tokens to keep per problem of
 *                 sequence s (the paper's ceil((1 - rho) n) for compression ratio rho is the
 *                 caller's).
 *   retained_out  [n_heads][T] uint8, receives the kept set as 0/1 (required).
 *   counts        [n_heads][T] int32, the Eq. 2 counts.  Nullable (then kept in workspace).
 *   scores        [n_heads][T] fp32, the Eq. 3 scores.  Nullable.
 *   stats         [n_heads * n_seqs][4] int32 = {tokens kept, count at the cut (-1 when the
 *                 cut falls inside the protected regions or nothing is cut), status, 0}.
 *                 A problem with a non-finite key (status NONFINITE) still keeps exactly its
 *                 budget, protected regions first; which other tokens is unspecified.
 *   workspace     twinkv_workspace_bytes(TWINKV_OP_SCORE_EVICT, ...) bytes.
 * Other arguments as in twinkv_twin_counts.
 */
int twinkv_score_evict(const void* keys, int dtype, int d, int n_heads, int n_seqs,
                       const int64_t* cu_seqlens, int64_t head_stride, int64_t token_stride,
                       const int64_t* budget, float tau, int w, int n_sink, int n_recent,
                       uint8_t* retained_out, int32_t* counts, float* scores, int32_t* stats,
                       void* workspace, int64_t workspace_bytes, void* stream);

/*
 * A score-based policy's retained set (Sec. 3.1: a policy keeps |S| = K positions per head
 * and layer; Sec. 3.2: the sink and recent regions take the maximum score): per problem,
 * the budget positions first in this order: protected positions (by position), then higher
 * scores, equal scores by lower position, NaN scores after every number (-0 equals +0).
 * With budget >= len every token is kept; with budget 0 none.  The result is the S0 that
 * twinkv_repair takes, so a wrapped policy that computes per-token scores on the GPU
 * (attention mass, an expected-attention estimate, a recency score) stays on the GPU.
 *
 *   scores        [n_heads][T] fp32 (any values, NaN and infinities included).
 *   budget        (host) [n_seqs] int64 in [0, 2^31 - 1]: tokens to keep per problem of
 *                 sequence s (values above the length keep everything).
 *   retained_out  [n_heads][T] uint8, receives the kept set as 0/1 (required).
 *   stats         [n_heads * n_seqs][4] int32 = {tokens kept, NaN scores, 0, 0}.  Nullable.
 *   workspace     twinkv_workspace_bytes(TWINKV_OP_REPAIR_FROM_SCORES, ...) bytes (the
 *                 sequence table).
 * Errors: NULL scores / budget / retained_out, a negative n_sink / n_recent or budget, or a
 * malformed cu_seqlens are rejected before anything is enqueued.
 */
int twinkv_select_topk(const float* scores, int n_heads, int n_seqs, const int64_t* cu_seqlens,
                       const int64_t* budget, int n_sink, int n_recent, uint8_t* retained_out,
                       int32_t* stats, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Twin prevalence (Sec. 2, Fig. 1b): for every problem q and threshold taus[k],
 *   out[q][k] = #{ tokens i of q : best_all[i] > taus[k] },
 * the number of tokens with at least one twin at that threshold (Eq. 2), from best_all as
 * produced by twinkv_nn_scores or twinkv_repair.
 *
 *   best_all  [n_heads][T] fp32.
 *   taus      (host) [n_taus] fp32, 1 <= n_taus <= TWINKV_MAX_TAUS.
 *   out       [n_heads * n_seqs][n_taus] int32.
 *   workspace  twinkv_workspace_bytes(TWINKV_OP_REPAIR_FROM_SCORES, ...) bytes (the sequence
 *              table).
 */
int twinkv_prevalence(const float* best_all, int n_heads, int n_seqs, const int64_t* cu_seqlens,
                      const float* taus, int n_taus, int32_t* out,
                      void* workspace, int64_t workspace_bytes, void* stream);

/*
 * KV compaction (Sec. 3.1): eviction keeps only the keys and values at the retained
 * positions.  For every problem (h, s) the rows of its retained tokens are copied, bit for
 * bit and in ascending position order, into the problem's `capacity[s]` reserved rows of a
 * dense cache; the usual caller passes S1 from twinkv_repair (or the scorer's retained set)
 * with capacity = the budget.
 *
 *   keys, values  [n_heads][T][d] bf16 or fp32 at (head_stride, token_stride) and
 *                 (v_head_stride, v_token_stride) elements (see Memory); d must be 64 or
 *                 128.  values may be NULL (keys only), and then values_out must be NULL.
 *   retained      [n_heads][T] uint8, nonzero = keep.
 *   capacity      (host) [n_seqs] int64, 0 <= capacity[s] <= length of sequence s: rows
 *                 reserved for each problem of sequence s.
 *   keys_out, values_out  [n_heads][C][d] dense, same dtype, 16-byte aligned,
 *                 C = sum of capacity.  Problem (h, s) owns rows [c_s, c_s + capacity[s]) of
 *                 head h, c_s = sum of capacity[s'] for s' < s.  Must not overlap the inputs.
 *   pos_out       [n_heads][C] int32: the position in the sequence of each row's token; -1
 *                 for unused rows.  Nullable.
 *   stats         [n_heads * n_seqs][4] int32 = {retained positions, capacity, status, 0};
 *                 status TWINKV_PROBLEM_BUDGET_MISMATCH when a problem retains more
 *                 positions than its capacity (then all its rows are zero, positions -1).
 *                 Reserved rows past the retained count are zero with position -1.
 *   workspace     twinkv_workspace_bytes(TWINKV_OP_COMPACT, ...) bytes.
 */
int twinkv_compact(const void* keys, const void* values, int dtype, int d, int n_heads,
                   int n_seqs, const int64_t* cu_seqlens, int64_t head_stride,
                   int64_t token_stride, int64_t v_head_stride, int64_t v_token_stride,
                   const uint8_t* retained, const int64_t* capacity, void* keys_out,
                   void* values_out, int32_t* pos_out, int32_t* stats, void* workspace,
                   int64_t workspace_bytes, void* stream);

/*
 * ---- The layer around the cache: what makes its keys, and what attends over it ----
 *
 * Rows of channels.  In the calls below q, k, v and their outputs are addressed like the keys above:
 * element (head, token, c) at p[head*head_stride + token*token_stride + c], pointer and byte strides
 * multiples of 16, so a projection's token-major output (head_stride = d, token_stride = heads*d) is
 * taken as it is.  An input may repeat one head (head_stride 0), outputs may not overlap (refused: a
 * head_stride below d, and heads that lie at least as far apart as tokens and meet; that the heads of a
 * token-major output end before its next token is the caller's to keep).  d is 64 or 128; bf16 or fp32, one
 * type in a call.  `group` query heads share a KV head: query head h*group + g reads KV head h.  These are
 * inference calls: none has a gradient.
 */

/*
 * Per-head RMS norm of queries and keys and the rotary position embedding (the keys as the cache
 * stores them, Sec. 3.2) in one pass.  With y = x * weight / sqrt(mean(x^2) + eps):
 *   out[c]       = y[c] * cos[c] - y[c + d/2] * sin[c]
 *   out[c + d/2] = y[c + d/2] * cos[c] + y[c] * sin[c],   c in [0, d/2).
 *
 *   q [n_q_heads][T][d], k [n_k_heads][T][d]; either may be NULL with 0 heads.  An output may be its
 *             input (same pointer and strides); any other overlap is not allowed.
 *   q_weight, k_weight  [d] fp32, 16-byte aligned.  Nullable, each: that side is not normalised (y = x).
 *   eps       finite, >= 0.
 *   rope      [n_pos][d] fp32, 16-byte aligned: cos for the d/2 channel pairs, then sin.  NULL: no
 *             rotation (positions is then not read).
 *   positions [T] int32: each token's row of the table.  A token whose position lies outside
 *             [0, n_pos) gets NaN in its outputs (its cache then reports TWINKV_PROBLEM_NONFINITE).
 * Everything is computed in fp32 and rounded once, to the output's type.
 */
int twinkv_qk_norm_rope(const void* q, const void* k, int dtype, int d, int n_q_heads, int n_k_heads,
                        int64_t T, int64_t q_head_stride, int64_t q_token_stride,
                        int64_t k_head_stride, int64_t k_token_stride, const float* q_weight,
                        const float* k_weight, float eps, const float* rope, int64_t n_pos,
                        const int32_t* positions, void* q_out, int64_t qo_head_stride,
                        int64_t qo_token_stride, void* k_out, int64_t ko_head_stride,
                        int64_t ko_token_stride, void* stream);

/*
 * Causal attention over a sliding window and the first tokens (sinks): the attention of a policy that
 * keeps n_sink leading and `window` trailing tokens.  Sequence s has query tokens [cu_q[s], cu_q[s+1])
 * and keys [cu_k[s], cu_k[s+1]); its queries are its last tokens: query i of m over n keys stands at
 * position p = n - m + i and sees the keys j <= p with p - j < window or j < n_sink.
 * A window >= n is plain causal attention; m = n a whole prompt, m = 1 a decode step.
 *
 *   out = softmax over the seen keys of (scale * q . k_j), times v_j.  A query that sees no key (window
 *         and n_sink 0, or p < 0) gets 0.
 *   lse   [n_heads*group][T_q] fp32: log of the sum of exp(scale * q . k_j); -inf where none is seen.
 *         Nullable.
 *   window, n_sink  >= 0.  scale finite.
 *   workspace  twinkv_attention_workspace_bytes(...) bytes (may be NULL when that is 0).
 * Scores, the running maximum and sums are fp32; for bf16 the weights are rounded to bf16 (to nearest)
 * for the product with v.  A key or value that a query does not see never changes its result, NaN and
 * infinities included.
 */
int twinkv_sink_attention(const void* q, const void* k, const void* v, int dtype, int d, int n_heads,
                          int group, int n_seqs, const int64_t* cu_q, const int64_t* cu_k,
                          int64_t q_head_stride, int64_t q_token_stride, int64_t k_head_stride,
                          int64_t k_token_stride, int64_t v_head_stride, int64_t v_token_stride,
                          int64_t window, int64_t n_sink, float scale, void* out,
                          int64_t out_head_stride, int64_t out_token_stride, float* lse,
                          void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Bytes of workspace twinkv_sink_attention needs for this batch; negative (-TWINKV_E_*) on invalid
 * arguments.  For twinkv_cache4_attention: cu_k = the cache's cu_rows, window = INT64_MAX, n_sink = 0.  One
 * figure serves both calls: the larger of what they may need.
 */
int64_t twinkv_attention_workspace_bytes(int dtype, int d, int n_heads, int group, int n_seqs,
                                         const int64_t* cu_q, const int64_t* cu_k, int64_t window,
                                         int64_t n_sink);

/*
 * A cache held in 4 bits.  Every 32 channels of a row share a scale 2^(byte - 127); an element is a
 * sign and one of 0, .5, 1, 1.5, 2, 3, 4, 6 (one sign, two exponent, one mantissa bit) times it:
 * 17/32 byte an element.  With a the largest magnitude of the 32, the byte is the smallest in [1, 252]
 * with a / scale < 7 (252 where none is); each element goes to the nearest value, ties to the even
 * code, magnitudes above 6 to 6.  32 channels of which one is NaN or infinite are stored as zeros, and the
 * problem reports TWINKV_PROBLEM_NONFINITE.
 *
 * Sequence s has rows [cu_rows[s], cu_rows[s+1]) of every head, a multiple of 32; how many of them are
 * in use is a count per problem (h, s), kept by the caller on the device (lengths may differ from head
 * to head).  C = cu_rows[n_seqs]; the four arrays are 16-byte aligned:
 *   k_codes   [n_heads][C][d/2]: byte b of a row holds channel 2b (low nibble) and 2b + 1
 *   k_scales  [n_heads][C][d/32]
 *   v_codes   [n_heads][C/8][d][4]: 8 rows a block; byte b of a channel holds rows 2b (low) and 2b + 1;
 *             place 64a + 4i + n holds channel 64a + 16n + i
 *   v_scales  [n_heads][C/8][d/32][8]
 * so that matrix operands are read 16 bytes a lane without reordering.  Unused rows may hold anything.
 */
typedef struct twinkv_cache4 {
  int d;                   /* 64 or 128 */
  int n_heads, n_seqs;
  const int64_t* cu_rows;  /* (host) [n_seqs + 1], consumed before the call returns */
  void* k_codes;
  void* k_scales;
  void* v_codes;
  void* v_scales;
} twinkv_cache4;

/* Bytes of workspace the three calls below need for n_seqs sequences (0 for small batches). */
int64_t twinkv_cache4_workspace_bytes(int n_seqs);

/*
 * twinkv_compact into a 4-bit cache: the keys and values at the retained positions of every problem,
 * in position order, as the first rows of its part of the cache.
 *
 *   keys, values  [n_heads][T][d] as in twinkv_compact; both required.  n_heads, n_seqs and d are the
 *                 cache's.
 *   retained      [n_heads][T] uint8, nonzero = keep.
 *   pos_out       [n_heads][C] int32: the position in the sequence of each row's token; -1 on rows not
 *                 in use.
 *   len_out       [n_heads * n_seqs] int32: rows in use (0 when the problem keeps more positions than
 *                 it has rows: TWINKV_PROBLEM_BUDGET_MISMATCH, nothing is stored).
 *   status        [n_heads * n_seqs] int32 TWINKV_PROBLEM_*.
 */
int twinkv_cache4_compact(const void* keys, const void* values, int dtype, const int64_t* cu_seqlens,
                          int64_t head_stride, int64_t token_stride, int64_t v_head_stride,
                          int64_t v_token_stride, const uint8_t* retained, const twinkv_cache4* cache,
                          int32_t* pos_out, int32_t* len_out, int32_t* status, void* workspace,
                          int64_t workspace_bytes, void* stream);

/*
 * Appends the keys and values of new tokens: those of sequence s, [cu_new[s], cu_new[s+1]), become rows
 * len .. of each of its problems.
 *
 *   len_in, len_out  [n_heads * n_seqs] int32: rows in use before and after.  May be the same array.
 *                    A problem whose new tokens do not fit (or whose len_in is negative) is left as it
 *                    is, len_out = len_in, with TWINKV_PROBLEM_BUDGET_MISMATCH.
 *   status           [n_heads * n_seqs] int32 TWINKV_PROBLEM_*.
 */
int twinkv_cache4_append(const void* keys, const void* values, int dtype, const int64_t* cu_new,
                         int64_t head_stride, int64_t token_stride, int64_t v_head_stride,
                         int64_t v_token_stride, const twinkv_cache4* cache, const int32_t* len_in,
                         int32_t* len_out, int32_t* status, void* workspace, int64_t workspace_bytes,
                         void* stream);

/*
 * The values that rows of the cache stand for (exact in both types), for a second repair of a cache
 * that has grown, or to move it: row r of sequence s in the output, r < cu_out[s+1] - cu_out[s], is
 * cache row first + r of the problem; rows outside [0, len) are zeros.
 *
 *   first     [n_heads * n_seqs] int32; NULL: 0.
 *   keys_out, values_out  [n_heads][cu_out[n_seqs]][d] dense, 16-byte aligned; either may be NULL.
 */
int twinkv_cache4_read(const twinkv_cache4* cache, const int32_t* len, const int32_t* first, int dtype,
                       const int64_t* cu_out, void* keys_out, void* values_out, void* workspace,
                       int64_t workspace_bytes, void* stream);

/*
 * Attention over a 4-bit cache: q [n_heads*group][T_q][d], the query tokens [cu_q[s], cu_q[s+1]) of
 * sequence s being the last tokens of its cache: query i of m sees rows [0, len - (m - 1 - i)) of each
 * problem (one query: all of them).  out and lse as in twinkv_sink_attention (0 and -inf where nothing
 * is seen); q and out are `dtype`.  len is taken as at most the problem's rows.
 * The products are exact in the cached values; scores, the running maximum and sums are fp32.  For bf16 the
 * weights, times the scales of their values, are rounded to bf16 (to nearest) for the product; for fp32 they
 * keep 24 bits.
 */
int twinkv_cache4_attention(const void* q, int dtype, int group, const int64_t* cu_q,
                            int64_t q_head_stride, int64_t q_token_stride, const twinkv_cache4* cache,
                            const int32_t* len, float scale, void* out, int64_t out_head_stride,
                            int64_t out_token_stride, float* lse, void* workspace,
                            int64_t workspace_bytes, void* stream);

/*
 * Profiling hook.  For calls made afterwards from the calling thread, record the given
 * hipEvent_t handles on the call's stream immediately before and immediately after the
 * launch of the call's main kernel -- the similarity kernel (the fused contraction +
 * reductions, with the short kernel that may follow it to write the results), or in twinkv_compact the row gather -- so its duration can be read with
 * hipEventElapsedTime.  The events stay owned by the caller; pass NULL, NULL to
 * stop recording.
 */
void twinkv_profile_sim_events(void* start_event, void* stop_event);

/* Static description of a return code (TWINKV_OK, TWINKV_E_*); never freed. */
const char* twinkv_status_string(int status);

/* Library version as major * 10000 + minor * 100 + patch. */
int twinkv_version(void);

#ifdef __cplusplus
}
#endif

#endif /* TWINKV_H */

/*
 * libe3 -- the per-token vocabulary pass, group advantages and temperature
 * scheduler of "E3" (arXiv 2505.18573) for AMD MI355X (gfx950).
 *
 * C ABI: plain pointers and sizes only.  Unless a parameter says "host", every
 * pointer is DEVICE memory on the current HIP device.  The caller owns all
 * buffers; the library never retains a pointer.  Device entry points only
 * enqueue work on `hip_stream` (a hipStream_t passed as void*, NULL = the
 * default stream) and return without synchronising: outputs are valid once the
 * stream has reached that point.  All argument checks happen on the host before
 * anything is launched; on error nothing is launched and outputs are untouched.
 * Results are bit-reproducible: the same call (same inputs, shapes and workspace
 * choice) gives the same bits in every run, since no floating-point atomics are
 * used and the order in which a row's columns are summed is fixed by the shape of
 * the launch.  A row that is part of a different batch (another number of rows, or
 * with / without a workspace) may run in a differently shaped launch: its token is
 * then the same except on near-ties, its entropy and log-prob the same up to fp32
 * rounding of the partial sums.
 *
 * Return value: 0 (E3_OK) or a negative e3_status.
 */
#ifndef E3_H
#define E3_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    E3_OK = 0,
    E3_ERR_NULL = -1,      /* a required pointer is NULL */
    E3_ERR_SHAPE = -2,     /* rows < 0, V < 1, row_stride < V, num_groups < 0 ... */
    E3_ERR_DTYPE = -3,     /* dtype is not an e3_dtype */
    E3_ERR_ALIGN = -4,     /* logits base or row pitch not 16-byte aligned */
    E3_ERR_VALUE = -5,     /* a scalar is outside its domain (tau <= 0, H <= 0, ...) */
    E3_ERR_WORKSPACE = -6, /* e3_sample_entropy_noalloc only: more rows than its scratch serves */
    E3_ERR_LAUNCH = -7     /* the HIP runtime refused a launch (see hipGetLastError) */
} e3_status;

typedef enum {
    E3_F32 = 0,
    E3_BF16 = 1,
    E3_E4M3 = 2            /* 8-bit floating point (OCP e4m3): the elements of an e3_cache only */
} e3_dtype;

/*
 * Column partition of the two-level sampler (see e3_sample_entropy).  Columns
 * are cut into chunks of E3_TILE_CHUNK; chunks are dealt round-robin to
 * E3_TILE_LANES slots; a tile is E3_TILE_DEPTH successive chunks of one slot:
 *   tile(i) = (i / (CHUNK*LANES*DEPTH)) * LANES + (i % (CHUNK*LANES)) / CHUNK.
 * These constants are part of the definition of the sampled token and are frozen:
 * the token drawn for a given (seed, row, logits) never changes with a later
 * version of the kernels (tests/golden/sampler_tokens.txt holds stored tokens).
 */
#define E3_TILE_CHUNK 8
#define E3_TILE_LANES 64
#define E3_TILE_DEPTH 8

/* Static, never-freed description of a status code (host). */
const char* e3_strerror(int status);

/*
 * Bytes of device workspace that e3_sample_entropy / e3_logprob_entropy can use
 * for a [rows, V] problem (pure host function; 0 for rows > 1024, at most 2 MiB).
 * The workspace is optional: with it, a small batch (too few rows to give every
 * compute unit whole rows of its own) is cut into runs of columns that are streamed
 * by many workgroups, their 32-byte partial results staged in the workspace and
 * merged by a second launch on the same stream; without it, or when it is smaller
 * than this bound or not 16-byte aligned, every row is streamed by one workgroup,
 * which is correct for any shape but slow for small batches.  Both ways compute the
 * same quantities; tokens can differ between them only on rows whose sampling race
 * is decided within fp32 rounding (the rows the near-tie rule below exempts).
 * The workspace holds no state between calls; calls that share one must be ordered
 * (same stream) because the merge reads what the first launch wrote.
 */
size_t e3_workspace_bytes(int64_t rows, int64_t V);

/*
 * Rollout side: sample one token per row at temperature tau_r and report its
 * log-probability and the entropy of the tau-scaled distribution.
 *
 *   a_i = z_i / tau_r,  p_i = exp(a_i) / sum_j exp(a_j)      (Appendix A, softmax)
 *   H   = -sum_i p_i ln p_i                                   (Appendix A, entropy;
 *         evaluated as ln S - W/S, the appendix's decomposition
 *         H = beta sum p_i Delta_i + ln Z(beta) in max-shifted form)
 *   tok ~ p by two-level Gumbel-max (the paper samples "at temperature tau",
 *         Section 5.1, without describing a sampler; this is the library's):
 *         tile T* = argmax_T ( ln sum_{i in T} exp(a_i) + g_T ),
 *         tok     = argmax_{i in T*} ( a_i + g_i ),  g = -ln(-ln u),
 *         u = ((w >> 9) + 1/2) 2^-23, w = word (index % 4) of
 *         Philox4x32-10( counter = (index/4, row lo, row hi, stream),
 *                        key = (seed lo, seed hi) ),
 *         stream 1 / index = tile id for g_T, stream 2 / index = column for g_i,
 *         row = row_base + r.  Exact ties go to the lowest index.  By
 *         max-stability of the Gumbel law P(tok = i) = p_i exactly.
 *   logp = a_tok - ln sum_j exp(a_j)
 *
 * logits      [rows, row_stride] elements of `dtype`, row-major, first V of each
 *             row used; base 16-byte aligned and row_stride*sizeof(elem) a
 *             multiple of 16 (else E3_ERR_ALIGN).  Values must be finite; a row
 *             holding NaN or +inf produces NaN outputs and an unspecified token
 *             in [0, V).  A row holding -inf produces a NaN entropy, and a
 *             log-prob and token that are unspecified unless it holds nothing
 *             else (NaN).  Mask with a finite value such as -1e9 instead.
 * tau_rows    [rows] fp32 or NULL; when NULL tau_scalar (host, finite, > 0, else
 *             E3_ERR_VALUE) applies to every row.  Per-row values are not checked:
 *             a row with tau <= 0 produces NaN outputs.
 * seed, row_base  host scalars; row_base is the global id of row 0, so results do
 *             not depend on how rows are batched.
 * token_out   [rows] int32;  logp_out, entropy_out [rows] fp32 (natural log).
 *             logp_out and entropy_out may be NULL.
 * workspace   device scratch of workspace_bytes bytes, or NULL (see
 *             e3_workspace_bytes); contents on entry are ignored.
 * V           at most 1,040,384 columns (per-workgroup tables must fit LDS),
 *             else E3_ERR_SHAPE.
 * rows == 0 is a no-op.  fp32 accumulation per lane, fp64 merges.
 */
int e3_sample_entropy(const void* logits, int dtype, int64_t rows, int64_t V, int64_t row_stride,
                      const float* tau_rows, float tau_scalar,
                      uint64_t seed, uint64_t row_base,
                      int32_t* token_out, float* logp_out, float* entropy_out,
                      void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * e3_sample_entropy for callers that cannot allocate device memory and therefore cannot
 * bring the optional workspace: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments (without the workspace pair), same
 * results bit for bit as e3_sample_entropy with a workspace of e3_workspace_bytes(rows, V):
 * the small-batch path stages its 32-byte row partials in a 2 MiB array that the library
 * holds in device memory for the life of the process (one copy per GPU it runs on, found
 * on this entry point's first call on that GPU).  The call allocates and frees nothing.
 *   rows  at most E3_NOALLOC_MAX_ROWS (what the array serves), else E3_ERR_WORKSPACE and
 *         nothing is launched; larger batches need no scratch at all: call
 *         e3_sample_entropy with workspace NULL.
 * All calls on one GPU share the array: calls that can overlap there (different streams,
 * different host threads) race on it and must be ordered by the caller; the array holds
 * no state between calls (every slot is written before it is read).
 */
#define E3_NOALLOC_MAX_ROWS 1024
int e3_sample_entropy_noalloc(const void* logits, int dtype, int64_t rows, int64_t V,
                              int64_t row_stride, const float* tau_rows, float tau_scalar,
                              uint64_t seed, uint64_t row_base,
                              int32_t* token_out, float* logp_out, float* entropy_out,
                              void* hip_stream);

/*
 * Rollout-side call with truncation: sample one token per row from the temperature-
 * scaled softmax restricted to the top-k and / or top-p (nucleus) part of the row.
 * The paper samples unrestricted (Section 5.1); this call covers the truncations that
 * rollout engines offer.  bf16 rows take every setting; fp32 rows need a count cut of
 * 1 <= top_k <= 256 (with or without top_p), anything else on fp32 rows is E3_ERR_VALUE.
 *
 * Definition (on value levels, so that it does not depend on the order of equal logits):
 *   a level is the set of columns storing one bit pattern; levels are ranked by value,
 *   highest first (-0 just below +0); level j has n_j columns and weight
 *   w_j = exp((z_j - z_1) / tau);  C_j = n_1 + .. + n_j,  M_j = n_1 w_1 + .. + n_j w_j.
 *   top_k >= 1: j_k = first j with C_j >= top_k (equal values at the cut are all kept);
 *               0, or >= V: no count cut.
 *   top_p < 1 : applied after top-k, to the distribution renormalised over levels
 *               1..j_k: j_p = first j <= j_k with M_j >= top_p * M_{j_k};  >= 1: j_p = j_k.
 *   The kept set is levels 1..j_p.  Draw: level = argmax_j n_j w_j / E_j with
 *   E_j = -ln u_j, u_j = uniform of Philox stream 3 at index = the level's bit pattern
 *   (same word -> uniform map as e3_sample_entropy; ties to the higher level); then
 *   with k the 23-bit integer of stream 4, index 0: pos = ((2k+1) n_j) >> 24 and the
 *   token is the pos-th column of the level in increasing column order.
 * Outputs: token_out [rows] int32; logp_out [rows] fp32 = ln of the token's probability
 *   under the truncated, renormalised distribution ((z_tok - z_1)/tau - ln M_{j_p});
 *   kept_out [rows] int32 = C_{j_p}.  logp_out and kept_out may be NULL.
 * Counts are exact; masses and the cuts are evaluated in fp64, the race scores in fp32.
 *   A row whose top_p target lies within 1e-9 (relative) of a cumulative mass may keep one
 *   level more or less than an fp64 reference with another summation order, and a row
 *   whose two best race scores lie within 1e-5 (relative) may draw the other level.
 * Logits must be finite (inf / NaN patterns are ignored as levels; a row without any
 *   finite logit gives token 0, logp NaN, kept 0).  Other arguments, alignment rules and
 *   errors as for e3_sample_entropy; top_k < 0 or top_p not in (0, inf): E3_ERR_VALUE.
 * One workgroup per row.  With 1 <= top_k <= 256 the row is read once (vectors that can hold
 * one of the k largest are listed in LDS while the row streams, exact selection among those); a
 * row with thousands of equal values at its cut is read several times.  Otherwise (bf16 only) the
 * row's stored patterns are counted in LDS: one counting sweep over a window of 31.5 binades of both signs, which ends at
 * 512 or at one binade above what a sample of the row shows, whichever is higher.  The sample is the row's first 16,384 columns,
 * or 32,768 where sixteen waves stream a row (at least 114,688 columns, at most one row per compute unit).  A second sweep over
 * a higher or lower window follows for a row with finite logits above the first one, or with more than 62 columns
 * nearer to zero than the window reaches (1.5 x 2^-23 in the usual one) without being zero.
 * The rare rows that take four to ten more sweeps, over all patterns: a second window that
 * does not hold them either; a level of 65,536 or more columns in a quarter of the row; columns below
 * -512 (or below the window) that still weigh something, i.e. that are less than 56 tau below the
 * largest logit; a count cut among columns there that are not all equal.
 */
int e3_sample_restricted(const void* logits, int dtype, int64_t rows, int64_t V, int64_t row_stride,
                         const float* tau_rows, float tau_scalar, int32_t top_k, float top_p,
                         uint64_t seed, uint64_t row_base,
                         int32_t* token_out, float* logp_out, int32_t* kept_out, void* hip_stream);

/*
 * e3_sample_restricted with an optional workspace (device, 16-byte aligned, contents on entry ignored, no
 * state between calls, to be used by one call at a time): with e3_restricted_workspace_bytes of it a small batch is
 * cut into slices of columns that many workgroups read, and a second launch on the same stream
 * finishes the rows.  Without it, or with less, every row is read by one workgroup as in
 * e3_sample_restricted.  Same tokens (but for the near-ties above), counts and log-probs up to rounding in either form.
 * The window of cut rows is chosen by 512 columns spread over the row, and also lies lower than the usual one where these
 * hold small values only; a row that does not fit it is swept once more by one workgroup.
 * e3_restricted_workspace_bytes: host only; 0 where a workspace would not be used.
 */
size_t e3_restricted_workspace_bytes(int dtype, int64_t rows, int64_t V, int32_t top_k);
int e3_sample_restricted_ws(const void* logits, int dtype, int64_t rows, int64_t V, int64_t row_stride,
                            const float* tau_rows, float tau_scalar, int32_t top_k, float top_p,
                            uint64_t seed, uint64_t row_base,
                            int32_t* token_out, float* logp_out, int32_t* kept_out,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Training side: log-probability of a given token and the entropy of each row,
 * with the logits divided by the temperature as in the policy forward pass (end
 * of the "Temperature Scheduler" paragraph of Section 4.2), plus the two numbers
 * from which the batch-mean entropy H_t of Eq. 4 follows.
 *
 * target_ids  [rows] int32 or NULL; an id outside [0, V) gives logp = NaN.
 *             NULL requires logp_out == NULL.
 * row_mask    [rows] uint8 or NULL; rows with mask 0 (padding) are still written
 *             to logp_out/entropy_out but excluded from the batch sum.
 * logp_out    [rows] fp32 or NULL;  entropy_out [rows] fp32 (required).
 * entropy_sum_out    one double or NULL: sum of entropy_out over kept rows,
 *             accumulated in fp64 in a fixed order.
 * entropy_count_out  one int64 or NULL: number of kept rows.
 *             These two are each written once, by one plain store at the end of the
 *             last kernel, so they may also point into pinned host memory that the
 *             device can address (hipHostMalloc): the host then reads H_t's two
 *             numbers after waiting on an event recorded behind this call, without a
 *             copy in between.
 * Other arguments as for e3_sample_entropy.
 */
int e3_logprob_entropy(const void* logits, int dtype, int64_t rows, int64_t V, int64_t row_stride,
                       const int32_t* target_ids, const uint8_t* row_mask,
                       const float* tau_rows, float tau_scalar,
                       float* logp_out, float* entropy_out,
                       double* entropy_sum_out, int64_t* entropy_count_out,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * e3_logprob_entropy that also measures, in the same pass, the logit gap Delta of
 * Appendix A on every row: the paper's update is tau1 = tau0 (1 + tau0 ln(alpha) /
 * Delta) and it replaces Delta by ln N + ln ln N only because measuring it would cost
 * another pass over the logits; here it is a by-product of the sums already taken.
 *   gap_r = sum_{i != i*} p_i (z_max - z_i) / sum_{i != i*} p_i        (logit units)
 * with i* one index attaining the row maximum and p = softmax(z / tau_r); it equals
 * Delta exactly on the appendix's two-level model and satisfies the appendix's
 * decomposition H = beta (1 - p_max) gap + ln Z.  A one-column row gives NaN.
 * gap_out      [rows] fp32 or NULL.
 * gap_sum_out  one double (device) or NULL (needs gap_out): sum of gap_out over kept
 *              rows, fp64, fixed order.  count_out as entropy_count_out.
 */
int e3_logprob_entropy_gap(const void* logits, int dtype, int64_t rows, int64_t V, int64_t row_stride,
                           const int32_t* target_ids, const uint8_t* row_mask,
                           const float* tau_rows, float tau_scalar,
                           float* logp_out, float* entropy_out, float* gap_out,
                           double* entropy_sum_out, double* gap_sum_out, int64_t* count_out,
                           void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Group-relative advantage, Eq. 2:  A_i = (r_i - mean(r)) / std(r) over the
 * rollouts of one prompt, groups stored CSR-style because Algorithm 1 gives each
 * prompt its own rollout budget.
 *
 * rewards        [N] fp32, N = group_offsets[num_groups].
 * group_offsets  [num_groups + 1] int32, non-decreasing, group_offsets[0] = 0
 *                (caller's contract; not checked on the device).  Empty groups
 *                write nothing.
 * ddof           0 = population standard deviation (the literal formula),
 *                1 = Bessel-corrected.
 * eps            >= 0, added to the standard deviation.
 * adv_out        [N] fp32.  A group whose rewards are all identical (exact
 *                compare; includes groups of one) gets 0 for every rollout
 *                (Section 4.2: identical rewards give zero advantage).
 * Sums are taken in fp64.  num_groups == 0 is a no-op.
 */
int e3_grpo_advantages(const float* rewards, const int32_t* group_offsets,
                       int32_t num_groups, int32_t ddof, float eps,
                       float* adv_out, void* hip_stream);

/*
 * e3_logprob_entropy and e3_grpo_advantages in one call: the two sets of statistics a
 * GRPO update needs of a batch of finished rollouts (Eq. 2's advantages from the
 * rewards; log-probabilities and entropies from the logits, Section 4.2).  Results are
 * bit for bit those of the two separate calls.  When the batch runs as whole rows per
 * workgroup and there are at most as many groups as workgroups, the groups are computed
 * inside the vocabulary pass's launch by waves that have time to spare, which saves a
 * launch; otherwise they get a launch of their own first.  Arguments as for the two
 * calls; num_groups == 0 makes it e3_logprob_entropy.
 */
int e3_logprob_entropy_advantages(const void* logits, int dtype, int64_t rows, int64_t V,
                                  int64_t row_stride, const int32_t* target_ids,
                                  const uint8_t* row_mask, const float* tau_rows, float tau_scalar,
                                  float* logp_out, float* entropy_out,
                                  double* entropy_sum_out, int64_t* entropy_count_out,
                                  const float* rewards, const int32_t* group_offsets,
                                  int32_t num_groups, int32_t ddof, float eps, float* adv_out,
                                  void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Forward value of the GRPO objective, Eq. 1 without the KL term (which the paper
 * drops, Section 3.1):
 *   J = mean_q (1/G_q) sum_{i in q} (1/|o_i|) sum_t min( r A_i , clip(r, 1-eps, 1+eps) A_i ),
 *   r = exp(logp_new[t] - logp_old[t]).
 * logp_new, logp_old  [T] fp32: log-probs of the rollout tokens under the current and
 *                     the sampling policy (e3_logprob_entropy / e3_sample_entropy).
 * seq_offsets    [num_seqs + 1] int32: token range of each rollout (CSR).
 * adv            [num_seqs] fp32: per-rollout advantage (e3_grpo_advantages).
 * group_offsets  [num_groups + 1] int32: rollout range of each question (CSR; the
 *                same array e3_grpo_advantages takes).  group_offsets[num_groups]
 *                must equal num_seqs (caller's contract).
 * clip_eps       >= 0 (E3_ERR_VALUE otherwise).
 * token_term_out [T] fp32 or NULL: the per-token min(...) term.
 * seq_mean_out   [num_seqs] fp64, required: per-rollout mean term (0 for an empty
 *                rollout); also the staging buffer of the two-stage reduction.
 * objective_out  one double (device), required.  An empty group contributes 0 and
 *                still counts in the mean over questions; num_groups == 0 gives 0.
 * Sums in fp64 in a fixed order.
 */
int e3_grpo_objective(const float* logp_new, const float* logp_old, const int32_t* seq_offsets,
                      const float* adv, int32_t num_seqs, const int32_t* group_offsets,
                      int32_t num_groups, float clip_eps, float* token_term_out,
                      double* seq_mean_out, double* objective_out, void* hip_stream);

/*
 * Temperature scheduler, host only (no GPU work, all pointers are HOST):
 *   H_target = H_init                                      for t < t_anneal or t_anneal < 0
 *            = H_init [eta + (1-eta)(1 + cos(pi x))/2]      otherwise (Eq. 5),
 *              x = clamp((t - t_anneal)/(t_max - t_anneal), 0, 1), x = 1 if t_max <= t_anneal
 *   alpha    = H_target / H_t
 *   tau_next = tau_t (1 + tau_t ln(alpha) / (ln|V| + ln ln|V|))               (Eq. 4)
 * then clamped to [tau_min, tau_max]; (0, +inf) leaves Eq. 4 untouched.
 * E3_ERR_VALUE if tau_t, H_t, H_init are not finite and > 0, vocab < 3, eta
 * outside [0,1], tau_min < 0, tau_max < tau_min, or the factor is <= 0 while
 * tau_min == 0.  On error the outputs are untouched.
 * tau_next_out required; H_target_out may be NULL.
 */
int e3_temperature_update(double tau_t, double H_t, double H_init, int64_t vocab,
                          int64_t t, int64_t t_anneal, int64_t t_max, double eta,
                          double tau_min, double tau_max,
                          double* tau_next_out, double* H_target_out);

/*
 * The same update with a measured gap instead of ln|V| + ln ln|V| (Appendix A, the
 * relation tau1 = tau0 (1 + tau0 ln(alpha) / Delta)); host only.  `gap` is the batch
 * mean of e3_logprob_entropy_gap's gap_out and must be finite and > 0; all else as
 * e3_temperature_update.
 */
int e3_temperature_update_gap(double tau_t, double H_t, double H_init, double gap,
                              int64_t t, int64_t t_anneal, int64_t t_max, double eta,
                              double tau_min, double tau_max,
                              double* tau_next_out, double* H_target_out);

/*
 * Difficulty ranking of the training questions, host only (Section 4.1): questions
 * are ranked by average reward cum_reward[i] / cum_rollouts[i] in descending order
 * and k_i = rank / num_questions, rank counted from 1, so the question answered worst
 * gets k = 1.  Equal averages rank in index order; a question with no rollouts yet
 * counts as average 0.  All pointers are HOST arrays of num_questions entries.
 * E3_ERR_VALUE for a negative rollout count or a NaN average.
 */
int e3_difficulty_ranks(const double* cum_reward, const int64_t* cum_rollouts,
                        int64_t num_questions, double* k_out);

/*
 * Algorithm 1 (Dynamic Rollout Budget), host only.  Given the normalised rankings
 * k[B] of a batch, the default budget G and the bounds G_min <= G <= G_max: every
 * question starts at G_min, the remaining B*G - B*G_min rollouts are split in
 * proportion to k_i (rounded down, capped at G_max), and what is left over is handed
 * out in passes over the questions in descending k (ties: lower index first), one
 * rollout per question per pass, skipping questions at G_max.  sum G_out = B*G.
 * G_out       [B] int32 (host).
 * offsets_out [B+1] int32 (host) or NULL: the CSR group offsets (prefix sums of
 *             G_out) in the form e3_grpo_advantages takes.
 * E3_ERR_VALUE unless G_min <= G <= G_max, k finite and >= 0 with a positive sum.
 */
int e3_allocate_budgets(const double* k, int32_t B, int32_t G, int32_t G_min, int32_t G_max,
                        int32_t* G_out, int32_t* offsets_out);

/*
 * Bounds curriculum, host only (end of Section 4.1): G_min and G_max start at G and
 * after each completed pass over the data move outwards by `step` until they reach
 * G_min_limit / G_max_limit (the paper's runs: G = 8, step 2, limits 4 and 12).
 */
int e3_budget_bounds(int32_t G, int32_t passes_done, int32_t step, int32_t G_min_limit,
                     int32_t G_max_limit, int32_t* G_min_out, int32_t* G_max_out);

/* ------------------------------------------------------------------------------------
 * The decode step in front of the sampler: a paged cache of keys and values, the
 * attention of rollouts that share their question's prompt, the verification of drafted
 * tokens.  (Section 4.1 gives every question its own number of rollouts, all of the same
 * prompt: the groups are the CSR groups that e3_grpo_advantages takes.)
 * ------------------------------------------------------------------------------------ */

/*
 * A paged cache (the struct itself is host memory, the arrays are device memory):
 *   k  [num_pages][kv_heads][page_size][head_dim]
 *   v  [num_pages][kv_heads][page_size / 8][head_dim][8]     (eight tokens of a column together)
 * of bf16, or of e4m3 codes with one exponent per token and head in
 *   k_scale, v_scale  [num_pages][kv_heads][page_size] uint8  (NULL for bf16):
 * element = code * 2^(scale - 127).  Token s of the cache ("slot") is token s % page_size of
 * page s / page_size.
 * page_size is a power of two of at least 32, head_dim 64 or 128 (else E3_ERR_SHAPE); k and v
 * are 16-byte, the scales 8-byte aligned (else E3_ERR_ALIGN).
 */
typedef struct {
    void* k;
    void* v;
    uint8_t* k_scale;
    uint8_t* v_scale;
    int64_t num_pages;
    int32_t page_size, kv_heads, head_dim;
    int32_t dtype;                 /* E3_BF16 or E3_E4M3 */
} e3_cache;

/*
 * Write the keys and values of `tokens` tokens into the cache, quantising them where it holds
 * 8 bits.  Per token, head and tensor, x being the head_dim elements:
 *   a = largest finite |x_i|,   e = smallest integer in [-126, 127] with a <= 448 * 2^e,
 *   code_i = e4m3(x_i * 2^-e), nearest, ties to even,   scale byte = e + 127.
 * Scaling by a power of two is exact, nothing saturates, and values that are read back and
 * written again keep their bits (but for magnitudes from 2^128 (1 - 2^-5) on, which round to
 * 2^128 and read back as inf).  Elements that are not finite become the NaN code and do
 * not enter a.  In a bf16 cache fp32 input is rounded (nearest, ties to even).
 *
 * k, v      [tokens][kv_heads][head_dim] of dtype (E3_BF16 / E3_F32), strides in elements,
 *           columns next to each other; base and strides multiples of 16 bytes (E3_ERR_ALIGN).
 * slots     [tokens] int64: where each goes.  A slot outside the cache (negative, say: padding)
 *           is skipped.  Slots are expected to differ within a call; which of two tokens with one
 *           slot is kept is not specified (elements and scale may then be of different tokens).
 * tokens == 0 is a no-op; tokens * kv_heads is at most 2^28 (E3_ERR_SHAPE), here and in e3_cache_read.
 */
int e3_cache_append(const e3_cache* cache, const void* k, const void* v, int dtype, int64_t tokens,
                    int64_t k_token_stride, int64_t k_head_stride,
                    int64_t v_token_stride, int64_t v_head_stride,
                    const int64_t* slots, void* hip_stream);

/*
 * Read tokens back: k_out, v_out [tokens][kv_heads][head_dim] contiguous, of dtype (E3_BF16 /
 * E3_F32), 16-byte aligned.  Exact in fp32, and in bf16 down to its smallest normal number.
 * A slot outside the cache reads as zeros.
 */
int e3_cache_read(const e3_cache* cache, const int64_t* slots, int64_t tokens,
                  void* k_out, void* v_out, int dtype, void* hip_stream);

/*
 * Rotary positions (the struct is host memory, its arrays device memory).  Pair i of rot_dim / 2 is turned by
 *   theta_i = positions[axis[i]][token] * freqs[i]:   y1 = x1 cos - x2 sin,  y2 = x2 cos + x1 sin.
 * freqs     [rot_dim / 2] fp64: radians per position.
 * axis      [rot_dim / 2] uint8, or NULL with axes == 1: which of the token's positions a pair goes by (a text's place; time,
 *           height and width of a picture's part).  Columns may be given to axes in blocks, in turn or in any other way.  A
 *           pair whose axis is not below `axes` stays as it is.
 * rot_dim   columns that are turned, the first ones: a multiple of 16, at most head_dim; those behind are copied.
 * axes      1 .. E3_MAX_AXES.
 * neighbours  0: pair i is columns i and i + rot_dim / 2;  1: columns 2 i and 2 i + 1.
 * Positions are int64, [axes][tokens], rows position_stride elements apart, and may be negative; angles are exact to far below fp32's
 * rounding for |position| < 2^52.
 */
#define E3_MAX_AXES 8
typedef struct {
    const double* freqs;
    const uint8_t* axis;
    int32_t rot_dim, axes, neighbours;
} e3_rotary;

/*
 * Turn rows of heads: out = R(theta) x, or with inverse = 1 R(-theta) x, which is R's transpose: the gradient with respect
 * to x where x stands for the gradient with respect to R x.
 *
 * x, out    [tokens][heads][head_dim] of dtype (E3_BF16 / E3_F32), strides in elements, columns next to each other (computed in
 *           fp32 and rounded once); bases and strides multiples of 16 bytes (E3_ERR_ALIGN).  out may be x with the same strides (other strides: E3_ERR_VALUE); they may not
 *           overlap in any other way.
 * tokens at most 2^25, heads at most 65,536, head_dim a multiple of 8 from 16 to 1024 (E3_ERR_SHAPE).
 */
int e3_rotate(const e3_rotary* rotary, const int64_t* positions, int64_t position_stride, const void* x, int dtype,
              int64_t tokens, int64_t heads, int64_t head_dim, int64_t x_token_stride, int64_t x_head_stride,
              void* out, int64_t out_token_stride, int64_t out_head_stride, int inverse, void* hip_stream);

/*
 * e3_cache_append with the keys turned on the way (in fp64, rounded or quantised once), and the same tokens' queries turned beside them
 * in the same launch.  Values are stored as they are.
 * q, q_out  [tokens][q_heads][head_dim] of dtype, as x and out of e3_rotate; q_heads == 0: keys and values only, both may be NULL.
 *           The queries of tokens whose slot is outside the cache are turned too.
 * tokens    at most 2^25; other arguments as for e3_cache_append and e3_rotate.
 */
int e3_cache_append_rotated(const e3_cache* cache, const e3_rotary* rotary, const int64_t* positions, int64_t position_stride,
                            const void* q, const void* k, const void* v, int dtype, int64_t tokens, int64_t q_heads,
                            int64_t q_token_stride, int64_t q_head_stride, int64_t k_token_stride, int64_t k_head_stride,
                            int64_t v_token_stride, int64_t v_head_stride, const int64_t* slots,
                            void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void* hip_stream);

/*
 * Attention of one decode step.  Row r belongs to group g (group_offsets[g] <= r <
 * group_offsets[g + 1]) and attends to the group's prefix, all of it, and to its own tokens, of
 * which the last `queries` are the step's own: query t sees the first
 * row_lens[r] - (queries - 1 - t).
 *   s_j = scale q . k_j,   out = sum_j softmax(s)_j v_j,   lse = ln sum_j exp(s_j)
 * Query head h reads key head h / (q_heads / kv_heads).  A query without any key (prefix and own
 * tokens empty) gives 0 and -inf.  The prefix is read once for all rows of the group.
 *
 * q             [rows][queries][q_heads][head_dim] bf16, strides in elements, columns next to
 *               each other; base and strides multiples of 16 bytes (E3_ERR_ALIGN).
 * rows, queries, q_heads   q_heads a multiple of kv_heads (E3_ERR_SHAPE); one query per row is
 *               the ordinary step, more are drafted tokens to be verified: few of them, since every tile
 *               of queries reads all of the row's tokens.  rows * kv_heads below 2^24.
 * group_offsets [num_groups + 1] int32, group_offsets[num_groups] = rows (the caller's contract);
 *               NULL with num_groups == 0: no prefixes.  A row in no group has none.
 * prefix_pages  [num_groups][prefix_width] int32, prefix_lens [num_groups] int32 (tokens).
 * row_pages     [rows][row_width] int32, row_lens [rows] int32 (tokens, the step's included).
 *               Lengths are cut to what the tables can hold; a page id outside the cache
 *               hides its tokens.  Table entries behind a length are not read.  Whatever the cache
 *               holds behind a length (NaN included) has no influence.
 * Elements that are not finite: one of V, infinite ones too, makes its column of every query that sees it NaN
 *               (or infinite), one of K or q the queries' rows NaN (a score of -inf is a weight of zero).
 *               Sums are divided at the end and weights reach 2^8 in them: a sum of 2^128 and more overflows,
 *               which values of V below 2^119 / (tokens that a query sees) cannot reach.
 * scale         host, finite and > 0 (E3_ERR_VALUE).
 * out           [rows][queries][q_heads][head_dim] bf16, contiguous, 16-byte aligned.
 * lse_out       [rows][queries][q_heads] fp32 or NULL.
 * workspace     device, 256-byte aligned (E3_ERR_ALIGN), at least
 *               e3_prefix_attention_workspace_bytes() (else E3_ERR_WORKSPACE); contents on entry
 *               ignored, no state between calls, to be used by one call at a time.
 * Scores, maxima, weights, sums and the output's sums in fp32.  Where the keys are cut into runs depends on the lengths, so a row in another
 * batch may differ in the last bits; the same call gives the same bits.
 * e3_prefix_attention_workspace_bytes: host only; 0 for a shape that is not served.
 */
size_t e3_prefix_attention_workspace_bytes(int64_t rows, int64_t queries, int64_t q_heads, int64_t kv_heads,
                                           int64_t head_dim, int64_t num_groups);
int e3_prefix_attention(const e3_cache* cache, const void* q, int64_t rows, int64_t queries, int64_t q_heads,
                        int64_t q_row_stride, int64_t q_token_stride, int64_t q_head_stride,
                        const int32_t* group_offsets, int64_t num_groups,
                        const int32_t* prefix_pages, int64_t prefix_width, const int32_t* prefix_lens,
                        const int32_t* row_pages, int64_t row_width, const int32_t* row_lens,
                        float scale, void* out, float* lse_out,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Attention with a sliding window and first tokens that stay visible, for rows of any numbers of queries: new tokens, drafted
 * ones, prompts or pieces of them, in one call.  Row r brings queries query_offsets[r] .. query_offsets[r + 1] - 1, the last ones of its row_lens[r]
 * tokens (whose keys are in the cache already); the one that is token p of the row sees token j <= p if
 *   j > p - window   or   j < sinks.
 * s_j, out and lse as for e3_prefix_attention.  Query head h reads key head h / (q_heads / kv_heads).  A query that sees nothing (of a row with
 * fewer tokens than queries) gives 0 and -inf.
 *
 * q             [tokens][q_heads][head_dim] bf16, strides in elements, columns next to each other; base and strides multiples of 16
 *               bytes (E3_ERR_ALIGN).
 * tokens, q_heads   q_heads a multiple of kv_heads, tokens * q_heads below 2^31, rows * kv_heads below 2^24 (E3_ERR_SHAPE).
 * query_offsets [rows + 1] int32, from 0 on, not falling, at most `tokens` (the caller's contract).  Rows without queries are allowed; out
 *               and lse_out of queries behind query_offsets[rows] are left as they are.
 * row_pages     [rows][row_width] int32, row_lens [rows] int32 (tokens, the queries' own included).  Lengths are cut to what the table can hold;
 *               a page id outside the cache hides its tokens.  Entries of pages of which no query of the row sees a token are not
 *               used: such pages may have been given to others.  Whatever the cache holds in tokens that a query does not see
 *               (NaN included) has no influence on it.
 * window        at least 1; sinks at least 0 (E3_ERR_VALUE).  A window of any row's length and more is plain causal attention.
 * Elements that are not finite, scale, out [tokens][q_heads][head_dim], lse_out [tokens][q_heads], workspace (at least
 *               e3_window_attention_workspace_bytes()): as for e3_prefix_attention.
 * Scores, maxima, sums and outputs' sums in fp32.  Weights enter their product with all of fp32's bits for rows of at most 32 queries
 * times (q_heads / kv_heads), with 16 of them at least (off by 2^-17 of themselves) for larger ones.  Where the keys are cut into runs depends on
 * the whole batch, so a row in another batch may differ in the last bits; the same call gives the same bits.
 * e3_window_attention_workspace_bytes: host only; 0 for a shape that is not served.
 */
size_t e3_window_attention_workspace_bytes(int64_t rows, int64_t tokens, int64_t q_heads, int64_t kv_heads, int64_t head_dim);
int e3_window_attention(const e3_cache* cache, const void* q, int64_t tokens, int64_t q_heads, int64_t q_token_stride, int64_t q_head_stride,
                        const int32_t* query_offsets, int64_t rows,
                        const int32_t* row_pages, int64_t row_width, const int32_t* row_lens,
                        int64_t window, int64_t sinks, float scale, void* out, float* lse_out,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Verification of drafted tokens (speculative sampling) with what a rollout keeps of every token.
 * A row brings `drafts` drafted tokens x_0 .. and the target's logits at drafts + 1 positions
 * (position t: given x_0 .. x_{t-1}).
 *   p_t = softmax(z_t / tau_r),   q_t = softmax(d_t / tau'_r), or the point mass on x_t when there are
 *         no draft logits (drafts looked up rather than sampled)
 *   draft t is accepted while u_t q_t(x_t) < p_t(x_t);   n = number of accepted drafts
 *   the token after them ~ (p_n - q_n)+ / sum (p_n - q_n)+ if draft n was rejected,  ~ p_n if none was
 *   (if p_n exceeds q_n nowhere, rounding aside they are equal: ~ p_n).
 * u_t is the uniform of e3_sample_entropy's map at Philox stream 5, index t; the draw is its two-level
 * race with r_i = (p_i - q_i)+ for exp(a_i), streams 6 (tiles) and 7 (columns):
 *   T* = argmax_T (sum_{i in T} r_i) / E_T,   token = argmax_{i in T*} r_i / E_i.
 * Random numbers are thus given by seed and row_base + r; a new step takes a new seed (or row_base).
 *
 * logits        [rows][drafts + 1][V] of dtype (E3_F32 / E3_BF16), strides in elements; base and
 *               strides multiples of 16 bytes (E3_ERR_ALIGN), position_stride >= V.
 * draft_logits  [rows][drafts][V] of the same dtype, or NULL.
 * draft_tokens  [rows][drafts] int32 (NULL only when drafts == 0).  An id outside [0, V) is rejected.
 * draft_lens    [rows] int32 or NULL: drafts of each row (cut to 0 .. drafts); positions behind a
 *               row's last draft and the one after it are not read.
 * drafts        0 .. E3_MAX_DRAFTS; rows * (drafts + 1) below 2^23 (E3_ERR_SHAPE).
 * tau_rows, tau_scalar  as for e3_sample_entropy;  draft_tau_rows [rows] or NULL: the drafts'
 *               temperature, NULL: the target's.
 * accepted_out  [rows] int32 = n.
 * token_out     [rows][drafts + 1] int32: the n drafts and the token after them, then -1.
 * logp_out, entropy_out  [rows][drafts + 1] fp32 or NULL: ln p_t of token t and the entropy of p_t for
 *               the n + 1 tokens, then 0: what e3_sample_entropy reports of a sampled token.
 * A logit of -inf, or of -1e30 and less, has no probability.  A position whose target logits hold
 * NaN or +inf, or no finite value, is rejected with an unspecified token in [0, V) and NaN outputs;
 * one whose draft logits do is rejected and drawn from p.
 * V             at most 1,040,384.
 * workspace     device, 256-byte aligned (E3_ERR_ALIGN), at least e3_verify_workspace_bytes()
 *               (else E3_ERR_WORKSPACE); contents on entry ignored, no state between calls, to be
 *               used by one call at a time.
 * Sums in fp32 per lane, merged in fp64; decisions in fp64.  A row whose decision or race lies within
 * fp32 rounding may fall the other way in a batch of another size; the same call gives the
 * same bits.
 */
#define E3_MAX_DRAFTS 63
size_t e3_verify_workspace_bytes(int64_t rows, int32_t drafts, int64_t V);
int e3_verify_drafts(const void* logits, int dtype, int64_t rows, int32_t drafts, int64_t V,
                     int64_t row_stride, int64_t position_stride,
                     const int32_t* draft_tokens, const int32_t* draft_lens,
                     const void* draft_logits, int64_t draft_row_stride, int64_t draft_position_stride,
                     const float* tau_rows, float tau_scalar, const float* draft_tau_rows,
                     uint64_t seed, uint64_t row_base,
                     int32_t* accepted_out, int32_t* token_out, float* logp_out, float* entropy_out,
                     void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Beam search: the best continuations of every sequence over its beams and the vocabulary.
 *   score(b, v) = scores[b] + z_bv / tau - ln sum_i exp(z_bi / tau)
 * The `keep` candidates with the largest scores, largest first; equal scores go to the lower beam, then to the lower token.  A finished beam
 * offers one candidate, eos_token with its score as it is.
 *
 * logits        [seqs][beams][V] of dtype (E3_F32 / E3_BF16), strides in elements; base and strides multiples of 16 bytes (E3_ERR_ALIGN),
 *               beam_stride >= V.  Rows of finished beams and of beams without a finite score are not read.
 * beams         1 .. E3_MAX_BEAMS;  keep  1 .. E3_MAX_KEEP (twice the beams where finished ones are sorted out behind the call);
 * V             at most 1,040,384; seqs below 2^22, and logits of at most 2^36 elements or so (E3_ERR_SHAPE: no workspace size).
 * scores        [seqs][beams] fp32: sums of log-probs so far; -inf (or NaN): the beam offers nothing (all but one in a first step).
 * tau           host, finite and > 0 (E3_ERR_VALUE).
 * finished      [seqs][beams] uint8 or NULL, with eos_token in [0, V) (E3_ERR_VALUE).
 * parent_out, token_out [seqs][keep] int32, score_out [seqs][keep] fp32.  Places without a candidate: -1, -1, -inf.
 * A logit of -inf, or of -1e30 and less, has no probability and is never chosen.  A beam whose logits hold NaN or +inf offers nothing, nor
 * does any that is not finished where log2(e) / tau is beyond fp32.
 * Scores are compared in fp64.  Where the order between two beams lies within 2e-6 the sums over their vocabularies are taken in
 * fp64 as well; beyond, fp32 sums decide, whose error is below that, wherever the logits lie, but for rows built to add up roundings.
 * workspace     device, 256-byte aligned (E3_ERR_ALIGN), at least e3_beam_workspace_bytes() (else E3_ERR_WORKSPACE); contents on entry ignored, no
 *               state between calls, to be used by one call at a time.
 */
#define E3_MAX_BEAMS 32
#define E3_MAX_KEEP 64
size_t e3_beam_workspace_bytes(int64_t seqs, int32_t beams, int64_t V);
int e3_beam_select(const void* logits, int dtype, int64_t seqs, int32_t beams, int64_t V, int64_t seq_stride, int64_t beam_stride,
                   const float* scores, int32_t keep, float tau, const uint8_t* finished, int32_t eos_token,
                   int32_t* parent_out, int32_t* token_out, float* score_out,
                   void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * The beams' pages after a selection: row r of a sequence goes on where its parent was.  Rows of one sequence share the pages that are
 * full and own the one that their next token goes to (entry row_lens[r] / page_size).  A parent's first child goes on in
 * that page; every other child takes over the page of a beam without children (there are as many), into which the parent's tokens are to be
 * copied: by e3_cache_copy, once for every layer's cache.
 * All other entries are the parent's, those behind that page too: rows with the same parent name the same pages there.  Where tables are
 * filled ahead they have to be set anew before a row's tokens reach them, to pages that no other row names (if a sequence's rows have the
 * same length: to those that the row had there before the call).
 *
 * parent        [seqs][beams] int32, within the sequence; an entry outside [0, beams) stands for the row itself.
 * row_pages     [seqs * beams][row_width] int32, row_lens [seqs * beams] int32 (tokens): before.
 * page_size     as the cache's (E3_ERR_SHAPE).
 * pages_out, lens_out   after: tables and lengths of the same shape, memory of their own (E3_ERR_VALUE where it is the input's).
 * src_out, dst_out, counts_out [seqs * beams] int32: for e3_cache_copy; -1, -1, 0 where there is nothing to copy.
 * A row whose table does not reach its next token has no such page: it has none to give and nothing is copied from it.
 */
int e3_beam_reorder(const int32_t* parent, int64_t seqs, int32_t beams, const int32_t* row_pages, int64_t row_width,
                    const int32_t* row_lens, int32_t page_size, int32_t* pages_out, int32_t* lens_out,
                    int32_t* src_out, int32_t* dst_out, int32_t* counts_out, void* hip_stream);

/*
 * Copy the first counts[i] tokens of page src_pages[i] to page dst_pages[i] (keys, values and scales, all heads), rounded up to a multiple
 * of eight and cut to the page.  Where either page is not in the cache or both are the same nothing is done.  No page may be a
 * destination twice, nor a source and a destination (the caller's contract).  [n] int32 each; n * kv_heads below 2^24 (E3_ERR_SHAPE).
 */
int e3_cache_copy(const e3_cache* cache, const int32_t* src_pages, const int32_t* dst_pages, const int32_t* counts, int64_t n,
                  void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* E3_H */

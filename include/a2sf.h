/*
 * liba2sf -- C ABI of the A2SF KV-cache pruning hot path on one NVIDIA B200 (sm_100a).
 *
 * A2SF (Accumulative Attention Score with Forgetting Factor) keeps, per attention
 * head, a score for every cached token: the forgetting-weighted sum over query
 * steps of the softmax probability that token received (paper Eq. 5), and evicts
 * the lowest-scoring tokens so the cache never exceeds a fixed budget (Sec. 3.1,
 * Sec. 4.1).  This library computes, per (batch, head) unit:
 *
 *   prefill : causal attention over the prompt, the score of every prompt token,
 *             and the set of tokens that stay in the cache;
 *   decode  : one generation step over the pruned, slot-indexed cache -- attention,
 *             the score recurrence S <- alpha*S + a_t, the eviction of one token
 *             and the in-place insertion of the new one.
 *
 * Conventions
 *   - Positions, slots and rows are 0-based.  n = prompt length, d = head size,
 *     M = budget (cache slots per head), R = recent (newest positions that are
 *     never evicted), U = B*H units.
 *   - Unless an argument says "host", every data pointer is a DEVICE pointer owned
 *     by the caller; the library never frees caller memory.  Rows of q/k/v/out
 *     must be 16-byte aligned (base pointer and strides).
 *   - Calls enqueue work on `cuda_stream` (a cudaStream_t passed as void*; NULL is
 *     the default stream) and return without synchronising, except where stated.
 *     The cache's resident count and length live on the device, so a decode step
 *     has no host-side data-dependent control flow.
 *   - Every function returns an a2sf_status.  Invalid arguments are rejected on
 *     the host before anything is launched; nothing is dereferenced on the host.
 *   - There is no CPU fallback.
 */
#ifndef A2SF_H
#define A2SF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { A2SF_F32 = 0, A2SF_BF16 = 1, A2SF_F16 = 2 } a2sf_dtype;

typedef enum {
    A2SF_OK = 0,
    A2SF_ERR_INVALID_ARG = -1,   /* null / misaligned pointer, bad shape or policy        */
    A2SF_ERR_UNSUPPORTED = -2,   /* dtype or head size without a kernel                   */
    A2SF_ERR_CUDA = -3,          /* a CUDA runtime call failed                            */
    A2SF_ERR_TIMEOUT = -4,       /* a bounded device-side wait ran out (kernel gave up)   */
    A2SF_ERR_WORKSPACE = -5      /* workspace / buffer smaller than the *_bytes() figure  */
} a2sf_status;

/* Shape and policy of a call.  `scale` = 0 selects 1/sqrt(d).  `alpha` is the
 * forgetting factor of Eq. 5; the paper states 0 < alpha < 1 and also runs
 * alpha = 0 (Sec. 4.4); alpha = 1 is the plain accumulative score of H2O (Eq. 4).
 * Accepted: 0 <= alpha <= 1 with alpha^0 = 1.  1 <= budget <= A2SF_MAX_BUDGET (one unit's
 * logits of a generation step are held in one CTA's shared memory), 0 <= recent <= budget,
 * d in {64, 128}.  Anything else: A2SF_ERR_INVALID_ARG, or A2SF_ERR_UNSUPPORTED for a dtype,
 * head size or budget outside the supported set. */
#define A2SF_MAX_BUDGET 49152
typedef struct a2sf_params {
    int32_t B, H, d;
    int32_t dtype;               /* a2sf_dtype of q, k, v, out and the cache rows */
    int32_t budget, recent;
    float alpha;
    float scale;
    int32_t flags;               /* 0 or A2SF_FLAG_* */
    int32_t score_window;        /* 0, or W > 0: see a2sf_score_window_bound */
} a2sf_params;

/* Scoring pass: Eq. 5 weighs query row i with alpha^(n-1-i).  Once that weight is below
 * 2^-127 (2^-152 on the CUDA-core path) the fp32 term is exactly zero, so with this flag the
 * pass leaves those rows out: O(n * window) instead of O(n^2) work with bit-identical scores.
 * Off by default; alpha = 1 has no such rows. */
#define A2SF_FLAG_SKIP_ZERO_WEIGHT_ROWS 1

/* Truncated scoring pass.  With score_window = W > 0 the sum of Eq. 5 runs over the last W
 * query rows only, S_j = sum_{i >= max(j, n-W)} alpha^(n-1-i) P_ij: O(n * W) work.  Every
 * probability is at most 1, so each score falls short of the full sum by at most
 *     sum_{a=W}^{n-1} alpha^a = alpha^W (1 - alpha^(n-W)) / (1 - alpha)      (n - W for alpha = 1),
 * which this function returns (0 when W = 0 or W >= n).  The attention output and lse are not
 * affected.  Unlike A2SF_FLAG_SKIP_ZERO_WEIGHT_ROWS this changes the scores: the kept set may
 * differ wherever two scores are closer than the bound. */
double a2sf_score_window_bound(float alpha, int32_t n, int32_t score_window);

typedef struct a2sf_cache a2sf_cache;   /* opaque, owned by the library */

/* ---------------------------------------------------------------------------
 * Prefill (prompt phase).
 *
 * For every unit, with s_ij = scale * q_i . k_j for j <= i (causal mask: Eq. 3 sets
 * the probability of a later key to zero) and P = row softmax of s:
 *     out_i    = sum_j P_ij v_j
 *     lse_i    = log sum_{j<=i} exp(s_ij)
 *     scores_j = sum_{i>=j} alpha^(n-1-i) P_ij           (Eq. 5, Eq. 6: the sum ends
 *                                                         at the diagonal term)
 *     kept_idx = every position >= n-R plus, of the others, all but the n-M lowest
 *                under the order (score, position) ascending; ascending positions.
 *                If n <= M every position is kept.  (Sec. 3.1, Sec. 4.1)
 *
 * q, k, v, out : [B][H][n][d] in `dtype`, element strides stride_b/stride_h/stride_t,
 *                d contiguous; out uses the same strides.
 * scores       : [B][H][n] fp32, contiguous.      kept_idx: [B][H][min(n,M)] int32.
 * lse_opt      : [B][H][n] fp32 or NULL (then it lives in the workspace).
 * workspace    : device scratch of at least a2sf_prefill_workspace_bytes() bytes,
 *                256-byte aligned; contents undefined afterwards.
 * Errors: INVALID_ARG, UNSUPPORTED, WORKSPACE, CUDA (launch failure).
 * ------------------------------------------------------------------------- */
size_t a2sf_prefill_workspace_bytes(const a2sf_params *p, int32_t n);

int a2sf_prefill(const a2sf_params *p, int32_t n,
                 const void *q, const void *k, const void *v,
                 int64_t stride_b, int64_t stride_h, int64_t stride_t,
                 void *out, float *scores, int32_t *kept_idx, float *lse_opt,
                 void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Scores and kept set only, from the log-sum-exp a prefill produced (the second
 * pass of the prefill alone).  Lets a sweep over alpha reuse one attention pass.
 * lse: [B][H][n] fp32 (input).  Other arguments as in a2sf_prefill; workspace may
 * be NULL when a2sf_rescore_workspace_bytes() is 0. */
size_t a2sf_rescore_workspace_bytes(const a2sf_params *p, int32_t n);

int a2sf_rescore(const a2sf_params *p, int32_t n,
                 const void *q, const void *k,
                 int64_t stride_b, int64_t stride_h, int64_t stride_t,
                 const float *lse, float *scores, int32_t *kept_idx,
                 void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Selection alone (Sec. 3.1, Sec. 4.1): kept_idx from a given score vector, exactly the last
 * step of a2sf_prefill / a2sf_rescore -- every position >= n-R plus, of the others, all but the
 * n-M lowest under (score, position) ascending.  scores [B][H][n] fp32 (input, non-negative),
 * kept_idx [B][H][min(n,M)] int32 (output, ascending).  Lets a caller re-select under another
 * budget or recent window without recomputing scores. */
int a2sf_select(const a2sf_params *p, int32_t n, const float *scores, int32_t *kept_idx,
                void *cuda_stream);

/* Per-head forgetting factors (the paper's Limitation section suggests a distinct factor per
 * layer and head instead of one uniform value).  `alphas` is a DEVICE array [B][H] fp32, one
 * factor per unit; p->alpha is ignored.  Values outside [0, 1] (or NaN) cannot be rejected on
 * the host and are clamped into [0, 1] on the device.  Everything else as in a2sf_prefill /
 * a2sf_rescore. */
int a2sf_prefill_per_head(const a2sf_params *p, int32_t n,
                          const void *q, const void *k, const void *v,
                          int64_t stride_b, int64_t stride_h, int64_t stride_t,
                          const float *alphas,
                          void *out, float *scores, int32_t *kept_idx, float *lse_opt,
                          void *workspace, size_t workspace_bytes, void *cuda_stream);

int a2sf_rescore_per_head(const a2sf_params *p, int32_t n,
                          const void *q, const void *k,
                          int64_t stride_b, int64_t stride_h, int64_t stride_t,
                          const float *lse, const float *alphas,
                          float *scores, int32_t *kept_idx,
                          void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Same as a2sf_prefill with HOST buffers: q, k, v, out contiguous [B][H][n][d];
 * scores, kept_idx as above, all in host memory (pinned memory makes the copies
 * asynchronous).  Inputs are copied to the device workspace, results copied back,
 * and the call returns after the stream has drained.  The device copies of k, v,
 * scores and kept_idx stay valid in the workspace for a2sf_cache_load: their
 * addresses are returned through dev_k, dev_v, dev_scores, dev_kept (any may be NULL).
 * With two or more batch rows the work is pipelined over chunks of rows on two internal
 * streams (created once per device on first use and kept): they start after what is already
 * queued on cuda_stream, and cuda_stream (and the call) continues only when they have drained.
 * Chunked calls on one device are serialised against each other. */
size_t a2sf_prefill_host_workspace_bytes(const a2sf_params *p, int32_t n);

int a2sf_prefill_host(const a2sf_params *p, int32_t n,
                      const void *q_host, const void *k_host, const void *v_host,
                      void *out_host, float *scores_host, int32_t *kept_idx_host,
                      void *workspace, size_t workspace_bytes,
                      void **dev_k, void **dev_v, float **dev_scores, int32_t **dev_kept,
                      void *cuda_stream);

/* Prefill without any allocation, for callers that cannot call cudaMalloc (an
 * engine whose own allocator owns the device, a plugin that only sees one layer's
 * tensors, a loop that must not hit an allocation's implicit synchronisation).
 * The paper has no counterpart: this is the same computation as a2sf_prefill, with
 * the per-row log-sum-exp scratch held in a fixed 4 MiB array inside the library's
 * device image (every GPU that loads the library carries it until the process
 * exits).  It runs the same kernels as a2sf_prefill except that, having no workspace
 * for an fp16 copy of V, bf16 storage multiplies P V with two bf16 terms.
 *   - Limit: B*H*n <= a2sf_prefill_static_scratch_max_rows() (1,048,576); larger
 *     calls return A2SF_ERR_WORKSPACE and launch nothing.
 *   - The first call on each device looks up the array's device address (a short
 *     host-side driver query with that device current); make that first call
 *     before starting any stream capture.
 *   - All calls on a device share the one array, which keeps the previous call's
 *     contents.  Each call overwrites every row it later reads, so nothing needs
 *     clearing, but two calls that overlap on the GPU (different streams without an
 *     event between them) race on it: keep them ordered.
 *   - It calls no cudaMalloc / cudaFree and takes no workspace; the log-sum-exp is
 *     not returned.  Other arguments, results and errors are those of a2sf_prefill. */
size_t a2sf_prefill_static_scratch_max_rows(void);

int a2sf_prefill_static_scratch(const a2sf_params *p, int32_t n,
                                const void *q, const void *k, const void *v,
                                int64_t stride_b, int64_t stride_h, int64_t stride_t,
                                void *out, float *scores, int32_t *kept_idx, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * The pruned cache.  Per unit: K and V rows [M][d] in `dtype`, scores [M] fp32,
 * positions [M] int32 (slot -> token position, -1 = empty), the resident count and
 * the number of tokens seen so far.  Slot order carries no meaning (softmax . V is
 * permutation invariant); positions exist for recency and the tie-break.
 *
 * a2sf_cache_create: `device_mem` NULL -> the library allocates a2sf_cache_bytes()
 * with cudaMalloc and frees it in a2sf_cache_destroy; otherwise it adopts the
 * caller's buffer (256-byte aligned, at least a2sf_cache_bytes(); WORKSPACE if
 * smaller), which the caller frees after destroy.  The cache starts empty.
 * Creation synchronises the device (it is not on the hot path).
 * ------------------------------------------------------------------------- */
size_t a2sf_cache_bytes(const a2sf_params *p);

int a2sf_cache_create(const a2sf_params *p, void *device_mem, size_t bytes, a2sf_cache **cache);

int a2sf_cache_destroy(a2sf_cache *cache);

/* Initial cache from a prefill: slot s <- token kept_idx[s] (its K and V row, score
 * and position); count = min(n, M); length = n; remaining slots emptied.
 * k, v: [B][H][n][d] with the given strides; scores [B][H][n]; kept_idx [B][H][min(n,M)]. */
int a2sf_cache_load(a2sf_cache *cache, int32_t n, const void *k, const void *v,
                    int64_t stride_b, int64_t stride_h, int64_t stride_t,
                    const float *scores, const int32_t *kept_idx, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * One generation step for every unit, fused in one kernel (Eq. 5 as a recurrence;
 * Sec. 3.1 eviction; the softmax runs over the pruned cache plus the new token,
 * cf. Sec. 2.2 on the changed denominator):
 *   a      = softmax over { scale*q.K[slot] : slot < count } and scale*q.k_new
 *   out    = sum_slot a_slot V[slot] + a_self v_new
 *   S[slot] <- alpha*S[slot] + a_slot,   S_new = a_self
 *   count < M : the new token goes to slot `count`; evicted_slot = -1.
 *   count = M : among the slots whose position is <= p - R (p = position of the new
 *               token) -- and the new token itself iff R = 0 -- the minimum under
 *               (S, position) is vacated and the new K/V/score/position are written
 *               there in place; evicted_slot = that slot, or -2 if the new token was
 *               the minimum (cache left as it was, apart from the updated scores).
 *   length += 1.
 * q, k_new, v_new, out: [B][H][d] contiguous in the cache's dtype; evicted_slot
 * [B][H] int32.  alpha overrides the value given at creation.
 * Steps on one cache must be ordered (same stream, or events between streams).
 * ------------------------------------------------------------------------- */
int a2sf_decode_step(a2sf_cache *cache, float alpha,
                     const void *q, const void *k_new, const void *v_new,
                     void *out, int32_t *evicted_slot, void *cuda_stream);

/* The same step with one forgetting factor per unit: `alphas` is a DEVICE array [B][H] fp32
 * (clamped into [0, 1] on the device).  See a2sf_prefill_per_head. */
int a2sf_decode_step_per_head(a2sf_cache *cache, const float *alphas,
                              const void *q, const void *k_new, const void *v_new,
                              void *out, int32_t *evicted_slot, void *cuda_stream);

/* The same step with HOST buffers.  Page-locked (pinned, mapped) buffers are read and written
 * by the step kernel directly over the bus; for any other host memory q, k_new, v_new are
 * copied into staging rows inside the cache, the step runs, out and evicted_slot are copied
 * back.  Either way the call returns after the stream has drained, with the results in place. */
int a2sf_decode_step_host(a2sf_cache *cache, float alpha,
                          const void *q_host, const void *k_new_host, const void *v_new_host,
                          void *out_host, int32_t *evicted_slot_host, void *cuda_stream);

/* Several tokens appended in one call (a draft that was accepted, a prompt continued in
 * chunks): exactly `steps` generation steps in order, token t taking row t of q, k_new,
 * v_new and writing row t of out -- DEVICE [B][H][steps][d] with element strides as in
 * a2sf_prefill.  evicted_opt: DEVICE [steps][B][H] int32 or NULL.  Runs as `steps` launches;
 * the result is bit-identical to calling a2sf_decode_step `steps` times. */
int a2sf_decode_multi(a2sf_cache *cache, float alpha, int32_t steps,
                      const void *q, const void *k_new, const void *v_new,
                      int64_t stride_b, int64_t stride_h, int64_t stride_t,
                      void *out, int32_t *evicted_opt, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Grouped query heads (GQA / MQA): `group` query heads share one K/V head, hence one pruned
 * cache.  The paper scores tokens per head and leaves grouping open (Limitation section);
 * the rule here: a token's score is the SUM over the group's query heads of Eq. 5, and one
 * selection / one eviction per K/V head serves the whole group.  a2sf_params.H counts K/V
 * heads; the query tensors have H * group heads, head h*group + g reading K/V head h.
 *
 * a2sf_prefill_group: q, out DEVICE [B][H*group][n][d] (q strides), k, v DEVICE [B][H][n][d]
 * (kv strides), scores [B][H][n] fp32 (summed over the group), kept_idx [B][H][min(n,budget)],
 * lse_opt [B][H*group][n] or NULL.  flags and score_window must be 0.  Workspace as for
 * a2sf_prefill, size from a2sf_prefill_group_workspace_bytes (0 = invalid arguments).
 *
 * a2sf_decode_step_group: the generation step for a cache built from those scores
 * (a2sf_cache_load).  q, out DEVICE [B][H*group][d] contiguous; k_new, v_new DEVICE [B][H][d];
 * evicted_slot [B][H].  Each query head attends over the cached tokens and the new one; the
 * cached scores become alpha * S + sum_g a_g, the new token's score sum_g a_g,self; eviction as
 * in a2sf_decode_step.  A2SF_ERR_UNSUPPORTED when group > A2SF_MAX_GROUP or (group + 2) * budget
 * is too large for one CTA's shared memory (about 47,000 for d = 128, group = 8).  For 16-bit
 * storage the products of the group run on the tensor cores (fp32 accumulation).
 * ------------------------------------------------------------------------- */
#define A2SF_MAX_GROUP 8
size_t a2sf_prefill_group_workspace_bytes(const a2sf_params *p, int32_t group, int32_t n);
int a2sf_prefill_group(const a2sf_params *p, int32_t group, int32_t n,
                       const void *q, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_t,
                       const void *k, const void *v,
                       int64_t kv_stride_b, int64_t kv_stride_h, int64_t kv_stride_t,
                       void *out, float *scores, int32_t *kept_idx, float *lse_opt,
                       void *workspace, size_t workspace_bytes, void *cuda_stream);
int a2sf_decode_step_group(a2sf_cache *cache, int32_t group, float alpha,
                           const void *q, const void *k_new, const void *v_new,
                           void *out, int32_t *evicted_slot, void *cuda_stream);

/* Empties the cache (count = length = 0, scores 0, positions -1), asynchronously. */
int a2sf_cache_reset(a2sf_cache *cache, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Streamed prompt: the cache is pruned WHILE the prompt is processed, row by row, the way
 * the paper's mask figures (Sec. 3.2, Sec. 4.3) draw it: token i attends only to what
 * is left of tokens 0..i-1, scores follow Eq. 5 as a recurrence and one token leaves per row
 * once the budget is full.  This is NOT a2sf_prefill followed by a2sf_cache_load (dense causal
 * attention, one selection at the end): the two give the same result only while n <= budget.
 *
 * Exactly: a2sf_cache_reset, then a2sf_decode_multi over the n prompt tokens (the generation
 * step with (q_i, k_i, v_i), out_i written to row i of `out`): n launches of the step kernel.
 * q, k, v, out: DEVICE [B][H][n][d] with the strides of a2sf_prefill.  evicted_opt: DEVICE
 * [n][B][H] int32 (each row as a2sf_decode_step's evicted_slot) or NULL.  On return (the work
 * is queued on the stream) the cache holds the pruned prompt and generation continues with
 * a2sf_decode_step.
 * ------------------------------------------------------------------------- */
int a2sf_prefill_streaming(a2sf_cache *cache, float alpha, int32_t n,
                           const void *q, const void *k, const void *v,
                           int64_t stride_b, int64_t stride_h, int64_t stride_t,
                           void *out, int32_t *evicted_opt, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Similarity with the ideal mask (Sec. 4.3: the mask figure and the similarity table).
 *
 * Runs a2sf_prefill_streaming and, for every row i, compares the attention the policy
 * actually uses -- the softmax over the cached tokens and token i itself -- with the ideal
 * row: the softmax over the budget + 1 largest logits of ALL tokens 0..i (equal logits: the
 * lower position first), i.e. the best any policy with that many tokens could do.
 *     cos_out[b][h][i] = <a_i, p_i> / (|a_i| |p_i|),   both rows as length-(i+1) vectors.
 * Rows i <= budget see every token and give 1.  Averaging (over rows, heads) is the caller's.
 * q, k, v, out, evicted_opt as in a2sf_prefill_streaming; cos_out DEVICE [B][H][n] fp32.
 * workspace: DEVICE, 256-byte aligned, a2sf_ideal_similarity_workspace_bytes (0 = invalid
 * arguments).  n <= A2SF_IDEAL_SIMILARITY_MAX_N (a row's logits are held in shared memory).
 * A diagnostic, not a hot path: 1 + 2n launches, O(n^2 d) CUDA-core work per unit.
 * ------------------------------------------------------------------------- */
#define A2SF_IDEAL_SIMILARITY_MAX_N 32768
size_t a2sf_ideal_similarity_workspace_bytes(const a2sf_params *p, int32_t n);
int a2sf_ideal_similarity(a2sf_cache *cache, float alpha, int32_t n,
                          const void *q, const void *k, const void *v,
                          int64_t stride_b, int64_t stride_h, int64_t stride_t,
                          void *out, float *cos_out, int32_t *evicted_opt,
                          void *workspace, size_t workspace_bytes, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Rotary positions.  A pair (x1, x2) of a row at position p is turned by the angle
 * p * f_k:  y1 = m (x1 cos - x2 sin),  y2 = m (x2 cos + x1 sin), k = 0 .. rotary_dim/2 - 1,
 * f_k = theta^(-2k / rotary_dim) before scaling.  Pairs are (k, k + rotary_dim/2), or the
 * neighbours (2k, 2k+1) with `interleaved`.  Elements from rotary_dim on are copied.
 *
 * a2sf_rotary_plan_init (host only) turns a configuration into a plan, which the caller keeps:
 * f_k / 2 pi as a 64-bit fixed-point fraction of a turn, so that  p * f_k  modulo one turn is
 * exact integer arithmetic on the device however far the position is.
 *   scaling LINEAR: f / factor.   NTK: theta * factor^(r / (r - 2)) instead of theta.
 *   BANDS: by wavelength 2 pi / f against the original length L: shorter than L / high is kept,
 *          longer than L / low is divided by factor, linear in L / wavelength between.
 *   RAMP : interpolation by parts (YaRN): the dimension at which `high` (beta fast) turns fit
 *          into L up to the one for `low` (beta slow), linear in the pair index between; the
 *          default magnitude is 0.1 ln(factor) + 1.
 *   magnitude: m; 0 selects the default (1 except for RAMP).
 * Accepted: even 2 <= rotary_dim <= 128 (NTK: >= 4), theta > 1, factor >= 1, and for BANDS and
 * RAMP original_length >= 1 and 0 < low < high.  INVALID_ARG otherwise.
 *
 * a2sf_rotary: x -> y, [B][H][n][d] in `dtype` with element strides of their own, d in {64, 128}
 * and >= rotary_dim.  y may be x itself (same strides); otherwise they must not overlap.  Row t of
 * sequence b stands at positions[b][t] (DEVICE [B][n] int32), or at start[b] + t (DEVICE [B]; NULL:
 * t) when `positions` is NULL.  lens (DEVICE [B] or NULL): rows t >= lens[b] of y are left as they
 * were.  flags: 0 or A2SF_ROTARY_TRANSPOSE, which applies the transposed matrix: the gradient of
 * the rotation, and for m = 1 its inverse.  Angles have an absolute error below 3e-8 at every position.
 * ------------------------------------------------------------------------- */
typedef enum {
    A2SF_ROTARY_PLAIN = 0, A2SF_ROTARY_LINEAR = 1, A2SF_ROTARY_NTK = 2, A2SF_ROTARY_BANDS = 3, A2SF_ROTARY_RAMP = 4
} a2sf_rotary_scaling;

typedef struct a2sf_rotary_config {
    int32_t rotary_dim, interleaved;
    int32_t scaling;             /* a2sf_rotary_scaling */
    int32_t original_length;     /* L: the length that the frequencies were made for */
    double theta, factor, low, high, magnitude;
} a2sf_rotary_config;

#define A2SF_ROTARY_MAX_PAIRS 64
typedef struct a2sf_rotary_plan {
    int32_t rotary_dim, interleaved;
    float magnitude;
    int32_t check;               /* written by a2sf_rotary_plan_init; other values are refused */
    uint64_t turn[A2SF_ROTARY_MAX_PAIRS];
} a2sf_rotary_plan;

#define A2SF_ROTARY_TRANSPOSE 1

int a2sf_rotary_plan_init(const a2sf_rotary_config *config, a2sf_rotary_plan *plan);

int a2sf_rotary(const a2sf_rotary_plan *plan, int32_t dtype, int32_t B, int32_t H, int32_t n, int32_t d,
                const void *x, int64_t x_stride_b, int64_t x_stride_h, int64_t x_stride_t,
                void *y, int64_t y_stride_b, int64_t y_stride_h, int64_t y_stride_t,
                const int32_t *positions, const int32_t *start, const int32_t *lens, int32_t flags,
                void *cuda_stream);

/* ---------------------------------------------------------------------------
 * The cache in pages.  A pool of pages, each holding page_size slots of every K/V head, and a
 * page table per sequence: slot s of sequence b is slot s % page_size of page
 * page_table[b][s / page_size].  Prompts of different lengths, prompts that arrive in chunks and
 * sequences that come and go share one pool.  A sequence uses the same number of slots in every
 * head, but each head evicts its own tokens: positions and scores are kept per slot and head, and
 * slot order carries no meaning.  A step of the cache is
 *     a2sf_paged_append   the chunk's keys and values into slots past .. past + len - 1
 *     a2sf_paged_attend   its attention over slots 0 .. past + len - 1, and the scores
 *     a2sf_paged_evict    back to the budget; past and start move on
 * for chunks of one token (generation) as for whole prompts.  All memory is the caller's; the
 * struct holds DEVICE pointers and is read during the call only.
 *   Per call, len[b] = min(lens[b], c), or c when lens is NULL.  A sequence with len 0 takes no
 *   part: nothing of it is read or written (a2sf_paged_evict still brings it to the budget).
 *   start[b] = tokens seen before the chunk = position of the chunk's first token (NULL: past).
 * Lengths and page tables are on the device and cannot be checked on the host: a page number
 * outside [0, num_pages) or a slot outside the table is never followed -- such slots are not
 * written, and where they would be read the sequence's results are undefined -- and
 * a2sf_last_device_status then returns A2SF_ERR_INVALID_ARG.  The first call on a device looks up
 * that status word and raises kernel limits: make it before a stream capture begins.
 * A page that two sequences share must not be written: by a2sf_paged_append, by a2sf_paged_evict in
 * place, nor by a2sf_paged_attend, which updates scores unless told not to.  Keys, values and
 * queries of resident tokens must be finite, their logits below 2^27 in magnitude (from 2^20 on the last place
 * of an fp32 logit is no longer small against a probability's exponent); values must be below
 * 2^113 / (past + len) in magnitude (fp16 always is), since up to 2^14 times their sum is held before
 * the division by the row sum, and keys and queries of 32-bit storage below 2^127.  Slots beyond
 * past + len may hold anything.  Calls on the same sequences must be ordered (same stream, or events
 * between streams).
 * ------------------------------------------------------------------------- */
#define A2SF_PAGED_MAX_SEQUENCES 1024
typedef struct a2sf_paged {
    int32_t B;                   /* sequences of the call, <= A2SF_PAGED_MAX_SEQUENCES */
    int32_t H;                   /* K/V heads */
    int32_t group;               /* query heads per K/V head, 1 .. A2SF_MAX_GROUP */
    int32_t d;                   /* 64 or 128 */
    int32_t dtype;               /* a2sf_dtype of the pages, q, k, v and out */
    int32_t page_size;           /* 16, 32, 64 or 128 */
    int32_t num_pages;           /* pages of the pool */
    int32_t max_pages;           /* entries of a page-table row */
    float scale;                 /* of the logits; 0 selects 1/sqrt(d) */
    int32_t reserved;            /* 0 */
    void *k_pages, *v_pages;     /* [num_pages][H][page_size][d], 16-byte aligned */
    float *scores;               /* [num_pages][H][page_size], 16-byte aligned */
    int32_t *positions;          /* [num_pages][H][page_size], 16-byte aligned */
    const int32_t *page_table;   /* [B][max_pages] */
    const int32_t *past;         /* [B] slots in use before the chunk */
    const int32_t *start;        /* [B] or NULL */
} a2sf_paged;

/* k, v [B][H][c][d], q and q_out [B][H*group][c][d], strides of their own (q and k, v have d
 * contiguous).  Token t of sequence b goes to slot past[b] + t with position start[b] + t and score
 * 0.  With a plan, keys (and queries, when q is not NULL) are rotated on the way; without one q must
 * be NULL.  q_out may be q itself with the same strides.  Nothing of past and start changes. */
int a2sf_paged_append(const a2sf_paged *cache, const a2sf_rotary_plan *rotary_opt, int32_t c, const int32_t *lens,
                      const void *k, const void *v, int64_t kv_stride_b, int64_t kv_stride_h, int64_t kv_stride_t,
                      const void *q_opt, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_t,
                      void *q_out, int64_t qo_stride_b, int64_t qo_stride_h, int64_t qo_stride_t,
                      void *cuda_stream);

/* Attention of the chunk (appended before): row i of query head h*group + g sees slots
 * 0 .. past[b] + i of K/V head h.
 *     out = softmax(scale q K^T) V,   lse = log sum exp   ([B][H*group][c] fp32, or NULL)
 *     score[slot] <- alpha^len * score[slot] + sum_{i,g} alpha^(len-1-i) P_ig,slot
 * which is Eq. 5 carried over chunks: any split of a prompt into chunks gives the scores of the
 * whole.  flags: 0, or A2SF_ATTEND_NO_SCORES (scores are neither read nor written).  out has strides
 * of its own and must not overlap q; rows i >= len[b] of out and lse are left as they were.  Rows whose weight alpha^age
 * is below 2^-126 (the smallest normal fp32 number) are left out of the sum.
 * workspace: DEVICE, 256-byte aligned, a2sf_paged_attend_workspace_bytes (0 = invalid arguments);
 * contents undefined afterwards; calls that may overlap in time need workspaces of their own.  Its size follows
 * the capacity of the page table, not what is cached: for c * group <= 16 it is mostly the logits, 4 bytes for
 * every sequence, head, slot of capacity and row (rows rounded up to a power of two), with scores or without. */
#define A2SF_ATTEND_NO_SCORES 1
size_t a2sf_paged_attend_workspace_bytes(const a2sf_paged *cache, int32_t c);
int a2sf_paged_attend(const a2sf_paged *cache, int32_t c, const int32_t *lens, float alpha,
                      const void *q, int64_t q_stride_b, int64_t q_stride_h, int64_t q_stride_t,
                      void *out, int64_t out_stride_b, int64_t out_stride_h, int64_t out_stride_t,
                      float *lse_opt, int32_t flags, void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Ends a step.  Of the n = past + len slots of every head min(n, budget) stay: those at the
 * `recent` newest positions (position >= start + len - recent) and of the others the best under
 * (score, position), the order of a2sf_select; equal pairs leave in slot order.  Then
 * past_out[b] = min(n, budget) and start_out[b] = start[b] + len[b] (may be past and start).
 *   dst_table NULL: in place.  The free slots below `budget`, in ascending order, take the
 *   survivors from above, in ascending order; nothing else moves.
 *   dst_table [B][dst_max_pages]: the survivors are copied, in ascending slot order, into those
 *   pages (none of them a page of page_table) and the old pages are left as they are -- for pages that
 *   other sequences share.  dst_max_pages * page_size >= min(budget, capacity) is required.
 * 0 <= recent <= budget, budget >= 1.  Scores may be any numbers (NaN of either sign sorts beyond
 * infinity).  workspace: as above, from a2sf_paged_evict_workspace_bytes. */
size_t a2sf_paged_evict_workspace_bytes(const a2sf_paged *cache, int32_t budget);
int a2sf_paged_evict(const a2sf_paged *cache, int32_t c, const int32_t *lens, int32_t budget, int32_t recent,
                     const int32_t *dst_table, int32_t dst_max_pages, int32_t *past_out, int32_t *start_out,
                     void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Snapshot / restore of the whole cache state into / from caller DEVICE buffers:
 * k, v [B][H][M][d] dtype; scores [B][H][M] fp32; pos [B][H][M] int32; count, len
 * [B][H] int32.  Any pointer may be NULL to skip that part. */
int a2sf_cache_export(const a2sf_cache *cache, void *k, void *v, float *scores,
                      int32_t *pos, int32_t *count, int32_t *len, void *cuda_stream);

int a2sf_cache_import(a2sf_cache *cache, const void *k, const void *v, const float *scores,
                      const int32_t *pos, const int32_t *count, const int32_t *len,
                      void *cuda_stream);

/* Number of kernels this library has launched in the calling process so far. */
int64_t a2sf_kernel_launch_count(void);

/* Synchronises the stream and returns the sticky device-side status (A2SF_OK,
 * A2SF_ERR_TIMEOUT if a kernel abandoned a bounded wait, or A2SF_ERR_INVALID_ARG if a paged-cache
 * kernel met a page number or length outside its bounds), then clears it.  While the
 * status is set the tensor-core prefill kernels return without working, so results
 * of calls made after a timeout and before this call are undefined. */
int a2sf_last_device_status(void *cuda_stream);

/* Self-test of the device-side failure path (the paper has no counterpart; a test hook, not
 * part of the method).  Every wait inside the kernels of this library is bounded: a wait that
 * runs out poisons its CTA, the kernel unwinds and raises the sticky status that
 * a2sf_last_device_status reports.  This call exercises exactly that, harmlessly: it launches one
 * CTA whose first thread waits -- through the library's own bounded wait, with `limit_cycles`
 * SM clocks as the limit -- on a barrier at which nobody ever arrives, then raises the status
 * word of the tensor-core prefill kernels (which = 0) or of the generation-step kernels
 * (which = 1).  Nothing traps and nothing waits without a bound.
 *   report : DEVICE int64[4], written by the kernel: [0] 1 if the wait reported failure,
 *            [1] SM clocks the wait took, [2] SM clocks of a second wait in the same CTA (it
 *            returns at once because the CTA is poisoned), [3] 1 if that second wait failed too.
 *   limit_cycles in [1, A2SF_SELFTEST_MAX_WAIT_CYCLES]; INVALID_ARG otherwise.
 * Afterwards a2sf_last_device_status returns A2SF_ERR_TIMEOUT once, then A2SF_OK. */
#define A2SF_SELFTEST_MAX_WAIT_CYCLES 2000000000ll
int a2sf_selftest_bounded_wait(int32_t which, int64_t limit_cycles, int64_t *report, void *cuda_stream);

/* Bounds-checked debug library (built with -DA2SF_DEBUG as liba2sf_debug.so; the paper has no
 * counterpart).  In it every slot, position, tile-row and ring-stage index that addresses global
 * or shared memory inside a kernel is range-checked; a violation is counted, the first one is
 * recorded, and the offending access is skipped (nothing traps).  a2sf_debug_build returns 1 in
 * that library and 0 in the release one.  a2sf_debug_violations synchronises the stream, writes
 * to the HOST array report[4] = { violations since the last call, (kernel id << 32) | source
 * line of the first one, its index, its bound } and clears the record; the release library
 * always reports zeros. */
int a2sf_debug_build(void);
int a2sf_debug_violations(int64_t *report, void *cuda_stream);

const char *a2sf_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* A2SF_H */

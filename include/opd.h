/*
 * opd.h - C ABI of the learner-time on-policy-distillation (OPD) loss for
 * AMD Instinct MI355X (gfx950).
 *
 * One call takes the student logits of N generated tokens over a vocabulary
 * of V entries, plus the finite teacher-score cache those tokens carry, and
 * returns the per-token loss and its gradient with respect to every logit
 * (Sec. 4.1, "Stage 3: Student update": the learner recomputes log p_theta
 * on the cached actions).  Further calls make what it reads: rows of logits from
 * 8-bit hidden states and head weights, draws, verified drafts, supports and
 * scores.  All work runs in HIP kernels on the caller's
 * stream; nothing is computed on the host.
 *
 * Conventions shared by every entry point
 *  - Array pointers are DEVICE pointers owned by the caller.  The library
 *    keeps no reference to them after the call returns and allocates no
 *    device memory.
 *  - Logit rows have stride `ld` elements (ld >= V).  logits, dlogits and
 *    teacher_logits must be 16-byte aligned and ld * element_size must be a
 *    multiple of 16 bytes (ld % 8 == 0 when any of them is bf16, else
 *    ld % 4 == 0).  Columns [V, ld) of dlogits are never written.
 *  - Calls are stream-ordered and asynchronous.  Argument errors are
 *    reported synchronously, before anything is launched; a HIP launch
 *    failure returns OPD_ERR_HIP.  Faults in the DATA (a cached id outside
 *    [0, V), NaN or infinite logits) never fault the device: an out-of-range
 *    id makes that row's loss NaN and fills its dlogits row with NaN, and
 *    NaN/Inf logits propagate into that row's outputs.
 *  - N may be as large as INT32_MAX: calls whose grid would exceed HIP's
 *    limit of 2^32 work-items launch over consecutive row chunks.
 *  - Results are deterministic: repeated calls with the same inputs produce
 *    bitwise-identical outputs (fixed-order reductions, no float atomics).
 *  - Entry points hold no mutable global state and are safe to call from
 *    several host threads (each call on its own stream and buffers).
 */
#ifndef OPD_H
#define OPD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OPD_VERSION 7
/* Largest cached support size k, and largest sample count M. */
#define OPD_K_MAX 256

typedef enum opd_status {
  OPD_OK = 0,
  OPD_ERR_NULL = -1,      /* a pointer the estimator needs is NULL */
  OPD_ERR_SHAPE = -2,     /* N < 0, V < 2, V >= 2^31, or ld < V */
  OPD_ERR_SUPPORT = -3,   /* k or M outside [1, min(V, OPD_K_MAX)], or RKL_MC1 with M != 1 */
  OPD_ERR_DTYPE = -4,     /* unknown logits or dlogits dtype, or scale type */
  OPD_ERR_ALIGN = -5,     /* a logit/gradient pointer or row stride is not 16-byte aligned */
  OPD_ERR_WORKSPACE = -6, /* split-vocabulary path forced with a missing or short workspace */
  OPD_ERR_ESTIMATOR = -7, /* unknown estimator */
  OPD_ERR_FLAGS = -8,     /* unknown or contradictory flag bits */
  OPD_ERR_HIP = -9,       /* a HIP runtime call or kernel launch failed */
  OPD_ERR_PARAM = -10,    /* invalid scalar option (clip_eps of a clipped estimator, block_rows), or
                             coverage_out for an estimator without a cached support */
  OPD_ERR_SCRATCH = -11   /* opd_loss_fwd_bwd_noalloc: the call needs more scratch than
                             OPD_NOALLOC_SCRATCH_BYTES */
} opd_status;

/*
 * Estimators.  Notation of Sec. 3: p_theta = softmax(z) the current student,
 * q the teacher, p_old the stale behaviour policy.  For token t with logits
 * z (row of `logits`), L = log sum_j exp(z_j) and log p_theta(j) = z_j - L.
 *
 * OPD_FKL_TOPK  Forward KL on the cached support S = {idx[t, 0..k)}, teacher
 *               and student both renormalised on S (Sec. 3, "Sparse and
 *               sampled implementations"; normalisers of App. A.1):
 *                 loss = sum_S q~ (log q~ - log p~),
 *                 dloss/dz_{a_i} = p~_i - q~_i, zero off S.
 * OPD_RKL_TOPK  Sparse reverse KL D_R^S = KL(p~ || q~) (App. A.1), support
 *               held fixed:  dloss/dz_{a_i} = p~_i ((log p~_i - log q~_i) - D_R^S).
 *               Renormalisation cancels L, so both top-k estimators read only
 *               the k cached logits unless lse_out is requested.
 * OPD_RKL_MC1   One-sample MC reverse KL with old-to-current importance
 *               ratio and the advantage recomputed under the current student,
 *               unclipped (Sec. 5.1, L_theta^noclip):
 *                 loss = -rho(a) sg(A_theta(a)),  A_theta = log q - log p_theta,
 *                 rho = p_theta(a) / p_old(a).   Requires M == 1.
 * OPD_RKL_MC    M-sample average of the same surrogate (Sec. 6.2; App. E):
 *                 loss = -(1/M) sum_i rho(a_i) sg(A_theta(a_i)),
 *                 dloss/dz_j = c p_theta(j) - (1/M) sum_{i: a_i = j} rho_i A_i,
 *               c = -loss.  Samples are iid with replacement; repeated ids are
 *               separate terms, accumulated in ascending i.
 * OPD_FKL_DENSE Full-vocabulary forward KL against dense teacher logits
 *               (Sec. 3, eq. dense-forward-kl): gradient p_theta - q.
 * OPD_RKL_DENSE Full-vocabulary reverse KL (Sec. 3, eq. dense-reverse-kl and
 *               eq. reverse-kl-gradient): gradient p_j ((log p_j - log q_j) - D_R).
 *
 * The remaining members of the surrogate ablation of Sec. 5.1, on the same
 * M behaviour samples as OPD_RKL_MC.  With rho_bar = clip(rho, 1 - eps,
 * 1 + eps), eps = opts->clip_eps, and A_old = log q - log p_old (rollout-time,
 * from teacher_logp and behav_logp):
 * OPD_RKL_MC_CLIP      L_theta^clip = -(1/M) sum_i min(rho_i A_theta,i, rho_bar_i A_theta,i)
 * OPD_RKL_MC_OLD       L_old^noclip = -(1/M) sum_i rho_i A_old,i
 * OPD_RKL_MC_OLD_CLIP  L_old^clip   = -(1/M) sum_i min(rho_i A_old,i, rho_bar_i A_old,i),
 *                      the PPO-style adaptation
 * The advantage is a stop-gradient weight.  Where the min selects the
 * clipped term outside [1 - eps, 1 + eps] the sample contributes no gradient;
 * ties (rho inside the range) count as unclipped.
 * OPD_RKL_MC_NOIS      MC without importance sampling (the App. F ablation):
 *                      the samples are used as if drawn from p_theta,
 *                      L = -(1/M) sum_i sg(A_theta,i) log p_theta(a_i), gradient
 *                      -(1/M) sum_i A_theta,i (1[j = a_i] - p_j).  behav_logp
 *                      is not read (may be NULL).
 *
 * Truncated top-k: the dense KLs of Sec. 3 with the action sum cut to the
 * cached support S = {idx[t, 0..k)} and no renormalisation (p_theta and q keep
 * their full-vocabulary normalisers, so teacher_logp must be normalised over
 * the full vocabulary).  Not a KL in general (can be negative); the gradient
 * is dense, so the row is read.
 * OPD_FKL_TOPK_TRUNC   sum_S q (log q - log p_theta);
 *                      dloss/dz_j = Z_q^S p_j - q_j 1[j in S], Z_q^S = q(S)
 * OPD_RKL_TOPK_TRUNC   sum_S p_theta (log p_theta - log q);
 *                      dloss/dz_j = p_j 1[j in S](log p_j - log q_j + 1)
 *                                   - p_j sum_S p (log p - log q + 1)
 */
typedef enum opd_estimator {
  OPD_FKL_TOPK = 0,
  OPD_RKL_TOPK = 1,
  OPD_RKL_MC1 = 2,
  OPD_RKL_MC = 3,
  OPD_FKL_DENSE = 4,
  OPD_RKL_DENSE = 5,
  OPD_RKL_MC_CLIP = 6,
  OPD_RKL_MC_OLD = 7,
  OPD_RKL_MC_OLD_CLIP = 8,
  OPD_RKL_MC_NOIS = 9,
  OPD_FKL_TOPK_TRUNC = 10,
  OPD_RKL_TOPK_TRUNC = 11
} opd_estimator;

typedef enum opd_dtype { OPD_F32 = 0, OPD_BF16 = 1 } opd_dtype;

/* Flags (opd_opts.flags). */
#define OPD_FLAG_SKIP_MASKED 1u   /* leave dlogits rows of masked tokens untouched */
#define OPD_FLAG_FORCE_ROWWISE 2u /* one workgroup per token row, whatever N is */
#define OPD_FLAG_FORCE_SPLITV 4u  /* split each row over several workgroups (needs workspace) */

/*
 * The teacher-score cache of N tokens (Sec. 4.1, Stage 1 and Stage 2).
 * Row-major device arrays; which fields are read depends on the estimator.
 *   idx            [N, k] int32  top-k support S (the top-k estimators, renormalised
 *                  and truncated); ids must be distinct within a row
 *                  (opd_validate_cache checks this)
 *   sampled_ids    [N, M] int32  behaviour-policy samples a_i ~ p_old (the
 *                  MC estimators, OPD_RKL_MC1 and OPD_RKL_MC_*); repeats allowed
 *   teacher_logp   [N, k] or [N, M] fp32  log q(a|s) at idx / sampled_ids,
 *                  normalised over the full vocabulary (the top-k estimators
 *                  renormalise on S, so any per-row constant cancels there)
 *   behav_logp     [N, M] fp32  log p_old(a|s) at sampled_ids (MC only),
 *                  recorded per token by the rollout policy
 *   teacher_logits [N, ld] dense teacher logits (dense estimators only),
 *                  same dtype and stride as the student logits
 */
typedef struct opd_cache {
  const int32_t* idx;
  const int32_t* sampled_ids;
  const float* teacher_logp;
  const float* behav_logp;
  const void* teacher_logits;
} opd_cache;

/*
 * grad_scale    gamma: dlogits[t, :] = gamma * mask[t] * dloss_t/dz_t; 1.0 gives
 *               the gradient of the masked sum of per-token losses.  Reductions
 *               over tokens (token mean, sequence mean) are the caller's: they
 *               are a choice of gamma.
 * dlogits_dtype OPD_F32 (default) or OPD_BF16 (round to nearest even).
 * flags         OPD_FLAG_* bits.
 * clip_eps      clip range eps of the clipped estimators; must be positive
 *               and finite for them (the paper uses 0.2, App. B, Table 3);
 *               ignored otherwise.
 * A NULL opts pointer means {1.0f, OPD_F32, 0, 0.2f}.
 */
typedef struct opd_opts {
  float grad_scale;
  int32_t dlogits_dtype;
  uint32_t flags;
  float clip_eps;
} opd_opts;

/*
 * Fused forward + backward of the OPD loss over N token rows.
 *
 *   logits        [N, ld] student logits, dtype OPD_F32 or OPD_BF16
 *   N, V, ld      tokens, vocabulary size, row stride (elements)
 *   cache         see opd_cache; must not be NULL
 *   estimator     opd_estimator
 *   k             support size for the top-k estimators (else ignored)
 *   M             samples per token for the MC estimators (else ignored)
 *   mask          [N] uint8, nullable (NULL = every token valid).  A masked
 *                 token (mask == 0) has loss 0, lse_out 0, gathered_out 0, and
 *                 a zero dlogits row (untouched with OPD_FLAG_SKIP_MASKED);
 *                 its logits are not read.
 *   opts          nullable, see opd_opts
 *   loss          [N] fp32 per-token loss (the MC loss is the surrogate value,
 *                 an unbiased estimate of the dense reverse KL, and can be
 *                 negative)
 *   dlogits       [N, ld] gradient, dtype opts->dlogits_dtype; may not alias
 *                 logits
 *   lse_out       [N] fp32 log sum_j exp(z_j), nullable.  For the top-k
 *                 estimators, requesting it adds one read of the logits.
 *   gathered_out  [N, k or M] fp32 student logits at the cached ids (exact
 *                 widening), nullable; not produced by the dense estimators.
 *   coverage_out  [N, 2] fp32 support coverage, nullable: the restricted
 *                 normalisers of App. A.1 on the cached support S,
 *                 Z_p^S = sum_{a in S} p_theta(a|s) (the student's mass on S)
 *                 and Z_q^S = sum_i exp(teacher_logp[t, i]) (the teacher's),
 *                 each cached entry counted once; 0 and 0 for a masked token.
 *                 A stale support (Sec. 6) shows as Z_p^S falling away from
 *                 Z_q^S.  Only the estimators that read a support (the
 *                 renormalised and truncated top-k) take it (else
 *                 OPD_ERR_PARAM); for the renormalised ones it adds one read
 *                 of the logits, as lse_out does.
 *   workspace     device scratch for the split-vocabulary path, nullable;
 *   workspace_bytes  its size.  The split path is taken for small N (unless the
 *                 rows are narrow enough to be faster whole) or when forced,
 *                 and only if workspace_bytes >= opd_workspace_bytes(...);
 *                 otherwise the row-per-workgroup path runs.
 *   stream        hipStream_t to launch on (NULL = default stream)
 * Returns OPD_OK or an opd_status error.  N == 0 is a no-op returning OPD_OK.
 */
int opd_loss_fwd_bwd(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
                     const opd_cache* cache, int32_t estimator, int32_t k, int32_t M,
                     const uint8_t* mask, const opd_opts* opts, float* loss, void* dlogits,
                     float* lse_out, float* gathered_out, float* coverage_out, void* workspace,
                     size_t workspace_bytes, void* stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * fused forward + backward as opd_loss_fwd_bwd, with the same arguments
 * except the workspace, the same kernels and bitwise the same results.  The
 * split-vocabulary path keeps its per-(row, chunk) statistics in a static
 * device array of OPD_NOALLOC_SCRATCH_BYTES that the library holds on each
 * GPU it runs on until the process ends (its address is looked up once per
 * device, on the first call that needs it, with that device current).  The
 * call allocates nothing: no hipMalloc, hipFree or allocating library call.
 *   - A call whose split path needs more than OPD_NOALLOC_SCRATCH_BYTES
 *     (opd_workspace_bytes(...) of the same arguments) returns
 *     OPD_ERR_SCRATCH when the split path is forced (OPD_FLAG_FORCE_SPLITV);
 *     unforced, such a call runs the row-per-workgroup path, which needs no
 *     scratch.  (Unforced split calls, below 64 rows, need at most 126 KiB.)
 *   - Every record the split path reads is written earlier in the same call,
 *     so nothing carries over from the previous call's contents.
 *   - All calls on one GPU share that GPU's array: calls that overlap in time
 *     on one GPU (on different streams, or from several host threads) race
 *     and may return wrong results.  Serialise them.
 * Other errors as for opd_loss_fwd_bwd.
 */
#define OPD_NOALLOC_SCRATCH_BYTES (1u << 20)
int opd_loss_fwd_bwd_noalloc(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
                             const opd_cache* cache, int32_t estimator, int32_t k, int32_t M,
                             const uint8_t* mask, const opd_opts* opts, float* loss,
                             void* dlogits, float* lse_out, float* gathered_out,
                             float* coverage_out, void* stream);

/* OPD_NOALLOC_SCRATCH_BYTES of the built library. */
size_t opd_noalloc_scratch_bytes(void);

/*
 * Bytes of workspace that let opd_loss_fwd_bwd take the split-vocabulary path
 * for these arguments: its per-(row, chunk) statistics records, N * P * 32
 * bytes, for calls below 64 rows or with OPD_FLAG_FORCE_SPLITV, else 0.  The
 * records need not all be used, and a call may not need them: narrow rows and
 * write-only top-k calls below 64 rows run the row-per-workgroup path, and
 * leave the workspace as it is, with or without one.  Pure host function: the
 * answer depends only on its arguments.  Invalid arguments return 0.
 */
size_t opd_workspace_bytes(int64_t N, int64_t V, int32_t dtype, int32_t estimator, int32_t k,
                           int32_t M, uint32_t flags);

/*
 * Checks a cache against the preconditions of the estimator and ADDS the
 * number of violations to *violations (a device int32 the caller zeroes):
 *   - ids outside [0, V);
 *   - repeated ids within a top-k row: a support S is a set of actions, and
 *     the restricted normalisers and renormalised distributions on S
 *     (App. A.1) count each action once.  Repeats within an MC row are legal,
 *     since the m samples are drawn iid with replacement (Sec. 6.2; App. E),
 *     and are not counted;
 *   - non-finite teacher_logp (and behav_logp for the estimators with an
 *     importance ratio or A_old): a log-probability the cache records for an
 *     action it holds is finite.
 * Each bad entry counts once, each repeated top-k pair once.  Stream-ordered;
 * read the counter after synchronising.  Dense estimators have no cache to
 * check (returns OPD_OK).  Errors: OPD_ERR_ESTIMATOR, OPD_ERR_SHAPE,
 * OPD_ERR_SUPPORT, OPD_ERR_NULL, OPD_ERR_HIP.
 */
int opd_validate_cache(const opd_cache* cache, int32_t estimator, int64_t N, int64_t V,
                       int32_t k, int32_t M, int32_t* violations, void* stream);

/*
 * Building the cache (Sec. 4.1, Stage 1 "Student rollout" and Stage 2
 * "Teacher scoring").  Each call reads N rows of logits (the rollout policy
 * p_old for Stage 1, the teacher for Stage 2) with the same dtype, ld and
 * alignment rules as opd_loss_fwd_bwd, and writes per-row results.  A masked
 * row (mask[t] == 0) is not read and gets 0 in every output.  lse_out, when
 * not NULL, receives log sum_j exp(z_j) per row.  No workspace.
 *
 * opd_sample_actions: M iid draws per row from softmax(z), as the rollout
 *   makes them (temperature 1, no top-p or top-k truncation; App. B), by
 *   inversion: draw i is the first index whose cumulative probability (index
 *   order) exceeds uniforms[t, i].  The uniforms are supplied by the caller
 *   ([N, M] fp32 in [0, 1)), so the draws are a deterministic function of
 *   them.  The CDF is evaluated in double precision (terms exp(z_j - max), or
 *   terms in proportion to them, to about 1.5e-15 relative, double sums), so a
 *   draw is the one exact arithmetic gives unless uniforms[t, i] lies within
 *   about 1e-14 of a cumulative value; terms follow double's gradual underflow
 *   below the row's maximum, -inf logits have exactly zero mass, and a drawn id
 *   always has nonzero probability.
 *     sampled_ids [N, M] int32 out; logp [N, M] fp32 out (nullable) =
 *     log softmax(z) at the draw, the rollout-time log-probability the MC
 *     estimators read as behav_logp.  A uniform outside [0, 1) (or NaN), or a
 *     row with a NaN or +inf logit or no finite logit, gives id -1, logp NaN.
 *     1 <= M <= OPD_K_MAX.
 *
 * opd_topk_support: the k largest logits of each row, S = TopK(softmax(z), k)
 *   (Sec. 5: S_old at rollout time, or a teacher-selected support at scoring
 *   time), in descending order; equal values are ordered by lower index.
 *   The order is the IEEE-754 total order of the values with -0 equal to +0
 *   (a +NaN ranks above +inf, a -NaN below -inf).
 *     idx [N, k] int32 out; logp [N, k] fp32 out (nullable) = log softmax(z)
 *     at idx.  1 <= k <= min(V, OPD_K_MAX).
 *
 * opd_score_actions: log softmax(z) at given ids (teacher scoring of cached
 *   actions, or rollout log-probs of a given support).
 *     ids [N, K] int32 in (repeats allowed); logp [N, K] fp32 out, NaN for an
 *     id outside [0, V).  1 <= K <= OPD_K_MAX.
 *
 * Errors as for opd_loss_fwd_bwd: OPD_ERR_DTYPE, OPD_ERR_SHAPE,
 * OPD_ERR_SUPPORT (M, k or K out of range), OPD_ERR_ALIGN, OPD_ERR_NULL (a
 * required pointer), OPD_ERR_HIP.  N == 0 is a no-op returning OPD_OK.
 */
int opd_sample_actions(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
                       int32_t M, const float* uniforms, const uint8_t* mask, int32_t* sampled_ids,
                       float* logp, float* lse_out, void* stream);
int opd_topk_support(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld, int32_t k,
                     const uint8_t* mask, int32_t* idx, float* logp, float* lse_out, void* stream);
int opd_score_actions(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t ld,
                      const int32_t* ids, int32_t K, const uint8_t* mask, float* logp,
                      float* lse_out, void* stream);

/*
 * The rows of logits (Sec. 4.1: Stage 1 draws from the rollout policy's rows,
 * Stage 2 scores on the teacher's): the product of hidden states and an output
 * head in 8-bit floating point, and the quantisation of both.  They serve
 * Stages 1 and 2, which have no backward pass.
 *
 * 8-bit values are OCP e4m3 (no infinities, largest 448, NaN 0x7F / 0xFF).  A
 * scale covers a block of 128 consecutive columns: [0, 128), [128, 256), ..; the
 * last block of a row may be shorter.  nb = ceil(H / 128).  Scales are fp32
 * (OPD_SCALE_F32) or powers of two held as OCP e8m0 (OPD_SCALE_E8M0: one byte,
 * the exponent plus 127; 255 is NaN), which the matrix cores apply themselves.
 *
 * opd_quantize_blocks: blocks of block_rows (1 for hidden states, 128 for head
 *   weights) rows by 128 columns, cut at the edges of x [N, H].  With a the
 *   largest magnitude in the block, the scale s is max(a / 448, 2^-126) in fp32,
 *   or the least power of two that is not below a / 448 (2^-127 at least), and
 *   q = x / s, divided in fp32 and rounded to the nearest e4m3 value, ties to
 *   even; what rounds to zero keeps its sign.  A block that holds a NaN or an
 *   infinity gets a NaN scale and values (0x7F).
 *     x [N, ldx] OPD_F32 or OPD_BF16; q [N, ldq] bytes, columns [H, ldq) are not
 *     written; scales [ceil(N / block_rows), nb].
 *   x and q are 16-byte aligned, ldx * element_size and ldq multiples of 16.
 *
 * opd_head_logits: logits[n, v] = sum_b sx[n, b] sw[v / 128, b] *
 *   sum_{h in block b} x[n, h] w[v, h], in fp32, rounded once to logits_dtype
 *   (OPD_F32 or OPD_BF16).  For fp32 logits products are exact; for bf16 ones
 *   the matrix cores cut each at 2^-13 of the largest of the 16 that they sum
 *   at once, at most 2^-6 of a block's largest product in all.  Of hidden states
 *   with a few channels far larger than the others that is 7e-5 of a logit, where
 *   the rounding to bf16 is 1.7e-3; where larger products cancel it is more, and
 *   such logits are better asked for in fp32.  (Two blocks' scales are multiplied
 *   first; their product should be finite in fp32.)  A NaN in a token's values
 *   or scales reaches its own row only, one in the weights its own vocabulary
 *   entries (a scale: those of its block).
 *     x [N, ldx], x_scales [N, nb]; w [V, ldw], w_scales [ceil(V / 128), nb];
 *     logits [N, ld], as every call here reads them; columns [V, ld) are not
 *     written.
 *   x, w and logits are 16-byte aligned; ldx, ldw and ld * element_size are
 *   multiples of 16.  Rows of x and w are read up to the next multiple of 16
 *   bytes; what is there past H may hold anything.
 *
 * Errors: OPD_ERR_DTYPE (dtype or scale_type), OPD_ERR_SHAPE (N < 0, N >=
 * 2^31, V outside [2, 2^29], H outside [1, 2^22], a row stride below its row's
 * length; in opd_head_logits also ldx or ldw above 2^22, N * V above 2^46),
 * OPD_ERR_PARAM (block_rows not 1 or 128), OPD_ERR_ALIGN, OPD_ERR_NULL,
 * OPD_ERR_HIP.  N == 0 is a no-op returning OPD_OK.
 */
typedef enum opd_scale { OPD_SCALE_F32 = 0, OPD_SCALE_E8M0 = 1 } opd_scale;

int opd_quantize_blocks(const void* x, int32_t dtype, int64_t N, int64_t H, int64_t ldx,
                        int32_t block_rows, int32_t scale_type, void* q, int64_t ldq,
                        void* scales, void* stream);
int opd_head_logits(const void* x, int64_t ldx, const void* x_scales, const void* w, int64_t ldw,
                    const void* w_scales, int32_t scale_type, int64_t N, int64_t V, int64_t H,
                    int32_t logits_dtype, void* logits, int64_t ld, void* stream);

/*
 * Verification of drafted tokens: Stage 1 with a drafter.  B sequences have up
 * to D drafted tokens each; the rollout policy's rows of logits at all of them,
 * and the one after, are at hand.  With p_i = softmax of target row i, q_i that of
 * draft row i, x_i the drafted token and u the uniforms (supplied by the caller,
 * as for opd_sample_actions), token i is kept while u[i] q_i(x_i) < p_i(x_i).  At
 * the first that is not, one token is drawn from max(p_i - q_i, 0) divided by
 * its sum; if all n are kept, from p_n.  If the drafts are draws from q, the
 * tokens that come out are draws from p, whatever q is.
 *
 * The draw is by inversion in index order at u[D]: the first index at which the
 * cumulative mass exceeds u[D] times the whole.  Tests and draw are evaluated in
 * double precision, wherever the logits lie (a row of the type's lowest value is
 * uniform), so they are those of exact arithmetic unless u[i] q_i(x_i) and
 * p_i(x_i) differ by less than about 1e-13 of p_i(x_i), or u[D] times the whole
 * lies within about 1e-13 of a cumulative mass.  (Masses of a residual are not
 * divided by its sum; the sums' part of the 1e-13 is a bound at V = 150,000 and
 * grows with V; probabilities below about 1e-280 may count as 0.)  Where a token
 * is refused and rounding leaves no residual at all (p and q are equal to double
 * precision but for it), the draw is from p.
 *
 *   target_logits  [B * (D + 1), ld], sequence b's rows b (D + 1) .. b (D + 1) + D
 *   draft_logits   [B * D, draft_ld], nullable, of the same dtype: NULL means
 *                  that the drafter is certain of its tokens (q_i is 1 at x_i,
 *                  as for drafts copied from the prompt)
 *   draft_ids      [B, D] int32
 *   draft_lens     [B] int32, nullable (NULL: all D): sequence b has drafts
 *                  [0, draft_lens[b]) and target rows [0, draft_lens[b]]; the
 *                  others are not read.  0 is a plain draw.
 *   uniforms       [B, D + 1] fp32 in [0, 1)
 *   mask           [B] uint8, nullable; a masked sequence (0) is not read
 *   accepted       [B] int32 out: the drafted tokens that were kept
 *   ids            [B, D + 1] int32 out: those, then the drawn token, then -1
 *   logp           [B, D + 1] fp32 out, nullable: log p at these tokens (what
 *                  the MC estimators read as behav_logp), 0 past them
 *   workspace      16-byte aligned, opd_verify_workspace_bytes(...) bytes, of any
 *                  content; calls (and captured graphs) that may overlap need
 *                  one each
 * Rows behind the first refusal have no part in the results and may stay unread.
 * Masked sequences get accepted 0, ids -1 and logp 0.  A sequence ends with id -1
 * and logp NaN, in place of the drawn token, at the first position whose
 * target row (or draft row, where its token is tested) has a NaN or +inf logit or
 * no finite one, whose uniform is outside [0, 1) or whose drafted id is outside
 * [0, V); and at position 0 if draft_lens[b] is outside [0, D].
 *
 * Errors: OPD_ERR_DTYPE, OPD_ERR_SHAPE (B < 0, B (D + 1) >= 2^31, V or a stride
 * out of range), OPD_ERR_SUPPORT (D outside [1, OPD_K_MAX]), OPD_ERR_ALIGN,
 * OPD_ERR_NULL, OPD_ERR_WORKSPACE, OPD_ERR_HIP.  B == 0 is a no-op returning
 * OPD_OK.
 */
int opd_verify_drafts(const void* target_logits, const void* draft_logits, int32_t dtype,
                      int64_t B, int32_t D, int64_t V, int64_t ld, int64_t draft_ld,
                      const int32_t* draft_ids, const int32_t* draft_lens, const float* uniforms,
                      const uint8_t* mask, int32_t* accepted, int32_t* ids, float* logp,
                      void* workspace, size_t workspace_bytes, void* stream);

/* Workspace bytes of opd_verify_drafts (0 for invalid arguments). */
size_t opd_verify_workspace_bytes(int64_t B, int32_t D, int64_t V, int32_t dtype);

/*
 * Token embeddings: rows of a vocabulary-sized table (often the output head's
 * too) for the tokens that Stages 1 to 3 run the model on, and the gradient that the
 * learner's update gives the table.
 *
 * opd_embed_tokens: out[n, :] = scale * table[ids[n], :], in fp32, rounded once.
 * opd_embed_grads: dtable[v, :] = scale * sum of dy[n, :] over the tokens n with
 *   ids[n] == v, summed in fp32 in the order of the tokens (where there is a workspace, an
 *   entry of more than 16 tokens in parts of 16 places of the sorted batch, then over the
 *   parts).  Every row of dtable is written, zeros among them; with accumulate = 1 the sums are
 *   added to what it holds, and the rows of entries without a token stay as they are, unread.
 *     table [V, ld], dtable [V, ldo], dy [N, ldy], out [N, ldo]: OPD_F32 or OPD_BF16, in
 *     any combination, 16-byte aligned rows; columns past H are not written.  Results may
 *     not overlap the inputs.
 *     ids [N] int32.  -1 (what opd_verify_drafts writes past a sequence's last token)
 *     gives a row of zeros and has no part in the gradient; any other id outside
 *     [0, V) gives a row of NaN and has no part in the gradient.
 *     workspace: opd_embed_workspace_bytes(N, V, H) bytes (0 for few tokens: may be
 *     NULL), 16-byte aligned, of any content; calls (and captured graphs) that may
 *     overlap need one each.
 * Errors: OPD_ERR_DTYPE, OPD_ERR_SHAPE (N, V >= 2^31, the gradient's V > 2^31 - 512 where
 * there is a workspace, V < 1, H outside [1, 2^22], a row stride below H), OPD_ERR_PARAM
 * (accumulate), OPD_ERR_ALIGN, OPD_ERR_NULL, OPD_ERR_WORKSPACE, OPD_ERR_HIP.  N == 0 looks
 * nothing up; the gradient is then zeros.
 */
int opd_embed_tokens(const void* table, int32_t dtype, int64_t V, int64_t H, int64_t ld,
                     const int32_t* ids, int64_t N, float scale, void* out, int32_t out_dtype,
                     int64_t ldo, void* stream);
int opd_embed_grads(const void* dy, int32_t dtype, int64_t N, int64_t H, int64_t ldy,
                    const int32_t* ids, int64_t V, float scale, void* dtable, int32_t out_dtype,
                    int64_t ldo, int32_t accumulate, void* workspace, size_t workspace_bytes,
                    void* stream);
size_t opd_embed_workspace_bytes(int64_t N, int64_t V, int64_t H);

/*
 * Low-rank adapters of many requests at once, beside a projection that they share:
 * the output head of opd_head_logits, whose rows of logits they change for each
 * student or teacher, or any other.  Token n has adapter g = adapter_ids[n]:
 *   t = x[n] a_g^T  (r numbers),  out[n] = y[n] + s_g t b_g
 * and the gradients of a loss, from dy = dloss/dout (of logits: what opd_loss_fwd_bwd
 * returns):
 *   u = dy[n] b_g^T,  dx[n] = dx_shared[n] + s_g u a_g,
 *   da_g = s_g sum_n u_n^T x[n],  db_g = s_g sum_n t_n^T dy[n]   (over its tokens)
 *     x [N, ldx], a [G, r, lda], b [G, r, ldb]: dtype.  (Both matrices are held as r
 *     rows of the long axis.)  y, out [N, ..], dy [N, lddy]: y_dtype, which is dtype or
 *     OPD_F32.  out may be y; results overlap no other input.  dx_shared (the shared
 *     projection's gradient; nullable: 0) and dx (nullable: not wanted) [N, ..]: dtype; they
 *     may be one.  da [G, r, ldda], db [G, r, lddb]: OPD_F32; adapters without a token get
 *     zeros.
 *     scales [G] fp32, nullable (1).
 *     adapter_ids [N] int32: -1 for a token without an adapter (out is y, dx is dx_shared);
 *     any other id outside [0, G) gives a row of NaN in out and dx, and no part in da and db.
 *     low_out [N, r] fp32, nullable: t, which opd_adapter_grads takes as low (nullable: it
 *     makes t again) for the same x and a.  Rows of tokens without an adapter are 0.
 *     workspace: opd_adapter_workspace_bytes(...) bytes, 16-byte aligned, of any
 *     content; calls (and captured graphs) that may overlap need one each.
 * Sums are fp32, each result is rounded once.  bf16 operands are multiplied exactly; t
 * and u enter the second product to 2^-25 of themselves.  A NaN or an infinity in a
 * token's x (dy) or in its adapter reaches its own row, and its adapter's da and db; no
 * other's.  (An infinity among bf16 values meets the other factor's parts, of either
 * sign: what would be infinite may then be NaN.)
 * All rows are 16-byte aligned, and read up to the next multiple of 16 bytes; what is there
 * past their end may hold anything, and is not written.
 * Errors: OPD_ERR_DTYPE, OPD_ERR_SHAPE (N > 2^24, H or O outside [1, 2^22], a row stride
 * below its row's length (or one of a or b above 2^22), strides of in-place rows that
 * differ, or a call whose launches would pass 2^32 work-items), OPD_ERR_SUPPORT (G outside
 * [1, OPD_ADAPTERS_MAX], r outside [1, OPD_RANK_MAX]), OPD_ERR_ALIGN, OPD_ERR_NULL, OPD_ERR_WORKSPACE, OPD_ERR_HIP.  N == 0
 * adds nothing; the gradients are then zeros.
 */
#define OPD_ADAPTERS_MAX 1000
#define OPD_RANK_MAX 128
int opd_add_adapters(const void* y, int32_t y_dtype, int64_t ldy, const void* x, int32_t dtype,
                     int64_t ldx, const void* a, int64_t lda, const void* b, int64_t ldb,
                     const float* scales, const int32_t* adapter_ids, int64_t N, int64_t H,
                     int64_t O, int32_t G, int32_t r, void* out, int64_t ldo, float* low_out,
                     void* workspace, size_t workspace_bytes, void* stream);
int opd_adapter_grads(const void* dy, int32_t y_dtype, int64_t lddy, const void* x, int32_t dtype,
                      int64_t ldx, const void* a, int64_t lda, const void* b, int64_t ldb,
                      const float* scales, const int32_t* adapter_ids, int64_t N, int64_t H,
                      int64_t O, int32_t G, int32_t r, const float* low, const void* dx_shared,
                      int64_t ldds, void* dx, int64_t lddx, float* da, int64_t ldda, float* db,
                      int64_t lddb, void* workspace, size_t workspace_bytes, void* stream);
size_t opd_adapter_workspace_bytes(int64_t N, int64_t H, int64_t O, int32_t G, int32_t r,
                                   int32_t dtype, int32_t y_dtype, int32_t backward);

/*
 * Beam search beside the draws: the continuations that a group of W beams goes on with,
 * and the beams' states in their new order.
 *
 * opd_beam_select: rows b W .. b W + W - 1 of the logits are group b's beams, with
 *   scores [B, W].  Candidate (w, v) has score scores[b, w] + log softmax(row)[v]; the k
 *   largest are returned in descending order, ties to the lower beam, then the lower token.
 *   Scores are made and compared in double precision.  A beam's log-sum is good to about 1e-8
 *   for rows of many different logits, and to 2e-7 for any: the order is that of exact arithmetic
 *   unless two beams' scores differ by about as little.
 *     finished [B, W] uint8, nullable: a finished beam (not 0) is one candidate, with its
 *     own score and id -1; its row is not read.  A beam of score -inf (one that does not
 *     exist yet) and a row without a finite logit have no candidates (a masked logit, -inf,
 *     is none either), and a beam of score -inf is not read.
 *     out_scores, parents, ids [B, k]: the scores in fp32, the beams [0, W), the tokens.
 *     Where a group has fewer candidates, the rest get score -inf, parent -1 and id -1.
 *     A group with a score that is NaN or +inf, or a row (that is read) with a NaN or a +inf
 *     logit, gets NaN, -1 and -1 throughout.
 *     workspace: opd_beam_workspace_bytes(B, W, V, dtype) bytes, 16-byte aligned, of any
 *     content; calls (and captured graphs) that may overlap need one each.
 * opd_reorder_beams: state j of group b becomes a copy of the group's state
 *   parents[b, j], for j < k; one whose parent is outside [0, W) becomes zeros.  A state is
 *   `outer` slices of inner_bytes bytes, outer_stride bytes apart; states lie `stride`
 *   bytes apart, b W + w of them before the state of beam w of group b (in out: b k + j).
 *   States of out do not overlap: they lie one after the other, or their slices do (all
 *   states' first slices, then all second ones).  Any element type.  out may be states
 *   (k == W, the same strides): the states are then moved in place, and those that are
 *   their own parent stay.  It may not overlap them otherwise.
 * Errors: OPD_ERR_DTYPE, OPD_ERR_SUPPORT (W or k outside [1, OPD_BEAM_MAX]), OPD_ERR_SHAPE,
 * OPD_ERR_ALIGN, OPD_ERR_NULL, OPD_ERR_WORKSPACE, OPD_ERR_HIP.  B == 0 is a no-op returning
 * OPD_OK.
 */
#define OPD_BEAM_MAX 64
int opd_beam_select(const void* logits, int32_t dtype, int64_t B, int32_t W, int64_t V, int64_t ld,
                    const float* scores, const uint8_t* finished, int32_t k, float* out_scores,
                    int32_t* parents, int32_t* ids, void* workspace, size_t workspace_bytes,
                    void* stream);
size_t opd_beam_workspace_bytes(int64_t B, int32_t W, int64_t V, int32_t dtype);
int opd_reorder_beams(const void* states, int64_t B, int32_t W, int64_t outer, int64_t inner_bytes,
                      int64_t stride, int64_t outer_stride, const int32_t* parents, int32_t k,
                      void* out, int64_t out_stride, int64_t out_outer_stride, void* stream);

/*
 * Diagnostics of the Monte-Carlo estimator: the importance-ratio tail that
 * Sec. 5.2 tracks (the p99 of rho_theta, Fig. 5) and the variance of the
 * m-sample estimator at a fixed prefix and over a sequence (App. E, Table 6).
 * Inputs are per token t what an MC loss call returns or reads: lse [N]
 * (lse_out, log sum_j exp z_j), gathered [N, M] (gathered_out, the student
 * logits at the M draws), teacher_logp and behav_logp [N, M] (the cache).
 * With log p = gathered - lse, A = teacher_logp - log p, rho = exp(log p -
 * behav_logp), the one-sample terms are X = -rho A (the loss is their mean).
 * Outputs (device fp32, each nullable):
 *   row_mean [N]     (1/M) sum_i X_i
 *   row_var [N]      unbiased variance of X_i over i (NaN when M = 1)
 *   row_rho_max [N]  max_i rho_i (NaN ratios ignored)
 *   rho_quantile [1] nearest-rank quantile of rho over all valid entries:
 *                    the r-th smallest, r = max(1, ceil(quantile * n)) (in
 *                    double, from the fp32 quantile); NaN ratios rank above
 *                    +inf
 *   clip_frac [1]    fraction of valid entries with |rho - 1| > clip_eps
 *   ratio_local [n_groups], ratio_seq [n_groups]
 *                    variance ratios for group sizes m = group_sizes[k]
 *                    (host array; M a multiple of m, M / m >= 2): the draws
 *                    of a token split into M / m groups of m consecutive
 *                    draws with means Y_g;
 *                      ratio_local = sum_t var_g(Y_g) / sum_t row_var_t,
 *                    and, with tokens [s seq_len, (s + 1) seq_len) forming
 *                    sequence s and S_g its valid-token average of Y_g,
 *                      ratio_seq = sum_s var_g(S_g) / sum_s var_i(S1_i)
 *                    (S1: the same with single draws).  var is unbiased.
 *                    ratio_seq needs seq_len > 0.
 * Masked tokens (mask[t] == 0) are excluded and get 0 in the per-token
 * outputs.  The workspace (size from opd_mc_diag_workspace_bytes, 16-byte
 * aligned) holds intermediates; the quantile is exact (radix selection with
 * integer histograms); sums run in a fixed order.
 * Errors: OPD_ERR_SHAPE (N < 0 or N >= 2^32 / 64: the batch reductions run
 * in one grid), OPD_ERR_SUPPORT (M outside [1, OPD_K_MAX]),
 * OPD_ERR_PARAM (quantile outside (0, 1], clip_eps negative or not finite,
 * more than 8 or invalid group sizes, seq_len < 0, ratio_seq without
 * seq_len), OPD_ERR_NULL, OPD_ERR_WORKSPACE, OPD_ERR_HIP.
 */
typedef struct opd_mc_diag {
  float* row_mean;
  float* row_var;
  float* row_rho_max;
  float* rho_quantile;
  float* clip_frac;
  float* ratio_local;
  float* ratio_seq;
} opd_mc_diag;

/* Workspace bytes of opd_mc_diagnostics (0 for invalid arguments). */
size_t opd_mc_diag_workspace_bytes(int64_t N, int32_t M, const int32_t* group_sizes,
                                   int32_t n_groups, int64_t seq_len);

int opd_mc_diagnostics(const float* lse, const float* gathered, const float* teacher_logp,
                       const float* behav_logp, int64_t N, int32_t M, const uint8_t* mask,
                       float quantile, float clip_eps, const int32_t* group_sizes,
                       int32_t n_groups, int64_t seq_len, const opd_mc_diag* out, void* workspace,
                       size_t workspace_bytes, void* stream);

/* Static description of a status code ("ok", "null pointer", ...); a code
 * outside opd_status gives "unknown status".  Never NULL. */
const char* opd_status_string(int status);

/* OPD_VERSION of the built library. */
int opd_version(void);

#ifdef __cplusplus
}
#endif
#endif /* OPD_H */

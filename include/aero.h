/*
 * aero.h - C ABI of the GPU library for the per-token hot path of a group-based RL update
 * (GRPO with AERO's curated rollout groups), written for AMD MI355X (gfx950).
 *
 * Conventions (all entry points)
 *   - Every array pointer is a DEVICE pointer owned by the caller.  The library never
 *     allocates or frees device memory; scratch comes from the caller's `workspace` (size it
 *     with aero_workspace_bytes; 256-byte aligned).  The one exception is stated at
 *     aero_grpo_loss_bwd_noalloc, which uses a fixed array inside the library instead.
 *   - Scalars, the parameter struct and the returned status live on the HOST.
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*, NULL = default stream)
 *     and the call returns without synchronising.  Calls that share a workspace must be
 *     ordered on one stream.
 *   - Outputs are fully overwritten (one exception, on request: dlogits rows of token rows marked
 *     AERO_ROW_UNTOUCHED).  Nullable arguments are marked.
 *   - Shape errors that can be seen from host scalars return a status code and enqueue
 *     nothing.  Errors that depend on device data never fault; a bit is OR-ed into the
 *     optional device word `err_flag`, which the caller zeroes:
 *       a sampled-token id >= V or a rollout index >= R: the token row is treated as ignored;
 *       a reward other than 0 or 1 where binary ones are required: the group is still
 *       processed, with every reward other than exactly 1 counted as incorrect.
 *   - "Ignored row": a token row with a negative sampled-token id, a negative rollout
 *     index, or row_active == 0.  It is not read, its outputs are 0 (gradient rows +0, or left as
 *     they are when the rollout index is AERO_ROW_UNTOUCHED), and nothing about it is flagged,
 *     whatever its other fields hold.
 *   - Logits (and hidden states / weights) of the calls up to aero_lmhead_logprob_fused must be
 *     finite.  An infinite or NaN logit gives NaN statistics for its row (the entropy term contains
 *     0 * inf); vocabulary masking with -inf is not part of the policy the paper defines (App. C).
 *     The calls around a drafter, at the end of this file, take masked logits.
 */
#ifndef AERO_H
#define AERO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t aero_status;
enum {
  AERO_OK = 0,
  AERO_ERR_NULL = 1,       /* a required pointer is NULL */
  AERO_ERR_SHAPE = 2,      /* negative size, ld < V, V or H outside the supported range */
  AERO_ERR_DTYPE = 3,      /* dtype code not supported by this call */
  AERO_ERR_ALIGN = 4,      /* pointer or leading dimension violates a stated alignment */
  AERO_ERR_WORKSPACE = 5,  /* workspace NULL, misaligned or smaller than aero_workspace_bytes */
  AERO_ERR_HIP = 6,        /* a HIP launch failed; hipGetLastError has the detail */
  AERO_ERR_LIMIT = 7       /* size beyond the fixed capacity of an entry point that owns its scratch */
};

/* Storage types.  AERO_F16 (IEEE binary16) and AERO_F8E4M3 are accepted by the calls that take logits (logits and
 * dlogits of aero_logprob_fwd, aero_grpo_loss_bwd, aero_topk_logprob, aero_distill_loss_bwd, aero_verify_draft),
 * AERO_F16 by the embedding calls as well (table, out, dout).  fp16 gradient entries round to the fp16 grid (subnormals
 * below 6.1e-5, zero below 3e-8): pass a grad_scale that lifts them, as with any fp16 gradient.
 * AERO_F8E4M3 is the 8-bit float with 4 exponent bits (bias 7) and 3 mantissa bits in the variant without
 * infinities (sign.1111.111 is NaN, largest finite value 448, subnormals are multiples of 2^-9); gradient
 * entries are rounded to nearest even on that grid and saturate at +-448, so a grad_scale is needed all the
 * more.  Arithmetic per element is fp32 whatever the storage type; what is formed in 64 bits is said at its call. */
enum { AERO_F32 = 0, AERO_BF16 = 1, AERO_F16 = 2, AERO_F8E4M3 = 3 };

/* OR-ed into the dweight_dtype argument of aero_lmhead_logprob_fused: dweight += dz^T hidden instead of
 * dweight = ..., i.e. the caller's buffer accumulates the gradient over the micro-batches of a step (the sum is
 * formed in fp32 per entry; with a bf16 buffer the running value is rounded after every call). */
enum { AERO_DW_ACCUMULATE = 0x100 };

/* token_rollout[t] of a token row that belongs to no rollout.  Both are ignored rows; AERO_ROW_UNTOUCHED
 * additionally tells aero_grpo_loss_bwd (and its _noalloc form) not to write the row's dlogits at all, for
 * callers whose consumer of the gradient skips padding rows or who keep those rows zero themselves.  Any other
 * negative value means AERO_ROW_PADDING. */
enum { AERO_ROW_PADDING = -1, AERO_ROW_UNTOUCHED = -2 };

/* bits of the device error word */
enum { AERO_DERR_NONBINARY_REWARD = 1, AERO_DERR_BAD_TARGET = 2, AERO_DERR_BAD_ROLLOUT = 4,
       AERO_DERR_BAD_TEACHER = 8, AERO_DERR_BAD_COUNT = 16 };

/* What a teacher's list says about the ids that are not on it (aero_distill_loss_bwd). */
enum { AERO_TAIL_RENORM = 0, AERO_TAIL_BUCKET = 1 };

/* group_category[q]: low two bits = four-way category by success rate u = c/n with
 * threshold tau (App. C, "Problem Categorization"); bit 2 = rescue stratum u <= S/n
 * (Sec. 4.2 Strategy 1, Alg. 1). */
enum { AERO_CAT_ZERO = 0, AERO_CAT_PARTIAL = 1, AERO_CAT_GOOD = 2, AERO_CAT_PERFECT = 3,
       AERO_CAT_RESCUE_BIT = 4 };

enum { AERO_OP_GROUP_ADVANTAGE = 0, AERO_OP_LOGPROB_FWD = 1, AERO_OP_GRPO_LOSS_BWD = 2,
       AERO_OP_LMHEAD_FUSED = 3, AERO_OP_TOPK_LOGPROB = 4, AERO_OP_DISTILL_LOSS_BWD = 5,
       AERO_OP_VERIFY_DRAFT = 6, AERO_OP_EMBEDDING_BWD = 7, AERO_OP_PREFERENCE_LOSS = 8,
       AERO_OP_PREFERENCE_LOSS_BWD = 9, AERO_OP_GRAD_NORM = 10 };

/* Hyper-parameters of the curation step (Table 8; Sec. 4.2). */
typedef struct {
  int32_t k_ratio;         /* Strategy 3: keep m = k*c incorrect rollouts, k >= 1 (paper: 1)      */
  int32_t s_rescue;        /* Strategy 1: rescue threshold S on the number of correct rollouts (0) */
  int32_t tau_num, tau_den;/* tau = tau_num/tau_den (1/2): u < tau is "partial", else "good"       */
  int32_t zero_keep;       /* Strategy 2: rollouts kept from an all-equal group (4)                */
  int32_t reject_enable;   /* 0 = plain GRPO grouping: every rollout is kept                       */
  int32_t posterior_mode;  /* 0 = all-equal groups get advantage 0; 1 = Beta posterior mean        */
  float alpha0, beta0;     /* Beta prior (1, 1)                                                    */
} aero_adv_params;

const char* aero_status_string(aero_status s);

/* Bytes of workspace the given call needs for these sizes (0 if it needs none).
 * Sizes that do not apply to an op are ignored. */
size_t aero_workspace_bytes(int32_t op, int64_t T, int32_t V, int32_t H, int32_t R, int32_t Q);

/*
 * Group statistics, kept subset, group-relative advantages and per-rollout loss weights.
 *
 * Defines: Eq. 1 (advantage = (r - mean) / std over the group, population std, no epsilon);
 * Sec. 3.2 (all rewards equal => advantage 0); Sec. 4.1 / Alg. 1 and App. C (strata);
 * Sec. 4.2 Strategy 2 (posterior mean u~ = (c + alpha0)/(n + alpha0 + beta0) replaces the
 * mean of all-fail / all-correct groups, zero_keep rollouts kept) and Strategy 3 (partial
 * groups keep all c correct rollouts and m = min(k c, n - c) incorrect ones); Theorem 4.1
 * (statistics are taken over the kept subset); Eq. 2 (weights 1/N and 1/|o_i|).
 *
 * Inputs   rewards[R] f32 (must be exactly 0 or 1 when reject_enable or posterior_mode is
 *          set), lengths[R] i32 (|o_i|, full valid response length), group_offsets[Q+1] i32
 *          (CSR, ascending, off[0] = 0, off[Q] = R, group q = rollouts [off[q], off[q+1]); every rollout
 *          belongs to exactly one group: a rollout outside all groups would be left unwritten), keep_priority[R] u32 or
 *          NULL (down-sampling keeps the smallest (key, index) pairs; NULL = index order).
 * Outputs  adv[R] f32, weight[R] f32 (1/(Q * kept_q * lengths[i]) for kept rollouts, else 0),
 *          keep_mask[R] u8, kept_index[R] i32 (first kept_offsets[Q] entries: kept rollout
 *          indices, ascending), kept_offsets[Q+1] i32 (CSR of kept counts),
 *          group_zero_var[Q] u8 (kept rewards all equal, or nothing kept),
 *          group_category[Q] u8 (AERO_CAT_*).
 * In posterior mode the advantage of an all-equal group is (r - u~)/sqrt(u~(1-u~)).
 * Q = 0 or R = 0 is valid.  p is a host pointer, read before the call returns.
 */
aero_status aero_group_advantage(
    const float* rewards, const int32_t* lengths, const int32_t* group_offsets,
    const uint32_t* keep_priority /*nullable*/, int32_t Q, int32_t R,
    const aero_adv_params* p,
    float* adv, float* weight, uint8_t* keep_mask, int32_t* kept_index, int32_t* kept_offsets,
    uint8_t* group_zero_var, uint8_t* group_category,
    int32_t* err_flag /*nullable*/, void* stream);

/*
 * Softmax policy statistics per token row (App. C: pi = softmax(f_theta); Sec. D: the
 * log-prob of the sampled token is what the update consumes; Table 8: an entropy term is used).
 *   lse[t] = log sum_j exp z[t,j],  logprob[t] = z[t, targets[t]] - lse[t],
 *   entropy[t] = lse[t] - sum_j softmax(z[t])_j z[t,j]          (natural log, temperature 1)
 *
 * logits   [T, ld] row-major, dtype AERO_BF16, AERO_F16, AERO_F8E4M3 or AERO_F32, ld >= V; columns >= V are never
 *          read.  Any alignment works; rows are read as 16-byte vectors between their ragged ends unless the base
 *          is not even a multiple of the element size.
 * targets  i32[T] sampled-token ids; row_active u8[T] or NULL.
 * Outputs  logprob[T], lse[T] f32; entropy[T] f32 or NULL.  Ignored rows get 0.
 * Accumulation is fp32.  T = 0 is valid.  1 <= V <= 2^24.
 */
aero_status aero_logprob_fwd(
    const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
    const int32_t* targets, const uint8_t* row_active /*nullable*/,
    float* logprob, float* entropy /*nullable*/, float* lse,
    int32_t* err_flag /*nullable*/, void* stream);

/*
 * Clipped-ratio surrogate loss (Eq. 2 with beta = 0, sign flipped: loss = -J) and its
 * gradient with respect to the logits (App. A.1).
 *   token t of rollout i = token_rollout[t] with A = adv[i] != 0 and w = weight[i] != 0:
 *     rho = exp(logprob[t] - old_logprob[t])
 *     loss -= w * min(rho A, clip(rho, 1 - eps_lo, 1 + eps_hi) A)
 *     g_t  = -grad_scale * w * A * rho   if the unclipped branch is active
 *            (A > 0: rho <= 1 + eps_hi;  A < 0: rho >= 1 - eps_lo), else 0
 *     dlogits[t, j] = g_t * (1[j == targets[t]] - exp(z[t,j] - lse[t]))
 *   every other row (padding, ignored, A == 0, w == 0, clipped): dlogits row = +0, except rows with
 *   token_rollout[t] == AERO_ROW_UNTOUCHED, whose dlogits row is neither read nor written (their
 *   scalar outputs are 0 like those of any ignored row).
 * Entropy bonus (Table 8 lists a coefficient; it is aggregated with Eq. 2's weights): with
 * entropy_coef = c != 0 every token of a rollout with w != 0, whatever A or the clip decision,
 *     loss -= c * w * H_t,   dlogits[t, j] += grad_scale * c * w * p_j * (ln p_j + H_t),
 *     p_j = exp(z[t,j] - lse[t]), H_t = entropy of row t.
 * KL penalty (the - beta D_KL(pi || pi_ref) term of Eq. 2; the paper names no estimator, the
 * per-token one of the GRPO literature is used): with kl_coef = beta != 0 every token of a rollout
 * with w != 0, clipped or not,
 *     d = ref_logprob[t] - logprob[t],  loss += beta * w * (exp(d) - d - 1),
 *     g_t += grad_scale * beta * w * (1 - exp(d)).
 *
 * logits / dlogits  [T, ld], same dtype and ld; dlogits may alias logits (in place).
 * lse      f32[T] from aero_logprob_fwd, or NULL: then the statistics are computed here.  With
 *          lse == NULL the whole call is one pass over the rows where logits are aligned to their element size and
 *          dlogits, if given, lies at the same offset from 16 bytes as logits, for
 *            rows of at most 320 KB (163840 2-byte logits, 81920 fp32, 327680 8-bit ones), which are held on chip: read once,
 *            written once.  fp32, fp16 and 8-bit rows of more than 128 KB with dlogits only, and from 1, 96 and 192 rows
 *            on; 8-bit rows of more than 64 KB without dlogits up to 512 rows;
 *            rows of at most 1280 KB with dlogits, of which 320 KB are held on chip and the rest is read a second time:
 *            from 256 MB of rows on, below that up to 256 rows of fp32 (at least 24 and 10 MB) and of 2-byte
 *            logits (at least one for every 6 KB of a row's length).
 *          Otherwise a forward pass into the workspace precedes the gradient pass, which stores element by element
 *          where logits and dlogits differ in that offset.
 * entropy  f32[T] from aero_logprob_fwd; read only when lse != NULL and entropy_coef != 0
 *          (AERO_ERR_NULL if missing then), may be NULL otherwise.
 * old_logprob f32[T]; token_rollout i32[T] (AERO_ROW_PADDING / AERO_ROW_UNTOUCHED = no rollout); adv, weight f32[R].
 * entropy_coef  c above; 0 switches the term off (NaN: AERO_ERR_SHAPE).
 * kl_coef, ref_logprob  beta above and f32[T] log pi_ref of the sampled tokens; ref_logprob is read
 *          only when kl_coef != 0 (AERO_ERR_NULL if missing then).
 * Outputs  loss f32[1] (deterministic: fixed-order reduction); clip_frac f32[1] or NULL
 *          (clipped tokens / tokens with A != 0 and w != 0); dlogits or NULL (loss only);
 *          logprob_out f32[T] or NULL: current log-prob of the tokens that carry signal, 0 elsewhere;
 *          entropy_out, lse_out f32[T] or NULL: allowed only with lse == NULL (AERO_ERR_NULL
 *          otherwise); when either is given, logprob_out / entropy_out / lse_out are written for
 *          every row with a valid rollout index and sampled token (as aero_logprob_fwd would),
 *          0 elsewhere.
 * workspace: aero_workspace_bytes(AERO_OP_GRPO_LOSS_BWD, T, V, 0, R, 0).
 */
aero_status aero_grpo_loss_bwd(
    const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
    const int32_t* targets, const float* lse /*nullable*/, const float* entropy /*nullable*/,
    const float* old_logprob, const int32_t* token_rollout,
    const float* adv, const float* weight, int32_t R,
    float eps_lo, float eps_hi, float grad_scale, float entropy_coef,
    float kl_coef, const float* ref_logprob /*nullable*/,
    float* loss, float* clip_frac /*nullable*/, float* logprob_out /*nullable*/,
    float* entropy_out /*nullable*/, float* lse_out /*nullable*/,
    void* dlogits /*nullable*/, int32_t* err_flag /*nullable*/,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * aero_grpo_loss_bwd for callers that cannot allocate device memory and so cannot bring a
 * workspace: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, results and status codes as aero_grpo_loss_bwd, minus `workspace` /
 * `workspace_bytes`: the scratch is a fixed array of device memory inside the library
 * (9 * 4 * AERO_NOALLOC_MAX_T + 256 bytes, about 2.3 MB, held on every GPU the library runs on
 * until the process ends).  The call allocates and frees nothing.
 *   - T > AERO_NOALLOC_MAX_T returns AERO_ERR_LIMIT and enqueues nothing.
 *   - All calls on one GPU share that GPU's array: calls that overlap in time on the same GPU
 *     (different streams, different threads) race; order them on one stream.  The array keeps the
 *     previous call's contents; the call clears what it needs cleared itself.
 *   - The first call on a device looks up the array's address on that device (and may load the
 *     code object): make it once outside any graph capture.
 */
#define AERO_NOALLOC_MAX_T 65536
aero_status aero_grpo_loss_bwd_noalloc(
    const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
    const int32_t* targets, const float* lse /*nullable*/, const float* entropy /*nullable*/,
    const float* old_logprob, const int32_t* token_rollout,
    const float* adv, const float* weight, int32_t R,
    float eps_lo, float eps_hi, float grad_scale, float entropy_coef,
    float kl_coef, const float* ref_logprob /*nullable*/,
    float* loss, float* clip_frac /*nullable*/, float* logprob_out /*nullable*/,
    float* entropy_out /*nullable*/, float* lse_out /*nullable*/,
    void* dlogits /*nullable*/, int32_t* err_flag /*nullable*/, void* stream);

/*
 * The same statistics, loss and gradients with the LM head fused in: logits are
 * z = hidden @ weight^T (no bias, fp32 accumulation of bf16 products) and are never
 * written to memory as a [T, V] tensor.
 *
 * Defines: App. C (the policy is the softmax of the model's final linear layer: pi = softmax(h W^T),
 * temperature 1, Table 8); Eq. 2 (clipped surrogate over the tokens of the kept rollouts, weights
 * 1/N and 1/|o_i|, optional - beta D_KL term); App. A.1 (grad rho = rho grad log pi, clipped tokens
 * contribute nothing, d log pi(y) / d z_j = 1[j = y] - pi_j), carried one step further through
 * z = h W^T: dhidden = dz W, dweight = dz^T h.
 *
 * hidden   bf16 [T, H] row-major, weight bf16 [V, H] row-major, both 16-byte aligned, H % 8 == 0.
 * Forward outputs  logprob[T], lse[T] f32, entropy[T] f32 or NULL.
 * Backward part (old_logprob .. dweight; pass old_logprob == NULL for forward only):
 *   loss f32[1]; dhidden bf16 [T, H] (16-byte aligned) = dz @ weight; dweight [V, H] = dz^T @ hidden in
 *   dweight_dtype (AERO_F32 or AERO_BF16, optionally | AERO_DW_ACCUMULATE), with dz as defined for aero_grpo_loss_bwd
 *   (entropy_coef and kl_coef / ref_logprob included: the entropy of the forward part is used,
 *   also when the `entropy` output is NULL).
 * Rows whose target or rollout index is negative take no part in the contraction (their outputs, the
 * dhidden row included, are 0; AERO_ROW_UNTOUCHED means the same as AERO_ROW_PADDING here); a
 * target >= V is treated the same way and raises AERO_DERR_BAD_TARGET in err_flag.
 * workspace: aero_workspace_bytes(AERO_OP_LMHEAD_FUSED, T, V, H, R, 0) bytes of device memory,
 * 256-byte aligned, owned by the caller, contents undefined before and after the call.
 * Errors: AERO_ERR_SHAPE (T < 0, V < 1 or > 2^24, H < 8, H % 8 != 0, or an operand too large for
 * 32-bit offsets: hidden, weight or 256 padded rows of a gradient operand of 4 GiB or more),
 * AERO_ERR_DTYPE (dweight_dtype), AERO_ERR_NULL, AERO_ERR_ALIGN, AERO_ERR_WORKSPACE,
 * AERO_ERR_HIP (launch failure).  Asynchronous on `stream`; nothing is allocated.
 */
aero_status aero_lmhead_logprob_fused(
    const void* hidden, const void* weight, int64_t T, int32_t H, int32_t V,
    const int32_t* targets,
    float* logprob, float* entropy /*nullable*/, float* lse,
    const float* old_logprob /*nullable => forward only*/, const int32_t* token_rollout,
    const float* adv, const float* weight_rollout, int32_t R,
    float eps_lo, float eps_hi, float grad_scale, float entropy_coef,
    float kl_coef, const float* ref_logprob /*nullable*/,
    float* loss, float* clip_frac /*nullable*/, void* dhidden, void* dweight, int32_t dweight_dtype,
    int32_t* err_flag /*nullable*/,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * The five calls below keep a drafter close to the policy and draft with it: the rollouts that this update is made
 * of are cheaper to generate when a small model proposes tokens and the policy's rows verify several of them at once.
 * Conventions of the three that take logits, besides those at the top of this file:
 *   - Temperature 1, as for the policy (Table 8).
 *   - Masked logits are allowed here: a logit at or below -AERO_LOGIT_LIMIT (-inf, the lowest value of fp32 or bf16, -1e10, as
 *     masks write it) has probability 0.  A row without any other logit is empty: its lse is -inf.  A NaN logit, or one at or
 *     above AERO_LOGIT_LIMIT (+inf), makes the row's lse NaN.
 *   - logits [T, ld] row-major in the four storage types, ld >= V, columns >= V never touched, any alignment; rows are
 *     moved as 16-byte vectors between their ragged ends unless a base is not a multiple of the element size.
 *     1 <= V <= 2^24, T < 2^22 rows.
 */

#define AERO_LOGIT_LIMIT 1.2e9f   /* logits at or below its negative are masked, at or above it make their row NaN */

/*
 * The K largest logits of each row: what a teacher's distribution is handed on as.
 *   index[t, 0 .. K) ids in descending order of the logit, the lower id first where logits are equal (+0 and -0
 *   are equal); logprob[t, k] = z[t, index[t, k]] - lse[t]; lse[t] as aero_logprob_fwd's.
 * Rows with fewer than K unmasked logits: the entries behind them are id -1, log-prob -inf (a NaN logit is not listed
 * and makes the row's log-probs NaN).  Rows with row_active == 0 are not read: ids -1, log-probs and lse 0.
 * 1 <= K <= AERO_TOPK_MAX (AERO_ERR_LIMIT beyond); K > V is valid.  T = 0 is valid.
 * row_active u8[T] or NULL; index i32[T, K], logprob f32[T, K], lse f32[T] or NULL.
 * workspace: aero_workspace_bytes(AERO_OP_TOPK_LOGPROB, T, V, K, 0, 0) (K in the place of H).
 */
#define AERO_TOPK_MAX 256
aero_status aero_topk_logprob(
    const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
    const uint8_t* row_active /*nullable*/, int32_t K,
    int32_t* index, float* logprob, float* lse /*nullable*/,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Distillation from a teacher's top logits: divergence of the student's rows from the lists, and its gradient.
 * Row t with weight w = token_weight[t] != 0, listed ids i_k (distinct, an id < 0 is an absent entry), their log-probs
 * l_k (at most 0; -inf: listed with probability 0), p_k = exp(l_k), q = softmax(z[t]):
 *   AERO_TAIL_RENORM  the teacher is its list: p'_k = p_k / sum p,
 *       L_t = sum_k p'_k (ln p'_k - ln q(i_k)),   dz_j = q_j - p'_j (p'_j = 0 for ids that are not listed)
 *   AERO_TAIL_BUCKET  all other ids are one event: p_r = max(0, 1 - sum p), q_r = sum of q over them,
 *       L_t = sum_k p_k (ln p_k - ln q(i_k)) + p_r (ln p_r - ln q_r),   P = sum p + p_r,
 *       dz_j = P q_j - p_j for listed ids,  (P - p_r / q_r) q_j for the others;
 *       a student without mass outside the list (q_r = 0) has no bucket: p_r counts as 0.
 *   row_loss[t] = L_t,  loss = sum_t w L_t,  dlogits[t, j] = grad_scale w dz_j.
 * Rows with w == 0 are not read; they, rows without a listed entry (in the first form: without teacher probability) and empty rows
 * of the student have L_t = 0 and a dlogits row of +0.  A row with an id >= V or the same id twice is treated alike
 * and raises AERO_DERR_BAD_TEACHER.  Teacher probability on a masked logit makes L_t +inf (the gradient stays finite).
 *
 * logits / dlogits [T, ld], same dtype and ld; dlogits may alias logits (in place), NULL: loss only.
 * teacher_index i32[T, K], teacher_logprob f32[T, K], 1 <= K <= AERO_TOPK_MAX (AERO_ERR_LIMIT beyond); token_weight f32[T].
 * loss f32[1] (fixed-order sum), row_loss f32[T] or NULL.
 * The lists' probabilities, what is added up across threads, logarithms and loss terms are formed in 64 bits, everything per logit in 32.
 * workspace: aero_workspace_bytes(AERO_OP_DISTILL_LOSS_BWD, T, V, 0, 0, 0).
 */
aero_status aero_distill_loss_bwd(
    const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld,
    const int32_t* teacher_index, const float* teacher_logprob, int32_t K,
    const float* token_weight, int32_t tail, float grad_scale,
    float* loss, float* row_loss /*nullable*/, void* dlogits /*nullable*/, int32_t* err_flag /*nullable*/,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Verification of drafted tokens: B sequences, up to G drafted tokens each, from given random numbers; what comes out is
 * distributed as if the policy had drawn every token itself.
 *   p_i = softmax of target_logits[b, i] (i = 0 .. G), q_i = softmax of draft_logits[b, i] (i = 0 .. G-1); with
 *   draft_logits == NULL the drafter has no probabilities (a copied token, say): q_i = 1 at the drafted token, else 0.
 *   Drafted token x_i = draft_tokens[b, i] is accepted while uniform[b, i] q_i(x_i) < p_i(x_i), up to the first refusal
 *   or draft_count[b] tokens: n of them.  The token behind them is the j with the largest r_j / noise[b, j] (the lowest
 *   where equal), r = max(0, p_n - q_n) after a refusal, r = p_n after draft_count[b] accepted tokens; with noise drawn
 *   from the exponential distribution that is a draw from r / sum r.  Where r vanishes, p_n takes its place.
 * Outputs  accepted i32[B] = n; tokens i32[B, G+1]: x_0 .. x_{n-1}, the drawn token, -1 behind it; logprob f32[B, G+1] or
 *          NULL: ln p_i(token) - the old_logprob that the update needs - and 0 behind the drawn token.
 * A drafted id outside [0, V) ends the sequence's drafted tokens in front of it (an id >= V raises AERO_DERR_BAD_TARGET).
 * draft_count[b] < 0: the sequence is idle (nothing read; accepted 0, tokens -1, logprob 0); > G: the same, and
 * AERO_DERR_BAD_COUNT.  A position whose target row is empty or has a NaN logit or one at or above the limit accepts nothing and draws
 * -1 (logprob 0); one whose draft row has is refused and drawn from p.
 *
 * target_logits [B, G+1, ld], draft_logits [B, G, ld] of the same dtype; draft_tokens i32[B, G], draft_count i32[B] or
 * NULL (= G for all), uniform f32[B, G] in [0, 1), noise f32[B, V], > 0 (normal numbers).  0 <= G <= AERO_DRAFT_MAX (AERO_ERR_LIMIT beyond);
 * with G = 0 draft_tokens, uniform and draft_logits may be NULL.  B = 0 is valid.
 * workspace: aero_workspace_bytes(AERO_OP_VERIFY_DRAFT, B * (G + 1), V, 0, 0, B).
 */
#define AERO_DRAFT_MAX 63
aero_status aero_verify_draft(
    const void* target_logits, const void* draft_logits /*nullable*/, int32_t dtype, int32_t B, int32_t G, int32_t V,
    int64_t ld, const int32_t* draft_tokens, const int32_t* draft_count /*nullable*/,
    const float* uniform, const float* noise,
    int32_t* accepted, int32_t* tokens, float* logprob /*nullable*/, int32_t* err_flag /*nullable*/,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * Embedding rows: out[t, :] = scale * table[ids[t], :], formed in fp32 and rounded once.
 * table [V, H] contiguous, out [T, ld_out] (ld_out >= H, columns >= H untouched: rows of a wider buffer), both of dtype AERO_F32, AERO_BF16
 * or AERO_F16; ids i32[T].  A negative id is padding: its row is +0; an id >= V likewise, and raises
 * AERO_DERR_BAD_TARGET.  T < 2^22, 1 <= V <= 2^24, 1 <= H <= 2^20; any element's alignment.
 */
aero_status aero_embedding_fwd(
    const void* table, int32_t dtype, int32_t V, int32_t H, const int32_t* ids, int64_t T, float scale,
    void* out, int64_t ld_out, int32_t* err_flag /*nullable*/, void* stream);

/*
 * Its gradient: dtable[v, :] = scale * sum over the tokens t with ids[t] == v of dout[t, :], rows without a token +0; with
 * AERO_DW_ACCUMULATE in dtable_dtype the sum is added to what dtable holds (for a table that is the LM head too: onto
 * the dweight of aero_lmhead_logprob_fused) and rows without a token are not touched.  A row's sum is formed in fp32 in an order
 * that the ids alone determine (the same bits every time) and rounded once.
 * dout [T, ld_dout] of dtype AERO_F32, AERO_BF16 or AERO_F16; dtable [V, H] contiguous, AERO_F32 or AERO_BF16.  ids, T, V, H as above
 * (ids outside [0, V) take no part).  T = 0 is valid.
 * workspace: aero_workspace_bytes(AERO_OP_EMBEDDING_BWD, T, V, H, 0, 0).
 */
aero_status aero_embedding_bwd(
    const void* dout, int32_t dtype, int64_t T, int32_t H, int64_t ld_dout, const int32_t* ids, int32_t V, float scale,
    void* dtable, int32_t dtable_dtype, int32_t* err_flag /*nullable*/,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * A loss on pairs of rollouts, the first of which is to be preferred (a right and a wrong one of the same query: with k_ratio = 1 the
 * curation keeps as many of either), and its gradient.
 *   log ratio of a rollout   s_r = sum over its tokens t of (logprob[t] - ref_logprob[t]), with `average` divided by their number;
 *                            ref_logprob == NULL counts as 0; a rollout without tokens has s_r = 0
 *   pair p, c = pair_chosen[p], j = pair_rejected[p]:  m_p = beta (s_c - s_j),  x_p = m_p - margin
 *   AERO_PAIR_LOGISTIC       l(x) = (1 - smoothing) ln(1 + e^-x) + smoothing ln(1 + e^x)
 *   AERO_PAIR_HINGE          l(x) = max(0, 1 - x)
 *   AERO_PAIR_SQUARE         l(x) = ((x - 1/2) / beta)^2
 *   loss = sum_p w_p l(x_p),  w_p = pair_weight[p], or 1 / P with pair_weight == NULL
 *   drollout[r] = dloss / ds_r (with `average` divided by the number of tokens: the derivative by each token's log-prob)
 *   dlogits[t, j] = grad_scale drollout[token_rollout[t]] (1[j == targets[t]] - softmax(z[t])_j)
 * A rollout may be in any number of pairs.  Pairs with w_p == 0 or a negative index take no part, nor do those with an index >= R, which raise
 * AERO_DERR_BAD_ROLLOUT; their pair_margin is 0.
 * Log ratios, margins, losses and derivatives are formed in 64 bits.  A token's difference and a pair's part of a derivative are rounded to 32 bits once; the
 * same bits every time.  Pairs in another order change nothing but the loss's last bit, tokens in another order (or other tokens beside them) no more than 2^-47 of the
 * sizes that are added up.
 * A token's logprob - ref_logprob that is infinite makes its rollout's s_r infinite, NaN (or infinities of both signs) NaN.  A
 * margin of +-inf has the loss's limit, and the derivative's; NaN makes the loss, the pair's margin and what derives from it NaN.
 *
 * token_rollout i32[T] (as elsewhere: negative = no rollout, an index >= R the same and raises AERO_DERR_BAD_ROLLOUT); tokens of a rollout may
 * stand anywhere.  pair_chosen, pair_rejected i32[P], pair_weight f32[P] or NULL, ref_logprob f32[T] or NULL.
 * T < 2^25 (2^22 rows of logits), 0 <= R < 2^22, 0 <= P < 2^22; T = 0, R = 0 and P = 0 are valid (arrays without entries may be NULL).
 * params is a host pointer, read before the call returns: beta > 0 and finite, 0 <= smoothing <= 1/2 (looked at by AERO_PAIR_LOGISTIC alone), margin finite.
 */
enum { AERO_PAIR_LOGISTIC = 0, AERO_PAIR_HINGE = 1, AERO_PAIR_SQUARE = 2 };
typedef struct {
  int32_t kind;      /* AERO_PAIR_* */
  int32_t average;   /* 0: log ratios are sums over a rollout's tokens, 1: means */
  float beta, smoothing, margin;
} aero_preference_params;

/*
 * The loss from log-probs (those of aero_logprob_fwd or aero_lmhead_logprob_fused over all micro-batches of a step: a rollout's log ratio needs all
 * of its tokens).  The gradient of a micro-batch is then aero_grpo_loss_bwd's, or aero_lmhead_logprob_fused's, with adv[r] = -drollout[r],
 * weight[r] = 1 and old_logprob the log-probs themselves (a ratio of 1).
 * logprob f32[T] (whatever it is where token_rollout is negative).  Outputs loss f32[1], pair_margin f32[P] (m_p) or NULL, rollout_ratio f32[R] (s_r) or
 * NULL, drollout f32[R] or NULL.
 * workspace: aero_workspace_bytes(AERO_OP_PREFERENCE_LOSS, T, 0, 0, R, P) (P in the place of Q).
 */
aero_status aero_preference_loss(
    const float* logprob, int64_t T, const float* ref_logprob /*nullable*/, const int32_t* token_rollout, int32_t R,
    const int32_t* pair_chosen, const int32_t* pair_rejected, const float* pair_weight /*nullable*/, int32_t P,
    const aero_preference_params* params,
    float* loss, float* pair_margin /*nullable*/, float* rollout_ratio /*nullable*/, float* drollout /*nullable*/,
    int32_t* err_flag /*nullable*/, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The same from logits, with the gradient, where all rollouts of a pair are in one batch of rows.  Conventions of the calls that take masked logits: a sampled token
 * whose logit is masked has log-prob -inf; rows without an unmasked logit take no part (log-prob 0, gradient +0); a row with a NaN or too
 * large logit has log-prob NaN, and NaN makes its gradient row NaN.  A sampled-token id >= V raises AERO_DERR_BAD_TARGET and its row is ignored, as rows with
 * a negative id or rollout index are; dlogits rows marked AERO_ROW_UNTOUCHED are left as they are, other ignored rows are +0.
 * logits / dlogits [T, ld], same dtype and ld; dlogits may alias logits (in place), NULL: loss only.  logprob_out f32[T] or
 * NULL (0 for rows that take no part).
 * workspace: aero_workspace_bytes(AERO_OP_PREFERENCE_LOSS_BWD, T, V, 0, R, P) (P in the place of Q).
 */
aero_status aero_preference_loss_bwd(
    const void* logits, int32_t dtype, int64_t T, int32_t V, int64_t ld, const int32_t* targets,
    const float* ref_logprob /*nullable*/, const int32_t* token_rollout, int32_t R,
    const int32_t* pair_chosen, const int32_t* pair_rejected, const float* pair_weight /*nullable*/, int32_t P,
    const aero_preference_params* params, float grad_scale,
    float* loss, float* pair_margin /*nullable*/, float* rollout_ratio /*nullable*/, float* logprob_out /*nullable*/,
    void* dlogits /*nullable*/, int32_t* err_flag /*nullable*/, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Many tensors at once: their description, laid out once.  aero_tensor_table writes an image of aero_tensor_table_bytes(list, count) bytes to HOST
 * memory; the caller keeps it and copies it to the device (16-byte aligned), and hands both to the calls below.  The image holds the
 * pointers, not what they point to; the device copy also holds a counter, so that calls on one table have to be ordered on one stream.
 *   - Tensors are contiguous, any element's alignment, 0 <= n < 2^32 elements each; count < 2^20.  They do not overlap.
 *   - grad and param f32, bf16 or fp16.  param == NULL: the gradient takes part in the norm alone (the moments are not looked at).
 *   - master f32[n] or NULL: the weights the step is made on; param is then its rounding.  fp16 parameters need one, fp32 ones have none
 *     (AERO_ERR_DTYPE).
 *   - Moments: f32[n] where the scales are NULL, otherwise 8 bits (see aero_adamw_step).  Both moments alike.
 *   - decay multiplies the step's weight_decay (0 for a tensor that does not decay).
 * NULL where a pointer is needed: AERO_ERR_NULL; element alignment: AERO_ERR_ALIGN; count or n out of range: AERO_ERR_SHAPE; an image too small:
 * AERO_ERR_WORKSPACE.
 */
typedef struct {
  void* param;
  const void* grad;
  float* master;
  void *exp_avg, *exp_avg_sq;               /* f32[n], or codes int8[n] and uint8[n] */
  float *exp_avg_scale, *exp_avg_sq_scale;  /* NULL, or f32[(n + 255) / 256] */
  int64_t n;
  int32_t param_dtype, grad_dtype;
  float decay;
} aero_tensor;
#define AERO_MOMENT_BLOCK 256
size_t aero_tensor_table_bytes(const aero_tensor* list, int32_t count);
aero_status aero_tensor_table(const aero_tensor* list, int32_t count, void* image, size_t image_bytes);

/*
 * Norm of all gradients of a table, and the factor that a step multiplies them with:
 *   norm[0] = |grad_scale| sqrt(sum of g^2),   factor[0] = grad_scale min(1, max_norm / norm), max_norm <= 0: grad_scale.
 * grad_scale undoes a scale that the loss was given.  A NaN or infinite gradient makes norm that and factor NaN, at
 * which aero_adamw_step leaves everything as it is.  Squares and sums in 64 bits, in an order that the table alone determines.
 * norm, factor f32[1], either may be NULL.  grad_scale finite, max_norm not NaN (AERO_ERR_SHAPE).  An empty table has norm 0.
 * workspace: aero_workspace_bytes(AERO_OP_GRAD_NORM, 0, 0, 0, 0, 0).
 */
aero_status aero_grad_norm(
    const void* image, void* table, float grad_scale, float max_norm, float* norm /*nullable*/, float* factor /*nullable*/,
    void* workspace, size_t workspace_bytes, void* stream);

/*
 * One step of Adam with decoupled weight decay on every tensor of a table that has parameters.  With t = step[0] + 1, per element:
 *   g = factor grad,   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2,
 *   p = p - rate (decay weight_decay p + (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)),   rate = lr lr_factor,
 * then step[0] = t.  factor f32[1] or NULL (1), lr_factor f32[1] or NULL (1), step i32[1] (>= 0) are device words, so that a captured call
 * follows a schedule and counts its replays.  factor NaN or infinite: the step does not take place, step included.
 * Per element in 32 bits, every product and sum of m and v rounded by itself, the weight's change (decay and step) formed before it meets the weight; 1 - beta^t in 64.
 *
 * Moments in 8 bits: blocks of 256 elements of a tensor share a scale S,
 *   m = c |c| S, c = -127 .. 127, S = max|m| / 127^2;    v = c^4 S, c = 0 .. 255, S = max v / 255^4
 * (steps that grow with the value: 1.6 % at the top of a block, 16 % at a hundredth of it, a smallest m of 6.2e-5 and a smallest sqrt(v) of 1.5e-5 of the
 * largest).  The parameters are stepped with the moments as formed; stored is the code next in value, or with `stochastic` one of the two neighbours at
 * random, so that the stored value's expectation is the moment: v changes by a thousandth a step, which rounding to nearest
 * loses.  A v > 0 is never stored as 0.  S below 2^-126 counts as 0 (all of the block's moments as 0), a block with a moment that is not finite has S = NaN.
 *   y = min(|m| (1 / S), 127^2), c the largest with c^2 <= y, one more if u (2 c + 1) < y - c^2;  for v alike with c^4;  u = 1/2, or at random
 * `stochastic` also rounds bf16 parameters without a master at random (to the neighbour that the added low bits carry to).
 * Random bits: h of the seed, t - 1, the tensor's place k in the list and the element's place i in it, with mix(x): x = (x ^ x >> 16) 0x6A09E667,
 * x = (x ^ x >> 15) 0xBB67AE85, x ^ x >> 16 (32 bits; fractions of sqrt 2 and sqrt 3):
 *   h = mix(mix(mix(seed_lo ^ mix(seed_hi ^ mix(t - 1))) + k) + i);   u = (low half of h + 1/2) / 2^16 for m, of the high half for v; the
 *   parameter's 16 bits are the high half of h 0x9E3779B1.
 * params is a host pointer, read before the call returns: 0 <= beta < 1, eps at least 2^-126 in fp32, lr >= 0 and weight_decay finite (AERO_ERR_SHAPE).
 */
typedef struct {
  double lr, beta1, beta2, eps, weight_decay;
  uint64_t seed;
  int32_t stochastic;
} aero_adamw_params;
aero_status aero_adamw_step(
    const void* image, void* table, const aero_adamw_params* params, int32_t* step,
    const float* factor /*nullable*/, const float* lr_factor /*nullable*/, void* stream);

/*
 * The moments of a table's tensors as numbers (for a checkpoint, say), one tensor behind the other in the list's order (those without parameters
 * have none): avg, avg_sq [sum of n], both of dtype AERO_F32 (exactly what is stored) or AERO_BF16 (rounded once).
 */
aero_status aero_adamw_moments(const void* image, void* table, int32_t dtype, void* avg, void* avg_sq, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AERO_H */

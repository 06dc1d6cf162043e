/*
 * oapl.h -- C ABI of the B200 (sm_100a) OAPL LM-head library.
 *
 * The library computes, for a batch of sampled responses, the trainer policy's
 * sequence log-probabilities ln pi(y_i|x) through the LM head, the group value
 * estimate of Eq. 2, the squared-regression objective of Eq. 3 of the OAPL paper
 * ("Method" section), and the gradient of Eq. 3 with respect to the hidden states
 * and the LM-head weight (Algorithm 1 takes gradient steps on Eq. 3), without ever
 * forming the [N, V] logits tensor.
 *
 * Conventions for every entry point
 *   - Pointers are DEVICE pointers unless the parameter comment says "host".
 *   - The caller owns every buffer.  The library allocates nothing, frees nothing
 *     and never synchronises the device (oapl_get_last_status excepted); all work
 *     is enqueued on `stream` (a cudaStream_t passed as void*).
 *   - Return value: OAPL_OK (0) or a negative oapl_status.  On an argument error
 *     nothing is enqueued.  Errors that only the device can see (a target outside
 *     [0,V) on a live row, decreasing seq_id, a pipeline wait that gave up) are
 *     recorded in the workspace and read back with oapl_get_last_status.
 *   - The current CUDA device must be the one that owns the buffers.
 */
#ifndef OAPL_H_
#define OAPL_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  OAPL_OK = 0,
  OAPL_ERR_INVALID_ARG = -1,         /* null pointer, non-positive size, beta <= 0 or not finite */
  OAPL_ERR_MISALIGNED = -2,          /* H, W, dH, dW or workspace not 16-byte aligned */
  OAPL_ERR_WORKSPACE_TOO_SMALL = -3, /* ws_bytes < oapl_workspace_bytes(problem, flags) */
  OAPL_ERR_UNSUPPORTED_SHAPE = -4,   /* d not a multiple of 64, or sizes beyond int32 index range */
  OAPL_ERR_BAD_TARGET = -5,          /* device: mask==1 and target outside [0,V) */
  OAPL_ERR_BAD_SEQ_ORDER = -6,       /* device: seq_id decreasing or outside [0,S) */
  OAPL_ERR_NONFINITE_INPUT = -7,     /* device: non-finite reward, logit or gradient norm, or group_id outside [0,P) */
  OAPL_ERR_DEVICE_TIMEOUT = -8,      /* device: a bounded pipeline wait expired */
  OAPL_ERR_CUDA = -9,                /* a CUDA runtime/driver call failed */
  OAPL_ERR_BAD_STATE = -10,          /* oapl_loss_bwd without a matching oapl_loss_fwd in ws */
  OAPL_ERR_SEQUENCE_TOO_LONG = -11,  /* device: oapl_loss_fwd_bwd met a sequence longer than its staging capacity */
  OAPL_ERR_OUT_OF_RANGE = -12,       /* device: a row's staged exponentials overflowed or vanished (single-call
                                        paths: some logit exceeds the target's by more than ~128, or H / W hold
                                        non-finite values); use oapl_loss_fwd + oapl_loss_bwd for such inputs */
  OAPL_ERR_BOUND_EXCEEDED = -13      /* device: the batch needs more ranges than the bounds passed in
                                        oapl_call_options allow (more live rows, or a longer sequence) */
} oapl_status;

/*
 * Environment variables, read by every call that uses them (tuning and testing; defaults in
 * parentheses):
 *   OAPL_STAGE_ROWS    rows of staged exponentials per range in the single-call paths (65536)
 *   OAPL_CHUNK_ROWS    rows per logit-gradient chunk of oapl_loss_bwd (18944)
 *   OAPL_SPLITS        vocabulary splits per wave of the logits sweeps (chosen from the L2 budget)
 *   OAPL_L2_BUDGET_MB  L2 budget for the hidden-state blocks of one wave of a sweep (48)
 *   OAPL_ACC_SKEW      K-steps by which the second accumulator of a sweep tile trails the first (4)
 *   OAPL_NVTX          1 = NVTX ranges around the phases a call enqueues, for a timeline profiler (0)
 *   OAPL_SYNC_EVERY    K-steps between the lock-step meetings of the CTA pairs (32; 0 = never)
 * They change workspace sizes and schedules, never results beyond summation order across splits.
 */

/* flags */
#define OAPL_FLAG_NONE 0
#define OAPL_FLAG_FUSED 1 /* oapl_workspace_bytes: size the workspace for oapl_loss_fwd_bwd */

/*
 * One batch, as the paper states the problem (Eq. 2 / Eq. 3): for every prompt x a
 * group of rollouts y_i with rewards r(x, y_i) and the inference engine's
 * log-probabilities; the trainer policy enters through the hidden states H and the
 * LM-head weight W.  Row n of H predicts targets[n]; rows of one sequence are
 * contiguous; only rows with mask==1 (response tokens) count in ln pi(y|x).
 */
typedef struct {
  int64_t N;               /* row positions (padded or packed; the mask decides)             */
  int32_t d;               /* hidden size, multiple of 64                                    */
  int32_t V;               /* vocabulary size, >= 1                                          */
  int32_t S;               /* sequences (rollouts)                                           */
  int32_t P;               /* prompts (groups)                                               */
  const void* H;           /* [N, d] bf16 row-major, 16-byte aligned                         */
  const void* W;           /* [V, d] bf16 row-major, 16-byte aligned; logits = H . W^T       */
  const int32_t* targets;  /* [N]; in [0,V) where mask==1; not read where mask==0            */
  const uint8_t* mask;     /* [N]; 1 = response token                                        */
  const int32_t* seq_id;   /* [N]; non-decreasing, in [0,S)                                  */
  const int32_t* group_id; /* [S]; in [0,P); members of a group need not be adjacent         */
  const float* reward;     /* [S]; finite                                                    */
  const float* logp_inf;   /* [N]; inference-policy token log-probs; read only where mask==1 */
  float beta_v;            /* temperature of Eq. 2 (the paper's beta_1), > 0                 */
  float beta_loss;         /* temperature of Eq. 3 (the paper's beta_2), > 0                 */
  float loss_scale;        /* lambda: 1 = Eq. 3's plain double sum; 1/S = mean per rollout   */
} oapl_problem;

/*
 * Bytes of device workspace the calls below need for `problem` (host call; reads
 * only N, d, V, S, P).  Returns 0 on invalid sizes.  The size grows with N*d and
 * with V (a bounded row-chunk of bf16 logit gradients), never with N*V.
 */
size_t oapl_workspace_bytes(const oapl_problem* problem /*host*/, int flags);

/*
 * ln pi(y_t | x, y_<t) for every row and ln pi(y_i|x) for every sequence: the log
 * of the policy's next-token distribution at the sampled token, summed over the
 * response tokens (the quantity pi(y_i|x) that enters Eq. 3).
 *   token_logp [N] f32: 0 where mask==0.       seq_logp [S] f32 or NULL.
 * Reads H, W, targets, mask, seq_id of `problem`; the other fields may be null.
 */
int oapl_token_logprobs(const oapl_problem* problem /*host*/, float* token_logp, float* seq_logp,
                        void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * Eq. 2: vhat[p] = beta_v * ln( (1/G_p) * sum_{i in group p} exp(reward[i]/beta_v) ),
 * evaluated in max-shifted form; G_p is the member count; a group without members
 * gets 0.  reward [S], group_id [S], vhat [P].  No workspace.
 */
int oapl_value_estimate(const float* reward, const int32_t* group_id, int32_t S, int32_t P,
                        float beta_v, float* vhat, void* stream);

/*
 * Eq. 3 forward: token log-probs -> masked per-sequence log-ratio D_i against
 * logp_inf -> Eq. 2 -> advantage A_i = r_i - vhat -> residual
 * delta_i = beta_loss*D_i - A_i -> loss = loss_scale * sum_i delta_i^2.
 *   loss [1], seq_logp [S], vhat [P], delta [S] (may be NULL), token_logp [N] (may be NULL).
 * Leaves in `ws` what oapl_loss_bwd needs (per-row log-sum-exp, per-sequence
 * coefficients 2*loss_scale*beta_loss*delta_i).
 */
int oapl_loss_fwd(const oapl_problem* problem /*host*/, float* loss, float* seq_logp, float* vhat,
                  float* delta, float* token_logp, void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * Gradient of Eq. 3: with p = softmax(logits) and c_i the coefficient of the row's
 * sequence, g[n,v] = c_i * mask_n * ([v == target_n] - p[n,v]);  dH = g . W,
 * dW = g^T . H.  Must follow oapl_loss_fwd on the same problem and workspace.
 *   dH [N, d] bf16 (rows with mask==0 are written as 0);
 *   dW [V, d] f32; overwritten, or added to when accumulate_dW != 0.
 */
int oapl_loss_bwd(const oapl_problem* problem /*host*/, void* dH, float* dW, int accumulate_dW,
                  void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * Eq. 3 forward and gradient in one call, without recomputing the logits in the backward.
 * Same inputs and outputs as oapl_loss_fwd followed by oapl_loss_bwd (same definitions:
 * Eq. 2, Eq. 3 and g = c_i * mask * (onehot - softmax)), but the work is organised by ranges
 * of whole sequences: for each range the logits pass stores e = exp(z - zref_row) as bf16
 * (zref_row = target logit + 40), the per-sequence coefficients of the range follow from
 * its log-probabilities, and since g = -c_i * e' / sum_v e (e' = e with the target entry
 * lowered by sum_v e) both gradient contractions read the staged e' directly:
 * dH = rowscale(e'.W), dW += e'^T.(scaled H).  Executed work is 6*N*d*V flops instead of 8.
 *
 * Workspace: oapl_workspace_bytes(problem, OAPL_FLAG_FUSED).  It holds e for 65536 rows
 * (2 bytes * round_up(V,512) each; OAPL_STAGE_ROWS in the environment changes the count), so
 * it does not grow with N*V; a sequence with more live rows than that cannot be staged and
 * raises OAPL_ERR_SEQUENCE_TOO_LONG in the status word (outputs are then not meaningful;
 * use the two separate calls).  A target whose probability under the policy is below
 * about e^-128 is outside the range of the staged exponentials: the row's sum overflows and
 * the status word becomes OAPL_ERR_OUT_OF_RANGE.
 */
int oapl_loss_fwd_bwd(const oapl_problem* problem /*host*/, float* loss, float* seq_logp, float* vhat,
                      float* delta /*may be NULL*/, float* token_logp /*may be NULL*/, void* dH, float* dW,
                      int accumulate_dW, void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * oapl_loss_fwd_bwd with what the caller knows about the batch on the host, and with a hook
 * for the data-parallel trainer step (the paper trains with a global batch spread over several
 * GPUs, "Experimental Details"; groups are independent in Eq. 2 / Eq. 3, so ranks hold whole
 * groups and exchange only the sum of dW).
 *
 * The number of live rows exists only on the device, so the call enqueues as many range slots
 * as the row count N could need; slots past the last range return at once.  A caller that
 * built the batch knows better:
 *   live_rows_bound     upper bound on the rows with mask==1 (0 = unknown: N is used);
 *   max_seq_rows_bound  upper bound on the live rows of any one sequence (0 = unknown).
 * They only reduce the number of (empty) launches.  Bounds that turn out too small are detected
 * on the device: the status word becomes OAPL_ERR_BOUND_EXCEEDED and the outputs are not
 * meaningful.
 *   dW_ready_event      a cudaEvent_t (as void*) or NULL.  It is recorded on `stream` right after
 *                       the last launch that writes dW; at that point the last range's dH
 *                       contraction has not started yet.  A second stream that waits for the event
 *                       can start the all-reduce of dW over the ranks under that contraction.
 *                       loss, seq_logp and dH are complete only when `stream` is.
 * options == NULL behaves like oapl_loss_fwd_bwd.
 */
typedef struct {
  int64_t live_rows_bound;
  int32_t max_seq_rows_bound;
  void* dW_ready_event;
} oapl_call_options;

int oapl_loss_fwd_bwd_ex(const oapl_problem* problem /*host*/, float* loss, float* seq_logp, float* vhat,
                         float* delta /*may be NULL*/, float* token_logp /*may be NULL*/, void* dH, float* dW,
                         int accumulate_dW, void* ws, size_t ws_bytes, int flags,
                         const oapl_call_options* options /*host, may be NULL*/, void* stream);

/*
 * The paper's baseline objective on the same LM-head pass: GRPO reweighted by token-level
 * importance ratios (the display in the Background section),
 *     J = 1/G sum_{y in group} 1/|y| sum_t  w_t * min( r_t A, clip(r_t, 1-eps, 1+eps) A ),
 *     w_t = pi_old(y_t|.) / pi_vllm(y_t|.)   (data: no gradient),
 *     r_t = pi(y_t|.) / pi_old(y_t|.),       A = the rollout's normalised advantage.
 *
 * oapl_group_advantage: A_i = (r_i - mean_p) / (std_p + eps) over the members of the
 * rollout's group p (population standard deviation; the paper only says "normalized
 * advantage").  reward [S], group_id [S], advantage [S]; a group without members writes
 * nothing.  eps >= 0.
 *
 * oapl_grpo_loss_fwd_bwd: loss = -loss_scale * sum_i 1/|y_i| sum_t w_t * min(...) (minimised),
 * and its gradient: per response token c_t = dloss/dlp_t = -loss_scale/|y_i| * w_t * A_i * r_t
 * where the unclipped branch is the minimum and 0 where the clipped (constant) branch is;
 * g[n,v] = c_n * ([v == target_n] - p[n,v]),  dH = g . W,  dW = g^T . H.  It runs on the
 * staged pipeline of oapl_loss_fwd_bwd (no logits tensor, no recompute) with per-token instead
 * of per-sequence coefficients.
 *   problem:    H, W, targets, mask, seq_id, logp_inf (= ln pi_vllm per token), loss_scale and
 *               the sizes are read; group_id, reward and the betas are not.
 *   logp_old    [N] f32: ln pi_old per token, read where mask==1.
 *   advantage   [S] f32.     clip_eps >= 0 (the paper's clip ratio 0.2).
 *   loss [1]; seq_logp [S] or NULL; token_logp [N] or NULL; clip_frac [1] or NULL: the fraction
 *   of response tokens on the clipped branch; dH [N,d] bf16; dW [V,d] f32 (overwritten, or
 *   added to when accumulate_dW != 0).
 *   ws: oapl_workspace_bytes(problem, OAPL_FLAG_FUSED) bytes; same limits as oapl_loss_fwd_bwd.
 */
int oapl_group_advantage(const float* reward, const int32_t* group_id, int32_t S, int32_t P, float eps,
                         float* advantage, void* stream);
int oapl_grpo_loss_fwd_bwd(const oapl_problem* problem /*host*/, const float* logp_old,
                           const float* advantage, float clip_eps, float* loss, float* seq_logp,
                           float* token_logp, float* clip_frac, void* dH, float* dW, int accumulate_dW,
                           void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * The optimizer step that follows the gradient in a trainer step, for the LM-head weight:
 * AdamW with gradient clipping by norm, the optimizer of the paper's "Experimental Details"
 * tables (math: lr 1e-6, betas 0.9/0.95, weight decay 1e-2, clip threshold 1e-3; code
 * generation: betas 0.9/0.999, threshold 1.0).  With g = dW * min(1, clip_norm / (||grad|| + 1e-6)),
 * where ||grad||^2 = sum(dW^2) + *other_sq_norm (the squared gradient norm of the model's other
 * parameters, device scalar or NULL), step t >= 1:
 *     m = beta1 m + (1-beta1) g;   v = beta2 v + (1-beta2) g^2;
 *     theta = theta (1 - lr weight_decay) - lr (m / (1-beta1^t)) / (sqrt(v / (1-beta2^t)) + eps).
 * theta is the fp32 `master` copy [n] when given (W then receives its bf16 rounding), else the
 * bf16 W itself.  W [n] bf16 (8-byte aligned), dW / m / v / master [n] f32 (16-byte aligned),
 * all updated in place; n = V*d.  clip_norm <= 0 disables clipping.  grad_norm [1] or NULL
 * receives ||grad||.  ws: oapl_adamw_workspace_bytes() bytes of device scratch (partial sums).
 * Two HBM-bound passes: dW is read twice, every other array once (34 bytes per element with a
 * master copy).
 */
size_t oapl_adamw_workspace_bytes(void);
int oapl_adamw_step(void* W, float* master, const float* dW, float* m, float* v, int64_t n, int64_t step,
                    float lr, float beta1, float beta2, float eps, float weight_decay, float clip_norm,
                    const float* other_sq_norm, float* grad_norm, void* ws, size_t ws_bytes, void* stream);

/*
 * Policy entropy of the trainer policy on the response tokens, the training-dynamics
 * diagnostic of the paper's experiments (the entropy curves of OAPL against GRPO in the
 * "Training dynamics" figure and the "sequence entropy" discussed beside it):
 *     H_n = - sum_v p[n,v] ln p[n,v] = lse_n - sum_v p[n,v] z[n,v],   p = softmax(z).
 * Every forward of this library (oapl_token_logprobs, oapl_loss_fwd, oapl_loss_fwd_bwd)
 * accumulates sum_v exp(z - ref) z next to the log-sum-exp in the same pass over the
 * logits and leaves H_n per response token in the workspace; this call only reads it back:
 *   token_entropy [N] f32 or NULL: H_n, 0 where mask==0;
 *   seq_entropy   [S] f32 or NULL: mean of H_n over the sequence's response tokens
 *                                  (0 for a sequence without any);
 *   mean_entropy  [1] f32 or NULL: mean of H_n over all response tokens of the batch.
 * `problem`, `ws`, `ws_bytes` and `flags` are those of the forward call (OAPL_FLAG_FUSED for
 * oapl_loss_fwd_bwd).  Without a preceding forward on `ws` the status word becomes
 * OAPL_ERR_BAD_STATE and nothing is written.
 */
int oapl_entropy(const oapl_problem* problem /*host*/, float* token_entropy, float* seq_entropy,
                 float* mean_entropy, void* ws, size_t ws_bytes, int flags, void* stream);

/*
 * Scalars a trainer logs next to the loss, from the quantities of Eq. 2 / Eq. 3 that the last
 * loss forward (oapl_loss_fwd, oapl_loss_fwd_bwd, oapl_loss_fwd_bwd_ex) left in `ws`; nothing is
 * recomputed.  With D_i = ln pi(y_i|x) - ln pi_vllm(y_i|x) and A_i = r_i - vhat[g_i]:
 *   stats[0] response tokens of the batch         stats[4] mean A_i over all rollouts
 *   stats[1] mean |D_i| over the rollouts with    stats[5] fraction of the groups (with members)
 *            response tokens                               whose rewards are all equal (A_i = 0)
 *   stats[2] max |D_i| over the same rollouts     stats[6] mean reward
 *   stats[3] sum_i D_i / response tokens          stats[7] 0
 * stats: 8 floats on the device; vhat [P]: the forward's output.  `problem`, `ws`, `ws_bytes`
 * and `flags` are those of the forward (OAPL_FLAG_FUSED for the single calls).  Without a
 * preceding loss forward on `ws` the status word becomes OAPL_ERR_BAD_STATE.
 */
int oapl_batch_stats(const oapl_problem* problem /*host*/, const float* vhat, float* stats, void* ws,
                     size_t ws_bytes, int flags, void* stream);

/* ------------------------------------------------------------------------------------------
 * The inference policy's side of the ratio in Eq. 3.  An engine that samples with lagged weights
 * produces logits, often through an 8-bit LM head; the calls below take ln pi_vllm(y_t|.) from such
 * logits (logp_inf of oapl_problem), give their gradient for objectives that are stated on logits,
 * and form the 8-bit products themselves.  They need no workspace and are one launch each.
 *
 * device_status: device int32 or NULL.  The caller clears it (0); a call only ever changes it from
 * OAPL_OK to the error it met.
 * ------------------------------------------------------------------------------------------ */

/* element types */
#define OAPL_TYPE_BF16 0
#define OAPL_TYPE_F16 1
#define OAPL_TYPE_F32 2
#define OAPL_TYPE_E4M3 3 /* 8-bit floating point, 3 bits of mantissa, largest value 448 */
#define OAPL_TYPE_E5M2 4 /* 2 bits of mantissa, largest value 57344 */

/* N rows of V logits; a row's distribution is softmax(scale * logits). */
typedef struct {
  const void* logits;     /* [N, V], rows ld elements apart; only the natural alignment of the type */
  int64_t N;              /* rows                                                                   */
  int64_t ld;             /* >= V, elements                                                         */
  int32_t V;              /* vocabulary size, >= 1                                                  */
  int32_t type;           /* OAPL_TYPE_BF16, _F16 or _F32                                           */
  const int32_t* targets; /* [N] or NULL; in [0,V) where mask==1                                    */
  const uint8_t* mask;    /* [N] or NULL (all rows live); rows with mask==0 are not read            */
  float scale;            /* in (0, 1e6]: 1 / sampling temperature                                  */
} oapl_logits;

/*
 * With p = softmax(scale * z) of a row z:
 *   token_logp    [N] f32 or NULL: ln p[target]                (needs targets)
 *   token_entropy [N] f32 or NULL: - sum_v p_v ln p_v
 *   token_lse     [N] f32 or NULL: ln sum_v exp(scale * z_v)
 *   top_id  [N,K] int32 or NULL, top_logp [N,K] f32 or NULL: the K largest logits (0 <= K <= 32; at
 *                 least one of the two for K > 0), largest first, equal ones by the lower index,
 *                 and their ln p.
 * Rows with mask==0: 0 in every f32 output, -1 in top_id.  A logit of -inf has probability 0 and is no
 * alternative; where fewer than K are left, top_id is -1 and top_logp -inf.  A row without a finite
 * logit: token_logp and token_lse -inf, token_entropy 0.  A row with a NaN or +inf logit: NaN in every
 * f32 output, status OAPL_ERR_NONFINITE_INPUT.  A target outside [0,V) on a live row: token_logp NaN,
 * status OAPL_ERR_BAD_TARGET.  Results do not depend on the order of execution.
 */
int oapl_logits_logprobs(const oapl_logits* logits /*host*/, float* token_logp, float* token_entropy,
                         float* token_lse, int32_t K, float* top_logp, int32_t* top_id,
                         int32_t* device_status, void* stream);

/*
 * Gradient of sum_n ( g_logp token_logp + g_entropy token_entropy + sum_k g_top ln p[top_id] ):
 *   dlogits_v = scale ( -p_v (G + g_entropy (ln p_v + entropy)) + g_logp [v == target]
 *                       + sum_k g_top_k [v == top_id_k] ),     G = g_logp + sum_k g_top_k.
 *   token_lse [N], token_entropy [N] (needed with g_entropy): as the forward left them.
 *   g_logp [N] or NULL (needs targets); g_entropy [N] or NULL; g_top [N,K] or NULL with top_id [N,K]
 *   (K = 0 without): any K token ids, not only the forward's; an id may occur twice.  Ids and targets
 *   outside [0,V) count for nothing (their share of G included).
 *   dlogits [N,V], the logits' type, rows ld_d elements apart; rows with mask==0 are written as 0.
 *   It may be the logits' own memory (then ld_d == ld) or, with ld_d == ld, lie between their rows; any other
 *   overlap is refused.
 * ln p_v is scale * z_v - token_lse in fp32, whose rounding costs |token_lse| 2^-24 of a probability.  A row whose
 * |token_lse| exceeds 1024 (a large common offset; nothing but a finite mask value such as -1e9) would lose its
 * probabilities that way: there the row's maximum and sum are formed again from its logits, by one CTA (34 us for a
 * row of 152064).  token_lse below -1e30 (no logit but -inf, or a type's lowest value used as a mask) counts
 * as p = 0 throughout: only the point terms are left.
 */
int oapl_logits_logprobs_bwd(const oapl_logits* logits /*host*/, const float* token_lse,
                             const float* token_entropy, const float* g_logp, const float* g_entropy,
                             int32_t K, const float* g_top, const int32_t* top_id, void* dlogits,
                             int64_t ld_d, void* stream);

/* A matrix of 8-bit floating point: element (i, j) stands for
 * data[i * ld + j] * scale[(i / block_rows) * scale_row_stride + (j / 128) * scale_col_stride]. */
typedef struct {
  void* data;               /* 16-byte aligned                              */
  float* scale;
  int64_t rows;
  int64_t cols;             /* the axis that a product contracts            */
  int64_t ld;               /* >= cols, multiple of 16                      */
  int64_t scale_row_stride; /* elements, >= 0; any layout.  Scales of one   */
  int64_t scale_col_stride; /* column block next to one another load best   */
  int32_t type;             /* OAPL_TYPE_E4M3 or OAPL_TYPE_E5M2             */
  int32_t block_rows;       /* 1: a scale per row and 128 columns; 128: per 128 x 128 block */
} oapl_scaled;

/*
 * Quantise x [rows, cols] (bf16, f16 or f32; rows ld_x elements apart) into `out`:
 *   amax = max(largest |x| of the block, 2^-100), scale = amax / top (top: the type's largest value),
 *   values = x * top / amax, correctly rounded to fp32 and then to the 8-bit type (nearest even).  top is 0.875 times
 *   a power of two, and fp32 inputs are multiplied by 0.875 in fp32 first: a quotient within 2^-23 of the middle between
 *   two 8-bit numbers may go to either of them.  16-bit inputs have no such rounding.
 * OAPL_QUANT_POW2: scale = 2^ceil(log2(amax / top)) instead, values = x / scale, rounded once.
 * OAPL_QUANT_TRANSPOSE: out is x turned, [cols, rows], with blocks of the turned matrix.
 * Only rows x cols values are written, never the padding behind a row.  A NaN makes its block's scale and values NaN,
 * an infinity the scale infinite.  Strides of out's scales that give two blocks one place (0 over several blocks, for
 * instance) are refused.
 */
#define OAPL_QUANT_TRANSPOSE 1
#define OAPL_QUANT_POW2 2
int oapl_quantize(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t ld_x,
                  const oapl_scaled* out /*host*/, int flags, void* stream);

/*
 * C [A.rows, B.rows] = A . B^T, or C += A . B^T when accumulate != 0.  A.cols == B.cols; the types and
 * block_rows of A and B may differ.  C: bf16, f16 or f32 (c_type), rows ldc elements apart, natural
 * alignment.  Products of a block of 128 are summed by the tensor cores in fp32, scaled blocks in fp32;
 * one rounding to c_type at the end (accumulate: of the sum with the old C).  Bitwise reproducible.
 * A pipeline wait that runs out (its limit is far above any healthy wait) sets OAPL_ERR_DEVICE_TIMEOUT in
 * device_status, and what was not computed is NaN in C, so that it shows without a status word too.
 *   logits = H . W^T:  A = H, B = W (128 x 128 blocks);
 *   dH = g . W:        A = g, B = W quantised with OAPL_QUANT_TRANSPOSE;
 *   dW = g^T . H:      A = g, B = H, both with OAPL_QUANT_TRANSPOSE (block_rows 1), accumulate.
 */
int oapl_scaled_matmul(const oapl_scaled* A /*host*/, const oapl_scaled* B /*host*/, void* C, int32_t c_type,
                       int64_t ldc, int accumulate, int32_t* device_status, void* stream);

/* ------------------------------------------------------------------------------------------
 * The two sides of the LM head in a model that trains: the embedding (whose table is the head's W where the two are
 * tied), the norms around a block, the last of which makes H, and the gradient norm over all parameters.  With tied
 * weights a step is oapl_embedding, the blocks with oapl_residual_norm, oapl_loss_fwd_bwd, oapl_residual_norm_bwd,
 * oapl_embedding_bwd with accumulate into dW, oapl_grad_norm over dW and the rest, oapl_adamw_step.
 * Matrices are row-major with rows ld elements apart and need only the natural alignment of their type; rows that start on
 * 16-byte boundaries are faster.  Results are the same in every run on one kind of GPU.  device_status as above.
 * ------------------------------------------------------------------------------------------ */

/* N token ids of a vocabulary of V. */
typedef struct {
  const int32_t* ids;  /* [N]; in [0,V) where mask==1                                        */
  const uint8_t* mask; /* [N] or NULL (all rows count); ids of rows with mask==0 may hold anything */
  int64_t N;
  int32_t V;
  float scale;         /* finite; a scaled embedding's factor, otherwise 1                   */
} oapl_lookup;

/*
 * out[n] = scale * table[ids[n]], rounded once; table [V,d] and out [N,d] of any of the three types.  Rows with mask==0
 * become 0.  An id outside [0,V) on a row that counts: 0, status OAPL_ERR_BAD_TARGET.  out does not overlap the table.
 */
int oapl_embedding(const oapl_lookup* lookup /*host*/, const void* table, int32_t table_type, int64_t ld_table, int32_t d,
                   void* out, int32_t out_type, int64_t ld_out, int32_t* device_status, void* stream);

/*
 * dtable[v] = scale * sum of dout[n] over the rows with ids[n] == v that count, or that added to dtable when
 * accumulate != 0 (rows of dtable without such a row are then not touched; they become 0 otherwise).
 * dout [N,d] bf16, f16 or f32; dtable [V,d] f32, apart from dout.  Sums are fp32, in the order of the rows, cut into
 * stretches of a batch.  An id outside [0,V) on a row that counts adds nothing and sets OAPL_ERR_BAD_TARGET.
 * N <= 2e9, d <= 2e9.  ws: oapl_embedding_workspace_bytes(N, V, d) bytes (0 for sizes that are refused), 16-byte aligned.
 */
size_t oapl_embedding_workspace_bytes(int64_t N, int32_t V, int32_t d);
int oapl_embedding_bwd(const oapl_lookup* lookup /*host*/, const void* dout, int32_t type, int64_t ld_dout, int32_t d,
                       float* dtable, int64_t ld_dtable, int accumulate, int32_t* device_status, void* ws,
                       size_t ws_bytes, void* stream);

/* kinds of a gate */
#define OAPL_GATE_NONE 0
#define OAPL_GATE_ROW 1    /* one factor per row: [N], ld_gate elements apart                     */
#define OAPL_GATE_COLUMN 2 /* one per channel: [d]                                                */
#define OAPL_GATE_FULL 3   /* [N,d], of the rows' type, rows ld_gate elements apart               */

/*
 * The end of a block with result y on the residual stream x, and the norm before what follows:
 *   u = w_post * y / rms(y) (u = y without w_post),   x' = residual_scale * x + branch_scale * gate * u,
 *   h = w_pre * x' / rms(x'),                         rms(v) = sqrt(mean v^2 + eps).
 * Without y: x' = residual_scale * x, the norm alone.  A weight counts as weight + weight_offset (1 where a model stores
 * the difference from 1).
 * Squares are added in fp32: a row whose sum of squares leaves its range (elements of 1.8e19 / sqrt(d) and more) has
 * 1 / rms = 0, and a row of zeros needs eps > 0.
 */
typedef struct {
  int64_t N;
  int32_t d;               /* 1 .. 16384                                                          */
  int32_t type;            /* of x, y, a full gate and all matrices below                         */
  const void* x;           /* [N,d]                                                               */
  int64_t ld_x;
  const void* y;           /* [N,d] or NULL                                                       */
  int64_t ld_y;
  const void* gate;        /* NULL with OAPL_GATE_NONE; otherwise needs y                         */
  int64_t ld_gate;         /* row and full gates                                                  */
  int32_t gate_kind;
  int32_t gate_type;       /* any of the three types; a full gate: the rows' type                 */
  const void* w_post;      /* [d] or NULL: no norm of y.  Needs y                                 */
  const void* w_pre;       /* [d] or NULL: no norm of x'                                          */
  int32_t weight_type;
  float weight_offset;
  float eps;               /* >= 0, finite                                                        */
  float residual_scale;    /* finite                                                              */
  float branch_scale;      /* finite                                                              */
} oapl_residual;

/*
 * Forward.  x_out [N,d]: x', or NULL; h [N,d]: with w_pre, NULL without; rstd_post [N], rstd_pre [N] f32 or NULL:
 * 1 / rms of y and of x' (with w_post, w_pre), which the gradient reads.  h and the statistics are formed from x' in
 * fp32, before it is rounded to its type.  x_out and h may each lie exactly over x, y or a full gate (the same rows);
 * other overlaps are refused.
 */
int oapl_residual_norm(const oapl_residual* residual /*host*/, void* x_out, int64_t ld_x_out, void* h, int64_t ld_h,
                       float* rstd_post, float* rstd_pre, void* stream);

/*
 * Gradient.  x_out (with w_pre), rstd_post (with w_post), rstd_pre (with w_pre): as the forward left them; x is not read
 * and may be NULL.  dh [N,d] (with w_pre) and dx_out [N,d] or NULL (0; needed without w_pre): the gradients of h and x'.
 *   dx [N,d], dy [N,d] (with y), or NULL; they may each lie exactly over x_out, dh, dx_out, y or a full gate;
 *   dgate or NULL: a row gate's [N] f32, ld_dgate elements apart; a channel gate's [d] f32; a full gate's [N,d], like dy;
 *   dw_post, dw_pre [d] f32 or NULL.
 * accumulate != 0: dw_post, dw_pre and a channel gate's dgate are added to what is there.
 * ws: oapl_residual_norm_workspace_bytes(N, d) bytes, 16-byte aligned; needed where one of those three sums is asked for.
 */
size_t oapl_residual_norm_workspace_bytes(int64_t N, int32_t d);
int oapl_residual_norm_bwd(const oapl_residual* residual /*host*/, const void* x_out, int64_t ld_x_out,
                           const float* rstd_post, const float* rstd_pre, const void* dh, int64_t ld_dh,
                           const void* dx_out, int64_t ld_dx_out, void* dx, int64_t ld_dx, void* dy, int64_t ld_dy,
                           void* dgate, int64_t ld_dgate, float* dw_post, float* dw_pre, int accumulate, void* ws,
                           size_t ws_bytes, void* stream);

/* One tensor of a list: n elements in a row. */
typedef struct {
  const void* data;  /* bf16, f16 or f32, natural alignment (16-byte alignment of data and out is faster) */
  void* out;         /* where the scaled elements go: data itself, memory of its own, or NULL for the norm alone */
  int64_t n;         /* >= 0; a tensor of none is passed over                                         */
  int32_t type;
  int32_t out_type;  /* type where out is data                                                       */
} oapl_tensor;

/*
 * sq_norm [1] f32 = sum of (scale * g)^2 over all elements of the list, norm [1] f32 its square root; one of them may be
 * NULL.  A thread adds 16 or 32 squares in fp32 where that is exact to fp32 rounding, else in fp64, as all sums from there, so
 * norm is right where sq_norm leaves the range of fp32: a norm above 1.8e19 makes sq_norm infinite.
 * OAPL_ERR_NONFINITE_INPUT: a norm that is not finite in fp32, or an infinite sq_norm where norm is NULL.  The list is read
 * during the call only.  ws: oapl_grad_norm_workspace_bytes(count) bytes, 16-byte aligned.  sq_norm is what
 * oapl_adamw_step takes as other_sq_norm; an infinite one makes the clipped gradient of that step 0.
 */
size_t oapl_grad_norm_workspace_bytes(int32_t count);
int oapl_grad_norm(const oapl_tensor* tensors /*host*/, int32_t count, float scale, float* sq_norm, float* norm,
                   int32_t* device_status, void* ws, size_t ws_bytes, void* stream);

/*
 * out = g * scale * min(1, clip_norm / (sqrt(*sq_norm) + 1e-6)) for every tensor of the list, rounded once.  sq_norm: of
 * oapl_grad_norm with the same scale, or such a sum over several ranks.  Where it is not finite the factor is scale
 * alone, so a norm above 1.8e19 is not clipped by its square: the caller leaves out the step, or calls the form below.
 * Elements that the factor 1 would leave in place are not read.  No out overlaps a tensor other than its own.
 */
int oapl_grad_clip(const oapl_tensor* tensors /*host*/, int32_t count, float scale, const float* sq_norm,
                   float clip_norm, void* stream);

/*
 * The same with the norm itself, which is finite wherever oapl_grad_norm reports no error: with norm [1] f32 the factor is
 * scale * min(1, clip_norm / (*norm + 1e-6)) and sq_norm, which may be NULL, is not read; without norm it is the call above.
 */
int oapl_grad_clip_ex(const oapl_tensor* tensors /*host*/, int32_t count, float scale, const float* sq_norm,
                      const float* norm, float clip_norm, void* stream);

/*
 * What a sampler does to logits before it samples, which a trainer that re-scores its tokens has to repeat.  For a token v
 * of row n, c: how often it is in the row's answer, seen: whether it is in the row's prompt or answer,
 *   z1 = seen ? (z > 0 ? z / repetition : z * repetition) : z,
 *   z2 = z1 - frequency * c - presence * [c > 0],   z3 = z2 + the sum of its biases,   result = allowed ? z3 : -inf.
 * Samplers differ in their order.  One that adds biases before the repetition penalty gives a token with both another logit;
 * its rows are had from two calls, the biases first (16-bit logits are rounded in between), gradients from the second's.
 */
typedef struct {
  const int32_t* tokens;    /* [T] or NULL: token ids of all rows' prompts and answers; ids outside [0,V) count for nothing */
  int64_t T;
  const int64_t* spans;     /* [N,3], with tokens: row n's prompt is tokens[s0 .. s1), its answer tokens[s1 .. s2);
                               rows may share tokens.  At most 2^30 - 1 tokens in an answer                             */
  const float* repetition;  /* [N] or NULL: > 0                                                                         */
  const float* frequency;   /* [N] or NULL                                                                              */
  const float* presence;    /* [N] or NULL                                                                              */
  const int64_t* bias_start;/* [N+1] or NULL: row n's biases are entries bias_start[n] .. bias_start[n+1) of the next two */
  const int32_t* bias_id;   /* [biases]; an id may occur several times in a row, ids outside [0,V) count for nothing     */
  const float* bias;        /* [biases]                                                                                 */
  int64_t biases;
  const uint32_t* allowed;  /* [allowed_rows, ld_allowed] or NULL: token v is allowed where bit v % 32 of word v / 32 is set */
  int64_t ld_allowed;       /* >= ceil(V / 32), words                                                                   */
  int64_t allowed_rows;
  const int32_t* allowed_row; /* [N] or NULL (row n of allowed, which then has N rows): a row of allowed; negative: all tokens */
} oapl_adjust;

/*
 * out [N,V], the logits' type, rows ld_out elements apart: the logits' own memory (then ld_out == ld, and only what
 * changes is touched) or memory apart.  Rows with the logits' mask==0 are neither read nor written; targets and scale of
 * `logits` are not used.  Unchanged logits keep their bits.  Spans that decrease or leave [0,T], biases that leave
 * [0,biases]: none for that row, status OAPL_ERR_BAD_SEQ_ORDER; an allowed_row past allowed_rows: no mask for that row,
 * OAPL_ERR_BAD_TARGET.  Each of a row's biases is compared with all of them: lists are meant to have up to a few hundred.
 */
int oapl_logits_adjust(const oapl_logits* logits /*host*/, const oapl_adjust* adjust /*host*/, void* out, int64_t ld_out,
                       int32_t* device_status, void* stream);

/*
 * Gradient: dlogits_v = allowed ? (seen ? (z > 0 ? d_out / repetition : d_out * repetition) : d_out) : 0.  `logits`: as
 * they were before the adjustment (read only at tokens that are seen).  d_out, dlogits [N,V] of the logits' type; dlogits
 * may lie exactly over d_out or the logits.  Rows with mask==0 are written as 0.
 */
int oapl_logits_adjust_bwd(const oapl_logits* logits /*host*/, const oapl_adjust* adjust /*host*/, const void* d_out,
                           int64_t ld_d_out, void* dlogits, int64_t ld_dlogits, int32_t* device_status, void* stream);

/* Synchronises `stream` and returns the status word the device recorded in `ws`
 * since the last forward call (OAPL_OK if none). */
int oapl_get_last_status(void* ws, void* stream);

/* Number of live rows (mask==1) counted by the last forward call on `ws`;
 * synchronises `stream`.  Negative oapl_status on error. */
int64_t oapl_get_live_rows(void* ws, void* stream);

/* Number of ranges of whole sequences the last single call (oapl_loss_fwd_bwd,
 * oapl_loss_fwd_bwd_ex, oapl_grpo_loss_fwd_bwd) on `ws` planned; synchronises `stream`. */
int oapl_get_range_count(void* ws, void* stream);

/* Kernel launches enqueued by this library in this process so far. */
uint64_t oapl_launch_count(void);

const char* oapl_status_string(int status);

/*
 * oapl_token_logprobs for callers that cannot provide a workspace.  (The paper has no
 * counterpart; this is a property of the library, not of the method.)
 *
 * Who needs it: code that is not allowed to allocate device memory where it calls us --
 * a plug-in inside a framework that owns the allocator, a serving loop whose memory was
 * fixed at start-up, or a section in which the CUDA allocator must not be entered.  The
 * scratch memory lives in a fixed device array inside the library (about 4.8 MB per GPU
 * that loads the library, held until the process exits), so sizes are limited:
 *     N <= 2048,  d <= 1024 (multiple of 64),  S <= 2048,  any V >= 1.
 * Larger problems return OAPL_ERR_UNSUPPORTED_SHAPE and print the limits to stderr.
 * The call itself allocates and frees nothing.
 *
 *   token_logp [N] f32, seq_logp [S] f32 or NULL: as in oapl_token_logprobs.
 *   device_status: device int32 or NULL; receives the device-detected status word
 *                  (OAPL_OK, OAPL_ERR_BAD_TARGET, OAPL_ERR_BAD_SEQ_ORDER, ...) in stream order.
 *
 * The first call on each device looks up the array's device address (with that device
 * current); make that first call before starting any stream capture.  All calls on one
 * GPU share the one array and it keeps the previous call's contents; the call clears the
 * parts that must start at zero, but two calls whose work overlaps on the GPU (different
 * streams without ordering, or several host threads) race on it and give wrong results:
 * order them.
 */
int oapl_token_logprobs_static(const oapl_problem* problem /*host*/, float* token_logp, float* seq_logp,
                               int32_t* device_status, void* stream);

/* ------------------------------------------------------------------------------------------
 * Testing and timing aids.  Nothing below is part of the method; a trainer does not need it.
 * ------------------------------------------------------------------------------------------ */

/*
 * Host logic only: the number of range slots the single call enqueues for a batch of at most
 * live_rows_bound live rows in S sequences of at most max_seq_rows_bound live rows each
 * (0 = unknown) and a staging capacity of stage_rows rows -- an upper bound on the number of
 * ranges the greedy packing of whole sequences can produce.
 */
int oapl_range_slots(int64_t live_rows_bound, int64_t max_seq_rows_bound, int32_t stage_rows, int32_t S);

/*
 * Optional timing of the contraction launches (off by default).  oapl_profile_enable(1)
 * switches it on for the CURRENT device: from then on every contraction launch on that device
 * is bracketed by a CUDA event pair on its stream (launches on other devices run untimed).
 * oapl_profile_read waits for those events and sums the elapsed milliseconds and the launch
 * counts per kind into host arrays of `kinds` entries: 0 = logits + online log-sum-exp,
 * 1 = logit-gradient chunk, 2 = dH, 3 = dW, 4 = bring-up GEMM, 5 = logits + staged
 * exponentials; then clears the record.  At most 65536 launches are recorded between two
 * reads; *launches_dropped (host, may be NULL) receives how many were not.  Not thread-safe.
 */
int oapl_profile_enable(int on);
int oapl_profile_read(float* ms_by_kind /*host*/, int* launches_by_kind /*host*/, int kinds,
                      int* launches_dropped /*host*/);
/*
 * While the timing is enabled, CTA 0 of every contraction launch also adds its SM cycle count
 * and its elapsed nanoseconds to two per-kind device counters.  This call (with the device the
 * timing was enabled on current) synchronises the device, writes cycles/nanoseconds as MHz per
 * kind (0 where the kind did not run) -- the SM clock that kind of launch ran at, which on a
 * power-capped part differs from kind to kind -- and clears the counters.  kinds <= 8.
 */
int oapl_profile_read_clocks(float* sm_mhz_by_kind /*host*/, int kinds);
/* The rule the launches apply (host logic only, no CUDA call): 1 when a launch on
 * `current_device` is timed given that the timing was enabled on `enabled_device` (-1 = off). */
int oapl_profile_applies(int enabled_device, int current_device);

/*
 * Bring-up aid for the tensor-core main loop shared by every contraction above:
 * C[M, N] (f32 row-major, ld = N) = A . B with bf16 operands, through the same
 * TMA/tcgen05 pipeline.  a_mn == 0: A is [M, K] row-major (K contiguous);
 * a_mn == 1: A is stored [K, M] row-major (M contiguous).  b_mn == 0: B is stored
 * [N, K] row-major; b_mn == 1: B is stored [K, N] row-major.  wide == 0: 256 x 256 tiles
 * with alternating accumulators; wide == 1: 256 x 512 tiles (the shape of every product
 * contraction).  K % 64 == 0, M % 8 == 0, N % 8 == 0.
 * `err` points to TWO device ints: err[0] (cleared by the caller) is set by the kernel to
 * OAPL_ERR_DEVICE_TIMEOUT when a pipeline wait gave up; err[1] is the counter of the CTA pairs'
 * lock-step meetings (cleared by the call; OAPL_SYNC_EVERY=0 switches the meetings off).
 *
 * Test of the give-up path: wait_cycles > 0 replaces the limit of every pipeline wait (SM
 * cycles; 0 = the product limit of 4e9), and skip_step = k > 0 makes the load warps leave out the
 * loads of pipeline step k - 1, so that the wait for them runs out: every role then leaves its
 * loop, the kernel frees its tensor memory and returns, and err[0] holds the timeout status
 * (C is not meaningful).  skip_step needs 0 < wait_cycles <= 1e8.  Nothing faults and the
 * context stays usable.
 */
int oapl_debug_gemm(const void* A, const void* B, float* C, int M, int N, int K, int a_mn,
                    int b_mn, int wide, long long wait_cycles, int skip_step, int* err, void* stream);

/*
 * oapl_scaled_matmul with the two arguments of the give-up path's test, as above: wait_cycles > 0 (at most 4e9, the
 * product limit) replaces the limit of every pipeline wait, and skip_step = k > 0 (with 0 < wait_cycles <= 1e8) leaves
 * out the loads of every CTA's pipeline step k - 1: a block of 128 of K, for at most 64 rows of A two or four of them.
 * device_status is needed.
 */
int oapl_debug_scaled_matmul(const oapl_scaled* A /*host*/, const oapl_scaled* B /*host*/, void* C, int32_t c_type,
                             int64_t ldc, int accumulate, int32_t* device_status, long long wait_cycles,
                             int skip_step, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* OAPL_H_ */

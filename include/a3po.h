/*
 * a3po.h — C ABI of the B200 (sm_100a) A-3PO log-prob + loss library.
 *
 * The library computes the data-parallel hot path of one A-3PO training step:
 *   hidden states --LM head + log-softmax + gather--> log pi_theta(a_t|s_t)
 *   --> A-3PO decoupled clipped loss with the staleness-interpolated proximal anchor
 *   --> dL/dlogp --> dL/dhidden, dL/dW_lmhead.
 *
 * Conventions for every entry point (unless an argument says otherwise):
 *   - Pointers are DEVICE pointers owned by the caller.  The library allocates no device
 *     memory: scratch space is the caller's `ws` buffer (size it with the *_workspace_bytes
 *     functions; 256-byte aligned).  Contents of `ws` are undefined before and after a call.
 *     Besides that, the library's device image holds two fixed arrays per GPU: 8 KB of
 *     counters with which the CTAs of a tensor-core launch keep in step (advisory, all zero
 *     between launches), and the scratch of a3po_loss_fwd_static.
 *   - Work is enqueued on `stream` (a cudaStream_t passed as void*; NULL = legacy default
 *     stream).  Calls never synchronise the device and are asynchronous w.r.t. the host.
 *     A call with device inputs is a fixed sequence of launches (row counts stay on the
 *     device), so it may be captured into a CUDA graph and replayed; make one uncaptured call
 *     per device first (it resolves kernel attributes and the addresses of the library's
 *     device arrays).
 *   - Return value: A3PO_OK or a negative a3po_error.  Argument errors are detected on the
 *     host before anything is launched; nothing is written in that case.
 *   - Conditions that only the device can see (a target index outside [0,V), a bounded wait
 *     that ran out) are OR-ed into the optional device word `status` (see A3PO_STATUS_*); the
 *     caller reads it after its own synchronisation.  An out-of-range target is clamped into
 *     range, never dereferenced.
 *   - N is the number of token rows.  Row-major layouts: hidden [N,H], W [V,H] (the LM head
 *     as stored by the model: one row per vocabulary entry), grad_hidden [N,H], grad_w [V,H].
 *   - `targets[t]` is the token whose probability is wanted at row t (the caller has already
 *     applied the next-token shift).
 *   - N = 0 is valid everywhere and is a no-op that still defines scalar outputs (loss = 0).
 */
#ifndef A3PO_H_
#define A3PO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  A3PO_OK = 0,
  A3PO_ERR_INVALID_ARG = -1,  /* NULL where a pointer is required, negative size, eps < 0 ...   */
  A3PO_ERR_UNSUPPORTED = -2,  /* dtype/shape/alignment the kernels do not handle                */
  A3PO_ERR_WORKSPACE = -3,    /* ws is NULL, misaligned or smaller than the minimum             */
  A3PO_ERR_CUDA = -4,         /* a CUDA runtime/driver call or a kernel launch failed           */
  A3PO_ERR_NO_DEVICE = -5,    /* no usable sm_100 device is current                             */
  A3PO_ERR_TOO_LARGE = -6     /* N exceeds the fixed scratch of a3po_loss_fwd_static            */
} a3po_error;

/* Storage type of hidden, W and grad_hidden.  Accumulation is always fp32. */
typedef enum { A3PO_F32 = 0, A3PO_BF16 = 1 } a3po_dtype;

/* Bits of the optional device status word. */
#define A3PO_STATUS_TARGET_OUT_OF_RANGE 1u /* some targets[t] was outside [0,V) and was clamped */
#define A3PO_STATUS_WAIT_TIMEOUT 2u        /* a bounded pipeline wait expired; results invalid  */
#define A3PO_STATUS_KEPT_RANGE 4u          /* keep-path only: some row's target probability is below
                                              about 1e-37, beyond what the kept ratios can express;
                                              that row's gradient contribution was dropped          */

/* Side outputs of the loss forward: the paper's per-step stability diagnostics
 * (importance-weight max/min, Fig. 5; number of clipped tokens, Fig. 6). */
typedef struct {
  int64_t n_valid;   /* M = number of tokens with mask != 0                                     */
  int64_t n_clipped; /* valid tokens whose clipped term is the strict minimum (zero gradient)   */
  float iw_max;      /* max over valid tokens of pi_prox/pi_behav (0 if M == 0)                 */
  float iw_min;      /* min over valid tokens of pi_prox/pi_behav (0 if M == 0)                 */
} a3po_stats;

const char* a3po_status_string(int code);

/* Library/ABI version: major*1000 + minor. */
int a3po_version(void);

/* --------------------------------------------------------------------------------------------
 * Policy forward, last stage (Sec. 2.2 "forward pass through the model"; Sec. 3: the engines
 * exchange token log-probabilities; Sec. 4.1: sampling temperature 1.0 => inv_temperature 1).
 *
 *   z[t,v]  = inv_temperature * sum_k hidden[t,k] * W[v,k]
 *   lse[t]  = log sum_v exp(z[t,v])
 *   logp[t] = z[t, targets[t]] - lse[t]
 *
 * The [N,V] logits are never written to memory: the contraction is fused with an online,
 * vocabulary-chunked log-sum-exp and the target gather.
 *
 * hidden [N,H], w [V,H]: dtype `dt`, 16-byte aligned, H % 8 == 0 for A3PO_BF16.
 * targets int32 [N].  row_mask uint8 [N] or NULL: rows with 0 report logp = lse = 0.
 * logp, lse: fp32 [N] outputs (lse is needed by the backward).
 * entropy: fp32 [N] or NULL; when given, receives the policy entropy -sum_v p_v log p_v of
 *          each row (the diagnostic of Fig. 4), computed in the same vocabulary sweep.
 * ws/ws_bytes: at least a3po_token_logprobs_min_workspace_bytes(N,H,V,dt,0).  With the larger
 * a3po_token_logprobs_workspace_bytes(N,H,V,dt,0) (bf16 inputs, row_mask given) the rows with
 * row_mask != 0 are gathered first and only they are multiplied; with less than that every row is
 * computed and the masked ones are discarded afterwards (same results, more work).
 * ------------------------------------------------------------------------------------------ */
size_t a3po_token_logprobs_workspace_bytes(int64_t N, int H, int V, a3po_dtype dt, int is_bwd);

int a3po_token_logprobs_fwd(const void* hidden, const void* w, const int32_t* targets,
                            const uint8_t* row_mask, int64_t N, int H, int V, a3po_dtype dt,
                            float inv_temperature, float* logp, float* lse, float* entropy,
                            void* ws, size_t ws_bytes, uint32_t* status, void* stream);

/* --------------------------------------------------------------------------------------------
 * Backward of the above (the derivative of log-softmax + gather; no counterpart formula in the
 * paper, which leaves the backward to autograd):
 *
 *   dz[t,v]          = grad_logp[t] * (1[v == targets[t]] - exp(z[t,v] - lse[t])) * inv_temperature
 *   grad_hidden[t,:] = sum_v dz[t,v] * W[v,:]                      (dtype dt, [N,H], overwritten)
 *   grad_w[v,:]      = sum_t dz[t,v] * hidden[t,:]                 (fp32 [V,H])
 *
 * lse: the forward's output.  grad_logp fp32 [N]: rows with 0 contribute nothing.
 * accumulate_grad_w != 0 adds into grad_w (gradient accumulation over the mini-batches of a
 * training step, Sec. 4.1); 0 overwrites it.
 * dz is materialised only for a chunk of rows at a time inside `ws` (bf16 for A3PO_BF16);
 * the chunk length adapts to ws_bytes.  a3po_token_logprobs_workspace_bytes(...,1) returns
 * the size that lets the library use its preferred chunk AND gather the rows with a non-zero
 * grad_logp first (bf16 inputs), so that padding and clipped tokens cost nothing; with less
 * than that they are multiplied as zero rows (same results, more work).  The call fails with
 * A3PO_ERR_WORKSPACE below a3po_token_logprobs_min_workspace_bytes(...).
 * ------------------------------------------------------------------------------------------ */
size_t a3po_token_logprobs_min_workspace_bytes(int64_t N, int H, int V, a3po_dtype dt, int is_bwd);

int a3po_token_logprobs_bwd(const void* hidden, const void* w, const int32_t* targets,
                            const float* lse, const float* grad_logp, int64_t N, int H, int V,
                            a3po_dtype dt, float inv_temperature, void* grad_hidden,
                            float* grad_w, int accumulate_grad_w, void* ws, size_t ws_bytes,
                            uint32_t* status, void* stream);

/* --------------------------------------------------------------------------------------------
 * Forward / backward pair that shares the softmax instead of recomputing the logits (bf16 inputs
 * only; no counterpart in the paper).  For callers whose forward and backward are separate calls,
 * as under an autograd engine:
 *
 *   a3po_token_logprobs_fwd_keep  = a3po_token_logprobs_fwd (same logp, lse, entropy; rows with
 *       row_mask 0 are skipped) that also fills `kept`.  For each row that took part it keeps the
 *       probability ratios q[t,v] = exp(z[t,v] - z[t,y_t]) = p[t,v] / p[t,y_t] in bf16 (a float
 *       ratio keeps bf16's relative precision whether the row is flat or peaked) and their sum
 *       s[t] over v != y_t, from which lse = z_y + log1p(s), logp = -log1p(s) and
 *       1 - p_y = s / (1 + s) follow without cancellation.
 *   a3po_token_logprobs_bwd_kept  = a3po_token_logprobs_bwd (same grad_hidden, grad_w within the
 *       gradient tolerance) that runs only the two gradient contractions, directly on q:
 *       dz[t,v] = a_t q'[t,v] with a_t = -grad_logp[t] inv_T / (1 + s[t]) and q'[t,y_t] = -s[t], so
 *       grad_hidden = diag(a) (q' W) and grad_w = q'^T (diag(a) hidden): 4 N V H flops instead of
 *       6 N V H for the backward, and no pass over an [N,V] matrix besides the contractions.
 *
 * `kept`: device buffer of a3po_kept_bytes(N, V) bytes (about 2 N V), 256-byte aligned, written by
 * the forward, read by the backward, which also writes the target entries q'[t,y_t] into it (the
 * same values on every call, so the backward may be repeated).  hidden, w, targets must be the
 * forward's; `lse` is accepted for symmetry with a3po_token_logprobs_bwd and not read.  Rows the
 * forward skipped get a zero gradient whatever their grad_logp.  A row whose target probability
 * is below about 1e-37 cannot be kept (A3PO_STATUS_KEPT_RANGE is raised, its contribution is
 * dropped).  Both calls return A3PO_ERR_UNSUPPORTED for shapes the tensor-core path does not take
 * (H % 8 != 0): use the plain pair then.  ws: at least the matching *_workspace_bytes.
 * ------------------------------------------------------------------------------------------ */
size_t a3po_kept_bytes(int64_t N, int V);
size_t a3po_token_logprobs_fwd_keep_workspace_bytes(int64_t N, int H, int V);
size_t a3po_token_logprobs_bwd_kept_workspace_bytes(int64_t N, int H, int V);

int a3po_token_logprobs_fwd_keep(const void* hidden, const void* w, const int32_t* targets,
                                 const uint8_t* row_mask, int64_t N, int H, int V,
                                 float inv_temperature, float* logp, float* lse, float* entropy,
                                 void* kept, size_t kept_bytes, void* ws, size_t ws_bytes,
                                 uint32_t* status, void* stream);

int a3po_token_logprobs_bwd_kept(const void* hidden, const void* w, const int32_t* targets,
                                 const float* lse, const float* grad_logp, void* kept,
                                 size_t kept_bytes, int64_t N, int H, int V, float inv_temperature,
                                 void* grad_hidden, float* grad_w, int accumulate_grad_w, void* ws,
                                 size_t ws_bytes, uint32_t* status, void* stream);

/* --------------------------------------------------------------------------------------------
 * A-3PO loss (Eq. 2 with the proximal policy of Eq. 3 and the coefficient of Eq. 4; argument
 * names follow Listing 1: behav_logp = old_logp, logp = logprobs, versions, current_version).
 *
 *   d_t     = current_version - versions[t]            (integer staleness)
 *   alpha_t = 1/d_t if d_t >= 1 else 1                 (d <= 0 gives 1, as the listing's where)
 *   lprox_t = alpha_t * behav_logp[t] + (1 - alpha_t) * logp[t]
 *   iw_t    = exp(lprox_t - behav_logp[t])             importance weight  pi_prox / pi_behav
 *   r_t     = exp(logp[t] - lprox_t)                   trust-region ratio pi_theta / pi_prox
 *   obj_t   = iw_t * min(r_t * adv[t], clip(r_t, 1-eps, 1+eps) * adv[t])
 *   loss    = - sum_t mask[t] * obj_t / max(M, 1),  M = sum_t mask[t]    (masked token mean)
 *
 * The kernels evaluate iw and r through the theorem's closed form r = w^alpha
 * (w = pi_theta/pi_behav), which is the same function with better fp32 conditioning.
 *
 * logp, behav_logp, adv: fp32 [N].  mask: uint8 [N] (0 = ignore; ignored tokens may hold any
 * bit pattern, NaN included: they are selected out, not multiplied).
 * versions: int32 [N] (one per token) when versions_per_seq == 0; int32 [B] (one per sequence)
 *   when versions_per_seq != 0, in which case cu_seqlens int32 [B+1] gives each sequence's row
 *   range [cu_seqlens[b], cu_seqlens[b+1]) with cu_seqlens[0] = 0 and cu_seqlens[B] = N.
 * clip_eps >= 0.
 * loss: fp32 device scalar.  stats: device struct or NULL.
 * The reduction is a fixed two-stage tree: results are bit-identical from run to run.  Where the
 * device supports cooperative launches the whole call is one kernel launch.
 * ws/ws_bytes: at least a3po_loss_workspace_bytes(N).
 * ------------------------------------------------------------------------------------------ */
size_t a3po_loss_workspace_bytes(int64_t N);

int a3po_loss_fwd(const float* logp, const float* behav_logp, const int32_t* versions,
                  int versions_per_seq, const int32_t* cu_seqlens, int B, int32_t current_version,
                  const float* adv, const uint8_t* mask, int64_t N, float clip_eps, float* loss,
                  a3po_stats* stats, void* ws, size_t ws_bytes, void* stream);

/* --------------------------------------------------------------------------------------------
 * dL/dlogp of the loss above.
 *
 *   act_t = 1 if r_t*adv_t <= clip(r_t)*adv_t (the unclipped term is the minimum) else 0
 *   detach_prox != 0 (default reading: the anchor is a constant, like the recomputed anchor of
 *   Sec. 2.2 which is "frozen"):      grad_logp[t] = -(gl * mask_t / M) * iw_t * adv_t * r_t * act_t
 *   detach_prox == 0 (differentiate through Eq. 3 too):
 *       grad_logp[t] = -(gl * mask_t / M) * ((1 - alpha_t) * obj_t + alpha_t * iw_t * adv_t * r_t * act_t)
 *
 * grad_loss: fp32 device scalar gl, or NULL for 1.
 * fwd_stats: the a3po_stats the forward wrote for the same inputs (supplies M), or NULL, in
 *   which case the mask is counted first (one extra byte per token of traffic).
 * grad_logp: fp32 [N] output; masked tokens get exactly 0.
 * ------------------------------------------------------------------------------------------ */
int a3po_loss_bwd(const float* logp, const float* behav_logp, const int32_t* versions,
                  int versions_per_seq, const int32_t* cu_seqlens, int B, int32_t current_version,
                  const float* adv, const uint8_t* mask, int64_t N, float clip_eps,
                  int detach_prox, const float* grad_loss, const a3po_stats* fwd_stats,
                  float* grad_logp, void* ws, size_t ws_bytes, void* stream);

/* Forward and backward in one pass over the inputs (mask counted first, then one stream that
 * reads 17 B/token and writes 4 B/token).  Outputs as in the two calls above; grad_loss = 1. */
int a3po_loss_fwd_bwd(const float* logp, const float* behav_logp, const int32_t* versions,
                      int versions_per_seq, const int32_t* cu_seqlens, int B,
                      int32_t current_version, const float* adv, const uint8_t* mask, int64_t N,
                      float clip_eps, int detach_prox, float* loss, a3po_stats* stats,
                      float* grad_logp, void* ws, size_t ws_bytes, void* stream);

/* --------------------------------------------------------------------------------------------
 * The decoupled clipped loss of Eq. 2 with an EXPLICIT proximal policy: the baseline the paper
 * calls "recompute" (Sec. 2.2: log pi_prox comes from an extra forward pass and is frozen), and,
 * with prox_logp = behav_logp, the coupled PPO-clip loss of Eq. 1 ("sync").  Same streaming
 * kernel as a3po_loss_fwd_bwd with the interpolation replaced by a load:
 *
 *   iw_t  = exp(prox_logp[t] - behav_logp[t]),   r_t = exp(logp[t] - prox_logp[t])
 *   obj_t = iw_t * min(r_t * adv[t], clip(r_t, 1-eps, 1+eps) * adv[t])
 *   loss  = - sum_t mask[t] * obj_t / max(M, 1)
 *   grad_logp[t] = -(mask_t / M) * iw_t * adv_t * r_t * act_t        (the anchor is a constant)
 *
 * prox_logp: fp32 [N].  grad_logp may be NULL (forward only).  Other arguments, outputs,
 * workspace and error codes as a3po_loss_fwd_bwd.
 * ------------------------------------------------------------------------------------------ */
int a3po_decoupled_loss_fwd_bwd(const float* logp, const float* behav_logp, const float* prox_logp,
                                const float* adv, const uint8_t* mask, int64_t N, float clip_eps,
                                float* loss, a3po_stats* stats, float* grad_logp, void* ws,
                                size_t ws_bytes, void* stream);

/* --------------------------------------------------------------------------------------------
 * Helpers for data-parallel training over sequences (no counterpart in the paper, which states E_t
 * of Eq. 2 for one batch).  The path is per token except the masked mean, so a job that shards its
 * sequences over ranks gets the whole-job loss and gradients from per-rank calls as
 *     L = sum_r (M_r / M) L_r,     grad = sum_r (M_r / M) grad_r,      M = sum_r M_r,
 * where L_r, grad_r are what rank r computes with its local mean.  a3po_mask_count gives M_r before
 * the step (the mask is an input), the caller all-reduces it, a3po_dp_loss_scale turns the two
 * counts into the weight M_r / M, and a3po_train_step takes that weight as `loss_scale`, so its
 * gradients come out already weighted and one sum all-reduce of grad_w (and of the weighted loss)
 * finishes the job; grad_hidden and grad_logp stay local.
 *
 * a3po_mask_count: *count (int64, device) = number of non-zero mask bytes; ws of
 *   a3po_mask_count_workspace_bytes() bytes.
 * a3po_dp_loss_scale: *scale = M_local / M_global (0 if M_global == 0), all device scalars; when
 *   loss_local is given, *weighted_loss = *scale * *loss_local as well.
 * ------------------------------------------------------------------------------------------ */
size_t a3po_mask_count_workspace_bytes(void);
int a3po_mask_count(const uint8_t* mask, int64_t N, int64_t* count, void* ws, size_t ws_bytes, void* stream);
int a3po_dp_loss_scale(const int64_t* m_local, const int64_t* m_global, const float* loss_local,
                       float* scale, float* weighted_loss, void* stream);

/* --------------------------------------------------------------------------------------------
 * GRPO advantages (Sec. 4.1: "estimate advantages using group reward normalization"; the paper
 * gives no formula, the customary one is used).  Sequences come in consecutive groups of
 * `group_size` responses to the same prompt:
 *
 *   A_i = (R_i - mean_group) / (std_group + norm_eps)        population standard deviation
 *   adv[t] = A_i for every row t of sequence i, i.e. cu_seqlens[i] <= t < cu_seqlens[i+1]
 *
 * rewards fp32 [B], cu_seqlens int32 [B+1] (cu_seqlens[0] = 0, cu_seqlens[B] = N), B a multiple
 * of group_size, adv fp32 [N] output.  ws: at least a3po_grpo_workspace_bytes(B).
 * ------------------------------------------------------------------------------------------ */
size_t a3po_grpo_workspace_bytes(int B);

int a3po_grpo_advantages(const float* rewards, int B, int group_size, const int32_t* cu_seqlens,
                         int64_t N, float norm_eps, float* adv, void* ws, size_t ws_bytes,
                         void* stream);

/* --------------------------------------------------------------------------------------------
 * Self-test of the bounded waits the pipelined kernels rely on (no counterpart in the paper).
 * Launches a one-warp kernel that waits on a barrier nothing ever signals; after timeout_ms
 * (1..2000) the wait gives up and ORs A3PO_STATUS_WAIT_TIMEOUT into *status (device word),
 * which is what a stuck pipeline stage does instead of hanging the GPU.
 * ------------------------------------------------------------------------------------------ */
int a3po_selftest_wait_timeout(uint32_t* status, unsigned timeout_ms, void* stream);

/* --------------------------------------------------------------------------------------------
 * a3po_loss_fwd for callers that have no way to hand over a workspace (the paper has no
 * counterpart: this is a packaging variant, the arithmetic is a3po_loss_fwd's).
 *
 * Who needs it: code that runs where device memory cannot be obtained at call time — a hook
 * inside a host framework whose memory pool is the only permitted allocator and is not exposed
 * to the hook, a latency-critical loop in which an allocation (an implicit device-wide
 * synchronisation) is forbidden, or a process whose device memory has been carved up in advance
 * and where cudaMalloc simply fails.  Such a caller still owns its inputs and outputs; what it
 * lacks is the few megabytes of scratch the loss kernels reduce through.
 *
 * Here that scratch is a fixed array inside the library's device image (about 4.2 MiB, sized
 * for A3PO_LOSS_FWD_STATIC_MAX_TOKENS tokens).  Every GPU on which the library is loaded holds
 * it from load until the process exits, whether or not this function is ever called.  The
 * function calls no cudaMalloc / cudaFree and no allocating library routine (with the optional
 * per-kernel profile left off, which is the default, it creates no CUDA objects at all).
 *
 * Arguments, outputs and error codes are those of a3po_loss_fwd without ws / ws_bytes, plus:
 *   - N > A3PO_LOSS_FWD_STATIC_MAX_TOKENS returns A3PO_ERR_TOO_LARGE before anything is
 *     launched or written; use a3po_loss_fwd with a caller workspace for larger batches.
 *   - The first call on each device looks up the array's device address (once per device, with
 *     that device current).  That first call should be made before any stream capture begins.
 *   - All calls on one device share the one array.  Nothing in it has to be zero on entry: a call
 *     reads only words it has written itself, so the previous call's leftovers are harmless.
 *     But two calls whose kernels overlap on the GPU (different streams, or different host
 *     threads without ordering) race on it and corrupt each other's result: serialise them.
 * ------------------------------------------------------------------------------------------ */
#define A3PO_LOSS_FWD_STATIC_MAX_TOKENS (1 << 20)

int a3po_loss_fwd_static(const float* logp, const float* behav_logp, const int32_t* versions,
                         int versions_per_seq, const int32_t* cu_seqlens, int B,
                         int32_t current_version, const float* adv, const uint8_t* mask, int64_t N,
                         float clip_eps, float* loss, a3po_stats* stats, void* stream);

/* --------------------------------------------------------------------------------------------
 * One whole training-step pass with every buffer on the device (no counterpart in the paper):
 *   logp, lse [, entropy]  = token_logprobs_fwd(hidden, w, targets, row_mask = mask)
 *   loss, stats, grad_logp = loss_fwd_bwd(logp, behav_logp, versions (per token), ...)   detach_prox = 1
 *   grad_hidden, grad_w    = token_logprobs_bwd(..., lse, grad_logp)
 * with the same results as the three calls.  For bf16 inputs and a workspace of at least
 * a3po_train_step_workspace_bytes(...) the step does not recompute the LM head in the backward
 * (6 N V H flops instead of 8 N V H): the rows with mask != 0 are gathered once (their number M
 * is then known on the device), and per chunk of those rows the forward keeps the softmax as
 * bf16 probability ratios (see a3po_token_logprobs_fwd_keep), the loss forward + backward runs
 * on the chunk's log-probs, and the two gradient contractions run on the kept ratios.  The
 * workspace holds one chunk of ratios at a time (chunk x V x 2 bytes; the recommended size is
 * for chunks of 65,536 rows, about 20 GB at V = 151,936, and a larger workspace gives larger
 * chunks) plus a gathered copy of hidden.  With a smaller workspace (at least
 * a3po_train_step_min_workspace_bytes) or fp32 inputs the three calls are made as they are.
 * logp, lse, grad_logp: fp32 [N] outputs.  entropy: fp32 [N] or NULL (policy entropy per row,
 * Fig. 4).  loss_scale: fp32 device scalar or NULL (= 1): every gradient (grad_logp, grad_hidden,
 * grad_w) is multiplied by it, the reported loss is not; data-parallel callers pass M_local /
 * M_global (see a3po_dp_loss_scale).  Other arguments as in the individual calls.
 * ------------------------------------------------------------------------------------------ */
size_t a3po_train_step_min_workspace_bytes(int64_t N, int H, int V, a3po_dtype dt);
size_t a3po_train_step_workspace_bytes(int64_t N, int H, int V, a3po_dtype dt);

int a3po_train_step(const void* hidden, const int32_t* targets, const float* behav_logp,
                    const int32_t* versions, const float* adv, const uint8_t* mask, int64_t N, int H,
                    int V, a3po_dtype dt, int32_t current_version, float clip_eps,
                    float inv_temperature, const void* w, float* grad_w, int accumulate_grad_w,
                    void* grad_hidden, float* logp, float* lse, float* entropy, float* grad_logp,
                    float* loss, a3po_stats* stats, const float* loss_scale, void* ws, size_t ws_bytes,
                    uint32_t* status, void* stream);

/* --------------------------------------------------------------------------------------------
 * The same pass with per-step inputs in HOST memory (no counterpart in the paper; this is the
 * end-to-end form of the call above):
 *   copies hidden, targets, behav_logp, versions, adv, mask host->device, runs a3po_train_step,
 *   copies loss + stats back.
 * Of `hidden`, only the runs of rows with mask != 0 are copied when the step keeps its softmax
 * (it reads no other row; the rest of the staged copy is then undefined); every row is copied
 * when the workspace or the shape sends the step down the recomputing calls.
 * h_* are host pointers (pinned memory recommended; pageable works but serialises); h_mask is
 * read by the host during the call.
 * d_w, d_grad_w (accumulated into when accumulate_grad_w != 0), d_grad_hidden ([N,H] dt) and
 * d_stage/d_ws are device buffers.  d_stage needs a3po_train_step_stage_bytes(N,H,dt) bytes and
 * d_ws a3po_train_step_workspace_bytes(N,H,V,dt).  h_loss (float) and h_stats are host outputs,
 * valid after the caller synchronises `stream`.
 * ------------------------------------------------------------------------------------------ */
size_t a3po_train_step_stage_bytes(int64_t N, int H, a3po_dtype dt);

int a3po_train_step_host(const void* h_hidden, const int32_t* h_targets, const float* h_behav_logp,
                         const int32_t* h_versions, const float* h_adv, const uint8_t* h_mask,
                         int64_t N, int H, int V, a3po_dtype dt, int32_t current_version,
                         float clip_eps, float inv_temperature, const void* d_w, float* d_grad_w,
                         int accumulate_grad_w, void* d_grad_hidden, void* d_stage,
                         size_t stage_bytes, void* d_ws, size_t ws_bytes, float* h_loss,
                         a3po_stats* h_stats, uint32_t* d_status, void* stream);

/* --------------------------------------------------------------------------------------------
 * Row operators in front of the LM head (the layers that produce `hidden`; no counterpart in the paper).  A trainer
 * that owns the last block of the policy runs them on the rows it then hands to a3po_token_logprobs_fwd or
 * a3po_train_step, and runs their backward on the grad_hidden it gets back.
 *
 * Common to all of them: matrices are row-major [N, H], contiguous, dtype `dt` (1 <= H <= 2^30; pointers aligned to their
 * elements, 16-byte aligned rows move in 16-byte pieces); arithmetic, statistics and weight gradients are fp32 and
 * each stored element is rounded once.  row_mask uint8 [N] or NULL: of rows with 0 nothing enters a result (they may
 * hold NaN), their outputs (gradients included) are 0 and they add nothing to a weight gradient.  N <= 2^31 - 1.  Outputs
 * must not overlap inputs.  N = 0 launches nothing, apart from the zeros of a weight gradient that is not accumulated.
 *
 * Norm:       xhat = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps),  y = xhat gamma + beta
 *   A3PO_NORM_LAYER: mean = sum(x) / H;  A3PO_NORM_RMS: mean = 0 (the argument mean must be NULL).  Either takes a beta.
 *   gamma [H], beta [H] or NULL: dtype dt.  mean, rstd: fp32 [N] outputs of the forward, or NULL if no backward
 *   follows; inputs of the backward.
 * Its backward:  gx = grad_y gamma;  grad_x = rstd (gx - [mean(gx)] - xhat mean(gx xhat))   ([.]: layer norm only)
 *   grad_gamma = sum_t grad_y xhat, grad_beta = sum_t grad_y: fp32 [H], added to what is there when
 *   accumulate_grad_w != 0, else overwritten; grad_beta may be NULL.  Sums are taken in a fixed order: results are
 *   bit-identical from run to run on the same GPU model.  ws: a3po_norm_bwd_workspace_bytes(N, H), 256-byte aligned.
 *
 * Dropout:    d(x)[t, c] = x[t, c] 65536 / (65536 - T) if u16(t, c) >= T else 0,   T = round(65536 p), 0 <= p <= 1
 *   (p is taken to the nearest multiple of 2^-16 and the scale is exact for that).  y = residual + d(x); residual
 *   [N, H] or NULL.  The mask is never stored: u16(t, c) is the (c mod 8)-th of the eight 16-bit halves (low half
 *   first) of Philox4x32-10 with key = seed and counter = (c / 8, t, low word of offset, high word of offset).
 *   rng: device pointer to {seed, offset} (two uint64, 8-byte aligned; NULL only if p = 0), read when the kernel
 *   runs, so a captured graph draws a new mask whenever the words have changed.  The backward (and any
 *   recomputation) passes the same p and words; calls that need different masks differ in offset or seed.
 *   Backward:  grad_x = d(grad_y).
 *
 * Join:       r = residual + d(x)  (stored),   y = norm(r)       dropout, add and norm in one pass
 *   Backward: grad_residual = norm's grad_x of (r, grad_y) + grad_r,   grad_x = d(grad_residual before rounding);
 *   grad_r [N, H] or NULL: the gradient that reaches r past the norm.  grad_x may be NULL (with p = 0: the backward of
 *   a norm on a residual stream that nothing joined there).
 * ------------------------------------------------------------------------------------------ */
typedef enum { A3PO_NORM_RMS = 0, A3PO_NORM_LAYER = 1 } a3po_norm_kind;

int a3po_norm_fwd(const void* x, const void* gamma, const void* beta, const uint8_t* row_mask, int64_t N, int H,
                  a3po_dtype dt, a3po_norm_kind kind, float eps, void* y, float* mean, float* rstd, void* stream);

size_t a3po_norm_bwd_workspace_bytes(int64_t N, int H);

int a3po_norm_bwd(const void* x, const void* gamma, const float* mean, const float* rstd, const uint8_t* row_mask,
                  const void* grad_y, int64_t N, int H, a3po_dtype dt, a3po_norm_kind kind, void* grad_x,
                  float* grad_gamma, float* grad_beta, int accumulate_grad_w, void* ws, size_t ws_bytes,
                  void* stream);

int a3po_dropout_fwd(const void* x, const void* residual, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt,
                     float p, const uint64_t* rng, void* y, void* stream);

int a3po_dropout_bwd(const void* grad_y, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt, float p,
                     const uint64_t* rng, void* grad_x, void* stream);

int a3po_dropout_norm_fwd(const void* x, const void* residual, float p, const uint64_t* rng, const void* gamma,
                          const void* beta, const uint8_t* row_mask, int64_t N, int H, a3po_dtype dt,
                          a3po_norm_kind kind, float eps, void* r, void* y, float* mean, float* rstd, void* stream);

int a3po_dropout_norm_bwd(const void* r, float p, const uint64_t* rng, const void* gamma, const float* mean,
                          const float* rstd, const uint8_t* row_mask, const void* grad_y, const void* grad_r,
                          int64_t N, int H, a3po_dtype dt, a3po_norm_kind kind, void* grad_residual, void* grad_x,
                          float* grad_gamma, float* grad_beta, int accumulate_grad_w, void* ws, size_t ws_bytes,
                          void* stream);

/* --------------------------------------------------------------------------------------------
 * Gated feed-forward block (no counterpart in the paper: the layer of the policy below the final norm).
 *
 *   g = x Wg^T,  u = x Wu^T,  h = act(g) u,  y = h Wd^T           act: SiLU g / (1 + exp(-g)), or the tanh form of GELU
 *   dh = grad_y Wd,  dg = dh u act'(g),  du = dh act(g)
 *   grad_x = dg Wg + du Wu,  grad_Wg = dg^T x,  grad_Wu = du^T x,  grad_Wd = grad_y^T h
 *
 * x, y, grad_x, grad_y [N, H]; w_gate_up [2 F, H] (the F rows of Wg, then the F rows of Wu); w_down [H, F]; dtype `dt`.
 * Any H and F: bf16 with H and F multiples of 8 runs on the tensor cores and wants every matrix 16-byte aligned, the rest
 * runs on the FP32 pipes and takes pointers aligned to their elements.
 * Both projections, the activation and the product are one kernel; dh never reaches memory either.  Accumulation is
 * fp32; for bf16 the intermediates that enter a matrix product (h, dg, du) are rounded to bf16.
 *
 * row_mask uint8 [N] or NULL: rows with 0 are skipped (of more than a few rows only the others are multiplied): nothing
 * of them enters a result (they may hold NaN); with finite weights their y and grad_x are 0 and they add nothing to a
 * weight gradient.
 * kept: device buffer of a3po_gated_ffn_kept_bytes(N, F, dt) bytes, 256-byte aligned, that receives g, u and h for the
 * backward (layout private; about 8 N F bytes for bf16), or NULL when no backward follows.  The backward takes it with
 * the forward's x, weights, row_mask, N, H, F, dt and act; it is not changed, so the backward may be repeated.
 * grad_w_gate_up [2 F, H], grad_w_down [H, F]: dtype grad_w_dt (A3PO_F32, or dt), overwritten; with
 * accumulate_grad_w != 0 added to (A3PO_F32 only, else A3PO_ERR_UNSUPPORTED).
 * ws: a3po_gated_ffn_workspace_bytes(N, H, F, dt, row_mask given, backward) bytes, 256-byte aligned.  On the tensor cores
 * 2 N F bytes forward and 4 N F backward (N to the next multiple of 128), with a row_mask two (backward three) times 2 N H
 * more, and up to 20 MB of partial sums while the output tiles are few; on the FP32 pipes 4 N F forward and 12 N F backward.
 * status: optional device word (A3PO_STATUS_WAIT_TIMEOUT).  Outputs must not overlap inputs.  N = 0 launches nothing
 * except the zeros of weight gradients that are not accumulated.  Results are bit-identical from run to run.
 * ------------------------------------------------------------------------------------------ */
/* A3PO_ACT_NONE is for the linear operator; the gated block refuses it. */
typedef enum { A3PO_ACT_SILU = 0, A3PO_ACT_GELU_TANH = 1, A3PO_ACT_NONE = 2 } a3po_activation;

size_t a3po_gated_ffn_kept_bytes(int64_t N, int F, a3po_dtype dt);
size_t a3po_gated_ffn_workspace_bytes(int64_t N, int H, int F, a3po_dtype dt, int has_row_mask, int is_bwd);

int a3po_gated_ffn_fwd(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask, int64_t N,
                       int H, int F, a3po_dtype dt, a3po_activation act, void* y, void* kept, size_t kept_bytes,
                       void* ws, size_t ws_bytes, uint32_t* status, void* stream);

int a3po_gated_ffn_bwd(const void* x, const void* w_gate_up, const void* w_down, const uint8_t* row_mask,
                       const void* kept, size_t kept_bytes, const void* grad_y, int64_t N, int H, int F, a3po_dtype dt,
                       a3po_activation act, void* grad_x, void* grad_w_gate_up, void* grad_w_down,
                       a3po_dtype grad_w_dt, int accumulate_grad_w, void* ws, size_t ws_bytes, uint32_t* status,
                       void* stream);

/* --------------------------------------------------------------------------------------------
 * Linear operator (no counterpart in the paper): projections onto the residual stream, biased layers, the logits of the next token.
 *
 *   z = x W^T + bias,   y = act(z) + residual                       act: none, SiLU or the tanh form of GELU
 *   dz = grad_y act'(z),  grad_x = dz W,  grad_w = dz^T x,  grad_bias = sum of the rows of dz,  grad_residual = grad_y
 *
 * x, grad_x [N, K]; w, grad_w [M, K]; bias [M] or NULL; residual [N, M] or NULL; y, grad_y [N, M]; dtype `dt`, y also A3PO_F32 (y_dt).
 * Any K and M up to 2,097,120: bf16 with K and M multiples of 8 runs on the tensor cores and wants every matrix 16-byte
 * aligned, the rest runs on the FP32 pipes and takes pointers aligned to their elements.  One kernel does the product, bias,
 * activation and residual (two where few output tiles are split along K).  Accumulation is fp32 and y is rounded once; for bf16
 * with an activation dz is rounded to bf16 as an operand of the products, not for grad_bias.
 *
 * row_mask uint8 [N] or NULL: rows with 0 are skipped (of more than a few rows only the others are multiplied): nothing of
 * them enters a result (they may hold NaN); with finite weights their y (residual included) and grad_x are 0 and they add
 * nothing to grad_w and grad_bias.  Their grad_residual is 0 too: callers that use grad_y for it mask it.
 * kept: device buffer of a3po_linear_kept_bytes(N, M, dt, act) bytes, 256-byte aligned, that receives z for the backward
 * (layout private, 4 N M bytes), or NULL when no backward follows or there is no activation (0 bytes).  The backward takes it
 * with the forward's row_mask, N, K, M, dt and act, and does not change it.
 * grad_x, grad_w, grad_bias: each may be NULL (not wanted), not all.  grad_w: dtype grad_w_dt (A3PO_F32, or dt); grad_bias: fp32.
 * Both are overwritten, or with accumulate != 0 added to (A3PO_F32 only, else A3PO_ERR_UNSUPPORTED).
 * ws: a3po_linear_workspace_bytes(N, K, M, dt, act, row_mask given, backward) bytes, 256-byte aligned.
 * status: optional device word (A3PO_STATUS_WAIT_TIMEOUT).  Outputs must not overlap inputs.  N = 0 launches nothing except the
 * zeros of gradients that are not accumulated.  Results are bit-identical from run to run.
 * ------------------------------------------------------------------------------------------ */
size_t a3po_linear_kept_bytes(int64_t N, int M, a3po_dtype dt, a3po_activation act);
size_t a3po_linear_workspace_bytes(int64_t N, int K, int M, a3po_dtype dt, a3po_activation act, int has_row_mask, int is_bwd);

int a3po_linear_fwd(const void* x, const void* w, const void* bias, const void* residual, const uint8_t* row_mask, int64_t N,
                    int K, int M, a3po_dtype dt, a3po_activation act, void* y, a3po_dtype y_dt, void* kept,
                    size_t kept_bytes, void* ws, size_t ws_bytes, uint32_t* status, void* stream);

int a3po_linear_bwd(const void* x, const void* w, const uint8_t* row_mask, const void* kept, size_t kept_bytes,
                    const void* grad_y, int64_t N, int K, int M, a3po_dtype dt, a3po_activation act, void* grad_x,
                    void* grad_w, a3po_dtype grad_w_dt, float* grad_bias, int accumulate, void* ws, size_t ws_bytes,
                    uint32_t* status, void* stream);

/* --------------------------------------------------------------------------------------------
 * Sampling of one token per row of logits (no counterpart in the paper: the rollout's side of the policy).  What it leaves in
 * `logp` is the behaviour log-prob that the loss takes as behav_logp, by the definition of a3po_token_logprobs_fwd with
 * inv_temperature = 1 / t (1 for a greedy row): a policy that is sampled at t is trained at t, or its importance weights are biased.
 *
 * A row with logits l (NaN counts as -inf) and temperature t, t <= 0 or NaN meaning greedy (with t = 1 below), above 1e30 as 1e30:
 *   w_i = exp((l_i - max l) / t);  tokens are ranked by l, of equal logits the lower index first
 *   top_k  keeps the k first ranks (k <= 0 or k >= V: all);
 *   top_p  keeps of those the fewest first ranks whose weights reach top_p times the sum of theirs (top_p >= 1: all);
 *   min_p  keeps of those the ones with w_i >= min_p (min_p <= 0: all);   the first rank is always kept, greedy keeps it alone
 *   token     = the first kept i, in index order, at which the running sum of the kept weights exceeds u times their sum
 *   logp      = log(w_token / sum of all w),   kept_logp = log(w_token / sum of the kept w)
 *   n_kept    = number of kept tokens with a logit above -inf
 * Weights carry 2^-31 of their value and sums 53 bits (the mass that top_p compares: multiples of 2^-43 of the largest weight),
 * added in a fixed order: results are bit-identical from run to run, and a token differs from the one that exact sums give
 * only where u lies within that of a border.  Weights of bf16 logits are off by up to 2^-24 |l_i - max l| / t more where one of the
 * two is that much smaller than the other (2^-15) that their difference is not an fp32 number.
 *
 * logits [N, V], dtype `dt`, rows row_stride >= V elements apart, pointer aligned to its elements.  temperature, top_k, top_p,
 * min_p: [N] or NULL (1, off, off, off); u fp32 [N] in [0, 1) (below 0 or NaN: 0; from 1 on: the last kept token whose
 * weight is not 0 in 64 bits).
 * token int32 [N]; logp, kept_logp fp32 [N] and n_kept int32 [N] or NULL.  A row with row_mask 0 (uint8 [N] or NULL) is not read;
 * it, and a row without a logit above -inf, gets token -1, logp 0, kept_logp 0, n_kept 0.
 * With any of top_k, top_p, min_p a row has to fit the shared memory of eight SMs: V <= 393,216 (fp32) or 786,432 (bf16), else
 * A3PO_ERR_UNSUPPORTED.  ws: a3po_sample_workspace_bytes(N, V), 256-byte aligned.  Outputs must not overlap inputs.
 * ------------------------------------------------------------------------------------------ */
size_t a3po_sample_workspace_bytes(int64_t N, int V);

int a3po_sample(const void* logits, int64_t row_stride, const uint8_t* row_mask, int64_t N, int V, a3po_dtype dt,
                const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, const float* u,
                int32_t* token, float* logp, float* kept_logp, int32_t* n_kept, void* ws, size_t ws_bytes,
                void* stream);

/* --------------------------------------------------------------------------------------------
 * AdamW over many tensors at once (no counterpart in the paper: what consumes the gradients of the step).
 *
 *   s  = min(1, max_grad_norm / (norm + 1e-6)),  norm over all gradients of the call;  s = 1 if max_grad_norm = 0
 *   t  = *step + 1,  g = s grad
 *   m' = beta1 m + (1 - beta1) g,   v' = beta2 v + (1 - beta2) g^2
 *   w' = w - lr (weight_decay w + (m' / (1 - beta1^t)) / (sqrt(v' / (1 - beta2^t)) + eps))
 *
 * One a3po_adamw_tensor per tensor, n elements each (contiguous; 0 is valid):
 *   weight   dtype weight_dt.  master: fp32 copy that is updated and then rounded into `weight` (weight_dt = A3PO_BF16 only), or
 *            NULL: the weight itself is read, updated in fp32 and rounded once
 *   grad     dtype grad_dt, not changed
 *   m, v     state_bits = 32: fp32.  state_bits = 8: one byte per element in blocks of 256, with fp32 scales of
 *            ceil(n / 256) blocks in m_scale and v_scale (all bytes and scales 0: states of 0).  A byte stands for
 *            q(c) scale with q(c) = c below 8, else (8 + c mod 8) 2^(c div 8 - 1); in m bit 7 is the sign and c the rest.
 *            New states become codes of scale = (largest of the block) / q(largest code).  Steps 1 to 32 take the nearest q, halves
 *            the even code.  Later steps take the q below or the one above it at random, with the probabilities that make
 *            the code right on average: the share of a step in an average is then down to 1 - beta, and a nearest code does not
 *            follow an average that moves by less than half a step between codes (1/32 to 1/16 of a value).  The random number
 *            of element e of a block is word e mod 4 of Philox4x32-10 with key 0 and counter (32 times the tensor's place in the call
 *            + e mod 128 div 4, block, t, upper bits of t xor 2^24 times the block's): its upper 16 bits are the first moment's for
 *            e < 128 and the second's for the others, its lower ones the other's; they and half of the last bit are added as a
 *            share of the step between the codes, and the rest is cut off.  A second moment above 0 is not stored as 0.
 *            The update itself uses the states before rounding.
 *   weight_decay   of this tensor
 * Pointers are aligned to their elements; tensors whose pointers allow it (four elements) move in wide pieces.  Tensors must not
 * overlap one another.  The table is read by the host during the call and travels in the kernels' arguments.
 * lr: fp32 device scalar.  step: int64 device scalar, steps taken so far, advanced by the call.  grad_norm: fp32 device
 * scalar or NULL (the norm before clipping).  When the norm is asked for (grad_norm given or max_grad_norm > 0) and is not
 * finite, nothing but grad_norm is written and *step stays.  beta1, beta2 in [0, 1), eps > 0.
 * ws: a3po_adamw_workspace_bytes(count), 256-byte aligned.  The norm is a sum in 64 bits in a fixed order; results are
 * bit-identical from run to run.
 *
 * a3po_adamw_state_values: what the bytes of an 8-bit state (is_signed: m) stand for, fp32 [n].
 * ------------------------------------------------------------------------------------------ */
typedef struct {
  void* weight;
  float* master;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  int64_t n;
  float weight_decay;
} a3po_adamw_tensor;

size_t a3po_adamw_workspace_bytes(int count);

int a3po_adamw_step(const a3po_adamw_tensor* tensors, int count, a3po_dtype weight_dt, a3po_dtype grad_dt, int state_bits,
                    double beta1, double beta2, float eps, float max_grad_norm, const float* lr, int64_t* step,
                    float* grad_norm, void* ws, size_t ws_bytes, void* stream);

int a3po_adamw_state_values(const uint8_t* codes, const float* scales, int64_t n, int is_signed, float* values, void* stream);

/* Bytes the host entries of this library have copied host->device in the calling process since
 * load (monotonic; for transfer accounting in benchmarks). */
int64_t a3po_host_to_device_bytes(void);

/* Number of kernels this library has launched in the calling process since load
 * (monotonic; for launch accounting in benchmarks). */
int64_t a3po_kernel_launch_count(void);

/* --------------------------------------------------------------------------------------------
 * Optional per-kernel timing (no counterpart in the paper).  While enabled, every kernel the
 * library launches is bracketed by a pair of CUDA events recorded on the launch stream.
 * a3po_profile_read waits for the recorded events, returns up to max_entries (kernel id,
 * milliseconds) pairs in launch order, and clears the record list; a3po_kernel_name maps an id
 * to a static string.  Host-side state is process-global and mutex-protected.  Leave it off
 * for production use: each launch costs two extra event records.
 * ------------------------------------------------------------------------------------------ */
int a3po_profile_enable(int on);
int a3po_profile_read(int max_entries, int* kernel_ids, float* milliseconds, int* count);
const char* a3po_kernel_name(int kernel_id);

#ifdef __cplusplus
}
#endif
#endif /* A3PO_H_ */

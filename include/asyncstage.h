/*
 * asyncstage.h - C ABI of one pipeline stage's training step under a one-step gradient delay,
 * for AMD Instinct MI355X (gfx950).
 *
 * The method (One-Step Gradient Delay is Not a Barrier for Large-Scale Asynchronous Pipeline
 * Parallel LLM Pretraining):
 *   - §2, Alg. 1 (Delayed Gradient Update): iteration t computes g_t at x_t, feeds g_{t-1} to the
 *     optimizer statistics and sets x_{t+1} = x_t - u_{t-1}(g_{t-1}); g_{-1} = 0, u_{-1} = 0.
 *   - §3.2, Error-Feedback equation: x_{t+1} = x_t - 2 u_{t-1}(g_{t-1}) + u_{t-2}(g_{t-2}) for
 *     t >= 2, and App. A.4 its lambda-scaled form x_{t+1} = x_t - u_{t-1} - lambda (u_{t-1} - u_{t-2}).
 *   - §2 and App. E.1: u is decoupled AdamW, betas (0.9, 0.95), weight decay 0.1, global-norm
 *     gradient clipping at 1.0; Alg. 2 (§4) puts the weight decay on the current weights x_t.
 *   - §2 / App. F.1: PipeDream-2BW keeps one stashed weight version, so a stage holds two compute
 *     copies of its weights (versions t mod 2) and two gradient buffers (g_t being accumulated,
 *     g_{t-1} being consumed).
 *   - App. C (delayed method with prev(k) = k - tau): a fixed delay tau >= 2 consumes g_{t-tau},
 *     with Error Feedback against the update formed tau iterations earlier, x_{t+1} = x_t - u -
 *     lambda (u - u_{t-tau}) (lambda = tau: the coefficients tau + 1 and tau of its proof); the
 *     stage then holds tau + 1 gradient buffers and tau EF buffers.
 *   - App. E.2: the stage is a stack of Llama-style decoder blocks (pre-norm RMSNorm, grouped-query
 *     causal attention with RoPE, SwiGLU feed-forward, no biases); a first stage owns the token
 *     embedding, a last stage the LM head with next-token cross-entropy (App. E) - tied to the
 *     embedding when one stage holds both ends, else its own matrix.
 *
 * Conventions
 *   - Every function returns a stage_status; no C++ exception crosses the ABI.  On error,
 *     stage_last_error() returns a message (thread-local, valid until the next call).
 *   - The library never allocates device memory.  The caller allocates one arena of
 *     stage_required_bytes() and every input/output buffer; all pointers stay owned by the caller.
 *   - All device work is enqueued asynchronously on the HIP stream given to stage_init (or to
 *     delayed_update_flat), with one exception: delayed_update runs its kernels on a stream of
 *     the stage's own (non-blocking, default priority).  It waits there only for the backwards
 *     whose gradient it consumes and for the last use of the weight version it overwrites, so
 *     it overlaps forward / backward work the caller enqueued before it; the stage stream then
 *     waits for it, so everything enqueued after delayed_update returns sees its results.
 *     Host pointers are never retained.  The caller synchronises.
 *   - The caller may write master weights and optimizer state (stage_tensor views) only when no
 *     update is in flight, and then calls stage_sync_weights() before the next delayed_update.
 *   - Device pointers must be 16-byte aligned.  Layouts are row-major, last index contiguous.
 *   - Token ids are int32; an id outside [0, vocab) is never used as an index (see
 *     stage_forward).
 *   - One stage_t per host thread; calls on one stage_t must not overlap.
 */
#ifndef ASYNCSTAGE_H
#define ASYNCSTAGE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct stage stage_t; /* opaque */

typedef enum {
  STAGE_OK = 0,
  STAGE_EINVAL = -1,     /* bad argument or shape                                  */
  STAGE_ENOSPACE = -2,   /* arena smaller than stage_required_bytes()              */
  STAGE_EHIP = -3,       /* a HIP runtime call failed                              */
  STAGE_ESTATE = -4,     /* call out of the documented order                       */
  STAGE_ENONFINITE = -5  /* reported by stage_poll_nonfinite                       */
} stage_status;

typedef enum { STAGE_DT_F32 = 0, STAGE_DT_BF16 = 1, STAGE_DT_I32 = 2 } stage_dtype;

/* Largest delay a stage can be shaped for (stage_shape_t.max_delay). */
enum { STAGE_MAX_DELAY = 8 };

/* Shape of one stage.  dtype 0: fp32 compute and storage; 1: bf16 compute copies, bf16
 * activations, fp32 accumulation, fp32 master weights / optimizer state / gradients.
 * vocab > 0 sizes the token embedding [vocab, d_model] of a first stage (vocab < 2^17) and the
 * head of a last stage (vocab < 2^20): logits = RMSNorm(x) W^T with W the embedding when
 * tie_embedding (which needs first_stage and last_stage), else the stage's "head" matrix
 * [vocab, d_model].  The head keeps fp32 logits [tokens, vocab] per activation slot.  head_dim in {32, 64, 128};
 * n_heads a multiple of n_kv_heads; d_model a multiple of 64.  max_inflight >= 1 is the number
 * of activation slots (microbatches whose backward is pending).  optimizer 0: AdamW only;
 * 1: the arena also holds the Newton-Schulz workspace of delayed Muon (Alg. 2 of §4), 8 to 12 (fp32
 * stage: 8) bytes per element of the blocks' weight matrices plus their Gram matrices, so that
 * delayed_update accepts update_hparams_t.optimizer = 1; 2: the arena also holds Adan's two extra
 * state vectors (8 bytes per parameter), so that delayed_update accepts optimizer = 4.  max_delay
 * in [0, 8] (0 is read as 1):
 * the largest delay delayed_update accepts; the arena holds max_delay + 1 gradient buffers and
 * max_delay EF buffers. */
typedef struct {
  int32_t n_blocks, d_model, n_heads, n_kv_heads, head_dim, d_ffn;
  int32_t vocab, first_stage, last_stage, tie_embedding;
  int32_t seq_len, micro_batch, max_inflight;
  int32_t dtype;
  float rms_eps, rope_theta;
  int32_t optimizer;
  int32_t max_delay;
} stage_shape_t;

/* Hyper-parameters of one update.  clip_norm <= 0 disables clipping.  ef_lambda = 0 is standard
 * delayed training, 1 the Error-Feedback equation of §3.2.  delay 1 is Alg. 1; delay 0 is the
 * synchronous optimizer (requires ef_lambda = 0); delay tau in [2, max_delay] consumes g_{t-tau}
 * with EF against the update formed tau iterations earlier (ef_lambda = tau reproduces the
 * appendix's x_k - (tau + 1) u_k + tau u_{k-tau}).  The delay of a stage stays fixed over a run.
 * optimizer 0: AdamW (beta1, beta2, eps) on every parameter.  optimizer 1: delayed Muon (Alg. 2
 * of §4) on every 2-D weight matrix of a block (wq, wk, wv, wo, wgate, wup, wdown, each on its
 * own) and AdamW on the embedding and the gains: M <- momentum M + (1 - momentum) c g;
 * O = Newton-Schulz(M) (ns_steps >= 1 quintic iterations on M / ||M||_F in the orientation with
 * rows <= cols, coefficients (3.4445, -4.7750, 2.0315); on a bf16 stage the iterate is held in
 * fp32 or as a hi + lo pair of bf16 matrices and the product P X uses the pair, while
 * A = hi hi^T and P = b A + c A A are bf16);
 * u = lr (update_rms sqrt(max(rows, cols)) O + weight_decay x_t); then the same standard or
 * Error-Feedback step as AdamW.  Needs a stage shaped with optimizer 1.
 * optimizer 2: Lion (§3.3's optimizer list) on every parameter, u = lr (sign(beta1 m + (1 - beta1)
 * c g) + weight_decay x_t), m <- beta2 m + (1 - beta2) c g (v unused).  optimizer 3: NAdam with the
 * momentum-decay schedule mu_k = beta1 (1 - 0.5 0.96^(k nadam_psi)): m, v as AdamW and u = lr
 * ((1 - mu_k) / (1 - P_k) c g + mu_{k+1} / (1 - P_k mu_{k+1}) m) / (sqrt(v / (1 - beta2^k)) + eps)
 * + lr weight_decay x_t, P_k = mu_1 ... mu_k.  optimizer 4: Adan (§3.3's optimizer list; the rule of
 * the cited Adan work, betas as averaging weights, the paper's beta1 = 0.98) on every parameter,
 * with diff = c g - c g_last (0 at the first update; g_last the clipped gradient the previous update
 * consumed): m <- beta1 m + (1 - beta1) c g, d <- beta2 d + (1 - beta2) diff, n <- beta3 n + (1 -
 * beta3) (c g + beta2 diff)^2 (n in the v slot), u = lr ((m / (1 - beta1^k) + beta2 d / (1 - beta2^k))
 * / (sqrt(n / (1 - beta3^k)) + eps) + weight_decay x_t); needs a stage shaped with optimizer 2.
 * predict 1 (AdamW, delay 1, ef_lambda 0 only): SAPipe weight prediction with the updated
 * optimizer state (App. B.1) - the master takes the standard delayed step x_{t+1} = x_t -
 * u_{t-1}(g_{t-1}) while the compute copy receives x_{t+1} - u_t(g_{t-1}), AdamW fed g_{t-1} once
 * more from the updated state (bias correction k + 1; the predicted state is not kept). */
typedef struct {
  float lr, beta1, beta2, eps, weight_decay, clip_norm, ef_lambda;
  int32_t delay;
  int32_t optimizer;
  float momentum, update_rms;
  int32_t ns_steps;
  int32_t predict;
  float nadam_psi;
  float beta3;
} update_hparams_t;

/* Bytes of device memory the stage needs (weights, optimizer state, max_delay + 1 gradient
 * buffers, max_delay EF buffers, two compute versions, the activation ring and scratch).  0 on an
 * invalid shape. */
size_t stage_required_bytes(const stage_shape_t* shape);

/* Carve the arena (device memory, >= stage_required_bytes, 256-byte aligned) and zero the
 * optimizer state.  The master weights are left for the caller to fill through stage_tensor(),
 * followed by stage_sync_weights().  hip_stream: a hipStream_t (NULL = default stream). */
int stage_init(const stage_shape_t* shape, void* arena, size_t arena_bytes, void* hip_stream,
               stage_t** out);

/* Number of named tensors exposed by stage_tensor. */
int stage_num_tensors(const stage_t* s, int32_t* count);

/* Tensor idx: name, device pointer, element count and dtype (stage_dtype).  Names:
 *   "embed", "blk{i}.attn_norm|wq|wk|wv|wo|ffn_norm|wgate|wup|wdown", "final_norm", "head" - fp32
 *   master weights [out, in]; the same names prefixed "m.", "v.", "u_prev." (fp32 optimizer
 *   state, EF buffer), "u_prev{j}." for j in [1, max_delay) (the further EF buffers: iteration t
 *   of a delay-tau run uses buffer t mod tau, "u_prev." being buffer 0), "grad{j}." for j in
 *   [0, max_delay] (gradient buffers: step s accumulates into buffer s mod (max_delay + 1)) and
 *   "w0.", "w1." (the two compute versions, bf16 or fp32); "flat.master|m|v|u_prev|u_prev{j}|
 *   grad{j}|w0|w1" for the whole flat vectors (padding between tensors is zero and stays zero);
 *   "act{slot}.blk{i}.{x|rstd1|n1|qkv|o|lse|h|rstd2|n2|gu|z}" (on a bf16 stage also "o32", the
 *   attention output in fp32) and "act{slot}.{x0|y|logits}"
 *   for the saved activations of an activation slot. */
int stage_tensor(const stage_t* s, int32_t idx, const char** name, void** dev_ptr,
                 int64_t* numel, int32_t* dtype);

/* Look a tensor up by name; STAGE_EINVAL if absent. */
int stage_tensor_by_name(const stage_t* s, const char* name, void** dev_ptr, int64_t* numel,
                         int32_t* dtype);

/* Copy the fp32 master weights into both compute versions (after the caller wrote them). */
int stage_sync_weights(stage_t* s);

/* Forward of one microbatch of optimizer step `step` at the weights x_step (compute version
 * step mod 2), saving activations in slot `slot` (0 <= slot < max_inflight).
 *   tokens  [micro_batch, seq_len] int32, device  (first stage; else NULL).  Ids outside
 *           [0, vocab) are not read: such a position embeds as a zero row and adds nothing to
 *           the embedding gradient.
 *   x_in    [micro_batch, seq_len, d_model] bf16/fp32 per dtype, device (non-first; else NULL)
 *   targets [micro_batch, seq_len] int32, device  (last stage; else NULL).  A target outside
 *           [0, vocab) is ignored: zero loss and zero gradient at that position (the mean still
 *           divides by micro_batch*seq_len).
 *   y_out   [micro_batch, seq_len, d_model] device (non-last; may be NULL to keep it in the slot)
 *   loss_dev one float, device (last stage: mean cross-entropy of this microbatch; else NULL)
 * STAGE_ESTATE if compute version step mod 2 does not hold x_step. */
int stage_forward(stage_t* s, int32_t slot, int64_t step, const int32_t* tokens, const void* x_in,
                  const int32_t* targets, void* y_out, float* loss_dev);

/* Backward of the microbatch saved in `slot`; its parameter gradient is added to gradient buffer
 * (step mod (max_delay + 1)) - the first backward of a step overwrites it; STAGE_ESTATE if that
 * buffer still holds a gradient no update has consumed.  dy: upstream gradient
 * [micro_batch, seq_len, d_model] (non-last stage; NULL on a last stage, whose loss is the mean
 * cross-entropy divided by microbatches_per_step).  dx_out: gradient w.r.t. x_in (non-first
 * stage; may be NULL).  STAGE_ESTATE if the slot holds no pending forward. */
int stage_backward(stage_t* s, int32_t slot, const void* dy, void* dx_out,
                   int32_t microbatches_per_step);

/* The last stage under a loss on the log-probabilities of its targets instead of the mean cross-entropy
 * (reward or preference fine-tuning; the losses are policy_loss and preference_loss below).
 * stage_forward_logprob is stage_forward up to the logits, then
 *   logp     [micro_batch, seq_len] fp32, device: log-probability of each target at inv_temperature in (0, 2^60]
 *            (token_logprob's rules; a target outside [0, vocab) is ignored: 0)
 *   entropy  the same shape, or NULL
 * and leaves the slot pending for stage_backward_logprob, which takes
 *   dlogp, dentropy  [micro_batch, seq_len] fp32, device: the loss's gradients (dentropy may be NULL), with
 *            whatever scale the caller's loss has; microbatches_per_step only places the chunks of overlap
 *            mode 2
 * and otherwise is stage_backward.  The two kinds of forward and backward do not mix on one slot
 * (STAGE_ESTATE). */
int stage_forward_logprob(stage_t* s, int32_t slot, int64_t step, const int32_t* tokens, const void* x_in,
                          const int32_t* targets, float inv_temperature, float* logp, float* entropy);
int stage_backward_logprob(stage_t* s, int32_t slot, const float* dlogp, const float* dentropy, void* dx_out,
                           int32_t microbatches_per_step);

/* The log-probabilities of stage_forward_logprob without a backward to follow (a reference policy, or the
 * policy an answer was sampled from): the logits are never all in memory (head_logprob).  `slot` must
 * hold no pending microbatch; its activations are overwritten and it stays free.  In the delayed update's
 * order this is a use of the weights of `step` like any forward. */
int stage_score_logprob(stage_t* s, int32_t slot, int64_t step, const int32_t* tokens, const void* x_in,
                        const int32_t* targets, float inv_temperature, float* logp, float* entropy);

/* Second half of iteration t of Alg. 1: with delay tau >= 1 consume g_{t-tau} (the gradient of
 * step t-tau, complete), with delay 0 consume g_t; clip by the global norm; AdamW (or Muon);
 * standard or lambda-EF update of the master weights (EF once tau earlier updates exist: the
 * "t <= 1" rule for tau = 1; the EF buffer of iteration t is t mod tau); write x_{t+1} to compute
 * version (t+1) mod 2.  Must be called once per t in increasing order; for t < tau (no pending
 * gradient) the weights are unchanged (u_{-1} = 0).  A non-finite
 * gradient norm leaves x, m, v and the EF buffer untouched (x_{t+1} = x_t, the compute copy is
 * written from x_t) and is counted on the device; see stage_poll_nonfinite.  Such an iteration still
 * counts as having consumed its gradient: the bias-correction index of every update is
 * k = t - tau + 1 (t + 1 with delay 0) whether or not earlier gradients were skipped, Error Feedback
 * starts once tau gradients have been consumed, and an EF buffer the skipped iteration would have
 * written keeps its contents.  The norm (two deterministic passes over the gradient) runs whether
 * or not clipping is on, since it is also the non-finite check.  STAGE_ESTATE on out-of-order t or
 * an incomplete gradient. */
int delayed_update(stage_t* s, int64_t t, const update_hparams_t* hp);

/* Resume a run at iteration next_t of a fixed-delay run (Alg. 1 carries x_t, the optimizer
 * statistics, the EF buffers and the gradients not yet consumed from one iteration to the next).
 * On a fresh stage (no delayed_update yet, no pending microbatch), after the caller has written
 * through stage_tensor views the master weights x_next_t, m, v, every EF buffer ("u_prev.",
 * "u_prev{j}.") and, for delay tau >= 1, the gradients g_s of steps s = next_t - tau .. next_t - 1
 * into their buffers "grad{s mod (max_delay + 1)}.": marks those gradients complete and unconsumed,
 * sets the count of consumed gradients to next_t - tau (next_t with delay 0) and copies the master
 * weights into both compute versions (stage_sync_weights).  The next calls are stage_forward(...,
 * step next_t, ...) and delayed_update(next_t).  delay in [0, max_delay] is the delay of the run
 * being resumed.  STAGE_ESTATE when the stage has run an update or holds a pending microbatch. */
int stage_resume(stage_t* s, int64_t next_t, int32_t delay);

/* Stateless fused update (AdamW, Lion, NAdam or the AdamW weight prediction of hp; not Muon) over
 * flat device vectors of n elements:
 * iteration t of a delay-tau run (tau = hp->delay >= 1) consumes g_prev (= g_{t-tau}; fp32, or
 * bf16 when g_is_bf16), with k = t - tau + 1 the AdamW bias-correction index and EF from
 * t >= 2 tau; t < tau only writes x_shadow.  x, m, v, u_prev fp32 (read and written; u_prev holds
 * the update formed tau iterations earlier - the caller keeps a ring of tau buffers, slot t mod
 * tau - and may be NULL when ef_lambda = 0); x_shadow (written, bf16 when shadow_is_bf16 else
 * fp32; may be NULL; required with predict, which writes the predicted point there).
 * clip_scale_dev: device float multiplying g_prev, or NULL for 1. */
int delayed_update_flat(int64_t n, float* x, const void* g_prev, int32_t g_is_bf16, float* m,
                        float* v, float* u_prev, void* x_shadow, int32_t shadow_is_bf16,
                        int64_t t, const update_hparams_t* hp, const float* clip_scale_dev,
                        void* hip_stream);

/* delayed_update_flat for Adan (hp->optimizer 4), whose rule keeps two more state vectors: d (the
 * average of gradient differences) and g_last (the clipped gradient of the previous update), fp32,
 * 16-byte aligned, read and written; v holds Adan's second moment n.  Every other argument and the
 * delay / EF / shadow conventions as delayed_update_flat. */
int delayed_update_flat_adan(int64_t n, float* x, const void* g_prev, int32_t g_is_bf16, float* m, float* v,
                             float* d, float* g_last, float* u_prev, void* x_shadow, int32_t shadow_is_bf16,
                             int64_t t, const update_hparams_t* hp, const float* clip_scale_dev, void* hip_stream);

/* Device bytes of the workspace grad_norm_flat needs (partial sums of the first pass). */
size_t grad_norm_flat_workspace_bytes(void);

/* Global L2 norm of a flat gradient vector and its clip coefficient (the gradient clipping of §2 /
 * App. E.1, c = min(1, clip_norm / (||g|| + 1e-6)), 1 when clip_norm <= 0 or the norm is not
 * finite), the pass delayed_update runs over the stage's gradient, for a caller-held flat vector
 * (with delayed_update_flat, whose clip_scale_dev can be out_dev + 1).  Two deterministic passes:
 * contiguous ranges summed in double per block, then the partials in a fixed order.
 *   g          n elements, fp32 or bf16 (g_is_bf16), device, 16-byte (bf16: 8-byte) aligned
 *   out_dev    two floats, device: ||g||, c
 *   nonfinite_dev  one int32, device, set to 1 when ||g|| is not finite and 0 otherwise; may be NULL
 *   workspace  device scratch of >= grad_norm_flat_workspace_bytes(), 8-byte aligned, owned by
 *              the caller; calls that share a workspace must not overlap
 * Enqueued on hip_stream. */
int grad_norm_flat(int64_t n, const void* g, int32_t g_is_bf16, float clip_norm, float* out_dev,
                   int32_t* nonfinite_dev, void* workspace, size_t workspace_bytes, void* hip_stream);

/* grad_norm_flat for callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same two passes, with the partial sums
 * in a static device array of the library (1024 doubles, 8 KiB per GPU, held until the process
 * ends) instead of a caller workspace.  It calls no hipMalloc, hipFree or allocating routine.  The
 * first pass runs at most 1024 blocks whatever n is, so n has no scratch-imposed maximum; a grid that
 * would need more partials is refused with STAGE_EINVAL.  Every call on a GPU shares that GPU's
 * array (each call overwrites every partial it reads): calls that overlap on one GPU race.
 * Arguments, results and alignment as grad_norm_flat. */
int grad_norm_flat_noalloc(int64_t n, const void* g, int32_t g_is_bf16, float clip_norm, float* out_dev,
                           int32_t* nonfinite_dev, void* hip_stream);

/* Measurement reference, not a step of the method: a streaming device copy of `bytes` (a multiple
 * of 16; both pointers 16-byte aligned) with 16-byte non-temporal loads and stores, four chunks in
 * flight per thread - the practical HBM ceiling the update pass's bandwidth is reported against. */
int hbm_stream_copy(void* dst, const void* src, size_t bytes, void* hip_stream);

/* A variant of the stage's blocks, beside the plain causal ones: attention scores capped by a tanh and lowered by
 * distance, rows that pack several documents (attention_key_ranges, attention_forward below say what each
 * is), and dropout on the outputs of a block's two branches before they join the residual stream (dropout_add). */
typedef struct {
  float softcap;         /* 0 (none) or in [2^-60, 2^100]                                            */
  const float* slopes;   /* [n_heads] device array or NULL; kept, owned by the caller                */
  double dropout;        /* p of both branches; a forward without a backward (stage_score_logprob) has none */
  uint64_t seed, offset; /* dropout_add's: block i of the n-th forward from here takes the offsets
                            offset + 2 (n_blocks n + i) (attention) and the next one (feed-forward)  */
  int32_t documents;     /* not 0: every forward takes the documents of its slot                     */
} stage_variant_t;
/* Sets (v NULL: takes back) the variant for the forwards from here on and their backwards; no slot may hold a
 * pending microbatch (STAGE_ESTATE).  workspace: device memory of stage_variant_bytes(), 256-byte aligned, kept
 * until the variant is replaced.  To continue a run, pass the offset its next forward would have taken. */
size_t stage_variant_bytes(stage_t* s, const stage_variant_t* v);
int stage_set_variant(stage_t* s, const stage_variant_t* v, void* workspace, size_t workspace_bytes);
/* The documents [micro_batch, seq_len] int32 packed in the slot's rows, and their prefixes (uint8 or NULL), for
 * its forwards until they are set again (attention_key_ranges, read on the stage stream).  RoPE positions
 * run along the row (only their differences count); targets of padding are the caller's (outside the
 * vocabulary: ignored).  A forward of a slot whose documents were never set is refused (STAGE_ESTATE). */
int stage_set_documents(stage_t* s, int32_t slot, const int32_t* documents, const uint8_t* prefix);

/* ---------------------------------------------------------------------------------------------
 * Log-probabilities and the losses on them: fine-tuning by rewards or preferences on the stage that
 * otherwise trains on next-token cross-entropy.  A last stage runs them in its own paths
 * (stage_forward_logprob, stage_backward_logprob, stage_score_logprob); these calls take a caller's
 * arrays.
 *
 * Common rules: every call is stateless, enqueues on hip_stream of the current device and allocates
 * nothing.  `workspace` is device scratch of at least the bytes the matching *_workspace_bytes call
 * gives (it may be NULL where that is 0), 256-byte aligned, written before it is read; calls that share
 * one must not overlap.  Arrays need the alignment of their element type only; an output may not
 * overlap an input unless said.  Sizes of 0 are allowed.  The *_workspace_bytes calls give 0 on sizes
 * their operator refuses.  Results are the same bit for bit from call to call.
 */

/* Log-probability of targets[r] under row r of logits, at inv_temperature s in (0, 2^60]: log p =
 * s (x_t - m) - log S with m the row's largest logit and S = sum_j exp(s (x_j - m)), and the entropy H = -sum p log p.
 *   logits      [rows, vocab] fp32, or bf16 when logits_bf16; rows ld >= vocab elements apart;
 *               vocab in [1, 2^24], ld <= 2^28
 *   targets     [rows] int32; a row whose target is outside [0, vocab) is ignored: its logits are not
 *               read and its outputs are 0
 *   logp        [rows] fp32;  entropy [rows] fp32, may be NULL
 *   stats       [rows, 2] fp32, m and log S (read by token_logprob_backward); may be NULL
 * A logit of -inf is a token that cannot occur (logp -inf for such a target); a row of only -inf has
 * logp -inf, entropy 0 and stats (-inf, 0).  A NaN or +inf among a row's logits makes its logp and
 * entropy NaN. */
size_t token_logprob_workspace_bytes(int64_t rows, int64_t vocab);
int token_logprob(int64_t rows, int64_t vocab, const void* logits, int64_t ld, int32_t logits_bf16,
                  const int32_t* targets, float inv_temperature, float* logp, float* entropy, float* stats,
                  void* workspace, size_t workspace_bytes, void* hip_stream);

/* Gradient in the logits of any function of the log-probabilities and entropies of token_logprob:
 * dlogits[r, j] = s (g (1[j = t] - p_j) - h p_j (log p_j + H)), g = dlogp[r], h = dentropy[r].
 * logits, targets and inv_temperature as in the forward, stats (and, with dentropy, entropy) what it
 * wrote; dentropy may be NULL (then entropy too).  dlogits: fp32, or bf16 (one rounding, to nearest)
 * when out_bf16, rows ld_out >= vocab elements apart, columns past vocab left as they are; it may be
 * logits itself (same type and row stride).  A row that is ignored, has only -inf, or has g = h = 0
 * gets zeros and its logits are not read. */
int token_logprob_backward(int64_t rows, int64_t vocab, const void* logits, int64_t ld, int32_t logits_bf16,
                           const int32_t* targets, const float* stats, const float* entropy,
                           const float* dlogp, const float* dentropy, float inv_temperature, void* dlogits,
                           int64_t ld_out, int32_t out_bf16, void* hip_stream);

/* token_logprob of the logits x W^T of a head, which are never all in memory: x [rows, d] hidden states
 * (after the final norm), W [vocab, d] the head's matrix, both fp32 or both bf16 (is_bf16), rows ldx and
 * ldw >= d elements apart; the products accumulate in fp32.  d in [1, 2^20], ldx and ldw <= 2^24; the other arguments as in
 * token_logprob.  For log-probabilities no gradient flows through: those of a reference policy, or
 * of the policy an answer was sampled from. */
size_t head_logprob_workspace_bytes(int64_t rows, int64_t vocab, int64_t d, int32_t is_bf16);
int head_logprob(int64_t rows, int64_t vocab, int64_t d, const void* x, int64_t ldx, const void* w, int64_t ldw,
                 int32_t is_bf16, const int32_t* targets, float inv_temperature, float* logp, float* entropy,
                 float* stats, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Policy loss of answers [seqs, len] against the policy they were sampled from, and its gradients.
 * Per token with mask != 0, x = logp - old_logp, r = e^x, A its advantage, d = ref_logp - logp:
 *   l = max(-r A, -clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (e^d - 1 - d) - entropy_coef H
 *   loss = sum w l, with w = 1 / N over the N tokens that count (reduction 0), or 1 / (B n_b) for a
 *   sequence of n_b > 0 such tokens among B sequences that have any (reduction 1); norm > 0 takes the
 *   place of N or B (a count over the whole step, where it is split into microbatches)
 *   dlogp = grad_scale w (-r A [not clipped] + kl_coef (1 - e^d)),  dentropy = -grad_scale w entropy_coef
 * A token is clipped where A > 0 and x > log(1 + clip_high), or A < 0 and x < log(1 - clip_low); it then
 * has no gradient from the first term.  A term is left out where its factor (A, kl_coef, entropy_coef) is 0,
 * also where it is infinite; e^d - 1 - d is infinite at d = +-inf. */
typedef struct {
  float clip_low, clip_high; /* clip_low in [0, 1], clip_high >= 0 */
  float kl_coef, entropy_coef;
  double norm;               /* 0: the counts of this call */
  double grad_scale;         /* multiplies the gradients, not the loss */
  int32_t reduction;         /* 0: mean over tokens, 1: mean over sequences of their means */
  int32_t advantage_per_token;
} policy_hparams_t;

/*   logp, old_logp      [seqs, len] fp32
 *   ref_logp            [seqs, len] fp32 or NULL (then kl_coef must be 0)
 *   entropy             [seqs, len] fp32 or NULL (then entropy_coef must be 0)
 *   advantages          [seqs] fp32, or [seqs, len] with hp->advantage_per_token
 *   mask                [seqs, len] uint8; where it is 0 the other arrays may hold anything, and the
 *                       gradients are 0
 *   loss                one fp32;  dlogp [seqs, len] fp32
 *   dentropy            [seqs, len] fp32 (NULL exactly when entropy is)
 *   metrics             6 fp32, sums of w times: the clipped surrogate, the KL term to ref_logp, the
 *                       entropy, whether the token is clipped, e^x - 1 - x, r
 *   counts              2 int64: tokens and sequences that count
 * seqs in [0, 2^31), len in [0, 2^31), seqs len < 2^40.  No token that counts: everything is 0. */
size_t policy_loss_workspace_bytes(int64_t seqs, int64_t len);
int policy_loss(int64_t seqs, int64_t len, const float* logp, const float* old_logp, const float* ref_logp,
                const float* entropy, const float* advantages, const uint8_t* mask, const policy_hparams_t* hp,
                float* loss, float* dlogp, float* dentropy, float* metrics, int64_t* counts, void* workspace,
                size_t workspace_bytes, void* hip_stream);

/* Preference loss of pairs of answers, and its gradient.  Rows 0 .. pairs - 1 of the arrays are the
 * chosen answers, row pairs + p the rejected one of pair p.  A row's score is the sum of logp - ref_logp
 * over its tokens with mask != 0 (divided by their number with length_normalize); for a pair,
 * delta = score(chosen) - score(rejected) and h = beta delta - margin:
 *   kind 0 (sigmoid)  l = -(1 - e) log sigmoid(h) - e log sigmoid(-h), e = label_smoothing
 *   kind 1 (hinge)    l = max(0, 1 - h)
 *   kind 2 (square)   l = ((h - 1/2) / beta)^2
 * loss = the mean of l over the pairs whose rows both have tokens; the others (padding of a batch) have
 * loss, rewards and gradients 0.  norm > 0 divides instead of their number. */
typedef struct {
  float beta; /* > 0 */
  float label_smoothing; /* [0, 1]; kind 0 only */
  float margin;
  int32_t kind, length_normalize;
  double norm, grad_scale;
} preference_hparams_t;

/*   logp       [2 pairs, len] fp32;  ref_logp the same or NULL (no reference: logp alone)
 *   mask       [2 pairs, len] uint8; where it is 0 the other arrays may hold anything
 *   loss       one fp32;  dlogp [2 pairs, len] fp32 = grad_scale dloss/dlogp
 *   pair_loss  [pairs] fp32;  rewards [2 pairs] fp32 = beta score
 *   metrics    4 fp32, means over the same pairs: delta > 0, reward of the chosen, of the rejected, h
 *   counts     1 int64: pairs that count
 * pairs in [0, 2^24], len in [0, 2^31), 2 pairs len < 2^40. */
size_t preference_loss_workspace_bytes(int64_t pairs, int64_t len);
int preference_loss(int64_t pairs, int64_t len, const float* logp, const float* ref_logp, const uint8_t* mask,
                    const preference_hparams_t* hp, float* loss, float* dlogp, float* pair_loss, float* rewards,
                    float* metrics, int64_t* counts, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Key ranges of packed documents.  documents [batch, length] int32: a document is a run of equal ids >= 0; ids
 * below 0 are padding.  Query i sees the keys [key_start[i], key_end[i]) of its row: from the first token of
 * its document to itself; with prefix [batch, length] uint8 (or NULL), the tokens from a document's first one on
 * whose flag is not 0 see that whole run of them.  Padding sees nothing (0, 0).  batch in [0, 2^24], length in [0, 2^30]; the
 * time grows with the square of a document's length beyond 2048 tokens. */
int attention_key_ranges(int64_t batch, int64_t length, const int32_t* documents, const uint8_t* prefix,
                         int32_t* key_start, int32_t* key_end, void* hip_stream);

/* Softmax attention over a range of keys per query, forward and backward, of grouped query heads (query head h
 * reads key/value head h / (heads / kv_heads)).  Query i of a sequence has position q_start + i and sees
 * keys [key_start[i], key_end[i]) (what lies outside [0, keys) is cut off), or, with key_start NULL, the
 * keys at or before its position.  With x = scale q.k the score of key j is
 *   cap tanh(x / cap) - slopes[h] |position - j|   (softcap 0: x; slopes NULL: no second term).
 * A launch bounds batch x (ceil(queries / 32) + 1) x heads + batch x (ceil(keys / 32) + 1) x kv_heads to below 2^25 (in
 * fp32 2^24) and, in the backward, batch x queries x heads x head_dim to about 2^34; a call beyond is refused.
 * A query that sees no key has o = 0, lse = -inf and no gradient; what a query does not see has no
 * influence on it, whatever it holds.  Products of bf16 accumulate in fp32; their operands P and dS
 * are rounded to bf16, but where o_f32 is kept the forward takes P in three bf16 parts (24 bits). */
typedef struct {
  int64_t batch, queries, keys;        /* [0, 2^24], [0, 2^30], [0, 2^30]                   */
  int32_t heads, kv_heads, head_dim;   /* kv_heads divides heads; head_dim 32, 64 or 128    */
  int32_t is_bf16;                     /* q, k, v, o and the gradients: bf16, else fp32     */
  int64_t q_strides[3], k_strides[3], v_strides[3]; /* elements between sequences, rows and heads; a head's
                                          elements are contiguous, strides and pointers whole 16 bytes  */
  const int32_t *key_start, *key_end;  /* [batch, queries] device arrays, or both NULL      */
  const int32_t* q_start;              /* [batch] device array; NULL: keys - queries        */
  const float* slopes;                 /* [heads] device array or NULL                      */
  float scale;                         /* [2^-60, 2^60]                                     */
  float softcap;                       /* 0 (none) or [2^-60, 2^100], scale / softcap >= 2^-126 */
} attention_params_t;

/*   q             [batch, queries, heads, head_dim];  k, v [batch, keys, kv_heads, head_dim], as strided
 *   o             [batch, queries, heads, head_dim], contiguous
 *   o_f32         the same in fp32 before its rounding, for the backward of a bf16 attention, or NULL
 *   lse           [batch, heads, queries] fp32: log of the sum of exp(score)
 *   workspace     attention_workspace_bytes(), 256-byte aligned (NULL where that is 0) */
size_t attention_workspace_bytes(const attention_params_t* p);
int attention_forward(const attention_params_t* p, const void* q, const void* k, const void* v, void* o, float* o_f32,
                      float* lse, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Gradients in q, k and v, from what the forward read and wrote (o, or better the o_f32 that it kept) and the
 * gradient dout in o.  No atomics: the same inputs give the same bits.  dq, dk and dv may interleave where they share
 * the strides that step over all of them: heads of one packed row, heads one by one ([B, S, kv_heads, 2, hd]), slices
 * of a [B, heads, S, hd] tensor.  Layouts that share an element, or of which that cannot be told, are refused. */
typedef struct {
  int64_t o_strides[3], dout_strides[3], dq_strides[3], dk_strides[3], dv_strides[3];
  void *dq, *dk, *dv;
  int32_t o_is_f32;   /* o is in fp32, whatever the type of the rest */
} attention_grads_t;
size_t attention_backward_workspace_bytes(const attention_params_t* p);
int attention_backward(const attention_params_t* p, const void* q, const void* k, const void* v, const void* o,
                       const float* lse, const void* dout, const attention_grads_t* g, void* workspace,
                       size_t workspace_bytes, void* hip_stream);

/* Dropout added to a residual: out = residual + keep x / (1 - p') over [rows, cols] with p' = t / 65536, t = p
 * 65536 rounded, p in [0, 1 - 2^-16].  Element e = row cols + col is kept when its 16-bit number is >= t:
 * bits 16 (e mod 2) .. of word (e mod 8) / 2 of Philox4x32-10 of the counter (e / 8, offset) under the key
 * seed.  The mask depends on nothing else, so the backward is the same call on the gradient with residual
 * NULL (nothing is added).  fp32 or bf16 (all three), rows ldx, ldr and ldo >= cols elements apart; out
 * may be x or residual itself.  Dropped elements of x may hold anything. */
int dropout_add(int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* residual, int64_t ldr, void* out,
                int64_t ldo, int32_t is_bf16, double p, uint64_t seed, uint64_t offset, void* hip_stream);

/* Ascending unique token ids of the microbatch in `slot` and their counts (after its backward
 * on a first stage).  ids, counts: device int32 arrays of >= micro_batch*seq_len entries;
 * n_unique: device int32. */
int stage_embed_indices(stage_t* s, int32_t slot, int32_t* ids, int32_t* counts,
                        int32_t* n_unique);

/* Synchronise the stream and report how many updates were skipped for a non-finite gradient
 * norm since the last poll (STAGE_ENONFINITE if any). */
int stage_poll_nonfinite(stage_t* s, int64_t* skipped);

/* Overlap mode (off by default).  Off: everything enqueued on the stage stream after
 * delayed_update(t) returns runs after that update.  On: the stage stream waits for update t only
 * where the one-step delay needs it - the first stage_forward of step t+1 (it reads compute
 * version (t+1) mod 2, which the update writes) and the first stage_backward that overwrites the
 * gradient buffer the update read (stage_sync_weights and stage_join_update wait for every
 * update).  A caller may then issue delayed_update(t) before step t's forwards and backwards, and
 * the update runs beside them on the stage's own stream (Alg. 1: x_{t+1} depends only on x_t and
 * g_{t-1}).  Reads of the master weights or optimizer state through stage_tensor() views must
 * follow stage_join_update() or a device synchronisation.  Turning it off joins.
 * on = 2: as 1, and the elementwise pass of each delayed_update (AdamW, Lion, NAdam, the
 * prediction; not Muon's or Adan's) is deferred in chunks, one per attention backward the stage
 * runs in a step (n_blocks x the microbatches_per_step of the last stage_backward; chunks of at
 * least 2^16 elements): each stage_backward launches the next chunk on the update stream as a
 * block's attention backward starts, so that the pass's HBM traffic runs beside work bound by the
 * matrix cores instead of beside the forward's products.  The results are those of mode 1
 * (elementwise pass, bit for bit).  Chunks not launched by then are launched by the first call that
 * needs the update: the forward that reads the version it writes, the backward that overwrites the
 * gradient buffer it reads, the next delayed_update, stage_join_update, stage_sync_weights, or a
 * change of mode; view reads must follow stage_join_update() (a device synchronisation alone does
 * not launch them).  Other values: STAGE_EINVAL. */
int stage_set_update_overlap(stage_t* s, int32_t on);

/* The stage stream waits for every delayed_update issued so far (no-op when none is owed). */
int stage_join_update(stage_t* s);

/* Global L2 norm of gradient buffer `which` (0 <= which <= max_delay), computed on device into
 * norm_dev (float). */
int stage_grad_norm(stage_t* s, int32_t which, float* norm_dev);

/* Kernel-class timing.  While enabled, the stage records a HIP event pair on the launching
 * stream around every launch of a class and, when read, adds up the elapsed times and the algorithmic work of
 * those launches: GEMM and attention in flops (2 M N K per product; causal attention forward
 * 4 B Hq hd s(s+1)/2, backward twice that, also where documents let a query see less), the delayed update and the gradient norm in bytes of
 * HBM traffic, the Newton-Schulz products of Muon (STAGE_PROF_NS) in flops.  Reading synchronises the stream and resets the counters.  Meant for measurement
 * passes; it adds two event records per launch. */
typedef enum {
  STAGE_PROF_GEMM = 0, STAGE_PROF_ATTN_FWD = 1, STAGE_PROF_ATTN_BWD = 2, STAGE_PROF_UPDATE = 3,
  STAGE_PROF_NORM = 4, STAGE_PROF_OTHER = 5, STAGE_PROF_NS = 6, STAGE_PROF_NCLASS = 7
} stage_prof_class;
int stage_profile_enable(stage_t* s, int32_t on);
int stage_profile_read(stage_t* s, int32_t cls, double* ms, int64_t* launches, double* work);

const char* stage_last_error(void);
void stage_destroy(stage_t* s);

#ifdef __cplusplus
}
#endif
#endif /* ASYNCSTAGE_H */

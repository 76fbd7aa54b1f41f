/*
 * libspo -- the data-parallel hot path of Single-stream Policy Optimization (SPO)
 * on NVIDIA B200 (sm_100a).  Plain C ABI.
 *
 * Conventions (every entry point):
 *   - Every pointer named d_* or documented "device" is device memory owned by the
 *     caller; the library allocates nothing and frees nothing.  Pointers must be
 *     16-byte aligned unless stated otherwise.  NULL is allowed only where marked
 *     "optional".
 *   - Work is enqueued on the caller's stream (`stream` is a cudaStream_t passed as
 *     void*; NULL = the default stream).  No call synchronises the host.
 *   - The return value is a host-side status (SPO_OK or a negative SPO_ERR_*),
 *     produced by argument checks and launch errors only.  Conditions found on
 *     the device (an id out of range, too few uniforms, a non-finite input, a
 *     bounded wait that ran out) are OR-ed as SPO_DEV_* bits into the caller's
 *     `d_status` word (device int32, must be zeroed by the caller beforehand);
 *     the offending element is skipped, nothing traps.  d_status may be NULL.
 *   - The device must be compute capability 10.x; otherwise SPO_ERR_UNSUPPORTED_ARCH.
 *   - Tracker table layout: `ab` is [N][2] fp32, interleaved (alpha, beta) per prompt.
 *   - Token rows are packed: sequence s owns rows cu_seqlens[s] .. cu_seqlens[s+1]-1.
 */
#ifndef SPO_H_
#define SPO_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* host-side status */
#define SPO_OK                        0
#define SPO_ERR_INVALID_ARG          -1   /* NULL where required, negative size, bad flag */
#define SPO_ERR_BAD_SHAPE            -2   /* size outside what the kernels support */
#define SPO_ERR_BAD_ALIGNMENT        -3
#define SPO_ERR_UNSUPPORTED_DTYPE    -4
#define SPO_ERR_UNSUPPORTED_ARCH     -5
#define SPO_ERR_WORKSPACE_TOO_SMALL  -6
#define SPO_ERR_CUDA                 -7   /* see spo_last_cuda_error() */

/* device-side status bits (OR-ed into *d_status) */
#define SPO_DEV_ID_OUT_OF_RANGE       1   /* prompt id or target token outside its table */
#define SPO_DEV_NONFINITE             2   /* NaN/Inf reward, divergence or table entry */
#define SPO_DEV_UNIFORMS_EXHAUSTED    4   /* fewer than B distinct prompts accepted */
#define SPO_DEV_TIMEOUT               8   /* a bounded wait inside a kernel ran out */
#define SPO_DEV_ZERO_TOTAL_WEIGHT    16   /* all sampling weights are zero */

/* element types of H / W / dH */
#define SPO_DTYPE_F32   0
#define SPO_DTYPE_BF16  1

/* token weights in the objective's expectation E_{s,t} (the paper does not say how responses of
 * different length are weighted): every unmasked token alike (default), or every response alike
 * with its tokens sharing the response's weight */
#define SPO_AGG_TOKEN_MEAN  0
#define SPO_AGG_SEQ_MEAN    1

/* objective evaluated by the loss calls.  Sec. 3.2 defines the first and names the other two as
 * compatible with the SPO advantage without writing them out; they follow their own publications:
 *   PPO_CLIP  sum_t u_t min(ratio_t a, clip(ratio_t, 1-clip_lo, 1+clip_hi) a)          (the default)
 *   CISPO     sum_t u_t w_t a logp_t with w_t = clip(ratio_t, 1-clip_lo, 1+clip_hi) held constant
 *             (no gradient through the weight): coef_t = -u_t w_t a for every unmasked token
 *   GSPO      one ratio per response, r_i = exp(mean over its unmasked tokens of logp_t - logp_old_t);
 *             (1/S_act) sum_i min(r_i a_i, clip(r_i) a_i); coef_t = -a_i r_i [unclipped_i] / (S_act n_i);
 *             agg_mode does not apply.  Needs every token of a response before any coef exists, so
 *             spo_loss_fwd_bwd runs it as forward-then-backward (see there) */
#define SPO_SUR_PPO_CLIP  0
#define SPO_SUR_CISPO     1
#define SPO_SUR_GSPO      2

/* selectors for spo_workspace_bytes */
#define SPO_WS_SAMPLE      0
#define SPO_WS_ADVANTAGES  1
#define SPO_WS_LOSS_FWD    2
#define SPO_WS_LOSS_BWD    3
#define SPO_WS_UPDATE_REPEATS 4
#define SPO_WS_ACTIVE_ROWS    5
#define SPO_WS_LOSS_BWD_ROWS  6
#define SPO_WS_LOSS_FWD_BWD   7
#define SPO_WS_LOSS_FWD_BWD_ROWS 8
#define SPO_WS_LOGPROBS       9
#define SPO_WS_LOGPROBS_BWD  10
#define SPO_WS_MUON          11   /* T = rows m, d = columns n, B = matrices */
#define SPO_WS_LAYERNORM_BWD 12
#define SPO_WS_GRAD_NORM     13

/*
 * Hyper-parameters.  Defaults (spo_default_params) are the values the paper prints:
 * rho_min 0.875, rho_max 0.96, clip_lo 0.2, clip_hi 0.28 (appendix "Training and
 * Evaluation Details"), eps_explore 0.05 (Sec. 3.3).  The paper names D_half but
 * gives no value; the default here is 0.1.  norm_eps and norm_ddof settle what the
 * paper leaves open about the batch standard deviation (population, +1e-8).
 */
typedef struct spo_params {
  float   rho_min;
  float   rho_max;
  float   d_half;
  float   eps_explore;
  float   clip_lo;
  float   clip_hi;
  float   norm_eps;
  int32_t norm_ddof;
  int32_t agg_mode;       /* SPO_AGG_*: how E_{s,t} of the objective weights tokens */
  /* Data-parallel training: when the mini-batch is spread over several ranks, the denominators of
   * the objective are those of the whole mini-batch.  0 = use this call's own counts. */
  int32_t global_tokens;     /* unmasked tokens of the whole mini-batch (n_tok) */
  int32_t global_responses;  /* responses with an unmasked token in the whole mini-batch (S_act) */
  int32_t surrogate;         /* SPO_SUR_*: which objective the loss calls evaluate */
  /* Second clip of dual-clip PPO (not in the paper; 0 = off, the default).  With c = dual_clip > 1 a
   * negative advantage's term becomes max(min(ratio a, clip(ratio) a), c a): once ratio > c the term
   * is the constant c a and carries no gradient.  Applies to SPO_SUR_PPO_CLIP (per token) and
   * SPO_SUR_GSPO (per response); SPO_SUR_CISPO has its own truncation and ignores it. */
  float   dual_clip;
  /* Tolerances of the near-zero-advantage counts (Sec. 4, signal efficiency: the share of raw
   * advantages with |A| <= tau, tracked at tau = 1e-4 and tau = 0.02). */
  float   near_zero_tau_lo;  /* 1e-4 */
  float   near_zero_tau_hi;  /* 0.02 */
} spo_params;

int32_t spo_default_params(spo_params* p /* host, out */);

/*
 * Algorithm 2 (SPO Initialization): N0 = 1/(1-rho_min); alpha0 = N0*v0; beta0 = N0*(1-v0).
 *   ab  device out [N][2];  v0  device in [N] initial estimates in [0,1].
 */
int32_t spo_tracker_init(float* ab, const float* v0, int64_t N,
                         const spo_params* params, void* stream);

/*
 * Prioritised sampling (Sec. 3.3, Eq. "sampling_coef"; Algorithm 1, the two
 * sampling steps): w(x) = sqrt(v(1-v)) + eps_explore with v = alpha/(alpha+beta)
 * (0.5 for an empty entry), then B distinct prompts drawn by weight.
 *
 * The draw is successive weighted sampling without replacement, made
 * reproducible bit for bit: weights are computed in fp32 by a fixed sequence of
 * individually rounded operations (nothing fused): n=a+b, t=a*b, x=t*(n*n);
 * for 2^-100 <= x <= 2^100 and a > 0 (any entry a tracker produces with both parameters
 * positive): y0 = the float with bits 0x5f3759df - (bits(x) >> 1), three Newton steps
 * y <- y*(1.5 - (0.5*x)*(y*y)), s = t*y (= sqrt(t)/n to 3e-7 relative); an empty entry has
 * s = 0.5, an entry with a or b zero s = 0, any other magnitude s = sqrt((a/n)*(b/n));
 * w = s+eps; q_i = floor(w_i * 2^32) (uint64); C_i = q_0+..+q_i; Wtot = C_{N-1};
 * for the k-th uniform U_k = floor(u_k * 2^32), t_k = floor(U_k*Wtot / 2^32),
 * candidate = first i with C_i > t_k; candidates are accepted in order k unless
 * already accepted, until B are accepted.
 *
 *   ab        device in  [N][2]
 *   uniforms  device in  [M] fp32 in [0,1); M >= B (M = 2B is ample for N >> B)
 *   out_ids   device out [B] int32, in acceptance order
 *   out_w     device out [N] fp32 weights, optional (the ids do not depend on whether it is given;
 *             given the same uniforms and these weights, the ids are fully determined by the
 *             integer arithmetic above)
 *   ws        device scratch, spo_workspace_bytes(SPO_WS_SAMPLE, ..., N, B, M) bytes (for tables of up
 *             to 2^20 prompts it includes 4 bytes per prompt: the call is organised for latency there,
 *             four short launches; larger tables are scanned at HBM speed)
 * Limits: 1 <= N < 2^31, 1 <= B <= M <= 2^20.
 * Device status: SPO_DEV_UNIFORMS_EXHAUSTED if fewer than B distinct candidates
 * (the tail of out_ids is then filled with -1), SPO_DEV_ZERO_TOTAL_WEIGHT,
 * SPO_DEV_NONFINITE for a negative or non-finite table entry (weight treated as 0).
 */
int32_t spo_sample_prompts(const float* ab, int64_t N, const float* uniforms, int32_t M, int32_t B,
                           int32_t* out_ids, float* out_w, void* ws, size_t ws_bytes,
                           const spo_params* params, int32_t* d_status, void* stream);

/*
 * Advantage with the pre-update baseline and global normalisation (Sec. 3.2;
 * Algorithm 1, "Compute raw advantage" and "Normalize advantages"):
 *   A_j = r_j - v(ids_j);  mu, sigma over the B values;  A~_j = (A_j - mu)/(sigma + norm_eps)
 * with sigma^2 = sum (A-mu)^2 / (B - norm_ddof).  Must be called BEFORE
 * spo_tracker_update for the same batch: the baseline is the table as it stood.
 *
 *   ids     device in  [B] int32 in [0,N)
 *   r       device in  [B] fp32 rewards
 *   a_raw   device out [B] fp32, optional
 *   a_norm  device out [B] fp32
 *   stats   device out [8] fp32 = (mu, sigma, B, M2 = sum (A-mu)^2, n_lo, n_hi, 0, 0), optional;
 *           n_lo / n_hi = how many raw advantages satisfy |A| <= near_zero_tau_lo / _hi (Sec. 4,
 *           signal efficiency; counts are exact up to 2^24).  (mu, M2, B) of several ranks merge
 *           exactly (pairwise: M2 = M2a + M2b + (mub-mua)^2 Ba Bb/(Ba+Bb)); the counts add.
 *   ws      device scratch, spo_workspace_bytes(SPO_WS_ADVANTAGES, ..., B, ...) bytes
 * An id outside [0,N) sets SPO_DEV_ID_OUT_OF_RANGE and contributes A = 0; a negative or non-finite
 * table entry sets SPO_DEV_NONFINITE and contributes A = 0 as well.
 */
int32_t spo_advantages(const float* ab, int64_t N, const int32_t* ids, const float* r, int32_t B,
                       float* a_raw, float* a_norm, float* stats, void* ws, size_t ws_bytes,
                       const spo_params* params, int32_t* d_status, void* stream);

/*
 * Second half of spo_advantages for a batch whose statistics were merged elsewhere (data-parallel
 * ranks each call spo_advantages for a_raw and stats, merge (mu, M2, B) on the host, then call
 * this): a_norm_j = (a_raw_j - mu) / (sigma + norm_eps)  (Sec. 3.2, global normalisation).
 * a_raw and a_norm may be the same buffer.
 */
int32_t spo_advantages_apply(const float* a_raw, int32_t B, float mu, float sigma, float* a_norm,
                             const spo_params* params, void* stream);

/*
 * spo_advantages with no scratch argument and no allocation anywhere.  (The paper has no
 * counterpart to this call: it computes exactly what spo_advantages computes and exists
 * only for the memory situation described here.)
 *
 * Who needs it: code that runs where device memory can no longer be obtained -- a
 * trainer whose framework has already handed every free byte of HBM to its own caching
 * allocator, a plug-in that is given input and output buffers but no allocator handle,
 * a step function that must never touch cudaMalloc because an allocation there would
 * synchronise the device or fail outright.  Such a caller cannot produce the `ws`
 * buffer that spo_advantages asks for large batches.
 *
 * Here the block partials of the two-pass path live in a fixed 32 KB array inside the
 * library's device image (each GPU that loads the library holds it until the process
 * exits).  Consequences the caller must know:
 *   - B may not exceed SPO_ADVANTAGES_STATIC_MAX_B; a larger B returns SPO_ERR_BAD_SHAPE
 *     and launches nothing.
 *   - The first call on a device looks up the array's device address (once per device,
 *     with that device current).  Make that first call outside any stream capture.
 *   - All calls share the one array.  Each call overwrites the part it later reads, so
 *     stale contents are harmless, but two calls whose kernels overlap on the GPU (two
 *     streams, two host threads) race on it: serialise them.
 *   - It calls no cudaMalloc/cudaFree or any allocating routine; inputs and outputs are
 *     still the caller's, with the same meaning, alignment and status bits as
 *     spo_advantages.  Always takes the two-kernel path, whatever B is.
 */
#define SPO_ADVANTAGES_STATIC_MAX_B  4194304
int32_t spo_advantages_static(const float* ab, int64_t N, const int32_t* ids, const float* r, int32_t B,
                              float* a_raw, float* a_norm, float* stats,
                              const spo_params* params, int32_t* d_status, void* stream);

/*
 * KL-adaptive tracker update (Sec. 3.1, the update equation; Algorithm 1, "Update tracker"):
 *   rho = clamp(2^(-D/D_half), rho_min, rho_max); alpha <- rho*alpha + r; beta <- rho*beta + (1-r)
 * at row ids[j], in place.  ids must be distinct within a call (what sampling
 * without replacement yields); duplicates race.
 *
 *   kl           device in: [B] per batch entry (kl_is_table = 0) or [N] per prompt,
 *                gathered by id (kl_is_table = 1)
 * A NaN divergence or reward sets SPO_DEV_NONFINITE and leaves the row untouched.
 */
int32_t spo_tracker_update(float* ab, int64_t N, const int32_t* ids, const float* r, const float* kl,
                           int32_t kl_is_table, int32_t B,
                           const spo_params* params, int32_t* d_status, void* stream);

/*
 * spo_advantages and spo_tracker_update for the same batch in one pass over the table (Algorithm 1:
 * "Compute raw advantage", "Update tracker", "Normalize advantages"): every entry ids[j] is read
 * once, A_j = r_j - v(ids_j) is formed from the value as read (the pre-update baseline of Sec. 3.2),
 * the entry is updated in place from that same value (Sec. 3.1) and the batch statistics and
 * normalised advantages follow as in spo_advantages.  Results equal the two calls made in the
 * paper's order; the table entry crosses the memory system once per step instead of twice.
 * ids must be distinct (as for spo_tracker_update).  Arguments, scratch size (SPO_WS_ADVANTAGES)
 * and status bits as in the two calls; an element with a bad id, table entry or reward contributes
 * A = 0 and leaves its entry untouched, a NaN divergence leaves the entry untouched.
 */
int32_t spo_advantages_update(float* ab, int64_t N, const int32_t* ids, const float* r, const float* kl,
                              int32_t kl_is_table, int32_t B, float* a_raw, float* a_norm, float* stats,
                              void* ws, size_t ws_bytes, const spo_params* params, int32_t* d_status, void* stream);

/*
 * Tracker update for batch SPO (appendix "Batch Extensions": every prompt rolled out G times per
 * batch against a shared baseline): like spo_tracker_update, but `ids` may repeat.  The entries
 * of one prompt are applied one after the other in batch order (the update equation of Sec. 3.1
 * composed G times), the same result as G successive calls; the outcome does not depend on
 * thread scheduling.  spo_advantages already accepts repeated ids (every copy reads the same
 * pre-update estimate), so a batch-SPO step is spo_advantages, then this call.
 *
 *   ws   device scratch, spo_workspace_bytes(SPO_WS_UPDATE_REPEATS, ..., B, ...) bytes
 * Limit: B <= 65536 (one thread block walks the rounds).  Status bits as spo_tracker_update.
 */
int32_t spo_tracker_update_repeats(float* ab, int64_t N, const int32_t* ids, const float* r, const float* kl,
                                   int32_t kl_is_table, int32_t B, void* ws, size_t ws_bytes,
                                   const spo_params* params, int32_t* d_status, void* stream);

/*
 * Policy loss forward (Sec. 3.2, the PPO-Clip objective with Clip-Higher bounds,
 * evaluated from final hidden states).  Per token row t:
 *   z = W h_t (never stored), lse = log sum_v exp z_v, logp = z[y_t] - lse,
 *   ratio = exp(logp - logp_old_t), a = a_norm[seq(t)],
 *   s_t = min(ratio*a, clip(ratio, 1-clip_lo, 1+clip_hi)*a),
 *   loss = - sum_t u_t s_t with token weights u_t that sum to one: u_t = mask_t / n_tok,
 *   n_tok = sum_t mask_t (SPO_AGG_TOKEN_MEAN), or u_t = mask_t / (S_act * n_seq(t)) with n_s the
 *   unmasked tokens of response s and S_act the responses that have any (SPO_AGG_SEQ_MEAN);
 *   loss = 0 if n_tok = 0.  With params->global_tokens / global_responses set, n_tok and S_act are
 *   those values (the whole data-parallel mini-batch) and `loss` is this rank's share: the ranks'
 *   losses and dW add up to the mini-batch's, dH rows are final;
 *   coef_t = d loss / d logp_t = -u_t * a * ratio * [gradient passes the clip].
 *   params->surrogate selects one of the other objectives (SPO_SUR_*, above) instead.
 *
 *   H           device in  [T][d], row-major, dtype as given (bf16: d % 64 == 0)
 *   W           device in  [V][d], row-major, same dtype
 *   y           device in  [T] int32 target token of each row
 *   logp_old    device in  [T] fp32
 *   mask        device in  [T] uint8, optional (NULL = all ones)
 *   cu_seqlens  device in  [S+1] int32, cu_seqlens[0] = 0, cu_seqlens[S] = T
 *   a_norm      device in  [S] fp32 normalised advantage per response
 *   loss        device out [1] fp32
 *   logp, lse, coef   device out [T] fp32 each
 *   seq_sums    device out [S][3] fp32 = per response (sum mask*logp,
 *               sum mask*(logp_old-logp), sum mask), optional
 *   entropy     device out [T] fp32, optional: entropy of each row's next-token distribution,
 *               -sum_v p log p = lse - sum_v p z, in nats (a diagnostic: Sec. 3.2 speaks of retaining
 *               policy entropy; it does not enter the objective).  Asking for it adds one multiply-add
 *               per logit to the contraction's epilogue; NULL costs nothing.
 *   ws          device scratch, spo_workspace_bytes(SPO_WS_LOSS_FWD, T, d, V, 0, S, 0) bytes
 *               (the B argument of that query carries the number of responses S)
 * A target outside [0,V) gives the row logp = -inf and coef = 0; it sets SPO_DEV_ID_OUT_OF_RANGE unless
 * the row is masked out (masked rows may carry an ignore-index target such as -100).
 */
int32_t spo_loss_fwd(const void* H, const void* W, int32_t dtype,
                     const int32_t* y, const float* logp_old, const uint8_t* mask,
                     const int32_t* cu_seqlens, const float* a_norm,
                     int64_t T, int32_t d, int32_t V, int32_t S,
                     float* loss, float* logp, float* lse, float* coef, float* seq_sums, float* entropy,
                     void* ws, size_t ws_bytes,
                     const spo_params* params, int32_t* d_status, void* stream);

/*
 * Policy loss backward: with p = exp(z - lse) recomputed tile by tile,
 *   g[t,v] = grad_loss * coef_t * (1[v = y_t] - p[t,v]);  dH = g W;  dW (+)= g^T H.
 * lse and coef are the forward's outputs for the same H, W, y.
 *
 *   dH        device out [T][d], dtype dH_dtype (bf16 or fp32)
 *   dW        device out [V][d] fp32; overwritten, or added to when dW_accumulate != 0
 *   ws        device scratch, spo_workspace_bytes(SPO_WS_LOSS_BWD, T, d, V, ...) bytes.
 *             For bf16 it holds a bounded chunk of g (a few thousand token rows
 *             by V, bf16), never the whole [T][V] matrix.
 */
int32_t spo_loss_bwd(const void* H, const void* W, int32_t dtype, const int32_t* y,
                     const float* lse, const float* coef, float grad_loss,
                     int64_t T, int32_t d, int32_t V,
                     void* dH, int32_t dH_dtype, float* dW, int32_t dW_accumulate,
                     void* ws, size_t ws_bytes,
                     const spo_params* params, int32_t* d_status, void* stream);

/*
 * Policy loss forward and backward in one pass: every output of spo_loss_fwd (loss, logp, lse,
 * coef, seq_sums; Sec. 3.2, the PPO-Clip objective) and of spo_loss_bwd (dH, dW) for the same
 * inputs, with three LM-head-sized contractions per token instead of four.  The loss is the last
 * node of the training graph, so its upstream gradient (`grad_loss`, e.g. 1 or a loss scale) is
 * known before the forward runs; that is what lets the two halves share their logits.
 *
 * bf16: token rows are processed in chunks (the chunk of spo_loss_bwd).  A short launch first
 * contracts every row with the first 512 vocabulary rows; the largest of those logits plus 40 binary
 * orders is the row's reference exponent ref_t.  The logits of a chunk are then contracted once; the
 * epilogue sums e = 2^(z log2(e) - ref_t) over the row (no running maximum is needed: fp32 and bf16
 * keep their relative precision at any magnitude) and stores every e as bf16.  With l_t = sum_v e the
 * softmax is e / l_t, so lse_t = (ref_t + log2 l_t) ln 2 and the logit gradient factors as
 *   g[t,v] = rowscale_t (e[t,v] - l_t 1[v = y_t]),   rowscale_t = -grad_loss coef_t / l_t:
 * after the chunk's rows are finalised the one target entry per row is patched in the stored chunk,
 * dH = rowscale (e W) takes the factor in its epilogue and dW = e^T (rowscale H) reads a scaled bf16
 * copy of the chunk's rows of H; the stored chunk is never rewritten.
 * loss, logp, lse and coef never see the bf16 rounding of e; dH and dW carry it
 * (and dW the rounding of rowscale H) in place of spo_loss_bwd's own bf16 rounding of g.
 * Range: a row whose largest logit exceeds the largest of its first 512 by more than 100 nats
 * overflows the stored exponentials; such a row sets SPO_DEV_NONFINITE, gets lse = Inf, logp = -Inf,
 * coef = 0 and takes no part in the gradients (use the two calls for such inputs).
 * fp32: the two SIMT halves run back to back (nothing to share).
 *
 *   arguments   as in spo_loss_fwd and spo_loss_bwd; lse and coef are outputs here.
 *               SPO_SUR_GSPO with bf16 inputs: a response's ratio needs the log-probs of all its tokens,
 *               which may lie in later chunks, so the call runs the forward to the end and then the
 *               chunked backward (four contractions, the cost of the two calls).
 *   ws          device scratch, spo_workspace_bytes(SPO_WS_LOSS_FWD_BWD, T, d, V, 0, S, 0) bytes:
 *               two chunk buffers (a few thousand token rows by V each, bf16), scaled bf16 copies of those
 *               chunks' rows of H, 36 bytes per token row and the forward's partials
 * Status bits as spo_loss_fwd.
 */
int32_t spo_loss_fwd_bwd(const void* H, const void* W, int32_t dtype,
                         const int32_t* y, const float* logp_old, const uint8_t* mask,
                         const int32_t* cu_seqlens, const float* a_norm,
                         int64_t T, int32_t d, int32_t V, int32_t S, float grad_loss,
                         float* loss, float* logp, float* lse, float* coef, float* seq_sums, float* entropy,
                         void* dH, int32_t dH_dtype, float* dW, int32_t dW_accumulate,
                         void* ws, size_t ws_bytes,
                         const spo_params* params, int32_t* d_status, void* stream);

/*
 * spo_loss_fwd_bwd for data-parallel ranks (Algorithm 1's mini-batch update spread over several GPUs:
 * every rank holds part of the responses, W is replicated, and the ranks' dW must be summed).  dW is
 * only final once its last contraction has run; this variant cuts that last launch into slabs of
 * vocabulary rows and records a CUDA event behind each, so that the caller can start reducing slab k
 * over the ranks on another stream (wait for events[k], then all-reduce rows row_begin[k] ..
 * row_begin[k+1]-1 of dW) while slab k+1 is still being contracted; only the last slab's reduction is
 * left exposed.  Results are those of spo_loss_fwd_bwd, bit for bit.
 *
 *   spo_dw_slab_rows   host only: writes row_begin[0..n] (row_begin[0] = 0, row_begin[n] = V) for a
 *                      request of n_wanted slabs (1 .. SPO_MAX_DW_SLABS) and returns n <= n_wanted
 *                      (slabs hold whole rounds of row tiles), or a negative status.
 *   events             host array of n_wanted cudaEvent_t (created by the caller, e.g. with timing
 *                      disabled); events[0..n) are recorded on `stream`.  Inputs for which the last
 *                      contraction is not cut (fp32, SPO_SUR_GSPO, T = 0) record them all at the end.
 * All other arguments as in spo_loss_fwd_bwd.  The library creates, waits on and destroys nothing.
 */
#define SPO_MAX_DW_SLABS 64
#define SPO_MAX_DW_SHARDS 16
int32_t spo_dw_slab_rows(int32_t V, int32_t d, int32_t n_wanted, int64_t* row_begin /* host, [n_wanted+1] */);
int32_t spo_loss_fwd_bwd_slabs(const void* H, const void* W, int32_t dtype,
                               const int32_t* y, const float* logp_old, const uint8_t* mask,
                               const int32_t* cu_seqlens, const float* a_norm,
                               int64_t T, int32_t d, int32_t V, int32_t S, float grad_loss,
                               float* loss, float* logp, float* lse, float* coef, float* seq_sums, float* entropy,
                               void* dH, int32_t dH_dtype, float* dW, int32_t dW_accumulate,
                               void* ws, size_t ws_bytes,
                               const spo_params* params, int32_t* d_status, void* stream,
                               int32_t n_wanted, void* const* events /* host, [n_wanted] */);

/*
 * spo_loss_fwd_bwd with the reduce-scatter of dW fused into its last contraction (data-parallel ranks whose
 * optimizer is sharded over the vocabulary rows of W; Algorithm 1's mini-batch update spread over GPUs).
 * The vocabulary rows are cut into n_shards equal shards of rows_per_shard rows (the last may be shorter);
 * shard k lives in the memory of rank k (shard[k]: fp32 [rows_per_shard][d]; for k != own rank a pointer to
 * PEER device memory mapped into this process).  The epilogue of the call's LAST dW contraction adds each
 * finished tile of dW (the sum over all chunks of this rank's tokens) straight into the shard that owns its
 * rows with vector store-reductions (`red.global.add` — over NVLink for a peer's shard; nothing is loaded
 * from a peer and nothing waits on a peer), so the exchange overlaps the contraction tile by tile and no
 * collective library call touches dW.  After every rank's call has completed (a barrier the caller
 * provides: stream synchronise + process-group barrier), shard[own rank] holds the mini-batch's dW rows.
 *   - Every shard must be zeroed by its owner, and that zeroing visible to all ranks, before any rank's call.
 *   - dW is scratch here (it ends up holding the partial sums of the chunks before the last); dW_accumulate
 *     still means "dW already holds a term to include".
 *   - Summation order across ranks is not fixed: results are reproducible up to fp32 addition order.
 *   - Inputs for which the last contraction is not this kernel (fp32, SPO_SUR_GSPO, T = 0) are followed by
 *     a plain kernel that adds dW into the shards the same way.
 * All other arguments and outputs as spo_loss_fwd_bwd.
 */
typedef struct spo_dw_shards {
  int32_t n_shards;                       /* 1 .. SPO_MAX_DW_SHARDS */
  int64_t rows_per_shard;                 /* n_shards * rows_per_shard >= V */
  float*  shard[SPO_MAX_DW_SHARDS];       /* device pointers (own or peer memory), 16-byte aligned */
} spo_dw_shards;
int32_t spo_loss_fwd_bwd_scatter(const void* H, const void* W, int32_t dtype,
                                 const int32_t* y, const float* logp_old, const uint8_t* mask,
                                 const int32_t* cu_seqlens, const float* a_norm,
                                 int64_t T, int32_t d, int32_t V, int32_t S, float grad_loss,
                                 float* loss, float* logp, float* lse, float* coef, float* seq_sums, float* entropy,
                                 void* dH, int32_t dH_dtype, float* dW, int32_t dW_accumulate,
                                 void* ws, size_t ws_bytes,
                                 const spo_params* params, int32_t* d_status, void* stream,
                                 const spo_dw_shards* shards /* host */);

/*
 * Diagnostic (no counterpart in the paper): runs the kernels' bounded mbarrier wait on a barrier
 * that nothing ever signals, with a limit of `limit_us` microseconds (1 .. 1 000 000).  A healthy
 * build sets SPO_DEV_TIMEOUT in *d_status, writes 1 to *reached_end (device int32, optional) and the
 * kernel returns normally; the context stays usable.  It shows that a stuck pipeline stage ends in a
 * status bit, not in a hang.  One tiny launch on `stream`.
 */
int32_t spo_selftest_bounded_wait(uint32_t limit_us, int32_t* reached_end, int32_t* d_status, void* stream);

/*
 * Backward over the rows that carry gradient only.  A token whose coef is zero -- masked out of the
 * loss (e.g. tool output inside a response) or clipped on the side that stops the gradient --
 * contributes nothing to dH or dW, so the three contractions of spo_loss_bwd can run on the other
 * rows alone; their cost falls in proportion.  Two calls, because the number of such rows has to
 * reach the host to size the second one (the library itself never synchronises):
 *
 *   spo_loss_active_rows: rows[0..count) = ascending indices t with coef[t] != 0, *d_count = count.
 *     rows    device out [T] int32;  d_count  device out [1] int32
 *     ws      device scratch, spo_workspace_bytes(SPO_WS_ACTIVE_ROWS, T, ...) bytes
 *   (the caller reads *d_count back, e.g. after a stream synchronise)
 *   spo_loss_bwd_rows: same results as spo_loss_bwd(H, W, ..., T, ...): dH[t] for the listed rows,
 *     zeros elsewhere; dW as in spo_loss_bwd.  bf16 H / W only.
 *     rows    device in [T_act] from the first call;  T_act  host value of *d_count
 *     ws      device scratch, spo_workspace_bytes(SPO_WS_LOSS_BWD_ROWS, T_act, d, V, ...) bytes
 *             (holds the gathered rows of H and dH besides the chunk buffer)
 */
int32_t spo_loss_active_rows(const float* coef, int64_t T, int32_t* rows, int32_t* d_count,
                             void* ws, size_t ws_bytes, void* stream);
int32_t spo_loss_bwd_rows(const void* H, const void* W, int32_t dtype, const int32_t* y,
                          const float* lse, const float* coef, float grad_loss,
                          int64_t T, int32_t d, int32_t V, const int32_t* rows, int64_t T_act,
                          void* dH, int32_t dH_dtype, float* dW, int32_t dW_accumulate,
                          void* ws, size_t ws_bytes, const spo_params* params, int32_t* d_status, void* stream);

/*
 * One-pass loss over the unmasked rows only.  In tool-integrated reasoning the tokens a tool wrote
 * sit inside the response but carry no loss (mask = 0): they enter neither the objective of Sec. 3.2
 * nor its gradients, so none of the three contractions has to see them and the cost of the call
 * falls in proportion to the masked share.  Two calls, because the number of unmasked rows has to
 * reach the host to size the second one (the library itself never synchronises):
 *
 *   spo_loss_mask_rows: rows[0..count) = ascending indices t with mask[t] != 0, *d_count = count.
 *     mask    device in [T] uint8;  rows  device out [T] int32;  d_count  device out [1] int32
 *     ws      device scratch, spo_workspace_bytes(SPO_WS_ACTIVE_ROWS, T, ...) bytes
 *   (the caller reads *d_count back, e.g. after a stream synchronise)
 *   spo_loss_fwd_bwd_rows: what spo_loss_fwd_bwd(H, W, ..., mask, ...) gives for loss, seq_sums,
 *     dW, and for logp / lse / coef / dH at the listed rows; at all other rows logp, lse, coef and
 *     dH are ZERO (spo_loss_fwd_bwd reports logp and lse of masked rows too; use it if you need them).
 *     The listed rows of H, y and logp_old are gathered into a packed batch of T_act rows whose
 *     sequence boundaries are the counts of listed rows per response, and the one-pass path runs on
 *     that batch.  bf16 H / W only.  Every listed row counts as unmasked.
 *     rows    device in [T_act] from the first call;  T_act  host value of *d_count
 *     ws      device scratch, spo_workspace_bytes(SPO_WS_LOSS_FWD_BWD_ROWS, T_act, d, V, 0, S, 0) bytes
 *             (holds the gathered rows of H and dH besides the one-pass scratch)
 */
int32_t spo_loss_mask_rows(const uint8_t* mask, int64_t T, int32_t* rows, int32_t* d_count,
                           void* ws, size_t ws_bytes, void* stream);
int32_t spo_loss_fwd_bwd_rows(const void* H, const void* W, int32_t dtype,
                              const int32_t* y, const float* logp_old,
                              const int32_t* cu_seqlens, const float* a_norm,
                              int64_t T, int32_t d, int32_t V, int32_t S,
                              const int32_t* rows, int64_t T_act, float grad_loss,
                              float* loss, float* logp, float* lse, float* coef, float* seq_sums,
                              void* dH, int32_t dH_dtype, float* dW, int32_t dW_accumulate,
                              void* ws, size_t ws_bytes,
                              const spo_params* params, int32_t* d_status, void* stream);

/*
 * Diagnostics of one policy update over the unmasked tokens, from the forward's logp (no counterpart
 * in the paper's equations; these are the quantities its training curves are read by, and none
 * enters the objective).  out (device, [8] fp32):
 *   [0] n_tok   [1] mean importance ratio   [2] share of tokens whose gradient the clip stops
 *   (ratio beyond the bound that matters for the sign of their advantage; zero advantage: not stopped)
 *   [3] mean of logp_old - logp (sampled estimate of KL(old || new))   [4] mean of ratio - 1 - log ratio
 *   (a non-negative estimate of the same)   [5] largest ratio   [6] smallest ratio
 *   [7] share of tokens whose ratio lies outside [1-clip_lo, 1+clip_hi].  All zeros when n_tok = 0.
 * One block, fixed reduction order; a few tens of microseconds at 250 k tokens.
 */
int32_t spo_loss_stats(const float* logp, const float* logp_old, const uint8_t* mask,
                       const int32_t* cu_seqlens, const float* a_norm, int64_t T, int32_t S,
                       float* out, const spo_params* params, void* stream);

/*
 * Log-probabilities of given tokens straight from hidden states: what a step needs before its loss (the
 * rollout policy's or a reference policy's logp_old of Sec. 3.2, the divergence D(x) that Sec. 3.1's tracker
 * update reads) and what a sampler reports about the tokens it drew.  Per token row t, s = inv_temperature:
 *   z = W h_t (not kept), lse = log sum_v exp(s z_v), logp = s z[y_t] - lse,
 *   entropy = -sum_v p log p = lse - s sum_v p_v z_v   (nats),
 *   top_ids / top_logp: the top_k largest z in descending order, equal ones by ascending id, and their
 *   log-probabilities.
 *
 *   H           device in  [T] rows of d elements, row pitch ldH >= d elements (bf16: d % 64 == 0, ldH % 8 == 0;
 *               fp32: d % 4 == 0, ldH % 4 == 0), so the last-token rows of a padded batch need no copy
 *   W           device in  [V][d], same dtype
 *   y           device in  [T] int32, optional together with logp (both NULL: no target)
 *   mask        device in  [T] uint8, optional: rows with mask 0 give logp = lse = entropy = 0, ids -1,
 *               top_logp 0, whatever their H and y hold (NaN included), and set no status bit
 *   inv_temperature   1e-4 .. 1e4
 *   top_k       0 .. SPO_MAX_TOP_K, at most V
 *   logp, lse   device out [T] fp32;  entropy  device out [T] fp32, optional
 *   top_ids     device out [T][top_k] int32;  top_logp  device out [T][top_k] fp32 (NULL when top_k = 0)
 *   ws          device scratch, spo_workspace_bytes(SPO_WS_LOGPROBS, T, d, V, 0, top_k, 0) bytes; a buffer of the size
 *               named for T rows serves every call of at most T rows (same d, V and top_k)
 * A target outside [0,V) gives logp = -inf and SPO_DEV_ID_OUT_OF_RANGE; a row whose lse is not finite sets
 * SPO_DEV_NONFINITE.  A logit of -inf (a banned token) has probability zero: it adds nothing to lse and entropy, and its
 * own log-prob is -inf.  Logits that are NaN or -inf are never listed; where fewer than top_k are left the
 * remaining ids are -1 with top_logp -inf.  A row with nothing but -inf has lse -inf.  T = 0 is allowed and launches nothing.
 */
#define SPO_MAX_TOP_K 20
int32_t spo_logprobs(const void* H, int64_t ldH, const void* W, int32_t dtype, const int32_t* y, const uint8_t* mask,
                     int64_t T, int32_t d, int32_t V, float inv_temperature, int32_t top_k,
                     float* logp, float* lse, float* entropy, int32_t* top_ids, float* top_logp,
                     void* ws, size_t ws_bytes, int32_t* d_status, void* stream);

/*
 * Gradients of spo_logprobs for upstream gradients of logp, lse and entropy (a loss of the caller's own over
 * the log-probabilities, an entropy bonus, a penalty on lse; the alternatives are constants):
 *   dz[t,v] = s ( g_logp_t (1[v = y_t] - p) + g_lse_t p - g_entropy_t p (log p + entropy_t) ),
 *   dH = dz W,  dW (+)= dz^T H,      p = exp(s z - lse_t) recomputed tile by tile.
 *
 *   lse         device in  [T] fp32, spo_logprobs' output for the same H, W, inv_temperature
 *   entropy     device in  [T] fp32, its entropy; required with g_entropy, otherwise optional
 *   g_logp, g_lse, g_entropy   device in [T] fp32, each optional (NULL = zero); y is required with g_logp
 *   mask        rows with mask 0 have dH = 0 and add nothing to dW, whatever their H holds
 *   dH          device out [T][d];  dW  device out [V][d], overwritten or (dW_accumulate) added to.  Types:
 *               bf16 H / W: dH and dW bf16 or fp32 each; fp32 H / W: both fp32.  A bf16 dW is summed over all
 *               tokens in fp32 and rounded once.  For the products dz is rounded to bf16, but for the target's
 *               entry, by far the largest of its row, whose rounding is put back in fp32.
 *   ws          device scratch, spo_workspace_bytes(SPO_WS_LOGPROBS_BWD, T, d, V, 0, 0, 0) bytes: a chunk of dz (a few
 *               thousand rows by V, bf16; fp32 for fp32 inputs), never all of it; it serves shorter calls too
 * dH and dW share no memory with H, W or each other (SPO_ERR_INVALID_ARG).
 * A target outside [0,V) contributes nothing through g_logp and sets SPO_DEV_ID_OUT_OF_RANGE (unless masked).
 * A token whose logit is -inf has dz = 0 (but for a target's g_logp).
 * T = 0 zeroes dW (unless accumulating).
 */
int32_t spo_logprobs_bwd(const void* H, int64_t ldH, const void* W, int32_t dtype, const int32_t* y, const uint8_t* mask,
                         const float* lse, const float* entropy, const float* g_logp, const float* g_lse,
                         const float* g_entropy, int64_t T, int32_t d, int32_t V, float inv_temperature,
                         void* dH, int32_t dH_dtype, void* dW, int32_t dW_dtype, int32_t dW_accumulate,
                         void* ws, size_t ws_bytes, int32_t* d_status, void* stream);

/*
 * Orthogonalised (Muon) weight updates, the step that consumes a gradient such as the loss calls' dW
 * (Algorithm 1, "update the policy parameters"; the paper leaves the optimiser open).  For each m x n matrix U:
 *   X_0 = U / (|U|_F + eps);  `steps` times:  A = X X^T,  X <- coef_a X + (coef_b A + coef_c A A) X
 * which drives the singular values of U towards one while keeping its singular vectors (for m > n the same
 * polynomial through X^T X).  spo_muon_update puts momentum in front and the weights behind it:
 *   M <- momentum M + G;  U = G + momentum M (nesterov) or M;
 *   W <- (1 - lr weight_decay) W - lr scale X,  scale = 1 (SPO_MUON_SCALE_NONE), sqrt(max(1, m/n))
 *   (SPO_MUON_SCALE_SPECTRAL) or 0.2 sqrt(max(m, n)) (SPO_MUON_SCALE_RMS).
 * Iterates are kept in fp32; the products' operands are fp16 with fp32 sums, whatever the types of G, W and out: a result is off by
 * about 1e-3 of its norm (matrices of two or three rows: up to 4e-3).  The Frobenius norm is summed in fp64 in a fixed order, so
 * results repeat bit for bit.
 *
 *   G         device in  [batch][m][n], fp32 or bf16 (dtype)
 *   out       device out [batch][m][n], fp32 or bf16; may be G itself when the types agree
 *   W         device in/out [batch][m][n], fp32 or bf16;  momentum  device in/out [batch][m][n] fp32
 *   ws        device scratch, spo_workspace_bytes(SPO_WS_MUON, m, n, 0, 0, batch, 0) bytes
 * A matrix whose U holds a NaN or an infinity sets SPO_DEV_NONFINITE; its out is zero, its W and momentum are
 * left as they were (the other matrices of the batch are not affected).  A zero U gives X = 0, whatever eps.
 * The default coefficients keep every singular value of X below 1.3.  Others may let X grow past fp16 (65504), in which case
 * the result, or W, holds NaN or infinities: SPO_DEV_NONFINITE is set, and nothing is taken back.
 * Limits: 1 <= m, n < 2^24, min(m, n) <= 65536, 0 <= batch <= 65535.
 * The scratch is what takes memory: 8 bytes an element of the batch, and 6 for each element of a min(m, n) square (5.1 GB
 * for a vocabulary matrix of 151936 x 4096, beside W, momentum and G).
 * More than one tile of work is one cooperative launch of clusters, which Nsight Compute (2025.2) does not replay: a program
 * profiled with it does not get past such a call, so leave the call out of what is profiled.
 */
#define SPO_MUON_SCALE_NONE      0
#define SPO_MUON_SCALE_SPECTRAL  1
#define SPO_MUON_SCALE_RMS       2
typedef struct spo_muon_params {
  float   lr;             /* 0.02 */
  float   momentum;       /* 0.95, in [0, 1) */
  float   weight_decay;   /* 0 */
  float   eps;            /* 1e-7, > 0 */
  float   coef_a, coef_b, coef_c;   /* 3.4445, -4.7750, 2.0315 */
  int32_t steps;          /* 5, 1 .. 16 */
  int32_t nesterov;       /* 1 */
  int32_t scale_mode;     /* SPO_MUON_SCALE_SPECTRAL */
} spo_muon_params;
int32_t spo_default_muon_params(spo_muon_params* p /* host, out */);
int32_t spo_orthogonalize(const void* G, int32_t G_dtype, int32_t batch, int64_t m, int64_t n,
                          void* out, int32_t out_dtype, void* ws, size_t ws_bytes,
                          const spo_muon_params* params, int32_t* d_status, void* stream);
int32_t spo_muon_update(void* W, int32_t W_dtype, float* momentum, const void* G, int32_t G_dtype,
                        int32_t batch, int64_t m, int64_t n, void* ws, size_t ws_bytes,
                        const spo_muon_params* params, int32_t* d_status, void* stream);

/*
 * Layer norm and RMS norm of hidden states, the step that makes the H of the loss and log-probability calls (and, with dH, takes their
 * gradient back to the residual stream).  Per row t:
 *   h = x, or x + residual rounded to the type of x;   mu = mean_j h (SPO_NORM_LAYER) or 0 (SPO_NORM_RMS);
 *   rstd = 1 / sqrt( mean_j (h_j - mu)^2 + eps );      y_j = (h_j - mu) rstd weight_j + bias_j.
 * Statistics in fp32, the squares about the mean; y is rounded once.
 *
 *   x         device in  [T] rows of d elements, fp32 or bf16 (dtype), row pitch ldx >= d elements: rows of a wider buffer (the last-token
 *             rows of a padded batch, a slice of columns) need no copy where the first of them begins on 16 bytes, as every pointer of
 *             these two calls has to
 *   residual  device in  [T][d], type of x, optional;   h  device out [T][d], type of x: required with residual and only then.
 *             h may be x (ldx = d) or residual
 *   weight, bias   device in [d], fp32 or bf16 (w_dtype), each optional (NULL: 1 and 0)
 *   mask      device in  [T] uint8, optional: rows with mask 0 give y = h = mean = rstd = 0, whatever they hold (NaN included), and set
 *             no status bit
 *   eps       > 0
 *   y         device out [T][d], fp32 or bf16 (y_dtype); may be x (ldx = d) where the types agree and there is no residual
 *   mean      device out [T] fp32, optional, SPO_NORM_LAYER only;   rstd  device out [T] fp32, optional
 * A row whose mean square is not finite sets SPO_DEV_NONFINITE; its y is what the formula gives.
 * Any d up to SPO_NORM_MAX_D: rows that begin on 16 bytes (d and ldx multiples of 8 in bf16, of 4 in fp32) are read fastest.  T = 0 is
 * allowed and launches nothing.
 */
#define SPO_NORM_LAYER  0
#define SPO_NORM_RMS    1
#define SPO_NORM_MAX_D  1048576
int32_t spo_layernorm_fwd(const void* x, int64_t ldx, const void* residual, int32_t dtype, const void* weight, const void* bias,
                          int32_t w_dtype, const uint8_t* mask, int64_t T, int32_t d, float eps, int32_t kind,
                          void* y, int32_t y_dtype, void* h, float* mean, float* rstd, int32_t* d_status, void* stream);

/*
 * Gradients of spo_layernorm_fwd.  With xh = (h - mu) rstd and a_j = weight_j dy_j:
 *   dx = rstd ( a - mean_j a [SPO_NORM_LAYER] - xh mean_j(a xh) ) + dh,    dweight (+)= sum_t dy xh,    dbias (+)= sum_t dy.
 * dx is the gradient of h, so of x and of residual alike; dh is what reaches h past the norm (the residual stream).
 *
 *   dy        device in  [T][d], fp32 or bf16 (dy_dtype)
 *   x         device in  the rows that were normalised (x of the forward call, or its h), row pitch ldx, dtype
 *   mean, rstd   device in [T] fp32, the forward's (mean: SPO_NORM_LAYER only)
 *   dh        device in  [T][d], type of x, optional
 *   mask      rows with mask 0 give dx = 0 and add nothing to dweight and dbias, whatever they hold
 *   dx        device out [T][d], type of x; may be dy (where the types agree), dh or x (ldx = d)
 *   dweight, dbias   device out [d], fp32 or bf16 (dw_dtype), each optional; overwritten, or added to when dw_accumulate != 0.  Summed
 *             over all rows in fp32, in an order that depends on T, d, ldx, the types of dy and x, whether there is a dh, and the device: the
 *             same call repeats bit for bit, and calls that differ in one of these may round differently
 *   ws        device scratch, spo_workspace_bytes(SPO_WS_LAYERNORM_BWD, T, d, 0, 0, 0, 0) bytes; it serves shorter calls too.  Optional
 *             where neither dweight nor dbias is wanted
 * T = 0 zeroes dweight and dbias (unless accumulating).  The call sets no status bit: what is not finite goes where the formula takes it.
 */
int32_t spo_layernorm_bwd(const void* dy, int32_t dy_dtype, const void* x, int64_t ldx, int32_t dtype, const void* weight,
                          int32_t w_dtype, const uint8_t* mask, const float* mean, const float* rstd, const void* dh,
                          int64_t T, int32_t d, int32_t kind, void* dx, void* dweight, void* dbias, int32_t dw_dtype,
                          int32_t dw_accumulate, void* ws, size_t ws_bytes, int32_t* d_status, void* stream);

/*
 * Global norm of many gradients and the factor that clips them (Algorithm 1, "update the policy parameters"; the paper leaves the
 * optimiser open): with s = grad_scale (1 / loss scale; 1),
 *   norm = |s| sqrt( sum over all tensors and elements of g^2 ),   factor = s min(1, max_norm / norm)    (max_norm <= 0: factor = s).
 * Summed in fp64 in a fixed order: results repeat bit for bit, and are the exact norm and factor rounded once (up to a near tie).
 *
 *   grads   host in [n_grads], read before the call returns; each g is a device pointer to n elements (n = 0 is allowed), aligned
 *           to its element (16 bytes is fastest)
 *   out     device out [4] fp32 = (norm, factor, 1 if norm is finite else 0, 0).  factor is NaN where norm is not finite:
 *           spo_adamw_update then takes no step.  Such a norm sets SPO_DEV_NONFINITE
 *   ws      device scratch, spo_workspace_bytes(SPO_WS_GRAD_NORM, ...) bytes (the same for all calls); neither it nor out may lie in a
 *           gradient
 * Up to 1200 tensors are one launch (and one small one behind it).
 */
typedef struct spo_grad_tensor {
  const void* g;
  int64_t     n;
  int32_t     dtype;
  int32_t     reserved;
} spo_grad_tensor;
int32_t spo_grad_norm(const spo_grad_tensor* grads /* host */, int32_t n_grads, float max_norm, float grad_scale, float* out,
                      void* ws, size_t ws_bytes, int32_t* d_status, void* stream);

/*
 * One AdamW step over many tensors (the vocabulary matrix with the loss's dW, norms, biases: what spo_muon_update is not used on).
 * With t the number of this step, f = *d_scale, lr_k = lr lr_scale and decay_k = weight_decay decay_scale of the tensor, per element:
 *   g~ = f g;   m <- beta1 m + (1 - beta1) g~;   v <- beta2 v + (1 - beta2) g~^2;
 *   w <- w - lr_k ( (m / (1 - beta1^t)) / ( sqrt(v / (1 - beta2^t)) + eps ) + decay_k w );   copy <- w rounded to bf16.
 * m and v are formed by individually rounded fp32 operations (every product and sum above; 1 - beta rounded to fp32 first).  bf16
 * weights are rounded to nearest after each step: at small lr they need fp32 weights with a bf16 copy to move at all.
 *
 *   tensors    host in [n_tensors], read before the call returns.  Device pointers, aligned to their elements (16 bytes is fastest):
 *     w        in/out [n], fp32 or bf16 (w_dtype);   g  in [n], fp32 or bf16 (g_dtype);   copy  out [n] bf16, optional
 *     state_bits 32:  m, v  in/out [n] fp32;  m_scale = v_scale = NULL
 *     state_bits 8:   m  in/out [n] int8, v  in/out [n] uint8;  m_scale, v_scale  in/out [ceil(n / 256)] fp32.  Elements 256 i ..
 *              256 i + 255 share scale i:  m = s sgn(c) (c/127)^2,  v = s (c/255)^4.  The new scale is the largest new magnitude of the
 *              block (at least 2^-100 for m, 2^-90 for v); a new code is the number of borders (j - 1/2)^2, j = 1 .. 127 (v: (j - 1/2)^4,
 *              j = 1 .. 255, as fp32), at or below the magnitude times the fp32 quotient 127^2 / s (255^4 / s); v > 0 takes code 1 at
 *              least.  Zeroed codes and scales are the start.  The update of w uses m and v before they are rounded to codes
 *     lr_scale, decay_scale   1 for the call's own
 *   No two tensors may share memory that is written, nor a gradient with what is written: the caller's to see to (the list of the Python
 *   binding checks it once).  d_scale, d_lr and d_step lie in no tensor that is written, d_step in no gradient, d_scale or d_lr:
 *   SPO_ERR_INVALID_ARG
 *   d_scale    device in [1] fp32, optional (1): spo_grad_norm's out + 1
 *   d_lr       device in [1] fp32, optional: replaces params->lr (a captured step whose rate changes)
 *   d_step     device in/out [2] int32 (steps taken, 0), optional: t is one more than d_step[0], and the call leaves it so (calls
 *              that share it run one after the other).  NULL: t = params->step
 * An element whose g~ is not finite or above 2^60 in magnitude keeps its w, m and v (in 8 bits up to the rounding to the block's new scale)
 * and sets SPO_DEV_NONFINITE.  A factor or rate that is not finite sets it too, and then the step is neither taken nor counted; so does a rate
 * that, times the largest lr_scale of the call and the largest decay_k above one, is beyond 2^100 in magnitude.
 * Up to 400 tensors are one launch.  Tensors without elements are allowed; a call without any launches nothing and counts no step.
 */
#define SPO_ADAMW_BLOCK 256
typedef struct spo_adamw_tensor {
  void*       w;
  const void* g;
  void*       m;
  void*       v;
  float*      m_scale;
  float*      v_scale;
  void*       copy;
  int64_t     n;
  int32_t     w_dtype;
  int32_t     g_dtype;
  int32_t     state_bits;   /* 8 or 32 */
  float       lr_scale;
  float       decay_scale;
  int32_t     reserved;
} spo_adamw_tensor;
typedef struct spo_adamw_params {
  float   lr;             /* 1e-6 */
  float   beta1;          /* 0.9, in [0, 1) */
  float   beta2;          /* 0.999, in [0, 1) */
  float   eps;            /* 1e-8, at least 2^-100 */
  float   weight_decay;   /* 0 */
  int32_t step;           /* 1, >= 1: the step that is taken, where d_step is NULL */
} spo_adamw_params;
int32_t spo_default_adamw_params(spo_adamw_params* p /* host, out */);
int32_t spo_adamw_update(const spo_adamw_tensor* tensors /* host */, int32_t n_tensors, const float* d_scale, const float* d_lr,
                         int32_t* d_step, const spo_adamw_params* params, int32_t* d_status, void* stream);

/*
 * Values of 8-bit states, for inspection or for going on in 32 bits: m_out[i], v_out[i] fp32 from the codes and scales of
 * spo_adamw_update.  m with m_scale and m_out, or v with v_scale and v_out, may be NULL together.  The outputs share memory with nothing.
 */
int32_t spo_adamw_decode(const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale, int64_t n,
                         float* m_out, float* v_out, void* stream);

/* Scratch size in bytes for one call of the selected entry point (host only, no CUDA call
 * except a device-property query).  Arguments that the selected call does not use are ignored. */
size_t spo_workspace_bytes(int32_t which, int64_t T, int32_t d, int32_t V,
                           int64_t N, int32_t B, int32_t M);

const char* spo_status_string(int32_t status);
int32_t     spo_last_cuda_error(void);   /* cudaError_t of the last SPO_ERR_CUDA on this thread */
int32_t     spo_version(void);

#ifdef __cplusplus
}
#endif
#endif  /* SPO_H_ */

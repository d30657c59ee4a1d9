/*
 * termezo.h -- C ABI of the MI355X (gfx950) TerMeZO sparse zeroth-order step.
 *
 * TerMeZO (Sec. 3 and Algorithm 1 of the paper) fine-tunes the latent weights
 * w of a BitNet model's ternary linear projections with two-point SPSA
 * (eq. spsa), perturbing and updating only a mask of latents that lie close
 * to the ternary quantiser's decision boundaries (eq. distance,
 * eq. selection_init, eq. selection_).  This library holds the hot path of one
 * step on one GPU: mask construction, seed-regenerated perturbation with
 * absmean requantisation, BitLinear forward (per-token absmax int8 activations
 * x ternary weights, int32 accumulation, rescale) and the masked update.
 *
 * Conventions shared by every call
 *   - All functions return a termezo_status; no C++ exception crosses the ABI.
 *     A call that fails validation changes no state; termezo_last_error()
 *     returns a message for the last failure on a context.
 *   - A context is not thread-safe.  All device work is ordered on the HIP
 *     stream given at creation.  Only the calls that return host values
 *     (build_mask, update with k_out, mse_loss, model_loss, sync and the
 *     exports) wait for the stream; they also report a deferred error
 *     raised by an earlier kernel on that context (NUMERIC, or INVALID_ARG for
 *     a token id out of range).
 *   - Device pointers are plain device addresses of memory owned by the
 *     caller (for example PyTorch tensors); host pointers are noted as such.
 *   - Latent weights are BORROWED: the caller owns them and they must outlive
 *     the context.  The library writes them only in termezo_update, and only
 *     at the active indices.
 *   - Global ids: layers are enumerated in registration order; inside a layer
 *     the latent matrix is row-major [d_out][d_in]; gid = (sum of the sizes
 *     of the earlier layers) + row * d_in + col.
 *   - Gaussian directions z are regenerated from the 64-bit seed with
 *     Philox4x32-10 (counter = (gid >> 2, stream 0)) and the Box-Muller
 *     transform; they are never stored.
 */
#ifndef TERMEZO_H_
#define TERMEZO_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TERMEZO_OK = 0,
  TERMEZO_ERR_INVALID_ARG = 1, /* bad argument; nothing was done            */
  TERMEZO_ERR_STATE = 2,       /* call not valid in the current state       */
  TERMEZO_ERR_DEVICE = 3,      /* no usable HIP device / HIP runtime error  */
  TERMEZO_ERR_OOM = 4,         /* device allocation failed                  */
  TERMEZO_ERR_NUMERIC = 5      /* non-finite value or |w| >= 4 in a latent  */
} termezo_status;

typedef enum {
  TERMEZO_F32 = 0,
  TERMEZO_BF16 = 1,
  TERMEZO_I8 = 2,
  TERMEZO_I32 = 3
} termezo_dtype;

/* One ternary linear projection (Sec. 3: q, k, v, o and every MLP linear).
 * latent: device pointer to d_out * d_in latent weights, row-major, 16-byte
 * aligned, of the context's latent dtype.  d_in must be a multiple of 16 and
 * d_out * d_in must not exceed 2^25 (the fixed-point |w| sum stays exact). */
typedef struct {
  void* latent;
  int64_t d_out;
  int64_t d_in;
} termezo_layer;

typedef struct termezo_ctx termezo_ctx;

/* Register the latent weights of n_layers projections (latent_dtype F32 or
 * BF16) and allocate the library-owned state: packed 2-bit ternary codes
 * (d_out * d_in / 4 bytes per layer), per-layer thresholds and fixed-point
 * sums, and mask storage.  hip_stream: a hipStream_t (NULL = default stream).
 * At most 2048 layers per context; each layer at most 2^25 weights.
 * Errors: INVALID_ARG (null pointers, n_layers <= 0 or > 2048, d_in % 16 != 0,
 * misaligned latent, layer too large, bad dtype), DEVICE, OOM. */
termezo_status termezo_create(const termezo_layer* layers, int32_t n_layers,
                              termezo_dtype latent_dtype, void* hip_stream,
                              termezo_ctx** out);

/* Free every library-owned buffer.  Never frees the latents.  NULL is a no-op. */
void termezo_destroy(termezo_ctx* ctx);

/* Message describing the last failure on ctx ("" if none).  Owned by ctx. */
const char* termezo_last_error(const termezo_ctx* ctx);

/* Initial mask (Sec. 3, eq. distance and eq. selection_init; the initial
 * threshold and selection of Algorithm 1).  Computes tau^l = 0.5 (mean|w^l| + delta) per layer,
 * the distance d_i = min(|w_i - tau|, |w_i + tau|) of every latent, the global
 * budget k0 = floor(rho0 * D) and xi0, the k0-th smallest distance over all
 * layers (ties at xi0 broken by ascending gid; tie_inclusive != 0 keeps every
 * distance <= xi0 instead).  Also sets the current codes to Q(w) (clean).
 * k0_out, xi0_out: host pointers (nullable) receiving the mask size and xi0.
 * Waits for the stream.  Rebuilding discards the previous mask.
 * Errors: INVALID_ARG (rho0 not in (0, 1], delta <= 0 or not finite),
 * STATE (k0 == 0), NUMERIC (a latent non-finite or |w| >= 4). */
termezo_status termezo_build_mask(termezo_ctx* ctx, float rho0, float delta,
                                  int32_t tie_inclusive, int64_t* k0_out,
                                  float* xi0_out);

/* Perturbed evaluation point (Algorithm 1: w +/- eps m (.) z).  Sets the
 * current ternary codes and scales of every layer to the requantisation of
 * w' = w + sign * eps * m (.) z(seed): w'_i = fma(sign * eps, z_i, w_i) on the
 * active set, w'_i = w_i elsewhere; tau' and beta' = 2 tau' are recomputed from
 * w' (the quantiser is applied on the fly to the perturbed latents, eq.
 * objective).  The latents themselves are not modified.  sign = 0 gives the
 * clean codes.  Registered theta tensors are perturbed too (see the theta
 * section below).  Records (seed, eps) for the following termezo_update.
 * Perturbation pairs: the first call with a (seed, eps) and sign +-1 also forms
 * the perturbed values of the other sign (list order, 4 bytes per active latent
 * of library memory; z itself is never stored); a following call with the same
 * seed and eps and either sign reuses them.  Any other seed or eps, sign 0, an
 * update or a mask rebuild starts afresh; the caller must not write the latents
 * in between (they are borrowed).
 * Errors: INVALID_ARG (sign not in {-1, 0, 1}; eps <= 0 or not finite),
 * STATE (no mask).  A perturbed |w'| >= 4 raises a deferred NUMERIC. */
termezo_status termezo_perturb(termezo_ctx* ctx, uint64_t seed, float eps,
                               int32_t sign);

/* Requantisation strategy of termezo_perturb (the codes are the same either way).
 * By default a perturbation rewrites only the codes of the active latents while
 * no frozen code can change: every frozen latent is tracked to lie at least a
 * bound m^l (exactly, from xi0 and the threshold drift) from the threshold its
 * code was computed with, and a layer whose perturbed threshold tau' moves by
 * less than m^l keeps its frozen codes (the actives' codes are rewritten one by
 * one, or, above 1/256 active, tile by tile over the code words); other layers
 * are requantised densely.
 * always_dense != 0 requantises every latent of every layer on each call
 * (for measurement).  Errors: INVALID_ARG (null ctx). */
termezo_status termezo_set_dense_requant(termezo_ctx* ctx, int32_t always_dense);

/* BitLinear forward of one projection on its current codes (Sec. 1 and 3:
 * ternary weights with 8-bit activations).  x: device [M][d_in] (F32 or BF16);
 * y: device [M][d_out] (F32 or BF16).  Per token row m: a_m = max_k |x[m][k]|,
 * s_m = 127 / max(a_m, 1e-5), x_q = clamp(round_half_even(x * s_m), -128, 127);
 * acc[m][n] = sum_k x_q[m][k] * c[n][k] exactly in int32;
 * y[m][n] = float(acc) * (beta' / s_m) (rounded to bf16 if y is BF16).
 * y may share memory with x: every row is quantised before y is written.
 * The call allocates scratch when M or M * d_in exceeds every earlier call's of the context, and not
 * otherwise: after one call of the largest size the smaller ones can be captured in a graph.
 * xq_out [M][d_in] int8, xscale_out [M] fp32 (s_m), acc_out [M][d_out] int32:
 * optional device outputs (nullable) for inspection.
 * Errors: INVALID_ARG (layer out of range, M <= 0, bad dtype, null x or y),
 * STATE (no current codes: before build_mask or after update). */
termezo_status termezo_bitlinear_forward(termezo_ctx* ctx, int32_t layer,
                                         const void* x, termezo_dtype x_dtype,
                                         int64_t M, void* y, termezo_dtype y_dtype,
                                         int8_t* xq_out, float* xscale_out,
                                         int32_t* acc_out);

/* For callers that cannot allocate device memory (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation): the same BitLinear
 * forward as termezo_bitlinear_forward (same kernels, same results) without the
 * inspection outputs, whose activation-quantisation scratch (int8 x_q, the
 * per-token scales and the per-token sums of x_q) lives in a fixed 16 MiB device
 * array inside the library instead of context buffers grown on demand.  The call
 * allocates nothing.  Limit: M * d_in bytes rounded up to 256, plus 4 * M rounded
 * up to 256, plus 4 * M, at most 16 MiB (for example M <= 6533 at d_in = 2560,
 * M <= 2424 at d_in = 6912).  Each GPU holds
 * one copy of the array, shared by every context and call on that GPU: calls
 * whose work overlaps on one GPU (different streams, or different host
 * threads) race on it; calls ordered on one stream do not.  Nothing in the
 * array needs to start at zero.  Errors: as termezo_bitlinear_forward, and
 * INVALID_ARG when M exceeds the limit; DEVICE if the array's address could
 * not be obtained at context creation. */
termezo_status termezo_bitlinear_forward_noalloc(termezo_ctx* ctx, int32_t layer, const void* x,
                                                 termezo_dtype x_dtype, int64_t M, void* y,
                                                 termezo_dtype y_dtype);

/* Masked projected-gradient update (Algorithm 1, last loop, K = 1) followed by
 * the shrink-only set update (eq. selection_).  With the seed of the last
 * termezo_perturb: for every active i, w_i <- round(fma(-(lr * g), z_i, w_i))
 * (round = to nearest-even bf16 for BF16 latents, identity for F32); unmasked
 * latents are untouched.  Then tau^l is recomputed from the updated latents and
 * the active set keeps only the i with d_i <= xi0 (order preserved).
 * Registered theta tensors are updated with the same g (theta section below).
 * proj_grad is g = (F+ - F-) / (2 eps) (eq. spsa).  k_out: host pointer
 * (nullable) receiving the new mask size; when non-NULL the call waits.
 * Invalidates the current codes.  Errors: INVALID_ARG (g or lr not finite),
 * STATE (no perturbation since the last update or mask build). */
termezo_status termezo_update(termezo_ctx* ctx, float proj_grad, float lr,
                              int64_t* k_out);

/* Device-side projected gradient and update (Algorithm 1: g = (F+ - F-) / (2 eps),
 * then the same update and shrink as termezo_update) without a host round
 * trip: loss_plus and loss_minus are device fp32 scalars (for example written
 * by termezo_model_loss).  g is formed in fp32 on the device as
 * (F+ - F-) / (2 eps).  A non-finite g skips the latent update and raises a
 * deferred NUMERIC.  Never waits.  Errors: INVALID_ARG (null pointers, eps or
 * lr not positive/finite), STATE as for termezo_update. */
termezo_status termezo_update_from_losses(termezo_ctx* ctx, const float* loss_plus,
                                          const float* loss_minus, float eps, float lr);

/* ---- memory-optimal storage (Sec. 5 eq. memory: frozen weights as 2-bit codes) ----
 * After the mask is built, termezo_compact copies the active latents into a
 * library-owned array in list order; from then on the context never reads or
 * writes the caller's latent tensors (they may be freed).  Frozen latents live
 * on only as their ternary codes.  Perturbation, update and shrink work on the
 * compact array (contiguous instead of scattered accesses).  The codes are
 * those of the dense semantics while every layer's threshold stays within its
 * frozen margin (see termezo_set_dense_requant); if a perturbed threshold ever
 * moves farther, the frozen codes are kept and a deferred NUMERIC error names
 * the condition.  termezo_build_mask then fails with STATE (it needs the full
 * latents).  Errors: STATE (no mask, already compact, pending perturbation),
 * OOM.  Waits for the stream. */
termezo_status termezo_compact(termezo_ctx* ctx);

/* Values (fp32, host) of one layer's active latents in list order (ascending
 * local index); *n receives the count.  Works with and without compact mode.
 * Errors: INVALID_ARG (layer, null n, cap below the count), STATE (no mask).
 * Waits for the stream. */
termezo_status termezo_active_values(termezo_ctx* ctx, int32_t layer, float* values,
                                     int64_t cap, int64_t* n);

/* Device memory of the method's state (host values, nullable): library_bytes =
 * the library-owned buffers (codes, mask lists, thresholds, tile tables, the
 * list-order copy of the active latents -- kept for sets of at most 1/8 of the
 * latents and in compact mode --, theta copies, the codes snapshot once taken,
 * scratch); latent_bytes = the caller's latent tensors the context still needs
 * (0 in compact mode). */
termezo_status termezo_memory_footprint(termezo_ctx* ctx, int64_t* library_bytes,
                                        int64_t* latent_bytes);

/* K perturbation directions per step (Algorithm 1: the K two-point estimates
 * are all taken at w_t, then the K updates are applied).  After the caller has
 * evaluated F+_k and F-_k for every seed s_k (termezo_perturb(s_k, eps, +1),
 * loss, termezo_perturb(s_k, eps, -1), loss), one call applies, at every active
 * latent (and every registered theta value),
 *   v = fma(a_K, z_K, ... fma(a_1, z_1, w) ...) in fp32,  w <- round(v),
 * with a_k = -((lr / K) * g_k) in fp32 and z_k regenerated from s_k, then the
 * shrink of termezo_update.  With fp32 storage this equals the K updates of
 * Algorithm 1 applied one after another; with bf16 storage the sum is rounded
 * once.  seeds, proj_grads: host arrays of K entries, 1 <= K <= 32.
 * k_out as for termezo_update.  Errors: INVALID_ARG (K out of range, null
 * arrays, non-finite g or lr), STATE (no perturbation since the last update). */
termezo_status termezo_update_multi(termezo_ctx* ctx, const uint64_t* seeds,
                                    const float* proj_grads, int32_t K, float lr,
                                    int64_t* k_out);

/* The same with the projected gradients formed on the device from the losses
 * (device fp32 [2K]: F+_1, F-_1, F+_2, F-_2, ...): g_k = (F+_k - F-_k) / (2 eps)
 * in fp32; seeds is a host array.  Never waits.  A non-finite g_k skips the
 * update and raises a deferred NUMERIC.  Errors as above (eps must be > 0). */
termezo_status termezo_update_multi_from_losses(termezo_ctx* ctx, const uint64_t* seeds,
                                                const float* losses, int32_t K, float eps,
                                                float lr);

/* ---- evolution strategies on the mask (appendix on RL-based fine-tuning) -------
 * The RL variant evaluates N one-sided perturbations w + sigma m (.) z_n
 * (termezo_perturb(s_n, sigma, +1), then the caller's reward R_n) and updates
 * with the reward-weighted sum of the directions, restricted to the mask:
 *   v = fma(a_N, z_N, ... fma(a_1, z_1, w) ...) in fp32,  w <- round(v),
 * a_n = (lr / N) * Rt_n in fp32 (lr / N one fp32 division), at every active
 * latent (and every registered theta value, stream 1), then the shrink of
 * termezo_update.  standardize != 0: Rt_n = fp32((R_n - mu) / sd) with mu and
 * the population deviation sd computed in fp64 in index order (all Rt zero when
 * sd = 0, so N = 1 or equal rewards leave the weights unchanged); standardize
 * = 0: Rt_n = R_n.  seeds: host array of N entries, 1 <= N <= 32.  A negative
 * lr descends instead of ascends (rewards = losses).
 * Errors: INVALID_ARG (N out of range, null arrays, non-finite reward, lr or
 * coefficient), STATE (no perturbation since the last update). */
termezo_status termezo_es_update(termezo_ctx* ctx, const uint64_t* seeds, const float* rewards,
                                 int32_t N, float lr, int32_t standardize, int64_t* k_out);

/* The same with the rewards in device memory (fp32 [N]); never waits.  A
 * non-finite coefficient skips the update and raises a deferred NUMERIC. */
termezo_status termezo_es_update_from_rewards(termezo_ctx* ctx, const uint64_t* seeds,
                                              const float* rewards, int32_t N, float lr,
                                              int32_t standardize);

/* ---- full-precision parameters theta (Sec. 3; Algorithm 1) ---------------------
 * Algorithm 1 perturbs and updates the full-precision parameters (embeddings,
 * normalisation weights, LM head) densely, together with the masked latents,
 * with directions drawn from the same seed.  Registering theta switches this on;
 * without registration theta is frozen.
 *   - theta ids: the registered tensors are enumerated in registration order,
 *     each flat; id = (sum of the sizes of the earlier tensors) + index.
 *     z_theta(id) is drawn like z (Philox4x32-10 + Box-Muller, same seed) on
 *     counter stream 1: counter = (id >> 2, stream 1).
 *   - termezo_perturb(seed, eps, sign != 0) makes the forward read
 *     theta' = round(fma(sign * eps, z_theta, theta)) (round = to nearest-even
 *     bf16 for BF16 tensors, identity for F32), held in library-owned copies;
 *     theta itself is not modified.  Both signs of a (seed, eps) pair are
 *     produced by the first of the two calls; sign = 0 reads theta itself.
 *   - termezo_update / termezo_update_from_losses apply, after the latent
 *     update, theta <- round(fma(-(lr * g), z_theta, theta)) in place (a
 *     non-finite g leaves theta untouched), and the forward reads theta again.
 * The tensors are BORROWED (caller-owned device memory that must outlive the
 * context); the caller must not write them while a perturbation is pending. */
typedef struct {
  void* data;              /* device pointer, 16-byte aligned                 */
  int64_t n;               /* number of elements                              */
  termezo_dtype dtype;     /* F32 or BF16                                     */
} termezo_theta;

/* Register n tensors as theta (once per context).  Allocates two copies of each
 * (the +eps and -eps values).  Errors: INVALID_ARG (null or misaligned data,
 * n <= 0, bad dtype), STATE (already registered), OOM. */
termezo_status termezo_theta_register(termezo_ctx* ctx, const termezo_theta* params,
                                      int32_t n);

/* *values receives the device pointer the forward pass must read for tensor i
 * now: the perturbed copy after termezo_perturb with sign +1 or -1, else the
 * caller's tensor.  Errors: INVALID_ARG (i out of range, null values). */
termezo_status termezo_theta_current(termezo_ctx* ctx, int32_t i, void** values);

/* Copy (device to device, ordered on the context's stream, no wait) the values
 * termezo_theta_current points to for tensor i into the caller's device buffer
 * dst (n elements of the tensor's dtype).  Inspection support.
 * Errors: INVALID_ARG (i out of range, null dst), DEVICE. */
termezo_status termezo_theta_copy(termezo_ctx* ctx, int32_t i, void* dst);

/* ---- BitNet decoder around the registered projections (Sec. 3) ----------------
 * The context's layers must be the ternary projections of n_blocks decoder
 * blocks in the order q, k, v, o, gate, up, down (shapes [n_heads*hd][d],
 * [n_kv_heads*hd][d] twice, [d][n_heads*hd], [d_ffn][d] twice, [d][d_ffn],
 * hd = d_model / n_heads).  The full-precision parameters are the token
 * embedding (tied to the LM head), the caller's device matrix [vocab][d_model]
 * in act_dtype, and the RMSNorm weights (one unless set with
 * termezo_model_set_norm_weights).  Either may be a registered theta tensor;
 * the forward then reads its current values.  Blocks are pre-norm:
 * h += o(attn(rope(q(x)), rope(k(x)), v(x))), x = rmsnorm(h); then
 * h += down(silu(gate(x)) * up(x)).  Attention is causal grouped-query with
 * scale 1/sqrt(hd); rotary pairs are (i, i + hd/2) with angle
 * p * rope_base^(-2i/hd).  Activations are stored in act_dtype between kernels;
 * BitLinear inputs are quantised per token as in termezo_bitlinear_forward. */
typedef struct {
  int32_t n_blocks, d_model, n_heads, n_kv_heads, d_ffn, vocab;
  float rope_base;          /* e.g. 10000 */
  float norm_eps;           /* e.g. 1e-5  */
  termezo_dtype act_dtype;  /* F32 or BF16 */
} termezo_model_config;

typedef struct termezo_model termezo_model;

/* Bind a decoder to ctx (which must outlive it).  embedding: device pointer,
 * 16-byte aligned, borrowed.  Errors: INVALID_ARG (shapes do not match the
 * registered layers, unsupported head_dim for BF16 (64, 96, 128), d_model or
 * d_ffn above 8192, bad dtype). */
termezo_status termezo_model_create(termezo_ctx* ctx, const termezo_model_config* cfg,
                                    const void* embedding, termezo_model** out);
/* RMSNorm weights of the model: norm_weights is a device [2 n_blocks + 1][d_model]
 * array in act_dtype, 16-byte aligned, borrowed (row 2 b scales the attention
 * input of block b, row 2 b + 1 its MLP input, the last row the LM-head input);
 * NULL restores weights one.  Errors: INVALID_ARG (misaligned pointer). */
termezo_status termezo_model_set_norm_weights(termezo_model* model, const void* norm_weights);

/* Free the model's activation buffers (it does not touch the context, which
 * may already have been destroyed).  NULL is a no-op. */
void termezo_model_destroy(termezo_model* model);

/* Batch loss of eq. objective_est with next-token cross-entropy: the mean over
 * the batch * (seq - 1) labelled positions of logsumexp(logits) - logit[next
 * token], with the current codes (clean or perturbed).  tokens: device int32
 * [batch][seq]; every id must lie in [0, vocab).  Outputs (all optional):
 * loss_dev (device fp32 scalar), row_loss_dev (device fp32 [batch*seq], 0 at
 * each sequence's last position), loss_host (host; the call then waits and
 * reports deferred errors).  An id outside [0, vocab) is read as id 0 (the
 * embedding is never read out of bounds) and raises a deferred INVALID_ARG,
 * reported by this call when loss_host is given, else by the next waiting
 * call (termezo_sync, ...); the losses of that call are then meaningless.
 * Errors: INVALID_ARG, STATE (no current codes), OOM. */
termezo_status termezo_model_loss(termezo_model* model, const int32_t* tokens, int32_t batch,
                                  int32_t seq, float* loss_dev, float* row_loss_dev,
                                  float* loss_host);

/* The two evaluations of a perturbation pair, F(w + eps z) and F(w - eps z) on the
 * same batch (Algorithm 1), depend on nothing but the pair's codes, so they may run
 * at the same time.  termezo_codes_snapshot copies the current codes and output
 * scales (those of the last termezo_perturb) into a library-owned buffer (allocated
 * on the first call: 4 bytes per 16 latents plus 4 per layer), stream-ordered on the
 * context's stream; a model set to read the snapshot (termezo_model_use_snapshot)
 * evaluates that perturbation while the next termezo_perturb rewrites the current
 * codes.  termezo_model_set_stream runs a model's forwards on a stream of the
 * caller's (NULL: the context's stream, the default): each termezo_model_loss then
 * starts after the work queued on the context's stream, and termezo_model_join
 * makes the context's stream wait for the model's work before anything queued after
 * it (the update that reads the losses).  A snapshot stays valid until the next
 * snapshot; the caller orders a snapshot after the forwards that read the previous
 * one (a join does).  Errors: INVALID_ARG (null), STATE (no current codes; a
 * snapshot model before any snapshot), OOM, DEVICE. */
termezo_status termezo_codes_snapshot(termezo_ctx* ctx);
termezo_status termezo_model_set_stream(termezo_model* model, void* hip_stream);
termezo_status termezo_model_use_snapshot(termezo_model* model, int32_t on);
termezo_status termezo_model_join(termezo_model* model);

/* Event timing of the model's matrix-core kernels, for measurement: with
 * enable != 0 every following termezo_model_loss records a HIP event pair on
 * the context's stream for each launch of class 0 (BitLinear int8 GEMM) and 2
 * (LM head with cross-entropy partials), whose events take the kernel's own
 * start and end (hipExtLaunchKernel), and around each launch pair of class 1
 * (attention: K/V preparation, then the attention kernel); enabling or
 * disabling clears the records.  termezo_model_timing waits for the stream and
 * returns, for one class, the summed kernel time in ms, the number of launches
 * and their algorithmic operation count (2 M K N per GEMM; 4 B H hd S(S+1)/2
 * for causal attention; 2 M d V for the LM head). */
termezo_status termezo_model_set_timing(termezo_model* model, int32_t enable);
termezo_status termezo_model_timing(termezo_model* model, int32_t cls, double* ms,
                                    int64_t* launches, double* ops);

/* ---- generation: 8-bit cache, attention over it, logits, beam selection ----------
 * The calls that a decoder needs to generate tokens with the current codes (the
 * rewards of the evolution-strategies variant are those of generated text).  They
 * return as soon as their work is queued on the context's stream and may be called
 * while another device is current.  Creating a cache allocates all that its calls need;
 * termezo_beam_select and termezo_model_decode allocate when a call needs more scratch
 * than every earlier one, so that after one of their size they can be captured in
 * graphs, as the other calls here can at once (a captured call that would have to allocate is
 * refused: STATE).  Graphs stay valid when a later call takes more: what they use is kept until the
 * context, model or cache is destroyed.  Work of one context or cache is ordered on
 * one stream: graphs of its calls must not run at the same time.
 *
 * A cache holds the keys and values of groups * beams sequences of up to max_len
 * tokens for n_layers attention layers.  The sequences of a group (the beams of a
 * search) have the same length.  Tokens are held in blocks of 64:
 *   - a complete block of a head holds 8-bit codes q = rne(x * s), s = 127 * (1 / a),
 *     and the step d = a * (1 / 127) (fp32, each operation rounded), a = max(max |x|,
 *     1e-30) over its 64 * head_dim values, keys and values apart; the cached value is
 *     q * d.  A block with a non-finite value has the step NaN;
 *   - the tokens of the incomplete last block are held in act_dtype.
 * So every value is rounded to 8 bits once, and what a cache holds does not depend
 * on how its tokens were split into calls.  With rope_base > 0 keys and queries are
 * given unrotated: pairs (i, i + head_dim / 2) are turned by
 * position * rope_base^(-2i/head_dim) (angles in fp64, cosine and sine in fp32) and
 * keys rounded to act_dtype; rope_base = 0 stores them as they are. */
typedef struct {
  int32_t n_layers, n_heads, n_kv_heads, head_dim;  /* head_dim 64, 96 or 128       */
  int32_t groups, beams;            /* beams: 1 to 64 sequences per group            */
  int64_t max_len;                  /* tokens per sequence, at most 2^24             */
  float rope_base;                  /* e.g. 10000; 0: no rotation                    */
  termezo_dtype act_dtype;          /* F32 or BF16: q, k, v and out                  */
} termezo_kvcache_config;

typedef struct termezo_kvcache termezo_kvcache;

/* Allocate a cache on ctx's device, empty.  Its calls run on ctx's stream; it must be
 * destroyed before ctx.  Errors: INVALID_ARG (sizes not positive, n_heads no multiple
 * of n_kv_heads, head_dim, beams, max_len, dtype, rope_base negative or not finite or
 * in (0, 1], more than 2^31 - 1 pages or more than 65535 rows or layers), DEVICE, OOM. */
termezo_status termezo_kvcache_create(termezo_ctx* ctx, const termezo_kvcache_config* cfg,
                                      termezo_kvcache** out);
/* Waits for the stream and frees the cache.  NULL is a no-op. */
void termezo_kvcache_destroy(termezo_kvcache* cache);

/* Empty one group (group >= 0; its sequences in use stay in use), or all of them (-1), which
 * also makes the first beam of every group the only one in use again.  Errors: INVALID_ARG (group out of range). */
termezo_status termezo_kvcache_reset(termezo_kvcache* cache, int32_t group);

/* Sequences in use: row r is sequence r.  After creation and a reset of all groups
 * only the first beam of each group is in use (rows = groups), so a prompt is taken
 * once per search; termezo_kvcache_fork gives every beam what the first one holds
 * (rows = groups * beams, beams of a group next to each other).  Complete blocks are
 * shared, not copied.  Errors: STATE (appended tokens not advanced; already forked;
 * beams = 1 never needs it). */
termezo_status termezo_kvcache_fork(termezo_kvcache* cache);

/* Append counts[g] tokens (device int32 [groups], each 0 .. n; NULL: n) to every
 * sequence of group g in one layer.  k, v: [rows][n][n_kv_heads][head_dim] in act_dtype;
 * the rows' tokens from counts[g] on are not read.  The tokens are pending: attention
 * and read see them, but the lengths stay until termezo_kvcache_advance (so that every
 * layer appends at the same place); appending again before that replaces them.
 * Counts outside 0 .. n and tokens past max_len raise a deferred INVALID_ARG and
 * append nothing to their group.  Errors: INVALID_ARG (layer out of range, n <= 0 or
 * > max_len, null or misaligned (16 bytes) pointers). */
termezo_status termezo_kvcache_append(termezo_kvcache* cache, int32_t layer, const void* k,
                                      const void* v, int64_t n, const int32_t* counts);

/* Causal attention of the pending tokens over the cache and themselves: query i of
 * a row (at position length + i) sees positions 0 .. length + i;
 * out = sum_t softmax_t(q . k_t / sqrt(head_dim)) v_t, head h reading key/value head
 * h / (n_heads / n_kv_heads).  q, out: [rows][n][n_heads][head_dim] in act_dtype; rows'
 * queries from the pending count on are neither read nor written.  k and v, both or
 * neither: when given, they are appended first (termezo_kvcache_append), for one token
 * a row and up to 32 heads a key/value head in the same launch.  counts: as in append; without k and v it may be NULL (the
 * pending counts), and counts that differ from the pending ones, as pending counts above n,
 * raise a deferred INVALID_ARG and leave their group's rows out.  A cached key or value
 * that is not finite makes the whole output (of its heads) NaN for every query that sees its
 * block, once that is complete, or its token, before; queries that do not are as without it.
 * A query that is not finite has NaN for its own output.
 * Blocks whose largest value is below 2^-80 of another's of the row may count as zeros in out (their weights
 * count in full).
 * out must not overlap q, k or v.  Errors: INVALID_ARG (as append; one of k, v null), STATE (k and v null and
 * nothing pending). */
termezo_status termezo_kvcache_attention(termezo_kvcache* cache, int32_t layer, const void* q,
                                         const void* k, const void* v, int64_t n,
                                         const int32_t* counts, void* out);

/* The pending tokens become part of the sequences.  Errors: STATE (nothing pending). */
termezo_status termezo_kvcache_advance(termezo_kvcache* cache);

/* Beam reordering: sequence b of group g continues what sequence parents[g * beams + b]
 * of the same group held (device int32 [groups * beams], 0 .. beams - 1 each; any other
 * value raises a deferred INVALID_ARG and keeps its sequence).  Complete blocks are
 * shared; of the tokens behind them only those of a parent's second and further
 * children are copied.  Errors: INVALID_ARG (null), STATE (pending tokens; not forked). */
termezo_status termezo_kvcache_reorder(termezo_kvcache* cache, const int32_t* parents);

/* Values of positions first .. first + n - 1 of every row of one layer, pending tokens
 * among them: k_out, v_out (nullable) [rows][n][n_kv_heads][head_dim] in dtype (F32: the
 * cached values exactly; BF16: rounded).  Positions behind a row's last token are not
 * written.  Errors: INVALID_ARG (layer, first < 0, n <= 0, first + n > max_len, dtype,
 * misaligned). */
termezo_status termezo_kvcache_read(termezo_kvcache* cache, int32_t layer, int64_t first, int64_t n,
                                    void* k_out, void* v_out, termezo_dtype dtype);

/* Host copy of the groups' lengths (without pending tokens).  Waits for the stream and
 * reports deferred errors.  Errors: INVALID_ARG (null). */
termezo_status termezo_kvcache_lengths(termezo_kvcache* cache, int32_t* lengths);

/* Logits of M rows of hidden states over the (tied) embedding: logits[m][t] =
 * sum_i x[m][i] E[t][i] in fp32.  x [M][d], E [vocab][d] in dtype (F32 or BF16), logits
 * [M][vocab] fp32, M = 1 .. 65535.  d must be a multiple of 16.  logits must not overlap x or E.
 * Errors: INVALID_ARG (sizes, dtype, null or misaligned (16 bytes) pointers). */
termezo_status termezo_logits(termezo_ctx* ctx, const void* x, const void* E, termezo_dtype dtype,
                              int64_t M, int64_t d, int64_t vocab, float* logits);

/* Beam search's selection: of all beams' continuations the n_out best per group.
 * logits: device fp32 [groups][beams][vocab]; scores: [groups][beams] fp32 summed log
 * probabilities.  Continuation (b, t) has the score scores[b] + logits[b][t] -
 * logsumexp(logits[b]); the best come first, equal ones by the lowest b * vocab + t.
 * finished (nullable, [groups][beams], nonzero: finished): a finished beam's logits are not
 * looked at, its only continuation is eos with its score unchanged.  A NaN logit counts as
 * -inf; beams whose logsumexp is not finite and NaN scores give continuations of score -inf.
 * Scores are compared in fp64, but a logsumexp's exponentials are fp32 (it is off by up to 2^-21),
 * so continuations of two beams closer than that may come in either order.
 * Outputs, [groups][n_out]: out_scores fp32, out_tokens and out_parents (the beam) int32,
 * out_finished (nullable; the parent was finished or the token is eos).  history (nullable,
 * int32 [groups][beams][hist_len]) and out_history [groups][n_out][hist_len + 1]: the
 * parent's tokens followed by the new one (hist_len 0: history may be null).  eos = -1: there
 * is none (finished must be null).  No output may overlap an input.  Errors: INVALID_ARG (groups 1 .. 65535, beams
 * 1 .. 64, vocab 1 .. 2^24, n_out 1 .. 64 and at most beams * vocab, hist_len 0 .. 2^24,
 * eos < -1 or >= vocab, null pointers, history without out_history or the
 * other way round, finished with eos -1), STATE (captured, with scratch to be allocated), OOM. */
termezo_status termezo_beam_select(termezo_ctx* ctx, const float* logits, const float* scores,
                                   const uint8_t* finished, int32_t groups, int32_t beams,
                                   int32_t vocab, int32_t n_out, int32_t eos, float* out_scores,
                                   int32_t* out_tokens, int32_t* out_parents,
                                   uint8_t* out_finished, const int32_t* history,
                                   int32_t* out_history, int64_t hist_len);

/* One generation step of the decoder with the current codes (clean or perturbed; a
 * snapshot model reads the snapshot): the n tokens of every row (device int32 [rows][n],
 * counts as in append) run through the blocks with attention over the cache, are
 * appended to it and advanced; logits [rows][vocab] fp32 (16-byte aligned) of each row's last
 * new token (0 for rows without one).  The cache's layers, heads, head size
 * and act_dtype must be the model's, its rope_base too.  Token ids are checked as in
 * termezo_model_loss; registered theta tensors are read at their values at the time of the call (a snapshot
 * holds codes and scales alone).  The call allocates activations when rows * n exceeds every earlier
 * call's.  A model with a stream of its own runs all of this there, the cache's work too:
 * termezo_model_join before other calls on the cache or the logits.
 * Errors: INVALID_ARG (2^24 tokens or more), STATE (no current codes; tokens pending; captured, with
 * activations to be allocated), OOM. */
termezo_status termezo_model_decode(termezo_model* model, termezo_kvcache* cache,
                                    const int32_t* tokens, int64_t n, const int32_t* counts,
                                    float* logits);

/* ---- inspection and support calls (not part of the four hot-path calls) ---- */

/* Wait for the context's stream; reports a deferred NUMERIC error. */
termezo_status termezo_sync(termezo_ctx* ctx);

/* Copy one layer's ascending active local indices (row * d_in + col) to the
 * host buffer idx (capacity cap entries); *n receives the count.
 * Errors: INVALID_ARG (layer range, null n, cap < count), STATE (no mask). */
termezo_status termezo_mask_export(termezo_ctx* ctx, int32_t layer, uint32_t* idx,
                                   int64_t cap, int64_t* n);

/* Unpack one layer's current ternary codes to host int8 [d_out][d_in]. */
termezo_status termezo_codes_export(termezo_ctx* ctx, int32_t layer, int8_t* codes);

/* Host copies of one layer's clean (tau, beta, fixed-point sum) and current
 * (tau', beta') scales; any pointer may be NULL. */
termezo_status termezo_layer_stats(termezo_ctx* ctx, int32_t layer, float* tau,
                                   float* beta, int64_t* abs_sum_fix,
                                   float* tau_cur, float* beta_cur);

/* Mean squared error of device fp32 y against device fp32 target over n
 * elements: e = y - t and e*e in fp32, the sum in fp64, mean rounded to fp32.
 * out: host pointer.  Waits for the stream. */
termezo_status termezo_mse_loss(termezo_ctx* ctx, const float* y, const float* target,
                                int64_t n, float* out);

/* The same mean squared error written to a device fp32 scalar (loss_dev), e.g.
 * for termezo_update_from_losses; never waits.  Errors: INVALID_ARG. */
termezo_status termezo_mse_loss_dev(termezo_ctx* ctx, const float* y, const float* target,
                                    int64_t n, float* loss_dev);

/* Gaussian directions z_i for n global ids (device uint64 gids, device fp32
 * z), exactly as the perturbation and the update regenerate them from seed.
 * hip_stream: a hipStream_t (NULL = default stream); no synchronisation. */
termezo_status termezo_gauss(void* hip_stream, uint64_t seed, const uint64_t* gids, int64_t n,
                             float* z);

/* Number of active latents (host value; waits for the stream). */
termezo_status termezo_active_count(termezo_ctx* ctx, int64_t* k);

#ifdef __cplusplus
}
#endif

#endif /* TERMEZO_H_ */

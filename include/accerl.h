/*
 * accerl.h -- C ABI of the MI355X actor-forward library.
 *
 * The one operation behind this boundary is the Actor's policy inference of the AcceRL paper
 * (Section 1: the agent maps each environment state s to an action a, and this step is the
 * bottleneck of data collection; Section 2.1: the Actors run the *compressed* policy; Section
 * 2.2, Eq. 1: the network yields an action distribution pi(.|s) and a value v(s)).  The
 * compressed ("student") policy is the post-training-quantized int8 network of Section 2.2
 * "Parameter Quantization" with the Conv+ReLU / FC+ReLU fusion described there, optionally of a
 * pruned or distilled shape (Section 2.2 "Structured Pruning", "Knowledge Distillation"); the
 * original ("teacher") policy in fp32 or bf16 sits alongside because the Corrector (Section 2.3,
 * Eq. 2: rho_t = min(rho, pi_original / pi_smaller)) and the Monitor (Section 2.4, Eq. 5) need
 * both distributions on the same states.  The behaviour logits are an output for the same reason.
 *
 * General rules
 *  - Every function returns an accerl_status (0 = OK, negative = error); nothing throws or
 *    aborts across this boundary.  accerl_last_error() gives a thread-local message.
 *  - "HOST" pointers are read during the call and never kept.  "DEVICE" pointers are HIP device
 *    memory owned by the caller, 16-byte aligned, valid until the work enqueued on `stream`
 *    has finished.  The library owns only its device copy of the weights and a per-policy
 *    workspace that it grows (hipMalloc, synchronising) when a call needs more than any
 *    earlier call did.
 *  - Forward calls only enqueue work on `stream` (a hipStream_t; NULL = the default stream) and
 *    return without synchronising; the status reports argument and launch errors only.
 *    B == 0 is valid and enqueues nothing.  One policy must not be used by two streams at once
 *    (the workspace is shared).
 *  - All tensors are dense and row-major in the logical order written below.
 */
#ifndef ACCERL_H
#define ACCERL_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct accerl_policy accerl_policy; /* opaque, library-owned */

typedef enum {
    ACCERL_OK = 0,
    ACCERL_EINVAL = -1,       /* NULL / mis-shaped / misaligned argument, inconsistent arch */
    ACCERL_ENOMEM = -2,       /* host or device allocation failed */
    ACCERL_EHIP = -3,         /* a HIP runtime call or kernel launch failed */
    ACCERL_EUNSUPPORTED = -4  /* valid request outside what the kernels cover */
} accerl_status;

typedef enum { ACCERL_OBS_U8 = 0, ACCERL_OBS_F32 = 1 } accerl_obs_dtype;

typedef enum {
    ACCERL_INT8 = 0, /* student: int8 weights and activations, int32 accumulation        */
    ACCERL_FP32 = 1, /* teacher: fp32 throughout                                           */
    ACCERL_BF16 = 2  /* teacher: bf16 operands and stored activations, fp32 accumulation  */
} accerl_precision;

typedef enum {
    ACCERL_CONV = 1,     /* cin cout k stride pad relu : square kernel, zero padding        */
    ACCERL_DENSE = 2,    /* cin cout relu                                                   */
    ACCERL_MAXPOOL = 3,  /* k stride pad : taps outside the image are ignored               */
    ACCERL_RESBLOCK = 4, /* cin == cout == channels : x + convB(relu(convA(relu(x)))), 3x3 pad 1 */
    ACCERL_RELU = 5,
    ACCERL_FLATTEN = 6,  /* C,H,W order                                                     */
    ACCERL_LSTM = 7      /* cin = input width, cout = hidden units; gate order i,f,g,o      */
} accerl_layer_kind;

typedef struct {
    int32_t kind;   /* accerl_layer_kind */
    int32_t cin, cout;
    int32_t k, stride, pad;
    int32_t relu;   /* conv / dense: ReLU fused after the layer */
    int32_t reserved;
} accerl_layer;

#define ACCERL_MAX_LAYERS 48

/* A network: observation, layer list, then two implicit heads on the last layer's flat output:
 * A = n_actions logits and one value (Section 2.2, Eq. 1: pi and v). */
typedef struct {
    int32_t obs_dtype;             /* accerl_obs_dtype */
    int32_t obs_c, obs_h, obs_w;   /* image observation [C,H,W]; vector observation: obs_c = D, obs_h = obs_w = 1 */
    int32_t n_actions;             /* 1 .. 64 */
    int32_t precision;             /* accerl_precision */
    int32_t n_layers;
    accerl_layer layers[ACCERL_MAX_LAYERS];
} accerl_arch;

/*
 * Sizes of the two host blobs accerl_policy_create expects for `arch` (so a caller can check its
 * packing).  Return ACCERL_EINVAL for an inconsistent arch.
 *
 * Weight blob: the parametrised tensors in layer order -- conv: W[cout,cin,k,k], b[cout];
 * dense: W[cout,cin], b[cout]; resblock: convA W,b then convB W,b; lstm: W_ih[4H,cin], b[4H],
 * W_hh[4H,H]; finally the heads W[A+1, F], b[A+1] (row A is the value head).  Each tensor
 * starts at the next multiple of 16 bytes.  Biases are always fp32.  W is int8 (already
 * quantized, values in -127..127) for every tensor of an ACCERL_INT8 policy except the LSTM
 * matrices and the heads of a network that contains an LSTM, which are fp32; W is fp32 for
 * teacher policies (an ACCERL_BF16 policy rounds it to bf16, ties to even, on upload).
 *
 * Scale array (ACCERL_INT8 only; n_scales = 0 for teachers): first the activation scales --
 * s_0 of the observation (uint8 observations: must be 1/255, the bytes enter as integers
 * 0..255), then in layer order one scale per quantized activation: conv and dense: their
 * output; resblock: the output of conv A, then the stream after the add -- followed by the
 * per-output-channel weight scales s_w of every int8 tensor in blob order.
 */
int accerl_blob_sizes(const accerl_arch* arch, int64_t* weights_bytes, int64_t* n_scales);

/*
 * Build a policy: validates `arch`, copies and re-lays the weights for the kernels, derives the
 * integer biases and fp32 requantization multipliers, uploads everything and fixes the launch
 * plan (the library's form of the static computational graph of Section 2.2).
 *
 * Derived constants (double arithmetic, then one rounding):
 *   biasq[n] = (int32) rint(b[n] / (s_in * s_w[n]))
 *   m[n]     = (float)((s_in * s_w[n]) / s_out)         requantization multiplier
 *   r        = (float)(s_x / s_out)                     residual-stream ratio
 *   d[n]     = (float)(s_in * s_w[n])                   head dequantization
 *   inv_s0   = (float)(1 / s_0)                         fp32 observation quantizer
 *
 * weights, quant_scales: HOST, copied.  quant_scales may be NULL iff n_scales == 0.
 * *out receives the policy; destroy it with accerl_policy_destroy.  Uses the current HIP device.
 */
int accerl_policy_create(const accerl_arch* arch, const void* weights, int64_t weights_bytes,
                         const float* quant_scales, int64_t n_scales, accerl_policy** out);

void accerl_policy_destroy(accerl_policy* p);

/*
 * Student forward (Section 1 / 2.1: the Actor's inference on the compressed policy; arithmetic:
 * Section 2.2 "Parameter Quantization").  The policy must be ACCERL_INT8 and contain no LSTM.
 *
 *   states     DEVICE [B, C, H, W] uint8 or [B, D] fp32, as the arch says
 *   uniforms   DEVICE [B] fp32 in [0, 1): one draw per state for the sampler
 *   out_logits DEVICE [B, A] fp32 behaviour logits
 *   out_value  DEVICE [B] fp32
 *   out_action DEVICE [B] int32: with m = max_a logit, e_a = exp(logit_a - m), Z = sum_a e_a
 *              (index order), the first a with e_0 + .. + e_a > u * Z, else A - 1
 *
 * Per layer: acc = sum Wq * xq + biasq (exact int32); y = (float)acc * m[n];
 * q = clamp(rint(y), relu ? 0 : -127, 127); residual join y = fma((float)acc, m[n], (float)xq * r);
 * heads logit = (float)acc * d[n].
 */
int accerl_actor_forward(accerl_policy* p, const void* states, int64_t B, const float* uniforms,
                         float* out_logits, float* out_value, int32_t* out_action, void* stream);

/* Teacher forward: same arguments and outputs; the policy must be ACCERL_FP32 or ACCERL_BF16 and
 * contain no LSTM (Section 3.1: the original network runs in fp32; Section 2.2: fp16-class
 * storage is the paper's other low-bit option).  uint8 observations enter as obs / 255. */
int accerl_actor_forward_teacher(accerl_policy* p, const void* states, int64_t B, const float* uniforms,
                                 float* out_logits, float* out_value, int32_t* out_action, void* stream);

/*
 * One environment step of a recurrent policy (the arch ends in an ACCERL_LSTM layer), any
 * precision.  done: DEVICE [B] uint8; rows with done != 0 have h and c zeroed before the cell.
 * h, c: DEVICE [B, H] fp32, updated in place.  The LSTM and the heads behind it use bf16 GEMM
 * operands (fp32 for an ACCERL_FP32 policy) with fp32 accumulation and fp32 gate arithmetic:
 * c' = sig(f) * c + sig(i) * tanh(g), h' = sig(o) * tanh(c').
 */
int accerl_actor_forward_recurrent(accerl_policy* p, const void* states, int64_t B, const float* uniforms,
                                   const uint8_t* done, float* h, float* c,
                                   float* out_logits, float* out_value, int32_t* out_action, void* stream);

typedef enum {
    ACCERL_TAP_ACC = 0,   /* int32 accumulator of a conv / dense layer (resblock: of conv B); layer = n_layers: of the heads */
    ACCERL_TAP_ACT = 1,   /* stored output of the layer: int8 (student), fp32 (teachers, converted) */
    ACCERL_TAP_ACC_A = 2, /* resblock: accumulator of conv A */
    ACCERL_TAP_ACT_A = 3  /* resblock: output of conv A */
} accerl_tap;

/*
 * Debug forward for parity tests: runs the network layer by layer up to and including layer
 * `layer` (kernels that the forward calls fuse run one by one: the same bits, except that an
 * ACCERL_FP32 policy's whole-network kernel adds in another order) and copies one intermediate
 * tensor to `out` (DEVICE, `out_bytes`
 * must equal the tensor's size).  Image tensors are written channels-last, [B, H, W, Cs] with
 * Cs = C rounded up to a multiple of 4 (padding channels are zero); flat tensors [B, N].  Accumulator taps are student-only and include the integer bias and are
 * zero-point free (uint8 observations count as 0..255).  Recurrent policies: layers before the
 * LSTM only.  Synchronises the stream before returning.
 */
int accerl_actor_forward_debug(accerl_policy* p, const void* states, int64_t B, int32_t layer, int32_t tap,
                               void* out, int64_t out_bytes, void* stream);

/*
 * Measurement aid (not part of the method).  Between accerl_profile_begin and accerl_profile_end
 * every forward call on the policy records one HIP event after each kernel launch of its plan (and
 * one before the first), on the stream of that call; a step's time is the span between the event
 * before it and the event after it.  A step whose work was done by the step before it (a conv or a
 * max-pool fused into the preceding conv kernel) records nothing and reports zero launches.
 * accerl_profile_end waits for the events and returns, per plan step, the summed elapsed time in
 * ms, the number of launches, the arch layer the step belongs to (n_layers = heads / sampler) and the step kind (0 fused MLP, 1 observation quantizer,
 * 2 convolution, 3 MFMA dense, 4 fp32 dense, 5 max pooling, 6 LSTM packing, 7 sampler, 8 heads + sampler).  All arrays
 * are HOST, `cap` entries each; *n_steps receives the number of plan steps (also on ACCERL_EINVAL
 * when cap is too small).
 */
int accerl_profile_begin(accerl_policy* p);
int accerl_profile_end(accerl_policy* p, int32_t cap, int32_t* n_steps, float* total_ms, int64_t* launches,
                       int32_t* layer, int32_t* kind);

/*
 * Host-only aid: builds the launch plan exactly as accerl_policy_create would (same arguments, no
 * GPU needed) and writes a one-line-per-kernel description of it into `text` (HOST, `cap` bytes,
 * always NUL-terminated, truncated if too small).
 */
int accerl_plan_describe(const accerl_arch* arch, const void* weights, int64_t weights_bytes,
                         const float* quant_scales, int64_t n_scales, char* text, int64_t cap);

/*
 * Policy mixture (Section 3.2, "Knowledge Distillation Results"): the actor sends a state through the
 * smaller network with probability alpha and through the original one otherwise.  The draw is the
 * caller's (use_smaller: HOST uint8 [B], non-zero = smaller network, read during the call); the
 * library compacts the rows of each subset, runs `smaller` on the first and `original` on the second
 * (any two non-recurrent policies: int8, fp32 or bf16) and writes every row's results to its place in the
 * outputs, so each row holds exactly what the chosen network alone would have produced for it.
 * Both policies must share observation shape and number of actions and be non-recurrent.  states,
 * uniforms and the outputs are DEVICE as in accerl_actor_forward.  Asynchronous on hip_stream; the
 * compaction buffers belong to `smaller` and grow on demand (a stream synchronisation when they do),
 * so calls that share `smaller` must not overlap.  Errors as accerl_actor_forward.
 */
int accerl_actor_forward_mixture(accerl_policy* smaller, accerl_policy* original, const void* states, int64_t B,
                                 const float* uniforms, const uint8_t* use_smaller,
                                 float* out_logits, float* out_value, int32_t* out_action, void* hip_stream);

/* Host-only: the mixture probability as a function of the Monitor's KL-mean indicator (same passage):
 * 1 up to kl_lo, 0 from kl_hi on, linear in between (the paper prints no constants). */
double accerl_mixture_alpha(double kl_mean, double kl_lo, double kl_hi);

/*
 * Monitor indicators (Monitor section, KL equation): for B states on which both the original and
 * the smaller (compressed) policy were evaluated,
 *     KL_b = sum_a pi_original(a|x_b) log(pi_original(a|x_b) / pi_smaller(a|x_b)),
 *     H_b  = -sum_a pi_smaller(a|x_b) log pi_smaller(a|x_b)     (the entropy indicator; Section 2.2 Eq. 1)
 * with pi = softmax of the logits.  logits_* : DEVICE fp32 [B, A] row-major, 16-byte aligned,
 * 1 <= A <= 64.  out_kl, out_entropy: DEVICE fp32 [B] or NULL.  out_stats: DEVICE double[4] =
 * {KL mean, KL max, KL variance (population: mean of squares minus squared mean), entropy mean},
 * the indicators the Monitor's strategies read.  Per-row arithmetic is fp32, the reductions are
 * fp64 in a fixed order (results do not depend on the launch).  Asynchronous on hip_stream; the
 * library keeps one small per-device buffer of partial sums, so calls that overlap on one device
 * must use the same stream.  B == 0 is a no-op.  Errors: ACCERL_EINVAL for NULL / misaligned /
 * out-of-range arguments, ACCERL_ENOMEM, ACCERL_EHIP.
 */
int accerl_monitor_kl(const float* logits_original, const float* logits_smaller, int64_t B, int A,
                      float* out_kl, float* out_entropy, double* out_stats, void* hip_stream);

/*
 * accerl_monitor_kl for callers that cannot allocate device memory: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels and the same results as
 * accerl_monitor_kl; the per-workgroup partial sums go to a fixed 40 KiB array inside the library's device
 * image (1024 records of 5 doubles; each GPU the library runs on holds its own copy until the process ends)
 * instead of a buffer allocated at first use, and the call makes no hipMalloc / hipFree and no allocating
 * library call.  B is limited to 16 777 216 (2^24) rows per call; a larger B returns ACCERL_EINVAL with a
 * message and enqueues nothing (split the batch).  Every call on a GPU uses that GPU's one array: calls that
 * overlap in time on one GPU (different streams or threads) race and must be serialised by the caller; calls
 * in sequence need no clearing in between, since a pass overwrites every record that its fold reads.
 * With more than 20 actions and more than 1024 x 256 rows the row pass runs over 1024 workgroups where
 * accerl_monitor_kl uses up to 2048, so the fp64 sums may differ from it in their last bits; out_kl and
 * out_entropy are identical.
 */
int accerl_monitor_kl_noalloc(const float* logits_original, const float* logits_smaller, int64_t B, int A,
                              float* out_kl, float* out_entropy, double* out_stats, void* hip_stream);

/*
 * Knowledge-distillation loss, forward value only (Section 2.2, Eq. 1): per state
 *     loss_b = KL(pi_original(.|s_b) || pi_smaller(.|s_b)) + (v_original(s_b) - v_smaller(s_b))^2 / 2
 *              - beta H(pi_smaller(.|s_b)),
 * the quantity the Compressor minimises when it transfers the original policy into the smaller
 * network (its gradient and the optimiser are outside this library).  logits_*: DEVICE fp32 [B, A]
 * (16-byte aligned, 1 <= A <= 64); value_*: DEVICE fp32 [B]; out_loss: DEVICE fp32 [B] or NULL;
 * out_mean: DEVICE double[1], the batch mean (fp64 reduction in a fixed order).  Same stream and
 * overlap rules as accerl_monitor_kl, whose per-device partial-sum buffer it shares.
 */
int accerl_distill_loss(const float* logits_original, const float* logits_smaller, const float* value_original,
                        const float* value_smaller, int64_t B, int A, float beta, float* out_loss, double* out_mean,
                        void* hip_stream);

/*
 * V-trace corrector (Corrector section, V-trace equation) for B trajectories of T steps collected
 * by the smaller policy and corrected towards the original one.  Time-major tensors, all DEVICE:
 *   logits_original, logits_smaller  fp32 [T, B, A], 16-byte aligned, 1 <= A <= 64
 *   actions int32 [T, B] (the a_t taken; clamped into 0..A-1), rewards, discounts, values fp32 [T, B]
 *   (discounts = gamma, or 0 where the episode ended at that step; values = V(x_t)),
 *   bootstrap fp32 [B] = V(x_T).
 *   rho_t = min(rho_bar, pi_original(a_t|x_t) / pi_smaller(a_t|x_t)),  c_t = min(c_bar, same ratio)
 *   delta_t = rho_t (r_t + gamma_t V(x_{t+1}) - V(x_t))
 *   v_s = V(x_s) + sum_{t=s}^{T-1} (prod_{i=s}^{t-1} gamma_i c_i) delta_t   (evaluated as a backward scan)
 * Outputs fp32 [T, B]: out_vs = v_s; out_rho = rho_t (also the importance weight of the Importance
 * Sampling corrector); out_pg_adv (may be NULL) = rho_t (r_t + gamma_t v_{t+1} - V(x_t)), v_T = V(x_T),
 * the advantage of the corrected actor-critic update.  out_rho is also used as scratch during the
 * call.  Asynchronous on hip_stream; allocates nothing.  T == 0 or B == 0 is a no-op.
 */
int accerl_vtrace(const float* logits_original, const float* logits_smaller, const int32_t* actions,
                  const float* rewards, const float* discounts, const float* values, const float* bootstrap,
                  int64_t T, int64_t B, int A, float rho_bar, float c_bar,
                  float* out_vs, float* out_pg_adv, float* out_rho, void* hip_stream);

/*
 * Operators of wide policies: an action set of up to 2^20 (tokens), dense layers whose inputs have no calibrated scale.
 *
 * Tensors here may have rows of any stride (`ld_*`: elements from one row to the next, at least the row's length) and any
 * alignment of whole elements, unless said otherwise; elements of a row are contiguous.
 */
typedef enum { ACCERL_DT_F32 = 0, ACCERL_DT_BF16 = 1, ACCERL_DT_F16 = 2 } accerl_dtype;

/*
 * Packed int8 rows: the layout in which the int8 product reads both of its operands.  Tiles of 16 rows by 64 columns of 1024 bytes,
 * [row / 16][column / 64][(column % 64) / 16][row % 16][column % 16], rows padded to a multiple of 16 and columns with zeros to a
 * multiple of 128.  accerl_packed_rows_bytes gives the size of the buffer (DEVICE, 16-byte aligned; negative: an accerl_status).
 * At most 2^24 rows and 2^16 columns (ACCERL_EUNSUPPORTED above).
 */
int64_t accerl_packed_rows_bytes(int64_t rows, int64_t cols);

/*
 * Quantises every row with a scale of its own (Section 2.2 "Parameter Quantization", symmetric, here with the scale found from
 * the row itself): with m_r = max_c |x[r,c]|,
 *     out_scale[r] = m_r / 127,    q[r,c] = rint(x[r,c] * 127 / m_r), ties to even, rounded once from the exact quotient
 * A row of zeros has scale 0.  A row that holds an infinity or a NaN has that (or NaN) as its scale and zeros, so that a product with
 * it is NaN.  x DEVICE [rows, cols] of x_dtype; out_scale DEVICE fp32 [rows].  Weights are quantised with the same call, a
 * channel being a row.  rows == 0 enqueues nothing.
 */
int accerl_quantize_rows(const void* x, int32_t x_dtype, int64_t rows, int64_t cols, int64_t ld_x, int8_t* out_packed,
                         float* out_scale, void* stream);

/* Rows that are int8 already (q DEVICE [rows, cols]) into the packed layout, and back. */
int accerl_pack_rows_i8(const int8_t* q, int64_t rows, int64_t cols, int64_t ld_q, int8_t* out_packed, void* stream);
int accerl_unpack_rows_i8(const int8_t* packed, int64_t rows, int64_t cols, int8_t* out_q, int64_t ld_q, void* stream);

/*
 * Int8 dense layer with a scale for each token and each channel:
 *     acc[m,n] = sum_k x[m,k] w[n,k] (exact int32),    y = ((float)acc * x_scale[m]) * w_scale[n] + bias[n],    ReLU if relu != 0
 * rounded once to out_dtype.  x_packed [M, K] and w_packed [N, K] packed rows; x_scale, w_scale, bias (NULL: none) DEVICE fp32; out
 * DEVICE [M, N], overlapping none of them (ACCERL_EINVAL).  M == 0 or N == 0 enqueues nothing.  Allocates nothing, does not synchronise.
 */
int accerl_dense_i8(const int8_t* x_packed, const float* x_scale, const int8_t* w_packed, const float* w_scale, const float* bias,
                    int64_t M, int64_t N, int64_t K, int32_t relu, void* out, int32_t out_dtype, int64_t ld_out, void* stream);

/*
 * The same layer on floating-point tokens, quantised as accerl_quantize_rows does (same results as the two calls).
 * workspace: DEVICE, 16-byte aligned, at least accerl_dense_i8_workspace(M, K) bytes, used until the work has finished, and by a graph that
 * captured the call as long as it is replayed: calls that may overlap, of several threads on one stream too, need a workspace each.  Its contents need not be kept or cleared.  out may lie over x, whose tokens are quantised before it is
 * written, and over nothing else; the workspace over neither (ACCERL_EINVAL).
 */
int64_t accerl_dense_i8_workspace(int64_t M, int64_t K);
int accerl_dense_i8_dynamic(const void* x, int32_t x_dtype, int64_t ld_x, const int8_t* w_packed, const float* w_scale, const float* bias,
                            int64_t M, int64_t N, int64_t K, int32_t relu, void* out, int32_t out_dtype, int64_t ld_out,
                            void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Log-probabilities of actions, and the entropy of the distribution they were drawn from, for a wide action set:
 *     out_logp[b] = log pi(a_b|x_b),    out_entropy[b] = H(pi(.|x_b))    (NULL: not wanted),    pi = softmax over the allowed actions
 * logits DEVICE [B, A] of `dtype`, 1 <= A <= 2^20; mask DEVICE uint8 [B, A], zero = not allowed, whatever its logit (NULL: all are
 * allowed; ld_mask == 0: one row for all); actions DEVICE int32 [B].  A logit of -inf is an action of probability 0.  An action that is not allowed
 * has log-probability -inf, and so has every action of a row that allows none (entropy 0).  An action outside 0 .. A-1 marks a row
 * without one: 0 and 0, and the row is not read.  workspace: DEVICE, 16-byte aligned, accerl_policy_loss_workspace() bytes (the same
 * for all sizes), used as accerl_dense_i8_dynamic's: calls that may overlap need one each.  Neither call allocates or synchronises;
 * B == 0 enqueues nothing; a call repeated gives the same bits.
 */
int64_t accerl_policy_loss_workspace(void);
int accerl_action_logprob(const void* logits, int32_t dtype, int64_t ld_logits, const uint8_t* mask, int64_t ld_mask, const int32_t* actions,
                          int64_t B, int64_t A, float* out_logp, float* out_entropy, void* workspace, int64_t workspace_bytes, void* stream);

typedef enum {
    ACCERL_KL_NONE = 0,
    ACCERL_KL_SAMPLED = 1,   /* exp(d) - d - 1 with d = ref_logp - log pi(a): the estimate from the action taken alone */
    ACCERL_KL_FORWARD = 2,   /* KL(pi_ref || pi) over all actions, the Monitor's and the distillation loss's */
    ACCERL_KL_REVERSE = 3    /* KL(pi || pi_ref) over all actions */
} accerl_kl_kind;

/*
 * Clipped policy loss with a KL term to a reference policy and an entropy term, and its gradient (the corrected actor-critic
 * update that accerl_vtrace's out_pg_adv feeds, Section 2.3; the KL and entropy terms of Section 2.2, Eq. 1).  Per row, with
 * pi = softmax of the allowed logits, r = exp(log pi(a) - old_logp):
 *     loss = -min(r adv, clip(r, 1 - clip_low, 1 + clip_high) adv) + kl_coef KL - entropy_coef H(pi)
 *     grad[b, j] = scale * weights[b] * d loss_b / d logits[b, j]
 *     out_stats  = scale * sum_b weights[b] * {loss, KL, H, 1 if r lies outside the borders}    (summed in 64 bits)
 * so that with scale = 1 / (number of rows that count) the first is the batch's loss and the gradient is its gradient.  A row of weight
 * 0, or whose action lies outside 0 .. A-1, is not read: its outputs and its gradient are 0.  A KL term of coefficient 0 is reported and
 * no part of the loss.  A row that allows no action has loss, KL,
 * entropy and gradient 0 and log-probability -inf.  An action of probability 0 has ratio 0.  The mask applies to both policies; where
 * the reference allows nothing, the forward KL is 0 and the reverse one infinite.  NaN and +inf among the allowed logits make the row NaN.
 * Arithmetic is fp32 or wider, gradients are rounded once to `dtype`.  grad_logits may be NULL (value only) or the logits themselves
 * (same stride); no other output may overlap an input.
 */
typedef struct {
    int64_t B, A;
    int32_t dtype;                 /* accerl_dtype of logits, ref_logits and grad_logits */
    int32_t kl_kind;               /* accerl_kl_kind */
    const void* logits;            /* DEVICE [B, A] */
    int64_t ld_logits;
    const void* ref_logits;        /* DEVICE [B, A] (FORWARD and REVERSE) */
    int64_t ld_ref;
    void* grad_logits;             /* DEVICE [B, A] or NULL */
    int64_t ld_grad;
    const uint8_t* mask;           /* as in accerl_action_logprob */
    int64_t ld_mask;
    const int32_t* actions;        /* DEVICE [B] */
    const float* old_logp;         /* DEVICE [B]: the behaviour's log-probabilities */
    const float* advantages;       /* DEVICE [B] */
    const float* weights;          /* DEVICE [B] or NULL (all 1) */
    const float* ref_logp;         /* DEVICE [B] (SAMPLED) */
    double clip_low, clip_high, kl_coef, entropy_coef, scale;
    float* out_loss;               /* DEVICE [B] each, or NULL */
    float* out_logp;
    float* out_kl;
    float* out_entropy;
    float* out_stats;              /* DEVICE [4] or NULL */
    void* workspace;               /* as in accerl_action_logprob */
    int64_t workspace_bytes;
} accerl_policy_loss_args;

int accerl_policy_loss(const accerl_policy_loss_args* args, void* stream);

/*
 * Operators of policies with a memory: linear attention with a decay for each head, and the norms around a block.  An actor carries the
 * memory from step to step, as it does the state of accerl_actor_forward_recurrent; a learner unrolls it over many steps and takes gradients.
 *
 * For a head h of decay g = exp(log_decay[h]) and its queries, keys and values, tokens in their order t = 0 .. n - 1:
 *     S_t = g S_{t-1} + k_t v_t^T,    o_t = scale q_t S_t        (S: [Dk, Dv]; S_{-1} = state, or zeros)
 * where reset[t] != 0 the token begins an episode: the state before it counts as zeros, whatever it holds.  H heads of queries share H / Hk heads
 * each: head h reads k and v of head h Hk / H (H is a multiple of Hk), and has a state of its own.  lengths[b] = n (taken as 0 .. T; NULL: T): the
 * tokens from n on are not read, their outputs and gradients are 0, and the state is that after n tokens.
 *
 * Tensors of tokens are [B, T, heads, D] with strides (elements) of their own for batch, token and head, of any alignment of whole elements;
 * elements of a head are contiguous: time-major tensors and parts of wider rows are taken as they are.  States are DEVICE fp32 [B, H, Dk, Dv], dense, 16-byte
 * aligned.  1 <= Dk, Dv <= 256.  log_decay holds numbers <= 0 or -inf.  State and sums are fp32.  With bf16 tokens the weights of
 * pairs of tokens and the state's copy that queries are multiplied with are rounded to bf16, as their partners are (fp16 tokens: both go through two bf16
 * parts each, and a term is 2^-15 off at most).  A state that is handed out, and those that segments of a long unroll hand on, are as exact as fp32; inside an unroll
 * whose last state is not wanted a key or value times its decay is held to 2^-16 (fp16: 2^-15).
 * A NaN or an infinity of a key or a value reaches the tokens behind it, of its episode and head, and no others; results that are not finite are those of
 * the recurrence in fp32, token by token.
 * out_state may be the state; otherwise outputs overlap neither inputs nor each other, and the workspace overlaps nothing (ACCERL_EINVAL; columns of
 * one buffer's rows that lie beside each other do not).
 */
typedef struct { int64_t batch, token, head; } accerl_token_stride;

typedef struct {
    int64_t B, T;
    int32_t H, Hk, Dk, Dv;
    int32_t dtype;                 /* accerl_dtype of the tokens, and of their outputs and gradients */
    const void *q, *k, *v;         /* DEVICE [B, T, H, Dk], [B, T, Hk, Dk], [B, T, Hk, Dv] */
    accerl_token_stride q_stride, k_stride, v_stride;
    const float* log_decay;        /* DEVICE [H] */
    double scale;
    const uint8_t* reset;          /* DEVICE [B, T] with strides, or NULL (no token resets) */
    int64_t reset_batch, reset_token;
    const int32_t* lengths;        /* DEVICE [B] or NULL */
    const float* state;            /* DEVICE [B, H, Dk, Dv] or NULL (zeros) */
    void* out;                     /* DEVICE [B, T, H, Dv] */
    accerl_token_stride out_stride;
    float* out_state;              /* DEVICE [B, H, Dk, Dv] or NULL (not wanted) */
    /* gradients (accerl_linear_attention_grad; out and out_state are not looked at) */
    const void* grad_out;          /* DEVICE [B, T, H, Dv] */
    accerl_token_stride grad_out_stride;
    const float* grad_out_state;   /* DEVICE [B, H, Dk, Dv] or NULL (zeros) */
    void *grad_q, *grad_k, *grad_v;    /* shapes of q, k, v */
    accerl_token_stride grad_q_stride, grad_k_stride, grad_v_stride;
    float* grad_state;             /* DEVICE [B, H, Dk, Dv] or NULL (not wanted) */
    void* workspace;               /* DEVICE, 16-byte aligned, of accerl_linear_attention_workspace's size; used as accerl_dense_i8_dynamic's */
    int64_t workspace_bytes;
} accerl_linear_attention_args;

/* Bytes of the workspace of an unroll (grad == 0) or of its gradients; negative: an accerl_status. */
int64_t accerl_linear_attention_workspace(int64_t B, int64_t T, int32_t H, int32_t Hk, int32_t Dk, int32_t Dv, int32_t grad);
/* The unroll: out, and out_state behind the last token.  B == 0 enqueues nothing. */
int accerl_linear_attention(const accerl_linear_attention_args* args, void* stream);
/* The gradients of sum(grad_out . out) + sum(grad_out_state . out_state) by q, k, v and state; the decay is a constant. */
int accerl_linear_attention_grad(const accerl_linear_attention_args* args, void* stream);
/* One token for each of B environments: T, lengths, token strides and the workspace are not looked at, state and out_state are needed (they may be the
 * same).  All arithmetic is fp32. */
int accerl_linear_attention_step(const accerl_linear_attention_args* args, void* stream);

typedef enum { ACCERL_NORM_RMS = 0, ACCERL_NORM_LAYER = 1 } accerl_norm_kind;             /* LAYER: the mean is taken off first */
typedef enum { ACCERL_GATE_NONE = 0, ACCERL_GATE_SIGMOID = 1, ACCERL_GATE_SILU = 2 } accerl_gate_kind;

/*
 * The end of a block and the beginning of the next one, in one pass over the rows: the norm behind the block, its gate, the residual with
 * its scales, and the norm before the next block.  For a row of D channels, y being the block's output and x the residual stream,
 *     u = skip x + branch act(gate) after(y),    h = before(u)
 *     norm(z)_i = weight_i (z_i - m) / sqrt(mean_j (z_j - m)^2 + eps),    m = 0 (RMS) or mean_j z_j (LAYER)
 * `after` works on each of `groups` equal parts of a row by itself (the heads of an attention); `before` on the whole row, and with it
 * groups is 1.  eps is positive, 2^-126 at least.  A NULL weight leaves its norm out (after(y) = y; no h), x NULL the residual, gate_kind NONE the
 * gate.  1 <= D <= 16384.
 * y, gate, h and their gradients have `dtype`; x, u and theirs `stream_dtype`, which is `dtype` or fp32.  Weights and their
 * gradients are DEVICE fp32 [D].  Arithmetic is fp32 (finite rows whose sum of squares leaves its range have norms of 0); h is taken from u before u
 * is rounded; results are rounded once.  Rows do not touch each other: a NaN stays in its row (and in the weights' gradients).  Rows of an output may
 * lie over rows of an input of the same type and stride, whole, and a weight's gradient over a weight; outputs and the workspace overlap nothing
 * else (ACCERL_EINVAL).
 * Gradients: of sum(grad_u . u) + sum(grad_h . h), by y, x, gate and both weights (a pointer of NULL: not wanted; grad_u or grad_h NULL: zeros).
 * They start from the forward's inputs: nothing is kept from the forward.  The weights' sums over rows have a fixed order.
 * workspace: of accerl_block_norm_workspace's bytes, needed where gradients of weights are asked for; used as accerl_dense_i8_dynamic's.
 */
typedef struct {
    int64_t N;                     /* rows */
    int32_t D, groups;
    int32_t kind, gate_kind;
    int32_t dtype, stream_dtype;
    double eps, skip, branch;
    const void* y; int64_t ld_y;               /* DEVICE [N, D] each, rows `ld` elements apart */
    const void* x; int64_t ld_x;
    const void* gate; int64_t ld_gate;
    const float *after, *before;
    void* out_u; int64_t ld_u;                 /* NULL: not wanted */
    void* out_h; int64_t ld_h;
    const void* grad_u; int64_t ld_grad_u;
    const void* grad_h; int64_t ld_grad_h;
    void* grad_y; int64_t ld_grad_y;
    void* grad_x; int64_t ld_grad_x;
    void* grad_gate; int64_t ld_grad_gate;
    float *grad_after, *grad_before;           /* [D] */
    void* workspace;
    int64_t workspace_bytes;
} accerl_block_norm_args;

int64_t accerl_block_norm_workspace(int64_t N, int32_t D, int32_t groups);
int accerl_block_norm(const accerl_block_norm_args* args, void* stream);
int accerl_block_norm_grad(const accerl_block_norm_args* args, void* stream);

/*
 * Measurement aids (not part of the method): the ceilings the kernels are compared with, as this machine
 * sustains them.  accerl_probe_mfma runs 2048 workgroups x 4 wavefronts, each issuing iters x 8 independent
 * 16x16 MFMAs on registers (int8 16x16x64, or bf16 16x16x32 if bf16 != 0): ops = 2048 * 4 * iters * 8 *
 * 2 * 16*16*K.  accerl_probe_copy streams `bytes` (a multiple of 16) from src to dst with 16-byte
 * loads and stores.  Both asynchronous on hip_stream; the caller times them.  sink: DEVICE int32[1].
 */
int accerl_probe_mfma(int32_t bf16, int32_t iters, int32_t* sink, void* hip_stream);
int accerl_probe_copy(const void* src, void* dst, int64_t bytes, void* hip_stream);
/* One launch of a kernel that does nothing (one wavefront): chains of it give the launch floor that the latency of
 * the small configured batches is quoted against. */
int accerl_probe_empty(void* hip_stream);

/* Message of the last error on this thread ("" if none). */
const char* accerl_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* ACCERL_H */

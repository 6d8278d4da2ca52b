/*
 * bmlp.h -- C-ABI of the GB300 (sm_103a) library that trains and evaluates
 * binary multi-layer perceptrons (BMLPs) with the fully binary, gradient-free
 * rule of "Training multi-layer binary neural networks with random local binary
 * error signals" (arXiv 2412.00119).
 *
 * What the library computes (paper notation; layers l = 1..L, widths K_0..K_L,
 * c classes):
 *   - H_l (K_{l-1} x K_l) integer "hidden metaplastic" weights, W_l = sign(H_l)
 *     the visible binary weights, P_l (K_l x c) a fixed random +-1 local
 *     classifier per layer (Sec. 3.1);
 *   - per mini-batch of bs patterns (Alg. 1): z_l = a_{l-1} W_l, a_l = sign(z_l),
 *     yhat_l = a_l P_l, the 01-loss of Eq. 1 and the robustness margin tau of
 *     Alg. 1 l.13-15 marking the patterns M_l to learn from;
 *   - the layer-level selection of Alg. 2: per group of gamma neurons the
 *     perceptron with the negative stability z_k rho_{k,y} closest to 0;
 *   - the perceptron-level CP + R rule of Alg. 3 with hidden weights clipped to
 *     [-h_max, h_max], W_l re-derived and re-packed in the same pass;
 *   - the end-of-epoch rescale p_r <- p_r sqrt(E^e) (Alg. 1 l.21);
 *   - forward-only evaluation: argmax of a_L P_L (Sec. 3.1).
 * Conventions where the paper is silent: sign(0) = +1; argmax ties go to the
 * lowest class; groups are contiguous (neuron k in group k / gamma); tuples are
 * applied in ascending pattern order with clipping after each; LayerUpdate runs
 * only when M_l is non-empty; the reinforcement events are drawn per block
 * of 64 inputs from 32-bit Philox4x32-10 draws against integer thresholds
 * (bmlp_reinforce_tables).  Every result is an integer or a bit and is
 * reproducible bit for bit.
 *
 * Data formats
 *   packed +-1 vectors: a vector of K values is ceil(K/64) little-endian uint64
 *     words; bit j of word w is element 64 w + j; a set bit means +1; pad bits
 *     must be 0.  A batch of n vectors is n such rows, row after row.
 *   labels: int32 in 0..c-1.
 *   H (state export): int16, K_l rows of K_{l-1} (neuron-major: element
 *     [k * K_{l-1} + i] is h_{ik}), odd values in [-h_max, h_max].
 *   W (state export): uint64, K_l rows of ceil(K_{l-1}/64) words, bit = (h > 0).
 *   P (state export): int8, K_l rows of c values rho_{kj} in {-1, +1}.
 *
 * Pointers and streams
 *   Batch inputs and outputs (x_packed, labels, labels_out) may be device or
 *   host pointers; the library asks the CUDA runtime which.  Host buffers are
 *   staged through library-owned device buffers with cudaMemcpyAsync on the
 *   given stream (pinned host memory makes the copies asynchronous).  The
 *   caller owns every buffer it passes in and must keep it alive until the
 *   work on `cuda_stream` has completed; the library owns the model state.
 *   `cuda_stream` is a cudaStream_t (NULL = the legacy default stream).
 *   Calls are asynchronous on that stream, except those that return host
 *   values (n_errors_out, BMLP_EPOCH_END, bmlp_get_state, bmlp_set_state),
 *   which synchronise it.
 *
 * Errors
 *   Every int-returning call returns BMLP_OK (0) or a negative BMLP_E* code and
 *   never throws or aborts; bmlp_last_error() gives a one-line reason.  Labels
 *   outside 0..c-1 in device memory are not read out of bounds: the kernels
 *   count them, and the next call that synchronises returns BMLP_EINVAL.
 *
 * One handle is used by one host thread at a time.
 */
#ifndef BMLP_H_
#define BMLP_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BMLP_OK 0
#define BMLP_EINVAL (-1)   /* bad argument or bad label values */
#define BMLP_ENOMEM (-2)   /* device or host allocation failed */
#define BMLP_ECUDA (-3)    /* a CUDA runtime call or kernel launch failed */
#define BMLP_ETIMEOUT (-4) /* a bounded device-side wait gave up */
#define BMLP_ESTATE (-5)   /* state blob inconsistent with the model */
#define BMLP_ENODEV (-6)   /* no usable sm_103 device */

#define BMLP_MAX_LAYERS 16
#define BMLP_MAX_BS 1024
#define BMLP_MAX_CLASSES 1024

/* bmlp_train flags */
#define BMLP_EPOCH_END 1u  /* after these n patterns, close the epoch (Alg. 1 l.21) */

/* forward-contraction engines (hparams.fwd_impl) */
#define BMLP_FWD_AUTO 0     /* library's choice: the tensor cores (bmlp_get_info reports
                             * BMLP_FWD_TCGEN05 up to bs = 128 and BMLP_FWD_POPC above) */
#define BMLP_FWD_POPC 1     /* CUDA-core XOR + popcount */
#define BMLP_FWD_TCGEN05 2  /* 5th-gen tensor cores, +-1 as e2m1, fp32 accumulate (exact) */
/* Further contraction units, measured by bmlp_engine_peak (and, for B1MMA,
 * bmlp_layer_forward_engine) for the engine comparison; training uses POPC or
 * TCGEN05.  tcgen05.mma.kind::i8 does not exist on sm_103a, so +-1 as int8 on
 * tensor cores is the legacy mma.sync path (S8MMA). */
#define BMLP_FWD_B1MMA 3    /* mma.sync m16n8k256 .b1 xor.popc (legacy tensor path) */
#define BMLP_FWD_S8MMA 4    /* mma.sync m16n8k32 .s8, +-1 as int8 (legacy tensor path) */

typedef struct bmlp bmlp_t;

/* Hyperparameters (Alg. 1 header).  Zero-initialise and set what you need:
 * a zero / negative field selects the paper's setting of Sec. 4.2. */
typedef struct bmlp_hparams {
  int32_t bs;            /* mini-batch size, 1..BMLP_MAX_BS; 0 -> 100 */
  int32_t r_num, r_den;  /* robustness r = r_num / r_den; r_den == 0 -> r = 1/4 */
  double p_r0;           /* initial reinforcement probability; < 0 -> 0.5 */
  const int32_t* gamma;  /* L group sizes, each dividing K_l; NULL -> Sec. 4.3 rule */
  int32_t fwd_impl;      /* BMLP_FWD_*; 0 -> auto */
  int32_t group_mode;    /* BMLP_GROUPS_*: group membership of Alg. 2 (Sec. 4.3); 0 -> contiguous */
} bmlp_hparams;

/* Group membership (Sec. 4.3: by the permutation symmetry of a hidden layer
 * its groups may be any fixed random partition, or one redrawn at every
 * step).  CONTIGUOUS: group g = neurons g*gamma .. (g+1)*gamma - 1.  FIXED /
 * RESHUFFLED: order the neurons k of layer l by the key u_k = word k%4 of
 * Philox4x32-10 at counter (k/4, 0, 32*2^16 + l, t') with the model's key,
 * ties to the smaller k; group g = the neurons at positions g*gamma ..
 * (g+1)*gamma - 1 of that order, with t' = 0 (FIXED) or t' = the step counter
 * (RESHUFFLED, a new partition every mini-batch).  Within a group the easiest
 * neuron is chosen with ties to the lowest neuron index.  FIXED and
 * RESHUFFLED need every K_l <= 16384. */
#define BMLP_GROUPS_CONTIGUOUS 0
#define BMLP_GROUPS_FIXED 1
#define BMLP_GROUPS_RESHUFFLED 2

/* Create a model and initialise H_l, P_l uniformly on {+-1} from `seed`
 * (Alg. 1 l.2).  widths: K_0..K_L (n_widths = L + 1, 2..BMLP_MAX_LAYERS + 1,
 * each 1..32767); classes: 2..BMLP_MAX_CLASSES; h_max: odd, 1..16383 (255 = 8-bit
 * hidden weights, Table 4); hp may be NULL (paper defaults).  Allocates the
 * model state on the current CUDA device.  On success *out owns it. */
int bmlp_create(const int32_t* widths, int32_t n_widths, int32_t classes, int16_t h_max,
                uint64_t seed, const bmlp_hparams* hp, bmlp_t** out);

/* Free the model (synchronises the device first).  NULL is accepted. */
void bmlp_destroy(bmlp_t* h);

/* One pass of NetworkUpdate (Alg. 1 l.4-20) over n patterns in the given
 * order, in mini-batches of bs (a last shorter batch is processed as a batch of
 * its own size).  x_packed: n packed rows of K_0 bits; labels: n int32.
 * flags & BMLP_EPOCH_END: afterwards set E = (last-layer 01-loss count since the
 * previous epoch end) / (patterns since then) and p_r <- p_r sqrt(E).
 * n_errors_out (host, may be NULL): last-layer 01-loss count of these n
 * patterns, measured in the training forward pass.  n == 0 is a no-op.
 * If a bounded device-side wait of a training forward pass expires (tensor-
 * core engine), that mini-batch and every later one until the expiry is
 * reported change neither H nor W (no marks, no update; the step counter
 * still advances); the next call that synchronises returns BMLP_ETIMEOUT.
 * While cuda_stream is being captured the call returns BMLP_ECUDA and puts
 * nothing into it (a replay would run past the host's step count). */
int bmlp_train(bmlp_t* h, const uint64_t* x_packed, const int32_t* labels, int64_t n,
               uint32_t flags, void* cuda_stream, int64_t* n_errors_out);

/* Forward-only evaluation (Sec. 3.1): labels_out[mu] = argmax_j (a_L P_L)_{mu j}
 * (lowest index on ties) for n packed rows of K_0 bits.  Does not change state.
 * With device x_packed and labels_out the call does not synchronise, and an
 * expired bounded device wait (tensor-core engine) is reported by the next
 * call that does (BMLP_ETIMEOUT). */
int bmlp_predict(bmlp_t* h, const uint64_t* x_packed, int64_t n, int32_t* labels_out,
                 void* cuda_stream);

/* Early-exit evaluation (Sec. 3.1: after training, the intermediate random
 * classifiers P_l may serve early-exit strategies).  For every layer
 * l = 1..L: labels_out[(l-1) n + mu] = argmax_j of yhat_l = a_l P_l for
 * pattern mu (ties to the lowest class), a_l from the same forward pass as
 * bmlp_predict; row L equals bmlp_predict's output.  x_packed: as for
 * bmlp_predict; labels_out: L x n int32, layer-major, caller-owned, host or
 * device.  Asynchronous on cuda_stream when both pointers are device
 * pointers; synchronises otherwise.  Errors as bmlp_predict. */
int bmlp_predict_layers(bmlp_t* h, const uint64_t* x_packed, int64_t n, int32_t* labels_out,
                        void* cuda_stream);

/* Local error counts (Eq. 1 for every layer, Alg. 1 l.12): errs_out[l-1] =
 * the number of training patterns whose layer-l local 01-loss was 1 in their
 * training forward pass (the weights of their mini-batch before its update),
 * counted since creation or the last reset; errs_out[L-1] counts what
 * bmlp_train's n_errors_out reports.  errs_out: host, L values.  Synchronises
 * the device; reset != 0 sets the counters to 0 after reading them.  The
 * counters are not part of the state that bmlp_get_state / bmlp_set_state
 * carry. */
int bmlp_layer_errors(bmlp_t* h, int64_t* errs_out, int32_t reset);

/* MedianBinarization (Alg. 1 l.5; Sec. 3.2: the median value is the
 * threshold) of real-valued patterns, for data that is not already +-1:
 * bit i of pattern mu is 1 (+1) iff x[mu][i] > m_mu, where m_mu is the
 * ceil(K/2)-th smallest of the pattern's K values (its lower median) and the
 * comparison is made in fp32 (-0 and +0 are equal); else 0 (-1).  Pad bits
 * are 0, so the output is bmlp_train / bmlp_predict input for K_0 = K.
 *   x: device, n x K fp32, row-major, 4-byte aligned, finite values (a NaN
 *      ranks by its bit pattern and compares false); caller-owned.
 *   out: device, n x ceil(K/64) words, 8-byte aligned, caller-owned.
 * Needs no handle (errors read with bmlp_last_error(NULL)); asynchronous on
 * cuda_stream.  BMLP_EINVAL for n < 0, K < 1, NULL, host or misaligned
 * pointers; BMLP_ECUDA if the launch fails. */
int bmlp_binarize_median(const float* x, int64_t n, int32_t K, uint64_t* out, void* cuda_stream);

/* Weights of a fixed random expansion layer (Sec. 3.2, footnote to the
 * binarisation step: a fixed random input layer with weights in {+-1} and
 * sign activation lets the BMLP take non-binary inputs directly):
 * e_k,i = +1 iff bit 31 of word i%4 of Philox4x32-10 at counter
 * (i/4, k, 33*2^16, 0) with key (seed mod 2^32, seed div 2^32), else -1.
 *   E_out: device, K x ceil(D/64) words (bit i % 64 of word i / 64 of row k
 *          = 1 <-> e_k,i = +1; pad bits 0), 8-byte aligned, caller-owned.
 * No handle (errors: bmlp_last_error(NULL)); asynchronous on cuda_stream.
 * BMLP_EINVAL for K < 1, D < 1, D > 2^23, NULL, host or misaligned E_out. */
int bmlp_expand_weights(uint64_t seed, int32_t K, int32_t D, uint64_t* E_out, void* cuda_stream);

/* The expansion layer itself, for unsigned 8-bit inputs (pixel
 * intensities): bit k of pattern mu is 1 (+1) iff
 * sum_i x[mu][i] e_k,i >= 0 (sign(0) = +1, as for every activation), the
 * sum taken exactly in integers; else 0 (-1).  Pad bits are 0, so the output
 * is bmlp_train / bmlp_predict input for K_0 = K.
 *   x: device, n x D uint8, row-major (row mu at x + mu D), caller-owned;
 *      any alignment.
 *   E: device, K x ceil(D/64) words as written by bmlp_expand_weights (any
 *      +-1 matrix in that layout; pad bits ignored), 8-byte aligned.
 *   out: device, n x ceil(K/64) words, 8-byte aligned, caller-owned.
 * No handle (errors: bmlp_last_error(NULL)); asynchronous on cuda_stream.  A
 * bounded device-side wait that expires costs time only: the affected tiles are
 * computed again without waits, so the output is always whole.
 * BMLP_EINVAL for n < 0, K < 1, D < 1, D > 2^23 (the int32 sum bound),
 * NULL, host or misaligned pointers; BMLP_ECUDA if the launch fails. */
int bmlp_expand_sign(const uint8_t* x, int64_t n, int32_t D, const uint64_t* E, int32_t K,
                     uint64_t* out, void* cuda_stream);

/* bmlp_expand_sign with that path forced, for tests: every CTA of the
 * tensor-core kernel takes its device-side wait for its tile number
 * expired_tile (0, 1, ..) as expired.  expired_tile < 0: none. */
int bmlp_debug_expand_sign(const uint8_t* x, int64_t n, int32_t D, const uint64_t* E, int32_t K,
                           uint64_t* out, void* cuda_stream, int64_t expired_tile);

/* ---------------------------------------------------------------------------
 * 8-bit front end for real-valued rows (hidden states of a language model,
 * features of an encoder): like the expansion layer, a fixed layer in front of
 * the BMLP (Sec. 3.2, footnote to the binarisation step), for real inputs and
 * integer weights.  bmlp_norm_quantize takes rows to 8-bit codes,
 * bmlp_quantize_rows a weight matrix, and bmlp_int8_sign their product to
 * bmlp_train / bmlp_predict input; bmlp_int8_matmul gives the product itself.
 * The learning rule passes no gradient below its first layer, so none of the
 * four has a backward form.
 *
 * Common to the four: no handle (errors: bmlp_last_error(NULL)); every pointer
 * is memory of the current device (or managed), caller-owned; asynchronous on cuda_stream, nothing is
 * allocated; may be captured.  Row strides (ld...) are in elements and at
 * least the row's length where there is more than one row; rows may start at
 * any element.  n == 0 is a no-op.  Outputs may not overlap inputs except where
 * said.  BMLP_EINVAL for bad arguments, BMLP_ECUDA if a launch fails.
 * ------------------------------------------------------------------------- */

/* element types of real-valued buffers (BMLP_I32: bmlp_int8_matmul's output only) */
#define BMLP_F32 0
#define BMLP_F16 1
#define BMLP_BF16 2
#define BMLP_I32 3

#define BMLP_INT8_MAX_K 131071  /* K 2^14 < 2^31: no sum leaves int32 */

/* Symmetric 8-bit quantisation of rows: with A = max_i |x_i| of a row (fp32),
 *   q_i = rint(x_i * (127 / A)),  scale = A / 127   (each operation rounded to
 *   fp32, ties of rint to even), so x_i is about q_i * scale, |q_i| <= 127.
 * A < 127 * 2^-126: q = 0 and scale = 0.  A row with an infinity or a NaN: q = 0
 * and scale = NaN (products scaled by it are NaN).
 *   x: n x K of x_type, row stride ldx.  q: n x K, row stride ldq.  scale: n.
 * For the channels of a weight matrix n is their number. */
int bmlp_quantize_rows(const void* x, int32_t x_type, int64_t ldx, int64_t n, int32_t K, int8_t* q,
                       int64_t ldq, float* scale, void* cuda_stream);

/* Root-mean-square norm of rows with the residual's addition, to 8 bits:
 *   h = x + res (fp32; h = x where res is NULL),  sum_out = h (rounded to x_type),
 *   u_i = h_i * gain_i,  A = max_i |u_i|,  rstd = 1 / sqrt(mean_i h_i^2 + eps),
 *   q_i = rint(u_i * (127 / A)),  scale = (A / 127) * rstd
 * so h_i rstd gain_i is about q_i * scale.  rstd is common to the row, so the
 * codes do not depend on it.  Sums are held in fp32.  A < 127 * 2^-126: q = 0 and
 * scale = 0; a row whose A or sum of squares is not finite: q = 0, scale = NaN.
 *   x, res, sum_out: n x K of x_type, row strides ldx, ldr, lds; res and sum_out
 *     may be NULL.  sum_out may be x or res itself (same pointer and stride).
 *   gain: K values of x_type, or NULL (1).  eps >= 0 and finite (below 2^-80, where a
 *     row's squares may be too small for fp32 beside it, fp32 and bf16 rows take a
 *     slower kernel).
 *   q: n x K, row stride ldq.  scale: n. */
int bmlp_norm_quantize(const void* x, int64_t ldx, const void* res, int64_t ldr, const void* gain,
                       int32_t x_type, int64_t n, int32_t K, float eps, void* sum_out, int64_t lds,
                       int8_t* q, int64_t ldq, float* scale, void* cuda_stream);

/* Product of 8-bit integers with scales for each row and channel:
 *   S_ij = sum_k a_ik w_jk, exact;  out_ij = (S_ij * a_scale_i) * w_scale_j + bias_j
 * in fp32 (one rounding per operation), rounded to out_type; with BMLP_I32 S
 * itself (scales and bias NULL).
 *   a: n x K, row stride lda.  w: N x K, row stride ldw.  All 256 values allowed.
 *   a_scale: n, w_scale: N, bias: N; each may be NULL (1, 1, 0).
 *   out: n x N of out_type, row stride ldo.
 * K in 1..BMLP_INT8_MAX_K, N in 1..2^30.
 * workspace, workspace_bytes: see bmlp_int8_workspace.  A bounded device-side wait that
 * expires costs time only: the affected sums are made again without waits. */
int bmlp_int8_matmul(const int8_t* a, int64_t lda, const float* a_scale, const int8_t* w, int64_t ldw,
                     const float* w_scale, const float* bias, int64_t n, int32_t K, int32_t N, void* out,
                     int32_t out_type, int64_t ldo, void* workspace, int64_t workspace_bytes, void* cuda_stream);

/* bmlp_int8_matmul with the path of an expired device-side wait forced, for tests:
 * every CTA of its tensor-core kernels takes one as expired (up to 8 rows run
 * without such waits).  The affected sums are made again on CUDA cores, so the
 * output is whole, as it is where a bounded wait does expire. */
int bmlp_debug_int8_matmul(const int8_t* a, int64_t lda, const float* a_scale, const int8_t* w, int64_t ldw,
                           const float* w_scale, const float* bias, int64_t n, int32_t K, int32_t N, void* out,
                           int32_t out_type, int64_t ldo, void* workspace, int64_t workspace_bytes,
                           void* cuda_stream);

/* Signs of the same product, packed: bit j of row i is 1 (+1) iff
 * S_ij >= threshold_j (threshold: N int32, or NULL for 0: sign(0) = +1); exact.
 * Scales are positive, so they do not matter here; a row that was not finite has
 * codes of 0 and with them sums of 0 (its NaN scale tells it).  out: n rows of ceil(N/64)
 * words, 8-byte aligned, pad bits 0: bmlp_train / bmlp_predict input for
 * K_0 = N. */
int bmlp_int8_sign(const int8_t* a, int64_t lda, const int8_t* w, int64_t ldw, const int32_t* threshold,
                   int64_t n, int32_t K, int32_t N, uint64_t* out, void* workspace, int64_t workspace_bytes,
                   void* cuda_stream);

/* bmlp_int8_sign with the path of an expired device-side wait forced, as
 * bmlp_debug_int8_matmul, for tests. */
int bmlp_debug_int8_sign(const int8_t* a, int64_t lda, const int8_t* w, int64_t ldw, const int32_t* threshold,
                         int64_t n, int32_t K, int32_t N, uint64_t* out, void* workspace, int64_t workspace_bytes,
                         void* cuda_stream);

/* Workspace with which bmlp_int8_matmul and bmlp_int8_sign run fastest for this
 * size, in bytes: 0 for few rows, else room for both operands in fp16 (rows in
 * slabs, so it does not grow past 65,536 of them).  The two calls take a device
 * buffer of at least this size, 16-byte aligned, written and read on cuda_stream
 * (not shared by calls that overlap), or NULL / a smaller one: the same results
 * without it, slower.  Host only; 0 for sizes that the calls refuse. */
int64_t bmlp_int8_workspace(int64_t n, int32_t K, int32_t N);

/* ---------------------------------------------------------------------------
 * Microscaled 4-bit front end (no counterpart in the paper): the real-valued rows
 * of the 8-bit front end at half the bytes, by the 4-bit kind of the tensor cores.
 * bmlp_mx4_norm_quantize takes hidden states, bmlp_mx4_quantize a weight matrix or
 * rows that are normed already, and bmlp_mx4_matmul gives their product (whose
 * fp32 rows bmlp_binarize_median takes to bmlp_train / bmlp_predict input),
 * bmlp_mx4_matmul_grouped that with a weight matrix for each group of rows, such as
 * the tokens of each expert.  bmlp_mx4_dequantize gives the values that codes
 * stand for.
 *
 * Format (the microscaling format MXFP4 of the Open Compute Project): a row of K
 * values is ceil(K/2) bytes of codes, value 2 i in the low four bits of byte i,
 * and ceil(K/32) scale bytes, one for each 32 values.  A code is e2m1: bit 3 the
 * sign, bits 2..0 = 0..7 the size 0, 1/2, 1, 3/2, 2, 3, 4, 6.  Scale byte s is
 * 2^(s - 127); 255 is NaN, and so is every value and sum that it scales.  For odd K
 * the high bits of a row's last byte are 0.
 *
 * Common to the five: no handle (errors: bmlp_last_error(NULL)); every pointer is
 * memory of the current device (or managed), caller-owned; asynchronous on
 * cuda_stream, nothing is allocated and no workspace needed; may be captured.
 * Row strides are in elements for real values and in bytes for codes and scales,
 * and at least the row's length where there is more than one row; rows may start
 * anywhere (which runs fastest: bmlp_mx4_matmul).  n in 0..BMLP_MX4_MAX_ROWS, 0 is a no-op.  Outputs may not
 * overlap inputs except where said.  BMLP_EINVAL for bad arguments, BMLP_ECUDA if a
 * launch fails.  None has a backward form, as the 8-bit front end.
 * ------------------------------------------------------------------------- */
#define BMLP_MX4_MAX_ROWS (1 << 30)
#define BMLP_MX4_MAX_GROUPS 4096

/* Rows to codes and scales.  Of each 32 values of a row (the last block may have fewer),
 * with m = max |x_i|:
 *   s = max(0, floor(log2 m) - 2 + 127),   code_i = e2m1(x_i 2^(127 - s))
 * where e2m1 rounds to the nearest (ties to the even code) and what is above 6
 * becomes 6; m = 0 gives s = 0.  A block with an infinity or a NaN: codes 0, s = 255.
 *   x: n x K of x_type, row stride ldx.  q: n x ceil(K/2), row stride ldq.
 *   scale: n x ceil(K/32), row stride lds. */
int bmlp_mx4_quantize(const void* x, int32_t x_type, int64_t ldx, int64_t n, int32_t K, uint8_t* q,
                      int64_t ldq, uint8_t* scale, int64_t lds, void* cuda_stream);

/* Root-mean-square norm of rows with the residual's addition, to the same codes:
 *   h = x + res (fp32; h = x where res is NULL),  sum_out = h (rounded to x_type),
 *   u_i = h_i * gain_i,   codes and scales of u as above,
 *   row_scale = 1 / sqrt(mean_i h_i^2 + eps)
 * so h_i row_scale gain_i is about code_i 2^(s - 127) row_scale: the factor that is
 * common to the row stays outside of the codes (bmlp_mx4_matmul takes it).  Sums are
 * held in fp32; a row whose sum of squares is not finite: row_scale = NaN; a row of
 * zeros with eps = 0: row_scale = 0.
 *   x, res, sum_out: n x K of x_type, row strides ldx, ldr, ldsum; res and sum_out
 *     may be NULL.  sum_out may be x or res itself (same pointer and stride).
 *   gain: K values of x_type, or NULL (1).  eps >= 0 and finite.
 *   q, scale: as for bmlp_mx4_quantize.  row_scale: n. */
int bmlp_mx4_norm_quantize(const void* x, int64_t ldx, const void* res, int64_t ldr, const void* gain,
                           int32_t x_type, int64_t n, int32_t K, float eps, void* sum_out, int64_t ldsum,
                           uint8_t* q, int64_t ldq, uint8_t* scale, int64_t lds, float* row_scale,
                           void* cuda_stream);

/* Values of codes: out = code 2^(s - 127), times row_scale where it is not NULL (fp32, one
 * rounding of the product), rounded to out_type (without row_scale exact in fp32 and bf16, but for
 * values of 2^128 on, which become infinite).
 *   q, scale: n rows of K codes and their scales.  row_scale: n, or NULL.
 *   out: n x K of out_type (BMLP_F32, BMLP_F16 or BMLP_BF16), row stride ldo. */
int bmlp_mx4_dequantize(const uint8_t* q, int64_t ldq, const uint8_t* scale, int64_t lds, const float* row_scale,
                        int64_t n, int32_t K, void* out, int32_t out_type, int64_t ldo, void* cuda_stream);

/* Product of such rows:
 *   S_ij = sum_b 2^(sa_ib - 127) 2^(sw_jb - 127) sum_{k in block b} a_ik w_jk
 *   out_ij = S_ij * row_scale_i + bias_j
 * with sums in fp32, the last two operations rounded one by one, and rounded to out_type.
 *   a, a_scale: n rows of K codes and their scales, row strides lda and ldas.
 *   w, w_scale: N rows (channels), row strides ldw and ldws.
 *   row_scale: n, bias: N (fp32); each may be NULL (1, 0).
 *   out: n x N of out_type (BMLP_F32, BMLP_F16 or BMLP_BF16), row stride ldo.
 * K in 1..2^31 - 1, N in 1..2^30; for odd K the unused four bits of a row of a or of w may
 * be anything if the other's are 0.
 * Buffers and strides (rows', and groups') of codes that are multiples of 16 bytes run fastest:
 * with codes at other places of either operand the product takes two to four times as long; with
 * scales at other places up to 1.25 times. */
int bmlp_mx4_matmul(const uint8_t* a, int64_t lda, const uint8_t* a_scale, int64_t ldas, const float* row_scale,
                    const uint8_t* w, int64_t ldw, const uint8_t* w_scale, int64_t ldws, const float* bias,
                    int64_t n, int32_t K, int32_t N, void* out, int32_t out_type, int64_t ldo, void* cuda_stream);

/* The same with E matrices of weights, rows offsets[e] <= i < offsets[e + 1] by the e-th.
 *   w, w_scale: E groups of N rows, group strides gw and gws (bytes).
 *   bias: E groups of N, group stride gb (elements), or NULL.
 *   offsets: E + 1 device integers, 0 <= offsets[0] <= .. <= offsets[E] <= n; read when the
 *     call runs, so they may be computed on the device.  Groups may be empty.  One that
 *     decreases or leaves 0..n is taken as the nearest value that does not.
 * Rows of no group (before offsets[0], from offsets[E] on) are left as they are, and
 * of their inputs nothing matters.  E in 1..BMLP_MX4_MAX_GROUPS. */
int bmlp_mx4_matmul_grouped(const uint8_t* a, int64_t lda, const uint8_t* a_scale, int64_t ldas,
                            const float* row_scale, const uint8_t* w, int64_t ldw, int64_t gw,
                            const uint8_t* w_scale, int64_t ldws, int64_t gws, const float* bias, int64_t gb,
                            const int32_t* offsets, int32_t E, int64_t n, int32_t K, int32_t N, void* out,
                            int32_t out_type, int64_t ldo, void* cuda_stream);

/* bmlp_mx4_matmul_grouped (offsets NULL: bmlp_mx4_matmul, E = 1) with the path of an expired
 * device-side wait forced, for tests: every CTA of its tensor-core kernels takes one as
 * expired.  The affected sums are made again on CUDA cores, so the output is whole,
 * as it is where a bounded wait does expire. */
int bmlp_debug_mx4_matmul(const uint8_t* a, int64_t lda, const uint8_t* a_scale, int64_t ldas,
                          const float* row_scale, const uint8_t* w, int64_t ldw, int64_t gw,
                          const uint8_t* w_scale, int64_t ldws, int64_t gws, const float* bias, int64_t gb,
                          const int32_t* offsets, int32_t E, int64_t n, int32_t K, int32_t N, void* out,
                          int32_t out_type, int64_t ldo, void* cuda_stream);

/* The same on the kernel of many rows (pairs of CTAs) whatever the sizes, for tests of it at its edges; expire:
 * as above, or 0.  BMLP_EINVAL for operands that it does not take: codes in rows (groups) that start
 * anywhere, or more than 256 groups. */
int bmlp_debug_mx4_pairs(const uint8_t* a, int64_t lda, const uint8_t* a_scale, int64_t ldas,
                         const float* row_scale, const uint8_t* w, int64_t ldw, int64_t gw,
                         const uint8_t* w_scale, int64_t ldws, int64_t gws, const float* bias, int64_t gb,
                         const int32_t* offsets, int32_t E, int64_t n, int32_t K, int32_t N, void* out,
                         int32_t out_type, int64_t ldo, int32_t expire, void* cuda_stream);

/* One layer of forward-only evaluation (Sec. 3.1; Alg. 1 l.8-9):
 * a_out = sign(a_in W_l), sign(0) = +1, for n packed rows.  a_in: n rows of
 * ceil(K_{l-1}/64) words (pad bits 0); a_out: n rows of ceil(K_l/64) words,
 * written with pad bits 0.  Both must be device pointers (else BMLP_EINVAL).
 * Runs the engine bmlp_predict uses for this handle; asynchronous on
 * cuda_stream.  An expired bounded device wait (tensor-core engine) is
 * reported by the next call that synchronises (BMLP_ETIMEOUT). */
int bmlp_layer_forward(bmlp_t* h, int32_t layer, const uint64_t* a_in, int64_t n,
                       uint64_t* a_out, void* cuda_stream);

/* bmlp_layer_forward on an engine chosen per call (the engine comparison of
 * the forward contraction, Alg. 1 l.8-9; Table 3 counts its XNOR/popcount
 * work): engine BMLP_FWD_POPC, BMLP_FWD_TCGEN05 or BMLP_FWD_B1MMA, whatever
 * the handle's own engine.  Same arguments, layouts and results as
 * bmlp_layer_forward (every engine gives the same bits); BMLP_EINVAL for
 * another engine (BMLP_FWD_S8MMA has no layer kernel). */
int bmlp_layer_forward_engine(bmlp_t* h, int32_t layer, int32_t engine, const uint64_t* a_in,
                              int64_t n, uint64_t* a_out, void* cuda_stream);

/* Copy layer `layer` (1..L) to host buffers (each may be NULL; formats above),
 * plus the current p_r and step counter t (mini-batches since creation). */
int bmlp_get_state(const bmlp_t* h, int32_t layer, int16_t* H_out, uint64_t* W_out,
                   int8_t* P_out, double* p_r_out, int64_t* step_out);

/* Resume: load H of layer `layer` (host, format above; NULL keeps it) and
 * re-derive W from it; set p_r and the step counter (step < 0 keeps both).
 * Values must be odd and within [-h_max, h_max], else BMLP_ESTATE and nothing
 * changes.  The epoch's error and pattern counters restart at 0. */
int bmlp_set_state(bmlp_t* h, int32_t layer, const int16_t* H_in, double p_r, int64_t step);

/* Model shape: any output may be NULL.  widths_out: L + 1 values; gamma_out: L. */
int bmlp_get_info(const bmlp_t* h, int32_t* n_layers, int32_t* widths_out, int32_t* classes,
                  int32_t* gamma_out, int32_t* bs, int32_t* fwd_impl);

/* One-line description of the last error on this handle ("" if none).  With
 * h == NULL: the last error of a call that had no handle (e.g. bmlp_create). */
const char* bmlp_last_error(const bmlp_t* h);

/* Group size chosen by the rule of Sec. 4.3 for a layer of K neurons: the
 * divisor of K closest to [75, 105], the largest among equally close ones;
 * -1 for K < 1.  Host only. */
int32_t bmlp_gamma_rule(int32_t K);

/* Thresholds of the reinforcement sampler (Alg. 3 l.5-12) for a block of n
 * inputs (1 <= n <= 64) of a layer of width K at p_r.  Each hidden weight is
 * reinforced independently with probability q = p_r sqrt(2 / (pi K)) (IEEE
 * double; >= 1 taken as 1).  The events of a neuron row are drawn per block
 * of 64 consecutive inputs (the last block shorter): the block has an event
 * iff its 32-bit draw U < any_out; its first event is at the least j with
 * V < first_out[j]; after an event at p the next is at p + 1 + g for the
 * least g <= n - 2 - p with V < gap_out[g], none if there is no such g (V the
 * block's successive 32-bit draws).  With thr(x) = ceil(x 2^32) (0 for
 * x <= 0, 2^32 for x >= 1) and (1-q)^m a left-to-right IEEE product:
 *   any_out = thr(1 - (1-q)^n), first_out[j] = thr((1 - (1-q)^(j+1)) /
 *   (1 - (1-q)^n)) for j < n, gap_out[g] = thr(1 - (1-q)^(g+1)) for g < n - 1.
 * first_out holds n values and gap_out n - 1 (caller-owned).  Host only;
 * BMLP_EINVAL for K < 1, n outside 1..64 or a NULL output. */
int bmlp_reinforce_tables(double p_r, int32_t K, int32_t n, uint64_t* any_out,
                          uint64_t* first_out, uint64_t* gap_out);

/* Debug view of the most recent training mini-batch (synchronises): for layer
 * `layer`, Z (bs x K_l int16 pre-activations), A (bs x ceil(K_l/64) packed
 * activations), mark (bs uint8, 1 = pattern in M_l), sel (bs x G_l int16,
 * selected neuron per group or -1).  Rows beyond the batch's size are stale.
 * Any output may be NULL. */
int bmlp_debug_last_step(const bmlp_t* h, int32_t layer, int16_t* Z, uint64_t* A,
                         uint8_t* mark, int16_t* sel);

/* Failure-path probe of the bounded device waits (no counterpart in the
 * paper): one CTA initialises an mbarrier and waits on its first phase with
 * the same bounded wait the tensor-core kernels use, limited to `seconds`
 * (0 < seconds <= 10) of SM clock.  arrive > 0: one arrival completes the
 * phase first, so the wait succeeds.  arrive <= 0: nothing arrives, the wait
 * gives up when the limit expires, the kernel counts it as a timeout and
 * returns (no trap, no fault; the context stays usable).  Synchronises; then,
 * for arrive >= 0, returns BMLP_ETIMEOUT if any timeout is pending (and clears
 * it), else BMLP_OK; for arrive < 0 returns BMLP_OK and leaves the expiry
 * pending, as an expired wait inside a training step would (the next call
 * that synchronises reports it). */
int bmlp_debug_wait_probe(bmlp_t* h, int32_t arrive, double seconds);

/* Per-kernel timing.  every = 0: off.  every = S > 0: every S-th training
 * mini-batch (counted by the step counter t) and every evaluation launch is
 * enqueued kernel by kernel between two CUDA events on the caller's stream; the
 * other mini-batches replay the captured step graph as usual.  Per kernel kind
 * the library accumulates the launch count and the summed device time when
 * the call ends (which then synchronises the stream).  kinds: 0 forward
 * (train), 1 local classifier + selection, 2 update (CP + R + repack),
 * 3 forward (predict), 4 predict output, 5 host-buffer copies, 6 drawing of
 * the reinforcement events by a kernel of its own (models of more than 20 M
 * hidden weights; in the replayed step graph it runs beside the forward
 * passes, in a sampled mini-batch alone; the update kernel of smaller models
 * draws them itself).
 * bmlp_launch_count: kernels this handle has launched since creation (graph
 * replays count each node). */
int bmlp_set_profiling(bmlp_t* h, int32_t every);
int bmlp_get_profile(const bmlp_t* h, int32_t kind, int64_t* launches, double* total_ms);
int bmlp_reset_profile(bmlp_t* h);
int64_t bmlp_launch_count(const bmlp_t* h);

/* Update-kernel statistics accumulated since creation or the last reset
 * (synchronises): neuron rows visited (layers with a non-empty M_l), rows
 * streamed (rows with at least one CP tuple; a row without tuple changes only
 * at its reinforcement events and keeps its W), and the algorithmic bytes the
 * rule touched: per streamed row its hidden weights read and written as the
 * library stores them (bit-sliced: the bits of h_max rounded up to a power of
 * two per weight, rows padded to 16 bytes) and its W row written, per group of
 * 32 weights with a reinforcement event in a row without tuple the group's
 * planes read and written.  Any output may be NULL; reset != 0 zeroes the
 * counters after reading them. */
int bmlp_update_stats(bmlp_t* h, int64_t* rows_out, int64_t* streamed_out, int64_t* bytes_out,
                      int32_t reset);

/* Failure injection for the allocation and launch paths (no counterpart in the
 * paper; it tests the library's clean-up without a GPU fault).  After
 * bmlp_debug_fail_alloc(n), n >= 1, the n-th memory allocation the library
 * makes from then on -- counting every cudaMalloc of a device buffer and the
 * pinned host block of bmlp_create, in any handle of the process -- fails as
 * if memory were exhausted: the call that needed it returns BMLP_ENOMEM
 * ("... (injected)"), a half-built handle is freed whole, and the injection
 * disarms itself.  n = 0 disarms it.  BMLP_EINVAL for n < 0.
 * bmlp_debug_alloc_stats: the number of allocations the library holds now,
 * over every live handle of the process, and their bytes (either output may
 * be NULL); a failed bmlp_create leaves both where they were.
 * bmlp_debug_fail_launch(n): the same for the n-th training mini-batch that is
 * launched kernel by kernel from then on (a call of one mini-batch, or one that
 * bmlp_set_profiling samples): its launch fails after the forward passes and
 * the call returns BMLP_ECUDA ("... (injected)"), with that mini-batch trained
 * on nothing.  Host only; none of these calls touches the device. */
int bmlp_debug_fail_alloc(int64_t nth);
int bmlp_debug_fail_launch(int64_t nth);
int bmlp_debug_alloc_stats(int64_t* live_allocs, int64_t* live_bytes);

/* Peak rate of one contraction unit on the current device (the engine
 * comparison for the forward XNOR/popcount term of Table 3; Alg. 1 l.8):
 * a kernel that keeps its operands on chip and issues only that unit's
 * instruction, `iters` iterations per thread (or per MMA-issuing thread),
 * timed between CUDA events after one untimed launch.  engine: BMLP_FWD_POPC
 * (32-bit XOR + popcount on CUDA cores, 32 bit-pairs each), BMLP_FWD_TCGEN05
 * (tcgen05.mma kind::f8f6f4 e4m3, M128 N256 K32), BMLP_FWD_B1MMA
 * (mma.sync m16n8k256 b1 xor.popc), BMLP_FWD_S8MMA (mma.sync m16n8k32 s8).
 * *bitpairs_per_s: multiply-accumulates (bit-pairs) per second over the whole
 * device; *ms_out (may be NULL): the timed launch.  Synchronises the device;
 * allocates a few bytes.  No handle (errors: bmlp_last_error(NULL));
 * BMLP_EINVAL for an unknown engine or iters outside 1..2^31; BMLP_ETIMEOUT
 * if the tcgen05 kernel's bounded completion wait expired. */
int bmlp_engine_peak(int32_t engine, int64_t iters, double* bitpairs_per_s, double* ms_out);

/* Forward-only evaluation that allocates no memory.  The paper has no
 * counterpart: this is bmlp_predict with its scratch moved into the library,
 * for callers that cannot call cudaMalloc -- code running in a host callback,
 * a real-time loop with a fixed memory plan, or a process whose device
 * allocator belongs to another runtime.  bmlp_predict allocates its
 * inter-layer activation buffers on first use; this call instead uses one
 * fixed 16 MiB device array inside the library (two buffers of 2^20 64-bit
 * words), which every GPU that loads the library holds until the process
 * exits.  Results equal bmlp_predict's.
 *   n * ceil(max_l K_l / 64) must not exceed 1,048,576 (n <= 8192 for
 *   8192-wide layers); a larger n returns BMLP_EINVAL before any work.
 *   x_packed and labels_out must be device pointers on the current device
 *   (or managed memory): staging host buffers would allocate; host pointers
 *   and other devices' pointers return BMLP_EINVAL.
 *   The first call on a device looks up the array's device address once
 *   (cudaGetSymbolAddress); make that first call before any stream capture.
 *   Every call shares the array and it keeps the last call's contents (each
 *   call writes every word it reads); calls whose GPU work overlaps -- on
 *   different streams, or from different handles -- race on it.
 *   Calls no cudaMalloc, cudaFree or allocating library routine. */
int bmlp_predict_noalloc(bmlp_t* h, const uint64_t* x_packed, int64_t n, int32_t* labels_out,
                         void* cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* BMLP_H_ */

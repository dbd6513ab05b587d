/*
 * adloco.h -- C ABI of the AdLoCo hot path on one B200 (sm_100a).
 *
 * The library computes, with hand-written CUDA kernels,
 *   - the approximate norm test that sizes the next local batch
 *     (paper, Section "Norm test": sigma^2_B, the batch rule b_{k+1}),
 *   - switch mode's accumulation of the test sums over micro-batches
 *     (Section "Mode switching"; first branch of Algorithm 3),
 *   - the outer step over K model instances (last loop of Algorithm 3),
 *   - the trainer merge (Algorithms 1 and 2).
 *
 * Conventions for every entry point
 *   - Returns an adloco_status (0 = ok, negative = error).  No exception, abort
 *     or trap crosses this boundary.  Argument errors are found on the host
 *     before anything is launched.
 *   - "dev" pointers are device memory owned by the caller; "host" pointers are
 *     host memory owned by the caller.  Base pointers of vector data must be
 *     16-byte aligned unless an entry point says otherwise (ADLOCO_ERR_ALIGNMENT
 *     if not).  The library owns only the workspace inside an adloco_ctx.
 *   - Work is enqueued on `stream` (a cudaStream_t passed as void*; NULL = the
 *     legacy default stream) and is asynchronous unless stated.  The streaming
 *     entry points (norm test, accumulate, finalize, inner-product test, host
 *     variants) share the ctx workspace: do not run two of them at the same
 *     time on one ctx.  The per-layer entry points (adloco_gram_sqnorm,
 *     adloco_linear_sqnorm, adloco_linear_sqnorm_group, adloco_embedding_sqnorm,
 *     adloco_vector_param_sqnorm), adloco_outer_step and adloco_merge use none of it and may be issued on
 *     several streams at once -- the layers of one micro-batch only add into
 *     n and into their own S, and alternating them on two streams overlaps
 *     one kernel's tail with the next one's start.  So may the operators between the
 *     linear layers (adloco_add_rmsnorm to adloco_blockscale_dequantize), of the linear layers in bf16
 *     and the loss (adloco_linear to adloco_token_logprobs_backward).
 *   - Sizes are int64_t element counts; all byte offsets are 64-bit inside.
 *   - There is no CPU fallback: without a usable CUDA device the calls fail
 *     with ADLOCO_ERR_CUDA.
 */
#ifndef ADLOCO_H
#define ADLOCO_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct adloco_ctx adloco_ctx;     /* device id and workspace */
typedef struct adloco_accum adloco_accum; /* switch-mode accumulator state */

typedef enum {
    ADLOCO_OK = 0,
    ADLOCO_ERR_INVALID_ARG = -1,
    ADLOCO_ERR_UNSUPPORTED = -2, /* a shape the kernels do not take; never a silent fallback */
    ADLOCO_ERR_ALIGNMENT = -3,
    ADLOCO_ERR_CUDA = -4,        /* a CUDA runtime/driver call failed; see adloco_last_cuda_error */
    ADLOCO_ERR_WORKSPACE = -5,
    ADLOCO_ERR_TIMEOUT = -6      /* a bounded wait inside a kernel ran out (device status word) */
} adloco_status;

typedef enum { ADLOCO_F32 = 0, ADLOCO_BF16 = 1 } adloco_dtype;

enum {
    ADLOCO_FLAG_GROW = 1,       /* b_req > b_cur */
    ADLOCO_FLAG_ACCUMULATE = 2, /* switch mode: b_req > switch_n * b_max */
    ADLOCO_FLAG_UNDEFINED = 4,  /* batch_count - ddof <= 0: no variance; b_req = max(1, b_cur) */
    ADLOCO_FLAG_ZERO_MEAN = 8,  /* ||gbar||^2 == 0: stat = +inf, b_req = b_cap or INT64_MAX */
    ADLOCO_FLAG_NONFINITE = 16  /* a sum is Inf or NaN (an overflowed gradient): variance = stat = 0
                                   are placeholders, b_req = max(1, b_cur); checked before the others */
};

/* Parameters of the batch rule and of switch mode.
 *   eta      threshold of the norm test, > 0 and finite
 *   ddof     variance normaliser is (b - ddof); 1 = unbiased sample variance
 *   b_cur    current batch size (only for the GROW flag and the UNDEFINED case)
 *   b_max    largest micro-batch the hardware holds (max_batch), >= 1
 *   b_cap    upper clamp on b_req, 0 = none
 *   switch_n switch multiplier n (the paper uses 2), >= 1 */
typedef struct {
    double eta;
    int32_t ddof;
    int32_t switch_n;
    int64_t b_cur;
    int64_t b_max;
    int64_t b_cap;
} adloco_test_params;

/* Sufficient statistics of one test (device memory, written by the kernels).
 *   sum_sqnorm  Q   = sum_i ||g_i||^2
 *   sum_sq_gsum      ||sum_i g_i||^2  (so ||gbar||^2 = sum_sq_gsum / b^2)
 *   centred_ss       sum_i ||g_i - gbar||^2 computed column-centred; valid iff has_centred
 *   batch_count b */
typedef struct {
    double sum_sqnorm;
    double sum_sq_gsum;
    double centred_ss;
    int64_t batch_count;
    int32_t has_centred;
    int32_t device_status; /* 0, or an adloco_status raised on the device */
} adloco_test_sums;

/* Outcome of the test.  mean_sqnorm = ||gbar||^2, variance = sigma^2_B,
 * stat = variance / (eta^2 mean_sqnorm), b_req = max(1, ceil(stat)) clamped by b_cap;
 * accum_steps / b_micro are the switch-mode plan. */
typedef struct {
    double sum_sqnorm;
    double mean_sqnorm;
    double variance;
    double stat;
    int64_t batch_count;
    int64_t b_req;
    int64_t accum_steps;
    int64_t b_micro;
    uint32_t flags;
    int32_t device_status;
} adloco_test_result;

/* ---- context ------------------------------------------------------------ */

/* Creates a context on CUDA device `device` (allocates about 10 MB of workspace, sized
 * for the largest batch the streaming entry points take, so that none of them allocates
 * or synchronises later; synchronous).  *out is NULL on failure. */
int adloco_create(adloco_ctx** out, int device);
/* Frees the workspace.  The caller must have synchronised every stream that used it. */
int adloco_destroy(adloco_ctx* ctx);
const char* adloco_status_string(int status);
/* Text of the last CUDA error seen by this ctx ("" if none); valid until the next call. */
const char* adloco_last_cuda_error(const adloco_ctx* ctx);
/* Number of kernel launches this ctx has enqueued so far. */
int64_t adloco_launch_count(const adloco_ctx* ctx);

/* The tensor-core kernels wait on hardware barriers (tile arrived, accumulator
 * drained).  Every such wait is bounded: when `limit_ns` of wall time pass the
 * kernel stops waiting, lets its copies in flight land, frees its tensor memory,
 * returns, and raises the context's device status word to ADLOCO_ERR_TIMEOUT; the
 * outputs of that call are then undefined but the context stays usable.  Default
 * 2 s.  adloco_device_status reads the word (synchronises `stream`) and
 * optionally clears it. */
int adloco_set_wait_limit(adloco_ctx* ctx, uint64_t limit_ns);
int adloco_device_status(adloco_ctx* ctx, int32_t* status_host, int clear, void* stream);

/* ---- norm test on materialised per-sample gradients ---------------------- */

/* Section "Norm test" (Eq. 1, sigma^2_B, b_{k+1}) followed by the switch-mode
 * plan (Section "Mode switching").
 *   grads              dev, [B, P] row-major, row i = g_i, row pitch `row_stride`
 *                      elements (>= P), dtype F32 or BF16 (widened exactly, fp32 arithmetic).
 *                      Vector loads are used when the base is 16-byte (F32) / 8-byte (BF16)
 *                      aligned and the pitch is a multiple of 4 (and grad_sum, if given, is
 *                      16-byte aligned); otherwise a slower element-wise path runs.
 *                      1 <= B <= 4096.
 *   per_sample_sqnorm  dev [B] float, receives n_i = ||g_i||^2; may be NULL
 *   grad_sum           dev [P] float, receives S = sum_i g_i; may be NULL
 *   sums_dev           dev, receives the sufficient statistics; may be NULL
 *   result_dev         dev, receives the decision; required
 *   result_host        host copy of the decision, valid after `stream` is synchronised; may be NULL.
 *                      Page-locked memory (cudaHostAlloc, cudaHostRegister) is written by the kernel
 *                      itself, which keeps a copy engine out of the stream (about 11 us per call);
 *                      pageable memory is filled by an async copy on `stream`.  The same holds for
 *                      every result_host of this library.
 * One pass over G: per-row sum of squares, per-column sum and column-centred
 * sum of squares, fp32 inside a thread, fp64 across threads and blocks (fixed
 * order: results are run-to-run deterministic).  B >= 1, P >= 1. */
int adloco_norm_test(adloco_ctx* ctx, const void* grads, adloco_dtype dtype, int64_t B, int64_t P,
                     int64_t row_stride, const adloco_test_params* params, float* per_sample_sqnorm,
                     float* grad_sum, adloco_test_sums* sums_dev, adloco_test_result* result_dev,
                     adloco_test_result* result_host, void* stream);

/* The batch rule and switch plan alone, from sufficient statistics already on
 * the device (e.g. to sweep eta without re-reading the gradients). */
int adloco_test_decide(adloco_ctx* ctx, const adloco_test_sums* sums_dev, const adloco_test_params* params,
                       adloco_test_result* result_dev, adloco_test_result* result_host, void* stream);

/* Same as adloco_norm_test with `grads_host` in HOST memory ([B, P], pitch
 * row_stride): the library stages column panels through device buffers it owns,
 * overlapping the copies with the reduction.  Synchronous: on return
 * *result_host (required) and the optional host outputs per_sample_sqnorm_host
 * [B] are valid. */
int adloco_norm_test_host(adloco_ctx* ctx, const float* grads_host, int64_t B, int64_t P, int64_t row_stride,
                          const adloco_test_params* params, float* per_sample_sqnorm_host,
                          adloco_test_result* result_host, void* stream);

/* Norm test for callers that must not allocate.  The paper has no counterpart:
 * this is adloco_norm_test (same kernel, same results) with the reduction
 * scratch in a device array built into the library (about 290 KB per GPU, held
 * from library load to process exit) instead of an adloco_ctx, for callers that
 * cannot call cudaMalloc where the test runs -- e.g. inside a step whose
 * allocator pool is frozen, or with the device-memory budget already spent.
 * It calls no cudaMalloc/cudaFree and no allocating library routine.
 *   - runs on the CURRENT device, on `stream`; grads/per_sample_sqnorm (may be
 *     NULL)/result_dev are caller-owned dev memory, result_host (may be NULL) is
 *     filled by an async copy as in adloco_norm_test
 *   - limit: B <= 64 rows (ADLOCO_ERR_UNSUPPORTED beyond); any P >= 1
 *   - the first call on each device looks up the array's device address; make
 *     that first call before any stream capture
 *   - every call shares the one array: calls that overlap on the GPU (different
 *     streams, or different threads) race and give wrong results; calls on one
 *     stream are safe back to back. */
int adloco_norm_test_noalloc(const float* grads, int64_t B, int64_t P, int64_t row_stride,
                             const adloco_test_params* params, float* per_sample_sqnorm,
                             adloco_test_result* result_dev, adloco_test_result* result_host, void* stream);

/* ---- inner-product test and augmented inner-product test ------------------ */

/* Parameters: theta and nu are the thresholds of the two tests (> 0, finite);
 * ddof, b_cur, b_cap as in adloco_test_params. */
typedef struct {
    double theta;
    double nu;
    int32_t ddof;
    int32_t reserved;
    int64_t b_cur;
    int64_t b_cap;
} adloco_ip_params;

/* var_ip = Var_i <g_i, gbar>, stat_ip = var_ip / (theta^2 ||gbar||^4), b_ip = max(1, ceil(stat_ip));
 * var_orth = Var_i (g_i - (<g_i, gbar> / ||gbar||^2) gbar), stat_orth = var_orth / (nu^2 ||gbar||^2),
 * b_aug = max(b_ip, ceil(stat_orth)).  Flags GROW (b_aug > b_cur), UNDEFINED, ZERO_MEAN, NONFINITE as for the
 * norm test. */
typedef struct {
    double var_ip;
    double stat_ip;
    double var_orth;
    double stat_orth;
    double mean_sqnorm;
    int64_t batch_count;
    int64_t b_ip;
    int64_t b_aug;
    uint32_t flags;
    int32_t device_status;
} adloco_ip_result;

/* Section "Inner product test": both batch rules for the batch whose norm test
 * has just run.  A second pass over G:
 *   grads, B, P, row_stride   as in adloco_norm_test (the same G)
 *   grad_sum                  dev [P] float: S = sum_i g_i, the grad_sum output of that norm test (required)
 *   sums_dev                  dev: the sums_dev output of that norm test (required)
 *   inner_products            dev [B] float, receives <g_i, gbar>; may be NULL
 *   result_dev / result_host  as in adloco_norm_test
 * Algorithmic traffic 4 B P + 4 P bytes. */
int adloco_inner_product_test(adloco_ctx* ctx, const void* grads, adloco_dtype dtype, int64_t B, int64_t P,
                              int64_t row_stride, const adloco_ip_params* params, const float* grad_sum,
                              const adloco_test_sums* sums_dev, float* inner_products,
                              adloco_ip_result* result_dev, adloco_ip_result* result_host, void* stream);

/* ---- per-sample norms of a linear layer via the Gram identity ------------ */

/* For a linear layer y = W x and a batch of B sequences of T tokens, sample i
 * has weight gradient G_i = sum_t delta_{i,t} x_{i,t}^T (Eq. 1 applied to W).
 * This call computes, on the tensor cores,
 *   n_i = ||G_i||_F^2 = sum_{t,s} (x_t . x_s)(delta_t . delta_s)     (Gram identity)
 *   S   = sum_i G_i = Delta^T X  ([d_out, d_in], fp32 accumulate)     (optional)
 *   X  dev bf16 [B, T, d_in]  row-major (features contiguous)
 *   D  dev bf16 [B, T, d_out] row-major
 *   per_sample_sqnorm  dev [B] float; overwritten, or += when accumulate_norms != 0
 *   grad_sum           dev [d_out, d_in] float, may be NULL; overwritten, or += when
 *                      accumulate_sum != 0
 * d_in and d_out must be multiples of 8 (ADLOCO_ERR_UNSUPPORTED otherwise); any
 * B, T >= 1.  bf16 x bf16 products are exact in fp32; accumulation is fp32. */
int adloco_gram_sqnorm(adloco_ctx* ctx, const void* X, const void* D, int64_t B, int64_t T, int64_t d_in,
                       int64_t d_out, float* per_sample_sqnorm, int accumulate_norms, float* grad_sum,
                       int accumulate_sum, void* stream);

/* Same outputs as adloco_gram_sqnorm (n_i and, optionally, S; same argument
 * meaning and limits) with a choice of route:
 *   ADLOCO_LINEAR_GRAM    the Gram identity (adloco_gram_sqnorm)
 *   ADLOCO_LINEAR_DIRECT  each sample's gradient tile G_i = D_i^T X_i (Eq. 1 applied to
 *                         W, before the mean) is formed in tensor memory, squared and
 *                         summed into n_i and added into S on chip; G_i never reaches HBM.
 *                         One GEMM of 2 B T d_in d_out flops gives both outputs.
 *   ADLOCO_LINEAR_DIRECT_PAIR  the direct route with 256 x 256 tiles, each shared by the two
 *                         SMs of a thread-block cluster (each loads half of the operands);
 *                         ADLOCO_ERR_UNSUPPORTED where cluster launches are not available.
 *   ADLOCO_LINEAR_GRAM_ONE_CTA / ADLOCO_LINEAR_GRAM_PAIR  the Gram identity by a named kernel: one CTA
 *                         per 128 x 256-token tile (what ADLOCO_LINEAR_GRAM and adloco_gram_sqnorm run), or
 *                         256 x 256-token tiles shared by the two SMs of a cluster (same result; a third less
 *                         traffic into shared memory and one read of the operands from HBM, for one unused
 *                         128 x 128 sub-block per diagonal tile; measured as fast as the one-CTA kernel at
 *                         T = 1024; ADLOCO_ERR_UNSUPPORTED where cluster launches are not available).
 *   ADLOCO_LINEAR_AUTO    whichever executes fewer tensor-core flops for the shape
 *                         (direct wins when T exceeds about d_in d_out / (d_in + d_out));
 *                         the direct route then runs in its pair form where available. */
enum { ADLOCO_LINEAR_AUTO = 0, ADLOCO_LINEAR_GRAM = 1, ADLOCO_LINEAR_DIRECT = 2, ADLOCO_LINEAR_DIRECT_PAIR = 3,
       ADLOCO_LINEAR_GRAM_ONE_CTA = 4, ADLOCO_LINEAR_GRAM_PAIR = 5 };
int adloco_linear_sqnorm(adloco_ctx* ctx, const void* X, const void* D, int64_t B, int64_t T, int64_t d_in,
                         int64_t d_out, float* per_sample_sqnorm, int accumulate_norms, float* grad_sum,
                         int accumulate_sum, int method, void* stream);

/* One linear layer of a group: X dev bf16 [B, T, d_in], D dev bf16 [B, T, d_out],
 * grad_sum dev float [d_out, d_in] or NULL; d_in, d_out multiples of 8. */
typedef struct {
    const void* X;
    const void* D;
    int64_t d_in;
    int64_t d_out;
    float* grad_sum;
} adloco_linear_layer;

/* All linear layers of one (micro-)batch in one call (Eq. 1 applied per weight matrix; a
 * sample's gradient is the concatenation over the layers, so its squared norm adds up):
 *   per_sample_sqnorm[i] (+)= sum over the layers of ||D_i^T X_i||_F^2,
 *   layers[l].grad_sum   (+)= sum_i D_i^T X_i   for every layer that gives a buffer.
 *   layers   HOST array of n_layers entries (read during the call); all layers share B and T
 *   method   ADLOCO_LINEAR_DIRECT, ADLOCO_LINEAR_DIRECT_PAIR or ADLOCO_LINEAR_AUTO (the pair
 *            kernel where available, else the direct one)
 * The direct route runs the whole group as one persistent launch per 48 layers: the work
 * items of all layers are dealt to the SMs from one list, so small layers pay no launch of
 * their own and layers whose tile count does not divide the SM count leave no SM idle.
 * accumulate_norms / accumulate_sum as in adloco_gram_sqnorm, applied to every layer. */
int adloco_linear_sqnorm_group(adloco_ctx* ctx, const adloco_linear_layer* layers, int32_t n_layers, int64_t B,
                               int64_t T, float* per_sample_sqnorm, int accumulate_norms, int accumulate_sum,
                               int method, void* stream);

/* Per-sample gradient norms of a vector parameter of width d that acts at every
 * token (Eq. 1 applied to that parameter): a bias, g_i = sum_t delta_{i,t} (X = NULL),
 * or an elementwise gain such as LayerNorm's, g_i = sum_t delta_{i,t} * x_{i,t}
 * (X = the normalised input).  n_i = ||g_i||^2 and, optionally, S = sum_i g_i.
 *   D, X               dev bf16 [B, T, d] row-major; d a multiple of 8, B <= 65535
 *   per_sample_sqnorm  dev [B] float; overwritten, or += when accumulate_norms != 0
 *   grad_sum           dev [d] float, may be NULL; overwritten, or += when accumulate_sum != 0
 * One streaming pass (2 B T d bytes per operand), fp32 accumulation. */
int adloco_vector_param_sqnorm(adloco_ctx* ctx, const void* D, const void* X, int64_t B, int64_t T, int64_t d,
                               float* per_sample_sqnorm, int accumulate_norms, float* grad_sum, int accumulate_sum,
                               void* stream);

/* Per-sample gradient norms of an embedding table E [V, d] looked up at every token
 * (Eq. 1 applied to E): row v of sample i's gradient is the sum of delta_{i,t} over the
 * tokens with token_ids[i, t] = v, and n_i = sum_v || sum_{t: id_t = v} delta_t ||^2.
 * Up to T = 4096 the tokens of a sample are grouped by id on chip and every delta row is
 * read once (a streaming pass; ids that occur once contribute their row's squared norm,
 * repeated ids the squared norm of their rows' sum); longer sequences take the equivalent
 * n_i = sum_{t,s} [id_t == id_s] (delta_t . delta_s) -- the Gram identity with a
 * token-equality mask in place of X X^T -- on the tensor cores.
 * With position indices as ids it covers a learned positional embedding.
 *   token_ids          dev int32 [B, T], values in [0, V) (others match nothing and are skipped)
 *   D                  dev bf16 [B, T, d]: gradient of the loss w.r.t. the looked-up rows; d % 8 == 0
 *   per_sample_sqnorm  dev [B] float; overwritten, or += when accumulate_norms != 0
 *   grad_sum           dev [V, d] float, may be NULL: S = sum_i G_i (scatter-add); overwritten
 *                      (V d floats are cleared first), or += when accumulate_sum != 0 */
int adloco_embedding_sqnorm(adloco_ctx* ctx, const int32_t* token_ids, const void* D, int64_t B, int64_t T, int64_t d,
                            int64_t V, float* per_sample_sqnorm, int accumulate_norms, float* grad_sum,
                            int accumulate_sum, void* stream);

/* ---- between the linear layers ------------------------------------------------ */

/* The operators of a decoder block around its linear layers: norm, residual and dropout,
 * rotary positions, and the linear layer in 8-bit floating point.  Their backward passes
 * produce the X and Delta that the per-sample norms above read; the norm's own gain
 * contributes its per-sample norms in the same pass.  None of them uses the ctx workspace, so
 * all may be issued on several streams at once.  Rows are addressed by a pitch in elements, the
 * same one where an output may be the same memory as an input and is;
 * 16-byte aligned rows (base and pitch) take vector loads; others are slower, the norm's through shared memory. */

/* h = residual + drop(x);  y = gain * h / sqrt(mean(h^2) + eps) over each row of d elements.
 *   x, y          dev [rows, d] in dtype
 *   residual, h   dev [rows, d] in stream_dtype (BF16 or F32; F32 x with a BF16 stream is UNSUPPORTED).
 *                 residual NULL: h = drop(x).  h may be NULL (not kept), or the same memory as residual.
 *   gain          dev [d] in gain_dtype
 *   rstd          dev [rows] float, receives 1 / sqrt(mean(h^2) + eps) for the backward pass; may be NULL
 *   q, q_scale    y in 8 bits as adloco_blockscale_quantize writes it (from the unrounded y); both or
 *                 neither.  q [rows, d] bytes with pitch q_stride (a multiple of 16, q 16-byte aligned),
 *                 q_scale [rows, ceil(d / 128)] bytes with pitch q_scale_stride (a multiple of 4, q_scale 4-byte aligned)
 *   y             may be NULL when q is given
 *   dropout_p, seed, offset   as in adloco_dropout, element index row * d + column; 0 = none
 * Sums, the root and the norm are formed in fp32 from the unrounded h; every output is rounded to its type
 * once.  Where x is dropped h is exactly the residual; elsewhere residual + x s takes two fused fp32 operations
 * with s as the sum of two numbers.  1 <= d <= 16384. */
typedef struct {
    adloco_dtype dtype, stream_dtype, gain_dtype;
    float eps;
    int64_t rows, d;
    const void* x;
    int64_t x_stride;
    const void* residual;
    int64_t residual_stride;
    const void* gain;
    void* h;
    int64_t h_stride;
    void* y;
    int64_t y_stride;
    float* rstd;
    void* q;
    int64_t q_stride;
    uint8_t* q_scale;
    int64_t q_scale_stride;
    double dropout_p;
    uint64_t seed, offset;
} adloco_rmsnorm_args;
int adloco_add_rmsnorm(adloco_ctx* ctx, const adloco_rmsnorm_args* args, void* stream);

/* Backward pass of adloco_add_rmsnorm over B samples of T rows (rows = B T, sample-major).
 * With xhat = h rstd and m = mean(gain dy xhat) over the row:
 *   dh = dh_residual + rstd (gain dy - xhat m)      gradient of h, hence of residual
 *   dx = drop(dh)                                   gradient of x (the forward call's mask)
 * and for the gain g_i = sum_t dy_{i,t} xhat_{i,t}:  n_i = ||g_i||^2,  S = sum_i g_i.
 *   dy             dev [rows, d] in dtype;  h (the forward pass's), dh_residual, dh: in stream_dtype
 *   dh_residual    the gradient that reaches h along the residual stream; NULL = 0; may be dh itself
 *   dx             dev [rows, d] in dtype, may be NULL (without dropout dx equals dh) or dy itself
 *   per_sample_sqnorm, accumulate_norms, grad_sum, accumulate_sum   as in adloco_vector_param_sqnorm;
 *                  both pointers may be NULL (a frozen gain)
 *   workspace      dev, 16-byte aligned, at least adloco_add_rmsnorm_backward_workspace bytes; not
 *                  needed (NULL) when neither norms nor sum are asked for.  One call at a time may use it.
 * B <= 2^27, B T <= 2^30.  All sums are fp32 in a fixed order; only the addition of a sample's n_i to what other calls put
 * there is an atomic. */
typedef struct {
    adloco_dtype dtype, stream_dtype, gain_dtype;
    int32_t accumulate_norms, accumulate_sum, reserved;
    int64_t B, T, d;
    const void* dy;
    int64_t dy_stride;
    const void* h;
    int64_t h_stride;
    const float* rstd;
    const void* gain;
    const void* dh_residual;
    int64_t dh_residual_stride;
    void* dh;
    int64_t dh_stride;
    void* dx;
    int64_t dx_stride;
    double dropout_p;
    uint64_t seed, offset;
    float* per_sample_sqnorm;
    float* grad_sum;
    void* workspace;
    int64_t workspace_bytes;
} adloco_rmsnorm_backward_args;
int64_t adloco_add_rmsnorm_backward_workspace(const adloco_ctx* ctx, int64_t B, int64_t T, int64_t d);
int adloco_add_rmsnorm_backward(adloco_ctx* ctx, const adloco_rmsnorm_backward_args* args, void* stream);

/* y = residual + drop(x) (residual NULL: y = drop(x)), the mask never stored: element e = row * cols + column
 * stays when 16 bits drawn for it are at least r = round(p 65536), and is then multiplied by
 * 65536 / (65536 - r).  The bits are those of the counter-based generator Philox-4x32-10 (Salmon,
 * Moraes, Dror, Shaw 2011) with key = seed and counter = (e / 8, offset), word (e mod 8) / 2, low half
 * first.  The same (p, seed, offset) gives the same mask in every call and in adloco_add_rmsnorm, so the
 * backward pass of dropout is this call on the gradient.  A dropped element is exactly 0 whatever x holds
 * there, and y exactly the residual; p = 1 drops all.  The sum is formed in fp32 as adloco_add_rmsnorm's h.
 *   x, residual, y   dev [rows, cols] in dtype, pitches in elements; y may be the same memory as x or residual
 *   0 <= p <= 1 */
int adloco_dropout(adloco_ctx* ctx, adloco_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride,
                   const void* residual, int64_t residual_stride, void* y, int64_t y_stride, double p, uint64_t seed,
                   uint64_t offset, void* stream);

/* Frequencies of rotary positions for rot_dim (even) rotated elements a head: turns[j], j < rot_dim / 2, is
 * w_j / (2 pi) in units of 2^-64, so that a position's phase is the low 64 bits of position * turns[j] --
 * exact for any position, with no reduction of large angles.  HOST output.  w_j = base^(-2 j / rot_dim), then
 *   NONE      as it is
 *   LINEAR    w_j / factor                                       (positions squeezed)
 *   NTK       base replaced by base factor^(rot_dim / (rot_dim - 2))   (the slowest pair slows by factor)
 *   BY_PARTS  u w_j + (1 - u) w_j / factor with u = clamp((w_j context / (2 pi) - low) / (high - low), 0, 1):
 *             pairs that turn more than `high` times within `context` positions keep their speed, pairs that
 *             turn fewer than `low` times are squeezed
 * base > 1 is not required, but base > 0, factor > 0, and for BY_PARTS high > low and context > 0. */
enum { ADLOCO_ROPE_NONE = 0, ADLOCO_ROPE_LINEAR = 1, ADLOCO_ROPE_NTK = 2, ADLOCO_ROPE_BY_PARTS = 3 };
int adloco_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double context, double low,
                            double high, uint64_t* turns_host);

/* One tensor of heads [B, T, heads, head_dim] with strides in elements (head_dim contiguous). */
typedef struct {
    const void* in;
    void* out;         /* the same memory and strides as `in`, or no overlap; its heads must not fall on one another */
    int64_t heads;
    int64_t in_batch, in_token, in_head;
    int64_t out_batch, out_token, out_head;
} adloco_rope_tensor;
/* Rotates the first rot_dim elements of every head by the phase of its token's position and copies the rest:
 *   (a, b) -> magnitude (a cos - b sin, a sin + b cos)
 * over the pairs (x_j, x_{j + rot_dim / 2}) or, interleaved, (x_{2j}, x_{2j+1}).  inverse != 0 turns the other
 * way, which is the backward pass (the rotation's transpose).
 *   tensors     HOST array of 1..4 entries (queries and keys of different head counts go in one call)
 *   turns_dev   dev copy of adloco_rope_frequencies' table
 *   positions   dev int32 [B, T] with pitch positions_stride, or NULL: position first_position + t
 * Phase arithmetic is exact, every output rounded once; sine and cosine are fp32's for F32 and those of the fast
 * instructions for BF16 (off by 2^-21, against the output's rounding of 2^-9). */
int adloco_rope(adloco_ctx* ctx, adloco_dtype dtype, const adloco_rope_tensor* tensors, int32_t n_tensors, int64_t B,
                int64_t T, int64_t head_dim, int64_t rot_dim, const uint64_t* turns_dev, float magnitude,
                const int32_t* positions, int64_t positions_stride, int64_t first_position, int interleaved, int inverse,
                void* stream);

/* ---- 8-bit floating point with a scale for each block of 128 --------------------- */

/* Values are e4m3 (largest 448); a block's scale is the power of two 2^(s - 127), s its byte, the smallest for
 * which the block's largest magnitude is at most 448 (a block of zeros has scale 1).  Multiplying by it is exact,
 * so the only rounding is the one to e4m3 (to nearest, ties to even).  A block that holds an Inf or NaN gets
 * s = 255, which stands for NaN: every product with it is NaN.
 *
 * Rows (activations and gradients): one scale for 128 consecutive elements of a row.
 *   x      dev [rows, cols] in dtype, pitch x_stride
 *   q      dev [rows, cols] bytes, pitch q_stride a multiple of 16, 16-byte aligned
 *   scale  dev [rows, ceil(cols / 128)] bytes, pitch scale_stride a multiple of 4, 4-byte aligned (the product
 *          reads whole aligned words; what a row's last word holds beyond its blocks does not matter) */
int adloco_blockscale_quantize(adloco_ctx* ctx, adloco_dtype dtype, int64_t rows, int64_t cols, const void* x,
                               int64_t x_stride, void* q, int64_t q_stride, uint8_t* scale, int64_t scale_stride,
                               void* stream);
/* Weights: one scale for each 128 x 128 block of W [rows, cols]; optionally the transposed copy too, which the
 * backward pass multiplies by (its scales are the same ones, transposed).
 *   q      dev [rows, cols] bytes, pitch q_stride;  q_t  dev [cols, rows] bytes, pitch q_t_stride, may be NULL
 *   scale  dev [ceil(rows / 128), ceil(cols / 128)] bytes, pitch scale_stride (any, >= its columns) */
int adloco_blockscale_quantize_weight(adloco_ctx* ctx, adloco_dtype dtype, int64_t rows, int64_t cols, const void* W,
                                      int64_t W_stride, void* q, int64_t q_stride, void* q_t, int64_t q_t_stride,
                                      uint8_t* scale, int64_t scale_stride, void* stream);

/* out [M, N] = A B^T (+ bias) with A [M, K] in rows' form and B [N, K] in weights' form:
 *   out_mn = sum_k 2^(sa(m, k / 128) - 127) a_mk 2^(sb(n / 128, k / 128) - 127) b_nk (+ bias_n)
 *   a, a_scale       as adloco_blockscale_quantize writes them (same pitch rules)
 *   b                dev [N, K] bytes, pitch b_stride a multiple of 16, 16-byte aligned
 *   b_scale          dev bytes; the block (n / 128, k / 128) is at n / 128 * b_scale_stride_n + k / 128 * b_scale_stride_k,
 *                    so the transposed copy of a weight uses the weight's own scales with the strides exchanged
 *   bias             dev [N] float, may be NULL
 *   out              dev [M, N] in out_dtype, pitch out_stride; rows that are 16-byte aligned take the fast stores
 * The layer y = x W^T is this call on (x, W); its input gradient dx = dy W on (dy, transposed copy of W).
 * Tensor cores apply the scales; accumulation is fp32, the output is rounded once. */
typedef struct {
    int64_t M, N, K;
    const void* a;
    int64_t a_stride;
    const uint8_t* a_scale;
    int64_t a_scale_stride;
    const void* b;
    int64_t b_stride;
    const uint8_t* b_scale;
    int64_t b_scale_stride_n, b_scale_stride_k;
    const float* bias;
    void* out;
    int64_t out_stride;
    adloco_dtype out_dtype;
    int32_t reserved;
} adloco_blockscale_matmul_args;
int adloco_blockscale_matmul(adloco_ctx* ctx, const adloco_blockscale_matmul_args* args, void* stream);

/* The values that rows in 8 bits stand for (adloco_blockscale_quantize's, or what the linear layers below keep), rounded to
 * dtype: exact but where a value leaves its range (a block with the byte 255 is all NaN).  This is how an activation kept
 * in 8 bits comes back as the X of adloco_linear_sqnorm.
 *   q, scale  as adloco_blockscale_quantize writes them (same rules);  x  dev [rows, cols] in dtype, pitch x_stride */
int adloco_blockscale_dequantize(adloco_ctx* ctx, adloco_dtype dtype, int64_t rows, int64_t cols, const void* q,
                                 int64_t q_stride, const uint8_t* scale, int64_t scale_stride, void* x, int64_t x_stride,
                                 void* stream);

/* ---- linear layers in bf16, alone and as the gated feed-forward -------------------- */

/* The products of a decoder's layers with what follows them in the same pass, forward and backward.  The gradients of the
 * weights, with their per-sample norms, are adloco_linear_sqnorm's, on the x and the gradients that these calls take and
 * return.  Operands of a product (x, w, dy) are bf16 with 16-byte aligned rows (base, and a pitch that is a multiple of 8);
 * other tensors may have any pitch, 16-byte aligned rows being the fast ones.  Products are exact, sums fp32: the tensor
 * cores' own in bf16 outputs (they cut off low bits: a relative error of 1e-6 after 1000 terms), with every 512 terms added
 * up to nearest where an output is F32 or what is kept goes to 8 bits; every output is rounded once.  An output may be the same
 * memory as an elementwise operand (residual, z, gate, up) of the same type and pitch; any other overlap of an output, scales
 * among them, is refused.
 * Activations and their derivatives have their limits at the infinities, and a NaN at a NaN.
 * None of them uses the ctx workspace. */
typedef enum {
    ADLOCO_ACT_NONE = 0,
    ADLOCO_ACT_RELU = 1,
    ADLOCO_ACT_GELU = 2,        /* z (1 + erf(z / sqrt 2)) / 2, to 2e-7 */
    ADLOCO_ACT_GELU_TANH = 3,   /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2 */
    ADLOCO_ACT_SILU = 4         /* z / (1 + exp(-z)) */
} adloco_activation;

/* A matrix that the forward pass keeps for the backward one: bf16 (scale NULL), or 8 bits with a power-of-two scale for each
 * 128 elements of a row, as adloco_blockscale_quantize writes them from the unrounded values (its rules for pitches and
 * alignment; bf16: 16-byte aligned rows).  p NULL: not kept. */
typedef struct {
    void* p;
    int64_t stride;
    uint8_t* scale;
    int64_t scale_stride;
} adloco_kept;

/* z = x w^T + bias;  y = residual + act(z)
 *   x [M, K], w [N, K] dev bf16;  bias dev [N] float, may be NULL
 *   residual, y  dev [M, N] in out_dtype;  residual may be NULL
 *   z            kept for adloco_linear_backward of the next layer, [M, N]; optional.  (With an activation and a residual together the
 *                next layer's input is their sum, whose way back these calls do not have.) */
typedef struct {
    int64_t M, N, K;
    const void* x;
    int64_t x_stride;
    const void* w;
    int64_t w_stride;
    const float* bias;
    const void* residual;
    int64_t residual_stride;
    void* y;
    int64_t y_stride;
    adloco_kept z;
    int32_t activation;
    adloco_dtype out_dtype;
} adloco_linear_args;
int adloco_linear(adloco_ctx* ctx, const adloco_linear_args* args, void* stream);

/* The way back through a layer y = a w^T and through the activation a = act(z) that made its input:
 *   dx = residual + (dy w) act'(z)          a = act(z), recomputed for the weight's gradient
 *   dy [M, N], w [N, K] dev bf16 (the forward call's w, as it lies)
 *   z         what the forward pass kept, [M, K]; may be NULL where activation is NONE
 *   residual, dx  dev [M, K] in out_dtype; residual may be NULL
 *   a         dev [M, K] bf16, may be NULL; needs z */
typedef struct {
    int64_t M, N, K;
    const void* dy;
    int64_t dy_stride;
    const void* w;
    int64_t w_stride;
    adloco_kept z;
    const void* residual;
    int64_t residual_stride;
    void* dx;
    int64_t dx_stride;
    void* a;
    int64_t a_stride;
    int32_t activation;
    adloco_dtype out_dtype;
} adloco_linear_backward_args;
int adloco_linear_backward(adloco_ctx* ctx, const adloco_linear_backward_args* args, void* stream);

/* The gated feed-forward's first half in one pass:  gate = x w_gate^T,  up = x w_up^T,  a = act(gate) up
 *   x [M, d], w_gate, w_up [f, d] dev bf16;  a dev [M, f] bf16
 *   gate, up  kept for the backward pass, [M, f], both or neither, in one form */
typedef struct {
    int64_t M, d, f;
    const void* x;
    int64_t x_stride;
    const void* w_gate;
    int64_t w_gate_stride;
    const void* w_up;
    int64_t w_up_stride;
    void* a;
    int64_t a_stride;
    adloco_kept gate, up;
    int32_t activation;
    int32_t reserved;
} adloco_gated_linear_args;
int adloco_gated_linear(adloco_ctx* ctx, const adloco_gated_linear_args* args, void* stream);

/* The way back through the layer y = a w_down^T after it and through the gate:  with da = dy w_down,
 *   d_gate = da up act'(gate)     d_up = da act(gate)     a = act(gate) up, recomputed
 *   dy [M, d], w_down [d, f] dev bf16;  gate, up as kept;  d_gate, d_up, a dev [M, f] bf16; a may be NULL
 * With [w_gate; w_up] as one matrix [2 f, d] and [d_gate | d_up] as one [M, 2 f], the input's gradient is
 * adloco_linear_backward of the two, and both weights' gradients and norms adloco_linear_sqnorm's. */
typedef struct {
    int64_t M, d, f;
    const void* dy;
    int64_t dy_stride;
    const void* w_down;
    int64_t w_down_stride;
    adloco_kept gate, up;
    void* d_gate;
    int64_t d_gate_stride;
    void* d_up;
    int64_t d_up_stride;
    void* a;
    int64_t a_stride;
    int32_t activation;
    int32_t reserved;
} adloco_gated_linear_backward_args;
int adloco_gated_linear_backward(adloco_ctx* ctx, const adloco_gated_linear_backward_args* args, void* stream);

/* ---- the loss ----------------------------------------------------------------------- */

/* Of each row of logits l: lse = log sum_j exp(l_j), the log-probability logp = l_t - lse of its given token t, the entropy
 * -sum_j p_j log p_j with p_j = exp(l_j - lse), and the log-probabilities and ids of its `top` most probable tokens, the
 * largest first, equal ones by the lower id.
 *   logits   dev [rows, V] in dtype, pitch logits_stride;  targets dev int32 [rows], may be NULL when logp is
 *   logp, entropy, lse   dev [rows] float, each may be NULL;  top_values float, top_ids int32 dev [rows, top]
 *            contiguous, both or neither, 0 <= top <= 64, top <= V.  No output may overlap anything else.
 * A row whose target is outside [0, V) has logp 0.  Logits of -Inf (tokens ruled out) have probability 0 and log-probability
 * -Inf; a row of nothing else has lse, logp and top_values -Inf and entropy 0.  A row with a NaN or +Inf has NaN in all of them,
 * and ids of some tokens of the vocabulary.  fp32 throughout, one pass over the logits (choosing the best tokens reads a few parts of a row again, a row of many equal logits once for
 * each of them). */
typedef struct {
    int64_t rows, V;
    const void* logits;
    int64_t logits_stride;
    const int32_t* targets;
    float *logp, *entropy, *lse;
    float* top_values;
    int32_t* top_ids;
    int32_t top;
    adloco_dtype dtype;
} adloco_token_logprobs_args;
int adloco_token_logprobs(adloco_ctx* ctx, const adloco_token_logprobs_args* args, void* stream);

/* The logits' gradient of sum_r d_logp_r logp_r + d_entropy_r entropy_r:
 *   d_logits_j = d_logp (delta_jt - p_j) - d_entropy p_j (log p_j + entropy),    p_j = exp(l_j - lse)
 *   logits, targets, lse, entropy  as given to and by the call above (entropy and d_entropy: both or neither); lse is a float: the
 *            probabilities are right to 2^-24 |lse|
 *   d_logits  dev [rows, V] in dtype, pitch d_logits_stride; may be logits itself, with the same pitch, and overlap nothing else
 * A row whose target is outside [0, V) takes no part in logp.  A row that takes part in nothing (and whose d_entropy is 0 or
 * not given), or with lse -Inf, gets zeros whatever its logits hold. */
typedef struct {
    int64_t rows, V;
    const void* logits;
    int64_t logits_stride;
    const int32_t* targets;
    const float *lse, *d_logp, *entropy, *d_entropy;
    void* d_logits;
    int64_t d_logits_stride;
    int32_t reserved;
    adloco_dtype dtype;
} adloco_token_logprobs_backward_args;
int adloco_token_logprobs_backward(adloco_ctx* ctx, const adloco_token_logprobs_backward_args* args, void* stream);

/* ---- switch-mode accumulation -------------------------------------------- */

/* Accumulator of the test sums over the micro-batches of one large batch:
 * Q = sum n_i, the batch count, and the gradient-sum buffers S (one per
 * parameter buffer; caller-owned dev float arrays that the accumulator borrows).
 * adloco_accum_create copies the n_bufs pointers/sizes (host arrays) and
 * allocates a small device state; synchronous. */
int adloco_accum_create(adloco_ctx* ctx, adloco_accum** out, float* const* sum_bufs, const int64_t* sum_sizes,
                        int32_t n_bufs);
/* Zeroes Q, the count and every S buffer (async on stream). */
int adloco_accum_reset(adloco_ctx* ctx, adloco_accum* acc, void* stream);
int adloco_accum_destroy(adloco_accum* acc);   /* before its ctx is destroyed */

/* Adds one micro-batch (Algorithm 3's g <- g + grad L(x; B), applied to the
 * test sums).  Two forms:
 *  (a) grads != NULL: materialised micro-batch [b_micro, P] float (pitch row_stride),
 *      P == sum_sizes[0] and n_bufs == 1.  One pass adds sum_i g_i into S, sum_i n_i
 *      into Q, and keeps the centred sum of squares exact across micro-batches by
 *      the pairwise update  css += css_mb + (c b/(c+b)) ||mean_mb - mean_so_far||^2.
 *      per_sample_sqnorm (dev [b_micro], may be NULL) receives this micro-batch's n_i.
 *  (b) grads == NULL: the caller has already added this micro-batch's gradient sums
 *      into the S buffers (adloco_gram_sqnorm with accumulate_sum) and passes its
 *      n_i in per_sample_sqnorm (dev [b_micro], required); only Q and the count move. */
int adloco_accumulate(adloco_ctx* ctx, adloco_accum* acc, const void* grads, adloco_dtype dtype,
                      int64_t b_micro, int64_t P, int64_t row_stride, float* per_sample_sqnorm, void* stream);

/* One test on everything accumulated: N = sum_bufs ||S/b||^2,
 * V = centred_ss/(b-ddof) when every micro-batch was materialised, otherwise
 * V = (Q - b N)/(b - ddof); then the batch rule and switch plan.  ||S||^2 is taken
 * from the last form-(a) call when that was the last change to S (the caller must
 * not modify S behind a form-(a) accumulation), else reduced here. */
int adloco_accum_finalize(adloco_ctx* ctx, adloco_accum* acc, const adloco_test_params* params,
                          adloco_test_sums* sums_dev, adloco_test_result* result_dev,
                          adloco_test_result* result_host, void* stream);

/* ---- outer step ----------------------------------------------------------- */

/* Last loop of Algorithm 3 for one trainer, fused in one pass:
 *   d      = (1/K) sum_k (theta - theta_k)
 *   v'     = momentum v + d
 *   u      = d + momentum v' (nesterov != 0)  |  v'
 *   theta' = theta - lr u
 *   inst_params  HOST array of K dev pointers, each [P] in inst_dtype (F32 or BF16),
 *                separate allocations allowed; 1 <= K <= 64
 *   theta_in/out, mom_in/out  dev [P] float; out may be the same pointer as in
 *                (exact aliasing only); instances must not overlap theta or mom
 *   inst_writeback  HOST array of K dev pointers (may be NULL, entries may be NULL):
 *                each receives theta' rounded to inst_dtype (Algorithm 3 resets every
 *                worker to the trainer's parameters at the next outer step)
 * The K differences (each exact in fp64) are summed in fp64 in the order k = 0..K-1 and the
 * update is carried in fp64; every output element is rounded to fp32 once. */
int adloco_outer_step(adloco_ctx* ctx, const void* const* inst_params, adloco_dtype inst_dtype, int32_t K,
                      int64_t P, const float* theta_in, float* theta_out, const float* mom_in, float* mom_out,
                      float lr, float momentum, int nesterov, void* const* inst_writeback, void* stream);

/* Same update with every buffer in HOST memory (inst_params_host: K host
 * pointers; theta_host and mom_host are updated in place): panels are staged
 * through device buffers the library owns, copies overlapped with the kernel.
 * Synchronous. */
int adloco_outer_step_host(adloco_ctx* ctx, const void* const* inst_params_host, adloco_dtype inst_dtype,
                           int32_t K, int64_t P, float* theta_host, float* mom_host, float lr, float momentum,
                           int nesterov, void* stream);

/* The outer step when every GPU holds ONE whole instance (and the shared starting point
 * theta) but only a slice of the momentum: the K pseudo-gradients are summed across the
 * GPUs by one reduce-scatter -- the single communication of the method (last loop of
 * Algorithm 3: the workers' differences are gathered and averaged) -- which the caller
 * performs between these calls, with whatever collective library it uses:
 *   1. adloco_pseudo_gradient    pseudo_grad = theta - theta_k, fp32 [P]      (every rank)
 *   2. reduce-scatter (sum) of pseudo_grad over the K ranks -> pseudo_grad_sum, this rank's slice
 *   3. adloco_outer_apply        d = pseudo_grad_sum / K; v' = momentum v + d;
 *                                u = d + momentum v' | v'; theta' = theta - lr u   (on the slice)
 *   4. all-gather of the theta' slices, then adloco_refresh_instance: theta_k = theta'
 *      rounded to the instance type (Algorithm 3 restarts every worker from theta).
 * All pointers dev, 16-byte aligned; theta/mom in and out may alias exactly.  The update is
 * carried in fp64 and rounded once, as in adloco_outer_step.  The K terms cross the exchange
 * as fp32 and are summed by the collective in fp32: against adloco_outer_step (which sums
 * them in fp64) the sum can be off by up to (K - 1/2) ulp of sum_k |theta - theta_k|, which
 * shows where the terms cancel and the update itself is small. */
int adloco_pseudo_gradient(adloco_ctx* ctx, const float* theta, const void* inst_params, adloco_dtype inst_dtype,
                           int64_t P, float* pseudo_grad, void* stream);
int adloco_outer_apply(adloco_ctx* ctx, const float* pseudo_grad_sum, int32_t K, int64_t P, const float* theta_in,
                       float* theta_out, const float* mom_in, float* mom_out, float lr, float momentum, int nesterov,
                       void* stream);
int adloco_refresh_instance(adloco_ctx* ctx, const float* theta, void* inst_params, adloco_dtype inst_dtype, int64_t P,
                            void* stream);

/* ---- trainer merge --------------------------------------------------------- */

/* CheckMerge (Algorithm 1), host only: writes into merge_idx (host, capacity >= w)
 * the indices of the w trainers with the smallest b_req (ties: lower index first)
 * and returns their number; 0 when w == 0, k <= 1 or w > k; negative status on
 * bad arguments. */
int adloco_check_merge(const int64_t* b_req, int32_t k, int32_t w, int32_t* merge_idx);

/* DoMerge (Algorithm 2): x_merge = sum_j b_j x_j / sum_j b_j over the K members
 * (HOST array of dev pointers, [P] each in `dtype`; weights HOST int64 > 0),
 * written to `out` (dev [P] in `dtype`; may be one of the members, exactly).
 * *rep (host, may be NULL) receives the member with the largest weight (lowest
 * index on ties), the trainer that is kept. 1 <= K <= 64. */
int adloco_merge(adloco_ctx* ctx, const void* const* members, const int64_t* weights, adloco_dtype dtype,
                 int32_t K, int64_t P, void* out, int32_t* rep, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ADLOCO_H */

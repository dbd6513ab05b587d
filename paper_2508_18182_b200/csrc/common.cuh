// Shared host-side declarations of the library: the context, error handling
// and the launch helpers that the entry points in api.cu use.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <cuda_bf16.h>
#include <atomic>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

// the library is built with hidden visibility; only the C ABI is exported
#pragma GCC visibility push(default)
#include "../../include/adloco.h"
#pragma GCC visibility pop

namespace adloco {

constexpr int kMaxInstances = 64;     // K of the outer step / merge (pointers travel as kernel arguments)
constexpr int kSchedCounters = 1024;   // launches of the grouped kernel that may be in flight at once
constexpr int64_t kMaxBatchRows = 4096;  // B of one materialised (micro-)batch (per-warp rows live in shared memory)

// Staging buffers for the host-memory entry points (allocated on first use).
struct HostStaging {
    void* dev[2] = {nullptr, nullptr};
    size_t bytes = 0;
    cudaStream_t copy_stream = nullptr;
    cudaEvent_t filled[2] = {nullptr, nullptr};
    cudaEvent_t drained[2] = {nullptr, nullptr};
    cudaEvent_t out_done[2] = {nullptr, nullptr};
};

}  // namespace adloco

struct adloco_ctx {
    int device = 0;
    int sm_count = 0;
    int64_t launches = 0;
    char cuda_err[384] = {0};

    // workspace of the streaming reductions
    float* n_partials = nullptr;   // [grid][B] per-block partial row sums of squares
    size_t n_partials_elems = 0;
    double* blk_scalars = nullptr; // [max_grid][4]
    unsigned* ticket = nullptr;    // "last block done" counter, left at zero by every kernel
    int max_grid = 0;
    adloco_test_sums* scratch_sums = nullptr;  // used when the caller passes no sums_dev
    int* gemm_status = nullptr;                // device status word of the tensor-core kernels
    uint64_t wait_limit_ns = 2000000000ull;    // bound of every in-kernel wait: 2 s, far beyond any legitimate wait
    float* n_scratch = nullptr;                // [kMaxBatchRows] per-sample norms when the caller wants none
    void* tensor_maps = nullptr;               // cache of encoded tensor maps (gram_kernels.cu owns the type)
    int pair_ok = -1;                          // CTA-pair launches possible on this device: -1 not asked yet
    int* sched_counters = nullptr;             // [kSchedCounters] work counters of the grouped tensor-core kernel
    std::atomic<unsigned> sched_next{0};       // next counter to hand to a launch

    adloco::HostStaging staging;
};

struct adloco_accum {
    adloco_ctx* ctx = nullptr;
    int32_t n_bufs = 0;
    float** bufs_host = nullptr;       // host copy of the S pointers
    int64_t* sizes_host = nullptr;
    float** bufs_dev = nullptr;        // device copies, for the squared-norm reduction
    int64_t* chunk_prefix_dev = nullptr;  // [n_bufs + 1] prefix sums of 4096-element chunks
    int64_t* sizes_dev = nullptr;
    int64_t total_chunks = 0;
    adloco_test_sums* state = nullptr; // device: Q, ||S||^2, centred ss, count
    bool sqnorm_current = true;        // state->sum_sq_gsum already equals ||S||^2 (kept by the materialised form)
};

namespace adloco {

inline int set_cuda_error(adloco_ctx* ctx, cudaError_t e, const char* where) {
    if (ctx) snprintf(ctx->cuda_err, sizeof(ctx->cuda_err), "%s: %s", where, cudaGetErrorString(e));
    return ADLOCO_ERR_CUDA;
}

#define ADLOCO_CUDA_TRY(ctx, expr)                                        \
    do {                                                                  \
        cudaError_t e__ = (expr);                                         \
        if (e__ != cudaSuccess) return adloco::set_cuda_error((ctx), e__, #expr); \
    } while (0)

// the ctx's device is current while an entry point runs
struct DeviceGuard {
    int prev = -1;                      // what to go back to, -1: nothing was changed
    bool ok = true;
    explicit DeviceGuard(int dev) {
        int now;
        if (cudaGetDevice(&now) != cudaSuccess) { ok = false; return; }
        if (now == dev) return;
        prev = now;
        if (cudaSetDevice(dev) != cudaSuccess) ok = false;
    }
    ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

// thread-block clusters of two CTAs need compute capability 9.0 or later and the launch attribute
inline bool cta_pairs_possible(adloco_ctx* ctx) {
    if (ctx->pair_ok < 0) {
        int v = 0;
        ctx->pair_ok = (cudaDeviceGetAttribute(&v, cudaDevAttrClusterLaunch, ctx->device) == cudaSuccess && v != 0) ? 1 : 0;
    }
    return ctx->pair_ok == 1;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_params(const adloco_test_params* p) {
    if (!p) return ADLOCO_ERR_INVALID_ARG;
    if (!(p->eta > 0.0) || !(p->eta < 1.0e300)) return ADLOCO_ERR_INVALID_ARG;  // also rejects NaN
    if (p->ddof < 0 || p->switch_n < 1 || p->b_max < 1 || p->b_cur < 0 || p->b_cap < 0) return ADLOCO_ERR_INVALID_ARG;
    return ADLOCO_OK;
}

// A launch that may begin while the kernel before it on the stream drains (programmatic dependent launch): the kernel
// calls after_predecessor() before it touches memory, which waits for that kernel's completion and its writes.  Only for
// kernels that do, and that take nothing through the non-coherent path (__ldg, __restrict__ on const): it is for data that
// does not change while the kernel runs, and this one runs while the kernel before it may still write any operand.
#ifdef __CUDACC__
__device__ __forceinline__ void after_predecessor() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
// An operand's address, not known to the compiler before after_predecessor() is through: loads that it may move as it likes
// (asm without volatile) stay behind the wait when they go by this address.
template <typename T>
__device__ __forceinline__ T* settled(T* p) {
    asm volatile("" : "+l"(p));
    return p;
}
template <typename... Params, typename... Args>
inline cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, unsigned cluster,
                                const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
#endif

// ---- launchers implemented in stream_kernels.cu --------------------------------
enum NtMode { NT_ONESHOT = 0, NT_PANEL = 1, NT_MICRO = 2 };

struct NtLaunch {
    const float* G = nullptr;     // rows of float, or of bfloat16 when bf16 != 0
    int bf16 = 0;
    int64_t B = 0, P = 0, stride = 0;
    float* n_out = nullptr;       // [B], may be null
    int n_accum = 0;              // n_out[i] += instead of =
    float* S = nullptr;           // [P]: written (ONESHOT/PANEL) or read-modify-written (MICRO); may be null unless MICRO
    adloco_test_sums* sums = nullptr;    // required (ctx scratch if the caller has none)
    adloco_test_result* result = nullptr;  // decision written by the last block when non-null
    adloco_test_result* result_mirror = nullptr;  // device-side address of a page-locked host copy of it, or null
    adloco_test_params params{};
    int mode = NT_ONESHOT;
    int first_panel = 1;          // PANEL: overwrite the sums on the first panel, add afterwards
};
int launch_norm_test(adloco_ctx* ctx, const NtLaunch& l, cudaStream_t st);
int launch_decide(adloco_ctx* ctx, const adloco_test_sums* sums, const adloco_test_params& p,
                  adloco_test_result* result, adloco_test_result* mirror, cudaStream_t st);

struct IpLaunch {
    const float* G = nullptr;
    int bf16 = 0;
    const float* S = nullptr;
    int64_t B = 0, P = 0, stride = 0;
    const adloco_test_sums* sums = nullptr;
    adloco_ip_params params{};
    float* dots_out = nullptr;
    adloco_ip_result* result = nullptr;
    adloco_ip_result* result_mirror = nullptr;
};
int launch_inner_product(adloco_ctx* ctx, const IpLaunch& l, cudaStream_t st);

int launch_vec_param(adloco_ctx* ctx, const void* D, const void* X, int64_t B, int64_t T, int64_t d, float* n,
                     int accumulate_norms, float* S, int accumulate_sum, cudaStream_t st);

struct OuterLaunch {
    const void* inst[kMaxInstances];
    void* wb[kMaxInstances];
    int K = 0;
    int has_wb = 0;
    int bf16 = 0;
    int64_t P = 0;
    const float* th_in = nullptr;
    float* th_out = nullptr;
    const float* v_in = nullptr;
    float* v_out = nullptr;
    float lr = 0, mu = 0;
    int nesterov = 1;
};
int launch_outer_step(adloco_ctx* ctx, const OuterLaunch& l, cudaStream_t st);

int launch_pseudo_grad(adloco_ctx* ctx, const float* theta, const void* inst, int bf16, float* g, int64_t P, cudaStream_t st);
int launch_outer_apply(adloco_ctx* ctx, const float* g_sum, int K, int64_t P, const float* th_in, float* th_out,
                       const float* v_in, float* v_out, float lr, float mu, int nesterov, cudaStream_t st);
int launch_refresh(adloco_ctx* ctx, const float* theta, void* inst, int bf16, int64_t P, cudaStream_t st);

struct MergeLaunch {
    const void* x[kMaxInstances];
    float coef[kMaxInstances];
    int K = 0;
    int bf16 = 0;
    int64_t P = 0;
    void* out = nullptr;
};
int launch_merge(adloco_ctx* ctx, const MergeLaunch& l, cudaStream_t st);

// sum over all S buffers of an accumulator of ||S||^2 -> state->sum_sq_gsum, then
// state->sum_sqnorm += sum(n[0..b)) and the count (form (b) of adloco_accumulate)
int launch_accum_add_norms(adloco_ctx* ctx, adloco_accum* acc, const float* n, int64_t b, cudaStream_t st);
int launch_accum_sqnorm(adloco_ctx* ctx, adloco_accum* acc, cudaStream_t st);
int launch_accum_zero(adloco_ctx* ctx, adloco_accum* acc, cudaStream_t st);

// ---- tensor-core path, implemented in gram_kernels.cu ---------------------------
int launch_gram_sqnorm(adloco_ctx* ctx, const void* X, const void* D, int64_t B, int64_t T, int64_t d_in,
                       int64_t d_out, float* n, int accumulate_norms, cudaStream_t st);
int launch_gram_pair(adloco_ctx* ctx, const void* X, const void* D, int64_t B, int64_t T, int64_t d_in,
                     int64_t d_out, float* n, int accumulate_norms, cudaStream_t st);
int launch_mean_grad(adloco_ctx* ctx, const void* X, const void* D, int64_t B, int64_t T, int64_t d_in,
                     int64_t d_out, float* S, int accumulate_sum, cudaStream_t st);
int launch_embedding(adloco_ctx* ctx, const int* ids, const void* D, int64_t B, int64_t T, int64_t d, int64_t V,
                     float* n, int accumulate_norms, float* S, int accumulate_sum, cudaStream_t st);
int launch_direct_sqnorm(adloco_ctx* ctx, const void* X, const void* D, int64_t B, int64_t T, int64_t d_in,
                         int64_t d_out, float* n, int accumulate_norms, float* S, int accumulate_sum, int pair,
                         cudaStream_t st);
int launch_direct_group(adloco_ctx* ctx, const adloco_linear_layer* layers, int n_layers, int64_t B, int64_t T,
                        float* n, int accumulate_norms, int accumulate_sum, int pair, cudaStream_t st);
void free_tensor_map_cache(adloco_ctx* ctx);
// the driver's encoder of TMA tensor maps, or null with the ctx's error text set
typedef CUresult (*TensorMapEncode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                    const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                    CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
TensorMapEncode tensor_map_encode(adloco_ctx* ctx);

// ---- between the linear layers, implemented in block_kernels.cu -------------------
// A dropout mask as the kernels take it: the generator's key schedule is formed once on the host, so that a round's
// key is an operand from the constant bank.
struct DropoutKey {
    uint32_t round[20] = {0};           // of round r: [2 r], [2 r + 1]
    uint32_t off_lo = 0, off_hi = 0;
    uint32_t on = 0;                    // any element is dropped at all
    float scale = 1.f;                  // 1 over the share that stays; 1 where none is dropped, or all are
    float high = 1.f, low = 0.f;        // the same beside a residual: the sum of two numbers, the first rounded down (low >= 0)
    // two 16-bit numbers are compared with the drop threshold at a time: the threshold in both halves, and the byte
    // selectors that spread a half's top bit over that half (of_pair), or over 32 bits (of_low, of_high); they select
    // zero bytes when all are dropped
    uint32_t limit = 0, of_pair = 0xBB99u, of_low = 0x9999u, of_high = 0xBBBBu;
};
int launch_add_rmsnorm(adloco_ctx* ctx, const adloco_rmsnorm_args& a, const DropoutKey& key, cudaStream_t st);
int64_t rmsnorm_backward_workspace(const adloco_ctx* ctx, int64_t B, int64_t T, int64_t d);
int launch_add_rmsnorm_backward(adloco_ctx* ctx, const adloco_rmsnorm_backward_args& a, const DropoutKey& key, cudaStream_t st);
int launch_dropout(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const void* r,
                   int64_t r_stride, void* y, int64_t y_stride, const DropoutKey& key, cudaStream_t st);
int launch_rope(adloco_ctx* ctx, int bf16, const adloco_rope_tensor* t, int n, int64_t B, int64_t T, int64_t D, int64_t R,
                const uint64_t* turns, float magnitude, const int32_t* pos, int64_t pos_stride, int64_t first, int interleaved,
                int inverse, cudaStream_t st);
int launch_blockscale_quantize(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* x, int64_t x_stride, void* q,
                               int64_t q_stride, uint8_t* scale, int64_t scale_stride, cudaStream_t st);
int launch_blockscale_quantize_weight(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* W, int64_t W_stride,
                                      void* q, int64_t q_stride, void* q_t, int64_t q_t_stride, uint8_t* scale,
                                      int64_t scale_stride, cudaStream_t st);
// implemented in blockscale_gemm.cu
int launch_blockscale_matmul(adloco_ctx* ctx, const adloco_blockscale_matmul_args& a, cudaStream_t st);
// implemented in dense_gemm.cu
int launch_linear(adloco_ctx* ctx, const adloco_linear_args& a, cudaStream_t st);
int launch_linear_backward(adloco_ctx* ctx, const adloco_linear_backward_args& a, cudaStream_t st);
int launch_gated_linear(adloco_ctx* ctx, const adloco_gated_linear_args& a, cudaStream_t st);
int launch_gated_linear_backward(adloco_ctx* ctx, const adloco_gated_linear_backward_args& a, cudaStream_t st);
// implemented in token_kernels.cu
int launch_blockscale_dequantize(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* q, int64_t q_stride,
                                 const uint8_t* scale, int64_t scale_stride, void* x, int64_t x_stride, cudaStream_t st);
int launch_token_logprobs(adloco_ctx* ctx, const adloco_token_logprobs_args& a, cudaStream_t st);
int launch_token_logprobs_backward(adloco_ctx* ctx, const adloco_token_logprobs_backward_args& a, cudaStream_t st);

}  // namespace adloco

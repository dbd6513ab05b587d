// What the tensor-core kernels of the linear layers share: the ring of stages, waits of a whole warp, tensor maps.
#pragma once

#include "common.cuh"
#include "ptx.cuh"

namespace adloco {
namespace {

using namespace ptx;

constexpr uint64_t kPairLeaveNs = 1000000ull;      // 1 ms: a CTA pair leaving after a time-out; copies in flight land long before
constexpr uint64_t kLeaveLimitNs = 50000000ull;    // 50 ms per barrier while leaving after a time-out

struct Ring {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void advance(uint32_t n) {
        if (++stage == n) { stage = 0; phase ^= 1u; }
    }
};

__device__ __forceinline__ uint32_t pack_bf16(uint32_t a, uint32_t b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(a), __uint_as_float(b));
    return *reinterpret_cast<const uint32_t*>(&h);
}

// A wait of the whole warp, which goes on (or gives up) together.
template <bool CLUSTER>
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abortp, uint64_t limit_ns) {
    return __all_sync(0xffffffffu, mbar_wait<CLUSTER>(bar, parity, abortp, limit_ns)) != 0;
}

// matrix [rows, cols] of `es`-byte elements with a pitch in elements, as a 2-D map with a box of box_rows rows of
// box_cols elements (as many bytes as the swizzle spans); elements outside the matrix read as zero and are not written
inline int make_map(adloco_ctx* ctx, CUtensorMap* m, CUtensorMapDataType type, int64_t es, const void* base, int64_t rows, int64_t cols,
             int64_t pitch, uint32_t box_cols, uint32_t box_rows, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
    TensorMapEncode fn = tensor_map_encode(ctx);
    if (!fn) return ADLOCO_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(pitch * es)};
    const cuuint32_t box[2] = {box_cols, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(m, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        snprintf(ctx->cuda_err, sizeof(ctx->cuda_err), "cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
        return ADLOCO_ERR_CUDA;
    }
    return ADLOCO_OK;
}

}  // namespace
}  // namespace adloco

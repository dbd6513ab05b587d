// out = A B^T for 8-bit operands with a power-of-two scale for each block of 128 (rows of A, 128 x 128
// blocks of B), on the tensor cores: TMA tiles, tcgen05.mma with the scales read from tensor memory,
// fp32 accumulators in tensor memory, one rounding in the epilogue.
#include <atomic>

#include "common.cuh"
#include "ptx.cuh"

namespace adloco {

using namespace ptx;

namespace {

constexpr uint64_t kLeaveLimitNs = 50000000ull;    // 50 ms per barrier while leaving after a time-out

struct Ring {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void advance(uint32_t n) {
        if (++stage == n) { stage = 0; phase ^= 1u; }
    }
};

struct MatArgs {
    int M, N, K, kb;                 // kb: blocks of 128 along K
    int tiles_m, tiles_n, tiles;
    const uint8_t* sa;
    int64_t sa_stride;
    const uint8_t* sb;
    int64_t sb_n, sb_k;
    const float* bias;
    void* out;
    int64_t out_stride;
    int out_bf16, out_vec;           // out_vec: 16-byte stores are possible
    int* status;
    uint64_t wait_ns;
};

// ---- 128 x 128 tiles, one CTA each --------------------------------------------------------------
// Persistent, 320 threads: warp 0 TMA, warp 1 MMA, warps 2-5 scales, warps 6-9 epilogue.  A stage is 128 of K (a
// 128-byte swizzle row of either operand): four MMAs of K = 32 that use the same byte of the scale words.  A scale
// word holds the bytes of four stages; the scale warps write the words of 512 of K at a time into a ring of slots
// in tensor memory (lane = row mod 32, column = row / 32, the same in all four lane quarters, which is how the
// MMA reads them).
constexpr int MT = 128;
constexpr int MT_STAGES = 6;
constexpr int MT_STAGE_BYTES = 2 * MT * 128;
constexpr int MT_SLOTS = 4;                                   // scale slots of 8 columns: 4 for A, 4 for B
constexpr int MT_SF_COL = 2 * MT;                             // tensor memory: two accumulators, then the slots
constexpr int MT_SMEM = MT_STAGES * MT_STAGE_BYTES + 1024 + 256;
constexpr int MT_THREADS = 320;

__global__ void __launch_bounds__(MT_THREADS, 1)
blockscale_tile_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const MatArgs a) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bars = smem_base + MT_STAGES * MT_STAGE_BYTES;
    auto full_bar = [&](uint32_t s) { return bars + 8u * s; };
    auto empty_bar = [&](uint32_t s) { return bars + 8u * (MT_STAGES + s); };
    auto sf_full = [&](uint32_t s) { return bars + 8u * (2 * MT_STAGES + s); };
    auto sf_empty = [&](uint32_t s) { return bars + 8u * (2 * MT_STAGES + MT_SLOTS + s); };
    auto acc_full = [&](uint32_t s) { return bars + 8u * (2 * MT_STAGES + 2 * MT_SLOTS + s); };
    auto acc_empty = [&](uint32_t s) { return bars + 8u * (2 * MT_STAGES + 2 * MT_SLOTS + 2 + s); };
    const uint32_t drain_bar = bars + 8u * (2 * MT_STAGES + 2 * MT_SLOTS + 4);
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (uint32_t s = 0; s < MT_STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (uint32_t s = 0; s < MT_SLOTS; ++s) { mbar_init(sf_full(s), 4); mbar_init(sf_empty(s), 1); }
        for (uint32_t s = 0; s < 2; ++s) { mbar_init(acc_full(s), 1); mbar_init(acc_empty(s), 4); }
        mbar_init(drain_bar, 1);
        fence_barrier_init();
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&tmem_slot), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    volatile int* abortp = &abort_flag;

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (lane == 0) {
            Ring ps;
            uint32_t issued = 0;
            bool ok = true;
            for (int tile = blockIdx.x; ok && tile < a.tiles; tile += gridDim.x) {
                const int m0 = (tile % a.tiles_m) * MT, n0 = (tile / a.tiles_m) * MT;
                for (int k = 0; k < a.kb; ++k) {
                    if (!mbar_wait(empty_bar(ps.stage), ps.phase ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
                    const uint32_t sA = smem_base + ps.stage * MT_STAGE_BYTES;
                    mbar_arrive_expect_tx(full_bar(ps.stage), MT_STAGE_BYTES);
                    tma_load_2d(sA, &tmA, full_bar(ps.stage), k * 128, m0);
                    tma_load_2d(sA + MT * 128, &tmB, full_bar(ps.stage), k * 128, n0);
                    ++issued;
                    ps.advance(MT_STAGES);
                }
            }
            if (!ok) {
                // leaving after a time-out: let the copies still in flight land first
                Ring q = ps;
                const uint32_t back = issued < MT_STAGES ? issued : MT_STAGES;
                for (uint32_t r = 0; r < back; ++r) {
                    if (q.stage == 0) { q.stage = MT_STAGES - 1; q.phase ^= 1u; } else { --q.stage; }
                    int never = 0;
                    mbar_wait(full_bar(q.stage), q.phase, &never, kLeaveLimitNs);
                }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer ----------------
        if (lane == 0) {
            Ring ps, sf;
            uint32_t n = 0;
            bool ok = true;
            for (int tile = blockIdx.x; ok && tile < a.tiles; tile += gridDim.x, ++n) {
                const uint32_t buf = n & 1u;
                if (!mbar_wait(acc_empty(buf), ((n >> 1) & 1u) ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
                tc_fence_after();
                for (int k = 0; k < a.kb; ++k) {
                    if ((k & 3) == 0 && !mbar_wait(sf_full(sf.stage), sf.phase, abortp, a.wait_ns)) { ok = false; break; }
                    if (!mbar_wait(full_bar(ps.stage), ps.phase, abortp, a.wait_ns)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sA = smem_base + ps.stage * MT_STAGE_BYTES, sB = sA + MT * 128;
                    const uint32_t sf_col = tmem + MT_SF_COL + sf.stage * 8u;
                    const uint32_t idesc = idesc_mxf8(MT, MT, (uint32_t)k & 3u);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)       // K-major, 128-byte swizzle: 32 elements further along K = 32 bytes
                        mma_mxf8(tmem + buf * MT, smem_desc_sw128(sA + kk * 32, 16, 1024), smem_desc_sw128(sB + kk * 32, 16, 1024),
                                 idesc, sf_col, sf_col + 4, (k == 0 && kk == 0) ? 0u : 1u);
                    mma_commit(empty_bar(ps.stage));
                    ps.advance(MT_STAGES);
                    if ((k & 3) == 3 || k == a.kb - 1) {
                        mma_commit(sf_empty(sf.stage));
                        sf.advance(MT_SLOTS);
                    }
                }
                if (ok) mma_commit(acc_full(buf));
            }
            if (!ok) {
                mma_commit(drain_bar);
                int never = 0;
                mbar_wait(drain_bar, 0, &never, kLeaveLimitNs);
            }
        }
    } else if (warp < 6) {
        // ---------------- scales into tensor memory ----------------
        const uint32_t quarter = (uint32_t)(warp & 3) << 21;       // lane 32 * (warp mod 4) of a tensor-memory address
        Ring sf;
        bool ok = true;
        for (int tile = blockIdx.x; ok && tile < a.tiles; tile += gridDim.x) {
            const int m0 = (tile % a.tiles_m) * MT, nb = (tile / a.tiles_m) * MT / 128;
            for (int g = 0; g * 4 < a.kb; ++g) {
                uint32_t w[4], b = 0x7f7f7f7fu;
                const int have = min(4, a.kb - g * 4);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int m = m0 + c * 32 + lane;
                    w[c] = 0x7f7f7f7fu;
                    if (m < a.M) {
                        const uint8_t* p = a.sa + (int64_t)m * a.sa_stride + g * 4;
                        if (have == 4) w[c] = *reinterpret_cast<const uint32_t*>(p);
                        else for (int j = 0; j < have; ++j) w[c] = (w[c] & ~(0xffu << (8 * j))) | ((uint32_t)p[j] << (8 * j));
                    }
                }
                for (int j = 0; j < have; ++j)
                    b = (b & ~(0xffu << (8 * j))) | ((uint32_t)a.sb[nb * a.sb_n + (g * 4 + j) * a.sb_k] << (8 * j));
                if (!__all_sync(0xffffffffu, mbar_wait(sf_empty(sf.stage), sf.phase ^ 1u, abortp, a.wait_ns))) { ok = false; break; }
                tc_fence_after();
                const uint32_t at = tmem + quarter + MT_SF_COL + sf.stage * 8u;
                tmem_st4(at, w[0], w[1], w[2], w[3]);
                tmem_st4(at + 4, b, b, b, b);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(sf_full(sf.stage));
                sf.advance(MT_SLOTS);
            }
        }
    } else {
        // ---------------- epilogue ----------------
        const uint32_t q = warp & 3;
        uint32_t n = 0;
        for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x, ++n) {
            const int m0 = (tile % a.tiles_m) * MT, n0 = (tile / a.tiles_m) * MT;
            const uint32_t buf = n & 1u;
            if (!__all_sync(0xffffffffu, mbar_wait(acc_full(buf), (n >> 1) & 1u, abortp, a.wait_ns))) break;
            tc_fence_after();
            const int m = m0 + (int)q * 32 + lane;
#pragma unroll 1
            for (int c = 0; c < MT; c += 32) {
                uint32_t r[32];
                tmem_ld32(tmem + ((q * 32u) << 16) + buf * MT + c, r);
                tmem_ld_wait();
                if (m >= a.M) continue;
                const int col = n0 + c;
                if (a.bias) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (col + e < a.N) r[e] = __float_as_uint(__uint_as_float(r[e]) + __ldg(a.bias + col + e));
                }
                if (a.out_bf16) {
                    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(a.out) + (int64_t)m * a.out_stride + col;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        if (a.out_vec && col + e + 8 <= a.N) {
                            uint32_t p[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(r[e + 2 * j]), __uint_as_float(r[e + 2 * j + 1]));
                                p[j] = *reinterpret_cast<const uint32_t*>(&h);
                            }
                            *reinterpret_cast<uint4*>(o + e) = make_uint4(p[0], p[1], p[2], p[3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                if (col + e + j < a.N) o[e + j] = __float2bfloat16_rn(__uint_as_float(r[e + j]));
                        }
                    }
                } else {
                    float* o = static_cast<float*>(a.out) + (int64_t)m * a.out_stride + col;
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        if (a.out_vec && col + e + 4 <= a.N) {
                            *reinterpret_cast<uint4*>(o + e) = make_uint4(r[e], r[e + 1], r[e + 2], r[e + 3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                if (col + e + j < a.N) o[e + j] = __uint_as_float(r[e + j]);
                        }
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty(buf));
        }
    }

    // ---------------- teardown ----------------
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0 && abort_flag) atomicExch(a.status, (int)ADLOCO_ERR_TIMEOUT);
}

// byte matrix [rows, cols] with a pitch, as a 2-D map with a box of box_rows rows of 128 bytes, 128-byte swizzle;
// bytes outside the matrix read as zero
int make_byte_map(adloco_ctx* ctx, CUtensorMap* m, const void* base, int64_t rows, int64_t cols, int64_t pitch, uint32_t box_rows) {
    TensorMapEncode fn = tensor_map_encode(ctx);
    if (!fn) return ADLOCO_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {128, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr,
                          CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        snprintf(ctx->cuda_err, sizeof(ctx->cuda_err), "cuTensorMapEncodeTiled (8-bit) failed with CUresult %d", (int)r);
        return ADLOCO_ERR_CUDA;
    }
    return ADLOCO_OK;
}

}  // namespace

int launch_blockscale_matmul(adloco_ctx* ctx, const adloco_blockscale_matmul_args& p, cudaStream_t st) {
    MatArgs a;
    a.M = (int)p.M; a.N = (int)p.N; a.K = (int)p.K; a.kb = (int)((p.K + 127) / 128);
    const int64_t tm = (p.M + MT - 1) / MT, tn = (p.N + MT - 1) / MT;
    if (tm * tn > 0x7fffffff) return ADLOCO_ERR_UNSUPPORTED;
    a.tiles_m = (int)tm; a.tiles_n = (int)tn; a.tiles = (int)(tm * tn);
    a.sa = p.a_scale; a.sa_stride = p.a_scale_stride;
    a.sb = p.b_scale; a.sb_n = p.b_scale_stride_n; a.sb_k = p.b_scale_stride_k;
    a.bias = p.bias; a.out = p.out; a.out_stride = p.out_stride;
    a.out_bf16 = p.out_dtype == ADLOCO_BF16;
    a.out_vec = aligned16(p.out) && (p.out_stride % (a.out_bf16 ? 8 : 4)) == 0;
    a.status = ctx->gemm_status; a.wait_ns = ctx->wait_limit_ns;
    CUtensorMap tmA, tmB;
    int rc = make_byte_map(ctx, &tmA, p.a, p.M, p.K, p.a_stride, MT);
    if (rc == ADLOCO_OK) rc = make_byte_map(ctx, &tmB, p.b, p.N, p.K, p.b_stride, MT);
    if (rc != ADLOCO_OK) return rc;
    static std::atomic<bool> attr_set[64];   // the attribute is per device
    if (!attr_set[ctx->device & 63].load()) {
        ADLOCO_CUDA_TRY(ctx, cudaFuncSetAttribute(blockscale_tile_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MT_SMEM));
        attr_set[ctx->device & 63].store(true);
    }
    blockscale_tile_kernel<<<a.tiles < ctx->sm_count ? a.tiles : ctx->sm_count, MT_THREADS, MT_SMEM, st>>>(tmA, tmB, a);
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    return ADLOCO_OK;
}

}  // namespace adloco

// out = A B^T for 8-bit operands with a power-of-two scale for each block of 128 (rows of A, 128 x 128
// blocks of B), on the tensor cores: TMA tiles, tcgen05.mma with the scales read from tensor memory,
// fp32 accumulators in tensor memory, one rounding in the epilogue.
#include <atomic>

#include "common.cuh"
#include "ptx.cuh"

namespace adloco {

using namespace ptx;

namespace {

constexpr uint64_t kPairLeaveNs = 1000000ull;      // 1 ms: a CTA pair leaving after a time-out; copies in flight land long before
constexpr uint64_t kLeaveLimitNs = 50000000ull;    // 50 ms per barrier while leaving after a time-out

struct Ring {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void advance(uint32_t n) {
        if (++stage == n) { stage = 0; phase ^= 1u; }
    }
};

struct MatArgs {
    int M, N, K, kb;                 // kb: blocks of 128 along K
    int tiles_n, tiles;              // tiles along N, and all
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

__device__ __forceinline__ uint32_t pack_bf16(uint32_t a, uint32_t b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(a), __uint_as_float(b));
    return *reinterpret_cast<const uint32_t*>(&h);
}
// The scale bytes of blocks 4 g .. 4 g + have - 1 of one row of A, or of one 128-row block of B; 127 (a scale of 1) where
// there is none
__device__ __forceinline__ uint32_t row_scale_word(const MatArgs& a, int m, int g, int have) {
    uint32_t w = 0x7f7f7f7fu;
    if (m >= a.M) return w;
    const uint8_t* p = a.sa + (int64_t)m * a.sa_stride + g * 4;
    if (have == 4) return *reinterpret_cast<const uint32_t*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < have) w = (w & ~(0xffu << (8 * j))) | ((uint32_t)p[j] << (8 * j));
    return w;
}
__device__ __forceinline__ uint32_t block_scale_word(const MatArgs& a, int nb, int g, int have) {
    uint32_t w = 0x7f7f7f7fu;
    if (nb * 128 >= a.N) return w;
    const uint8_t* p = a.sb + nb * a.sb_n + (int64_t)(g * 4) * a.sb_k;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < have) w = (w & ~(0xffu << (8 * j))) | ((uint32_t)p[j * a.sb_k] << (8 * j));
    return w;
}
// A scale warp's loop: the scale words of 512 of K at a time, for 128 rows of A and NB 128-row blocks of B, from global
// memory into a ring of SLOTS slots of COLS columns of tensor memory.  Lane l of every lane quarter holds, in column c,
// the word of row 32 c + l (the MMA reads each quarter's copy), so each of the four warps writes the same words.  The
// words of the next 512 of K are loaded before the wait for a free slot: without that the loads' latency, once for
// every four stages, held the MMAs up (85 us instead of 44 us at 32768 x 768 x 2304).
template <int NB, int SLOTS, int COLS, bool PAIR>
__device__ __forceinline__ void write_scales(const MatArgs& a, uint32_t tmem_sf, int worker, int workers, int tile_side, int row_offset,
                                             uint32_t sf_full, uint32_t sf_empty, volatile int* abortp) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t at0 = tmem_sf + ((uint32_t)(warp & 3) << 21);      // lane 32 * (warp mod 4) of a tensor-memory address
    const int groups = (a.kb + 3) / 4;
    uint32_t w[4], b[NB];
    auto load = [&](int tile, int g) {
        const int have = min(4, a.kb - g * 4);
        const int m0 = (tile / a.tiles_n) * tile_side + row_offset, nb = (tile % a.tiles_n) * NB;
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = row_scale_word(a, m0 + c * 32 + lane, g, have);
#pragma unroll
        for (int i = 0; i < NB; ++i) b[i] = block_scale_word(a, nb + i, g, have);
    };
    Ring sf;
    int tile = worker, g = 0;
    if (tile < a.tiles) load(tile, 0);
    while (tile < a.tiles) {
        uint32_t w0[4], b0[NB];
#pragma unroll
        for (int c = 0; c < 4; ++c) w0[c] = w[c];
#pragma unroll
        for (int i = 0; i < NB; ++i) b0[i] = b[i];
        if (++g == groups) { g = 0; tile += workers; }
        if (tile < a.tiles) load(tile, g);
        if (!__all_sync(0xffffffffu, mbar_wait(sf_empty + 8u * sf.stage, sf.phase ^ 1u, abortp, a.wait_ns))) break;
        tc_fence_after();
        const uint32_t at = at0 + sf.stage * COLS;
        tmem_st4(at, w0[0], w0[1], w0[2], w0[3]);
#pragma unroll
        for (int i = 0; i < NB; ++i) tmem_st4(at + 4 + 4 * i, b0[i], b0[i], b0[i], b0[i]);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
            if (PAIR) mbar_arrive_cluster(sf_full + 8u * sf.stage);
            else mbar_arrive(sf_full + 8u * sf.stage);
        }
        sf.advance(SLOTS);
    }
}
// 16 accumulator columns of row m to the output one by one, for outputs whose rows are not 16-byte aligned
__device__ __forceinline__ void store_elements(const MatArgs& a, int m, int col, const uint32_t (&r)[16]) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        if (col + e >= a.N) continue;
        const float v = __uint_as_float(r[e]) + (a.bias ? __ldg(a.bias + col + e) : 0.f);
        const int64_t at = (int64_t)m * a.out_stride + col + e;
        if (a.out_bf16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(a.out)[at] = v;
    }
}

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
                const int m0 = (tile / a.tiles_n) * MT, n0 = (tile % a.tiles_n) * MT;
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
        write_scales<1, MT_SLOTS, 8, false>(a, tmem + MT_SF_COL, (int)blockIdx.x, (int)gridDim.x, MT, 0, sf_full(0), sf_empty(0), abortp);
    } else {
        // ---------------- epilogue ----------------
        const uint32_t q = warp & 3;
        uint32_t n = 0;
        for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x, ++n) {
            const int m0 = (tile / a.tiles_n) * MT, n0 = (tile % a.tiles_n) * MT;
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

// ---- 256 x 256 tiles shared by a CTA pair ---------------------------------------------------------
// One MMA over the two CTAs of a cluster (cta_group::2): CTA r holds rows 128 r .. + 127 of the tile in its tensor
// memory and loads those rows of A and one half of the rows of B, 32 KB a stage for 512 clocks of tensor work --
// 64 bytes a clock, what L2 delivers to an SM; a 128 x 128 tile of its own asks for 128, a 128 x 256 one for 96.
// The accumulator takes 256 of the 512 columns of tensor memory and the scale slots need some of the rest, so there
// is no room for a second one: 16 epilogue warps empty it in one go, each 32 rows x 64 columns, into shared memory
// (rounded to the output type), hand it back, and TMA stores write the boxes while the next tile's MMAs run.
constexpr int MP_STAGES = 5;
constexpr int MP_STAGE_BYTES = 2 * MT * 128;                  // 128 rows of A and 128 of B
constexpr int MP_EPI_WARPS = 16;
constexpr int MP_BOX_BYTES = 32 * 128;                        // 32 rows of 128 bytes: one epilogue warp's store
constexpr int MP_SLOTS = 8;                                   // scale slots of 16 columns: 4 for A, 8 for B
constexpr int MP_SF_COL = 256;
constexpr int MP_SMEM = MP_STAGES * MP_STAGE_BYTES + MP_EPI_WARPS * MP_BOX_BYTES + 1024 + 256;
constexpr int MP_THREADS = 32 * (6 + MP_EPI_WARPS);           // warp 0 TMA, warp 1 MMA, warps 2-5 scales, the rest epilogue

__global__ void __launch_bounds__(MP_THREADS, 1)
blockscale_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                       const __grid_constant__ CUtensorMap tmO, const MatArgs a) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t boxes = smem_base + MP_STAGES * MP_STAGE_BYTES;
    const uint32_t bars = boxes + MP_EPI_WARPS * MP_BOX_BYTES;
    auto full_bar = [&](uint32_t s) { return bars + 8u * s; };
    auto empty_bar = [&](uint32_t s) { return bars + 8u * (MP_STAGES + s); };
    auto sf_full = [&](uint32_t s) { return bars + 8u * (2 * MP_STAGES + s); };
    auto sf_empty = [&](uint32_t s) { return bars + 8u * (2 * MP_STAGES + MP_SLOTS + s); };
    const uint32_t acc_full = bars + 8u * (2 * MP_STAGES + 2 * MP_SLOTS);
    const uint32_t acc_empty = acc_full + 8u, drain_bar = acc_full + 16u;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_cta_rank();                  // 0: the CTA that issues the MMAs
    const int worker = (int)(blockIdx.x >> 1), workers = (int)(gridDim.x >> 1);
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (uint32_t s = 0; s < MP_STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (uint32_t s = 0; s < MP_SLOTS; ++s) { mbar_init(sf_full(s), 8); mbar_init(sf_empty(s), 1); }
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, 2 * MP_EPI_WARPS);                // the epilogue warps of both CTAs
        mbar_init(drain_bar, 1);
        fence_barrier_init();
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
        prefetch_tmap(&tmO);
    }
    if (warp == 1) { tmem_alloc_pair(smem_u32(&tmem_slot), 512); tmem_relinquish_pair(); }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                        // the peer's barriers exist before anything is signalled on them
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    volatile int* abortp = &abort_flag;

    if (warp == 0) {
        // ---------------- TMA producer, one per CTA ----------------
        if (lane == 0) {
            Ring ps;
            bool ok = true;
            for (int tile = worker; ok && tile < a.tiles; tile += workers) {
                const int m0 = (tile / a.tiles_n) * 256 + (int)rank * MT, n0 = (tile % a.tiles_n) * 256 + (int)rank * MT;
                for (int k = 0; k < a.kb; ++k) {
                    if (!mbar_wait(empty_bar(ps.stage), ps.phase ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
                    const uint32_t sA = smem_base + ps.stage * MP_STAGE_BYTES;
                    const uint32_t bar = map_to_cta(full_bar(ps.stage), 0);
                    if (rank == 0) mbar_arrive_expect_tx(full_bar(ps.stage), 2 * MP_STAGE_BYTES);
                    tma_load_2d_pair(sA, &tmA, bar, k * 128, m0);
                    tma_load_2d_pair(sA + MT * 128, &tmB, bar, k * 128, n0);
                    ps.advance(MP_STAGES);
                }
            }
            if (!ok) {
                // leaving after a time-out: the byte counts of copies in flight complete on the even CTA's barriers, which the
                // odd CTA cannot wait on: both sit out a grace period far beyond the flight time of a copy
                st_cluster_u32(map_to_cta(smem_u32(&abort_flag), rank ^ 1u), 1u);
                const uint64_t t0 = globaltimer_ns();
                while (globaltimer_ns() - t0 < kPairLeaveNs) { }
            }
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (even CTA only) ----------------
        if (lane == 0 && rank == 0) {
            Ring ps, sf;
            uint32_t n = 0;
            bool ok = true;
            for (int tile = worker; ok && tile < a.tiles; tile += workers, ++n) {
                if (!mbar_wait<true>(acc_empty, (n & 1u) ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
                tc_fence_after();
                for (int k = 0; k < a.kb; ++k) {
                    if ((k & 3) == 0 && !mbar_wait<true>(sf_full(sf.stage), sf.phase, abortp, a.wait_ns)) { ok = false; break; }
                    if (!mbar_wait(full_bar(ps.stage), ps.phase, abortp, a.wait_ns)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sA = smem_base + ps.stage * MP_STAGE_BYTES, sB = sA + MT * 128;
                    const uint32_t sf_col = tmem + MP_SF_COL + sf.stage * 16u;
                    const uint32_t idesc = idesc_mxf8(256, 256, (uint32_t)k & 3u);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_mxf8_pair(tmem, smem_desc_sw128(sA + kk * 32, 16, 1024), smem_desc_sw128(sB + kk * 32, 16, 1024),
                                      idesc, sf_col, sf_col + 4, (k == 0 && kk == 0) ? 0u : 1u);
                    mma_commit_pair(empty_bar(ps.stage), 3);
                    ps.advance(MP_STAGES);
                    if ((k & 3) == 3 || k == a.kb - 1) {
                        mma_commit_pair(sf_empty(sf.stage), 3);
                        sf.advance(MP_SLOTS);
                    }
                }
                if (ok) mma_commit_pair(acc_full, 3);
            }
            if (!ok) {
                st_cluster_u32(map_to_cta(smem_u32(&abort_flag), 1u), 1u);
                mma_commit_pair(drain_bar, 1);
                int never = 0;
                mbar_wait(drain_bar, 0, &never, kLeaveLimitNs);
            }
        }
    } else if (warp < 6) {
        // ---------------- scales into this CTA's tensor memory ----------------
        write_scales<2, MP_SLOTS, 16, true>(a, tmem + MP_SF_COL, worker, workers, 256, (int)rank * MT, map_to_cta(sf_full(0), 0), sf_empty(0),
                                            abortp);
    } else {
        // ---------------- epilogue ----------------
        const uint32_t q = warp & 3, slice = (uint32_t)(warp - 6) >> 2;      // 32 rows, 64 columns of this CTA's 128 x 256
        const uint32_t acc_empty_0 = map_to_cta(acc_empty, 0);
        const uint32_t box = boxes + (uint32_t)(warp - 6) * MP_BOX_BYTES;
        const uint32_t row_addr = box + lane * 128u, taddr = tmem + ((q * 32u) << 16) + slice * 64u;
        uint32_t n = 0;
        for (int tile = worker; tile < a.tiles; tile += workers, ++n) {
            const int row0 = (tile / a.tiles_n) * 256 + (int)rank * MT + (int)q * 32;
            const int col0 = (tile % a.tiles_n) * 256 + (int)slice * 64;
            const bool some = row0 < a.M && col0 < a.N;                      // uniform across the warp
            if (!__all_sync(0xffffffffu, mbar_wait(acc_full, n & 1u, abortp, a.wait_ns))) break;
            tc_fence_after();
            if (some && a.out_vec) {
                if (lane == 0) bulk_wait_read_all();                         // the last store has read the box
                __syncwarp();
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t r[16];
                    tmem_ld16(taddr + c * 16, r);
                    tmem_ld_wait();
                    if (a.bias) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int col = col0 + c * 16 + e;
                            if (col < a.N) r[e] = __float_as_uint(__uint_as_float(r[e]) + __ldg(a.bias + col));
                        }
                    }
                    // 128-byte swizzle of the store's box: piece j of row i at piece j ^ (i mod 8)
                    if (a.out_bf16) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint32_t p[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) p[e] = pack_bf16(r[8 * j + 2 * e], r[8 * j + 2 * e + 1]);
                            st_shared_v4(row_addr + ((((uint32_t)(2 * c + j)) ^ (lane & 7u)) << 4), p[0], p[1], p[2], p[3]);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            st_shared_v4(row_addr + ((((uint32_t)(4 * (c & 1) + j)) ^ (lane & 7u)) << 4), r[4 * j], r[4 * j + 1], r[4 * j + 2],
                                         r[4 * j + 3]);
                        if (c == 1) {                                        // fp32: a box holds 32 columns, the slice is two
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) {
                                tma_store_2d(&tmO, box, col0, row0);
                                bulk_commit_group();
                                bulk_wait_read_all();
                            }
                            __syncwarp();
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acc_empty_0);             // the next tile's MMAs need not wait for the store
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    const int col = a.out_bf16 ? col0 : col0 + 32;
                    if (col < a.N) {
                        tma_store_2d(&tmO, box, col, row0);
                        bulk_commit_group();
                    }
                }
                continue;
            }
            if (some) {
                const int m = row0 + lane;
#pragma unroll 1
                for (int c = 0; c < 4; ++c) {
                    uint32_t r[16];
                    tmem_ld16(taddr + c * 16, r);
                    tmem_ld_wait();
                    if (m < a.M) store_elements(a, m, col0 + c * 16, r);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acc_empty_0);
        }
        if (lane == 0) bulk_wait_all();                                      // this warp's stores are complete
        __syncwarp();
    }

    // ---------------- teardown ----------------
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                        // neither CTA frees tensor memory or leaves while its peer still works
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem, 512);
    }
    if (threadIdx.x == 0 && abort_flag) atomicExch(a.status, (int)ADLOCO_ERR_TIMEOUT);
}

// matrix [rows, cols] of `es`-byte elements with a pitch in elements, as a 2-D map with a box of box_rows rows of
// box_cols elements (128 bytes), 128-byte swizzle; elements outside the matrix read as zero and are not written
int make_map(adloco_ctx* ctx, CUtensorMap* m, CUtensorMapDataType type, int64_t es, const void* base, int64_t rows, int64_t cols,
             int64_t pitch, uint32_t box_cols, uint32_t box_rows) {
    TensorMapEncode fn = tensor_map_encode(ctx);
    if (!fn) return ADLOCO_ERR_CUDA;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)(pitch * es)};
    const cuuint32_t box[2] = {box_cols, box_rows};
    const cuuint32_t estr[2] = {1, 1};
    const CUresult r = fn(m, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        snprintf(ctx->cuda_err, sizeof(ctx->cuda_err), "cuTensorMapEncodeTiled failed with CUresult %d", (int)r);
        return ADLOCO_ERR_CUDA;
    }
    return ADLOCO_OK;
}

}  // namespace

int launch_blockscale_matmul(adloco_ctx* ctx, const adloco_blockscale_matmul_args& p, cudaStream_t st) {
    MatArgs a;
    a.M = (int)p.M; a.N = (int)p.N; a.K = (int)p.K; a.kb = (int)((p.K + 127) / 128);
    a.sa = p.a_scale; a.sa_stride = p.a_scale_stride;
    a.sb = p.b_scale; a.sb_n = p.b_scale_stride_n; a.sb_k = p.b_scale_stride_k;
    a.bias = p.bias; a.out = p.out; a.out_stride = p.out_stride;
    a.out_bf16 = p.out_dtype == ADLOCO_BF16;
    // whole 16-byte pieces of every row: a TMA store writes a row's last piece in full, beyond the matrix too
    const int64_t piece = a.out_bf16 ? 8 : 4;
    a.out_vec = aligned16(p.out) && p.out_stride % piece == 0 && p.N % piece == 0;
    a.status = ctx->gemm_status; a.wait_ns = ctx->wait_limit_ns;
    const int64_t pair_tiles = ((p.M + 255) / 256) * ((p.N + 255) / 256);
    const bool pair = pair_tiles >= ctx->sm_count / 2 && cta_pairs_possible(ctx);
    const int64_t side = pair ? 256 : MT;
    const int64_t tm = (p.M + side - 1) / side, tn = (p.N + side - 1) / side;
    if (tm * tn > 0x7fffffff) return ADLOCO_ERR_UNSUPPORTED;
    a.tiles_n = (int)tn; a.tiles = (int)(tm * tn);
    CUtensorMap tmA, tmB, tmO;
    int rc = make_map(ctx, &tmA, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.a, p.M, p.K, p.a_stride, 128, MT);
    if (rc == ADLOCO_OK) rc = make_map(ctx, &tmB, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.b, p.N, p.K, p.b_stride, 128, MT);
    if (rc != ADLOCO_OK) return rc;
    static std::atomic<bool> attr_set[64];   // the attributes are per device
    if (!attr_set[ctx->device & 63].load()) {
        ADLOCO_CUDA_TRY(ctx, cudaFuncSetAttribute(blockscale_tile_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MT_SMEM));
        ADLOCO_CUDA_TRY(ctx, cudaFuncSetAttribute(blockscale_pair_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MP_SMEM));
        attr_set[ctx->device & 63].store(true);
    }
    if (pair) {
        tmO = tmA;                           // not looked at when the output takes no TMA stores
        if (a.out_vec) {
            rc = a.out_bf16 ? make_map(ctx, &tmO, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.out, p.M, p.N, p.out_stride, 64, 32)
                            : make_map(ctx, &tmO, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, p.out, p.M, p.N, p.out_stride, 32, 32);
            if (rc != ADLOCO_OK) return rc;
        }
        const int workers = a.tiles < ctx->sm_count / 2 ? a.tiles : ctx->sm_count / 2;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(2 * workers));
        cfg.blockDim = dim3(MP_THREADS);
        cfg.dynamicSmemBytes = MP_SMEM;
        cfg.stream = st;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 2; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        ADLOCO_CUDA_TRY(ctx, cudaLaunchKernelEx(&cfg, blockscale_pair_kernel, tmA, tmB, tmO, a));
    } else {
        blockscale_tile_kernel<<<a.tiles < ctx->sm_count ? a.tiles : ctx->sm_count, MT_THREADS, MT_SMEM, st>>>(tmA, tmB, a);
        ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    }
    ctx->launches++;
    return ADLOCO_OK;
}

}  // namespace adloco

// out = A B^T for 8-bit operands with a power-of-two scale for each block of 128 (rows of A, 128 x 128
// blocks of B), on the tensor cores: TMA tiles, tcgen05.mma with the scales read from tensor memory,
// fp32 accumulators in tensor memory, one rounding in the epilogue.
#include <atomic>

#include "common.cuh"
#include "e4m3.cuh"
#include "gemm_parts.cuh"
#include "ptx.cuh"

namespace adloco {

using namespace ptx;

namespace {

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

// An epilogue warp's box of shared memory: 32 rows of 128 bytes (64 bf16 or 32 fp32 columns), piece j of row i at piece
// j ^ (i mod 8), so that a thread's row written and a row's pieces read by neighbouring lanes fall on all banks.
constexpr int kBoxBytes = 32 * 128;
__device__ __forceinline__ uint32_t box_piece(uint32_t box, int row, int piece) { return box + row * 128u + ((uint32_t)(piece ^ (row & 7)) << 4); }

// 16 accumulator columns, col .. col + 15 of the output, of this lane's row into the box from column `at` of it on
__device__ __forceinline__ void fill_box(const MatArgs& a, uint32_t box, int lane, int at, int col, uint32_t (&r)[16]) {
    if (a.bias) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (col + e < a.N) r[e] = __float_as_uint(__uint_as_float(r[e]) + a.bias[col + e]);
    }
    if (a.out_bf16) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = pack_bf16(r[8 * j + 2 * e], r[8 * j + 2 * e + 1]);
            st_shared_v4(box_piece(box, lane, at / 8 + j), p[0], p[1], p[2], p[3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) st_shared_v4(box_piece(box, lane, at / 4 + j), r[4 * j], r[4 * j + 1], r[4 * j + 2], r[4 * j + 3]);
    }
}
// The box to the output at (row0, col): whole pieces where rows are 16-byte aligned, else element by element, both along rows.
__device__ __forceinline__ void flush_box(const MatArgs& a, uint32_t box, int lane, int row0, int col) {
    __syncwarp();
    const int es = a.out_bf16 ? 2 : 4;
    char* out = static_cast<char*>(a.out) + ((int64_t)row0 * a.out_stride + col) * es;
    const int64_t pitch = a.out_stride * es;
    if (a.out_vec) {
        const int piece = lane & 7;
        if (col + piece * (16 / es) < a.N) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = i * 4 + (lane >> 3);
                uint4 v;
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(box_piece(box, row, piece)) : "memory");
                if (row0 + row < a.M) __stcs(reinterpret_cast<uint4*>(out + row * pitch + piece * 16), v);
            }
        }
    } else {
        const int rows = min(32, a.M - row0);
#pragma unroll 4
        for (int row = 0; row < rows; ++row) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int c = h * 32 + lane;                                    // bf16: two sweeps of 32 columns; fp32: one
                if (h * 32 * es >= 128 || col + c >= a.N) continue;
                const uint32_t from = box_piece(box, row, c * es / 16) + (uint32_t)(c * es & 15);
                if (es == 2) {
                    unsigned short v;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(from) : "memory");
                    reinterpret_cast<unsigned short*>(out + row * pitch)[c] = v;
                } else {
                    uint32_t v;
                    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
                    reinterpret_cast<uint32_t*>(out + row * pitch)[c] = v;
                }
            }
        }
    }
    __syncwarp();
}

// The tiles of one worker: dealt round, the tiles along N fastest, so that all workers sit on the same few rows of A at a
// time -- a tile of A is then read from HBM once and from L2 by the rest.  (Runs of tiles along M instead let a tile's uses
// drift apart, past what L2 keeps beside the output's stream: 37888 x 768 x 2304 took 76 us, 55 without the stores.)
struct TileWalk {
    int left, m, n, step_m, step_n, line;                  // no division on the way
    __device__ __forceinline__ TileWalk(const MatArgs& a, int worker, int workers) : line(a.tiles_n) {
        left = worker < a.tiles ? (a.tiles - worker - 1) / workers + 1 : 0;
        m = worker / line;
        n = worker % line;
        step_m = workers / line;
        step_n = workers % line;
    }
    __device__ __forceinline__ bool more() const { return left > 0; }
    __device__ __forceinline__ void next() {
        --left;
        m += step_m;
        n += step_n;
        if (n >= line) { n -= line; ++m; }
    }
};

// The four scale warps' loop: the scale words (four blocks' bytes) of 512 of K at a time, for 128 rows of A and TILE_N
// rows of B, from global memory into a ring of slots in shared memory: 512 bytes for A, then 512 for each 128 rows of B,
// the word of row r at 16 (r mod 32) + 4 (r / 32), which is how tcgen05.cp spreads them over tensor memory.  A's words
// come by cp.async, each warp's own 32 rows; B's bytes lie anywhere and come by one load of 8 lanes.  A turn issues its
// loads, then finishes the turn before, so that loads have a turn's time and a slot is ready two turns before it is used.
// The MMA thread copies a slot to tensor memory in front of the MMAs that read it.  (Written into tensor memory by these
// warps instead, a turn took 2400 clocks: tcgen05.st queues behind the MMAs in flight.  32768 x 768 x 2304: 84 us.)
// Rows of A's scales are whole aligned words; what a row's last word holds beyond its blocks is not used.
constexpr int kScaleSlots = 4;
template <int TILE_N>
__host__ __device__ constexpr int scale_slot_bytes() { return 512 * (1 + (TILE_N + 127) / 128); }
template <int TILE_M, int TILE_N>
__device__ __forceinline__ void fetch_scales(const MatArgs& a, uint32_t ring, TileWalk walk, int row_offset, uint32_t sf_full,
                                             uint32_t sf_empty, volatile int* abortp) {
    constexpr int BLOCKS = (TILE_N + 127) / 128, SLOT = scale_slot_bytes<TILE_N>();
    const int quarter = __shfl_sync(0xffffffffu, (threadIdx.x >> 5) & 3, 0), lane = threadIdx.x & 31;
    const int groups = (a.kb + 3) / 4;
    uint32_t byte[2], shift[2];                           // lanes 0-3, 4-7: B's bytes of the two 128-row blocks
    int g = 0, m0 = 0, n0 = 0;                            // of the next fetch
    Ring fill, done;
    auto fetch = [&](int i) -> bool {                     // turn's loads into slot fill.stage
        if (!wait_warp<false>(sf_empty + 8u * fill.stage, fill.phase ^ 1u, abortp, a.wait_ns)) return false;
        if (g == 0) { m0 = walk.m * TILE_M + row_offset; n0 = walk.n * TILE_N; }
        const int m = m0 + quarter * 32 + lane, nb = (n0 >> 7) + ((lane >> 2) & 1), k = g * 4 + (lane & 3);
        const uint32_t to = ring + fill.stage * SLOT + (uint32_t)(lane * 16 + quarter * 4);
        if (m < a.M)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(a.sa + (int64_t)m * a.sa_stride + g * 4) : "memory");
        asm volatile("cp.async.commit_group;" ::: "memory");
        byte[i] = 127u;
        if (lane < 8 && nb * 128 < a.N && k < a.kb) byte[i] = a.sb[nb * a.sb_n + k * a.sb_k];
        shift[i] = (uint32_t)(n0 & 127);                  // rows of the tile's first 128-row block before the tile
        if (++g == groups) { g = 0; walk.next(); }
        fill.advance(kScaleSlots);
        return true;
    };
    if (!walk.more() || !fetch(0)) return;
    for (;;) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool last = !walk.more();
            if (!last && !fetch(i ^ 1)) {                 // leaving after a time-out: the turn before has copies in flight
                asm volatile("cp.async.wait_all;" ::: "memory");
                return;
            }
            if (last) asm volatile("cp.async.wait_group 0;" ::: "memory");
            else asm volatile("cp.async.wait_group 1;" ::: "memory");
            const uint32_t part = byte[i] << (8 * (lane & 3));
            if (quarter < BLOCKS) {                       // warp q: the q-th 128 rows of B's part
                const uint32_t b0 = __reduce_or_sync(0xffffffffu, lane < 4 ? part : 0u);
                const uint32_t b1 = BLOCKS > 1 ? __reduce_or_sync(0xffffffffu, lane >= 4 && lane < 8 ? part : 0u) : b0;
                uint32_t v[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = shift[i] + 128u * quarter + 32u * c < 128u ? b0 : b1;
                st_shared_v4(ring + done.stage * SLOT + (uint32_t)(512 + quarter * 512 + lane * 16), v[0], v[1], v[2], v[3]);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(sf_full + 8u * done.stage);
            done.advance(kScaleSlots);
            if (last) return;
        }
    }
}
// ---- 128 x 128 tiles, one CTA each --------------------------------------------------------------
// Persistent, 320 threads: warp 0 TMA, warp 1 MMA, warps 2-5 scales, warps 6-9 epilogue.  A stage is 128 of K (a
// 128-byte swizzle row of either operand): four MMAs of K = 32 that use the same byte of the scale words.  A scale
// word holds the bytes of four stages: the scale warps bring the words of 512 of K at a time.
constexpr int MT = 128;
constexpr int MT_STAGES = 6;
constexpr int MT_STAGE_BYTES = 2 * MT * 128;
constexpr int MT_SF_COL = 2 * MT;                             // tensor memory: two accumulators, then the slots
constexpr int MT_SMEM = MT_STAGES * MT_STAGE_BYTES + 4 * kBoxBytes + 1024 + 256 + kScaleSlots * scale_slot_bytes<MT>();
constexpr int MT_THREADS = 320;

__global__ void __launch_bounds__(MT_THREADS, 1)
blockscale_tile_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB, const MatArgs a) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t boxes = smem_base + MT_STAGES * MT_STAGE_BYTES, bars = boxes + 4 * kBoxBytes, sf_ring = bars + 256;
    auto full_bar = [&](uint32_t s) { return bars + 8u * s; };
    auto empty_bar = [&](uint32_t s) { return bars + 8u * (MT_STAGES + s); };
    auto sf_full = [&](uint32_t s) { return bars + 8u * (2 * MT_STAGES + s); };
    auto sf_empty = [&](uint32_t s) { return bars + 8u * (2 * MT_STAGES + kScaleSlots + s); };
    auto acc_full = [&](uint32_t s) { return bars + 8u * (2 * MT_STAGES + 2 * kScaleSlots + s); };
    auto acc_empty = [&](uint32_t s) { return bars + 8u * (2 * MT_STAGES + 2 * kScaleSlots + 2 + s); };
    const uint32_t drain_bar = bars + 8u * (2 * MT_STAGES + 2 * kScaleSlots + 4);
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // warp: known to be uniform
    TileWalk walk(a, (int)blockIdx.x, (int)gridDim.x);
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (uint32_t s = 0; s < MT_STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (uint32_t s = 0; s < kScaleSlots; ++s) { mbar_init(sf_full(s), 4); mbar_init(sf_empty(s), 1); }
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
    after_predecessor();
    const uint32_t tmem = tmem_slot;
    volatile int* abortp = &abort_flag;

    if (warp == 0) {
        // ---------------- TMA producer ----------------
        if (lane == 0) {
            Ring ps;
            uint32_t issued = 0;
            bool ok = true;
            for (; ok && walk.more(); walk.next()) {
                const int m0 = walk.m * MT, n0 = walk.n * MT;
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
        // ---------------- MMA issuer (the whole warp keeps step, one lane issues) ----------------
        const bool leader = elect_one();
        const uint64_t desc0 = smem_desc_sw128(0, 16, 1024);
        Ring ps, sf;
        uint32_t n = 0;
        bool ok = true;
        for (; ok && walk.more(); walk.next(), ++n) {
            const uint32_t buf = n & 1u;
            if (!wait_warp<false>(acc_empty(buf), ((n >> 1) & 1u) ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
            for (int k = 0; k < a.kb; ++k) {
                if ((k & 3) == 0 && !wait_warp<false>(sf_full(sf.stage), sf.phase, abortp, a.wait_ns)) { ok = false; break; }
                if (!wait_warp<false>(full_bar(ps.stage), ps.phase, abortp, a.wait_ns)) { ok = false; break; }
                tc_fence_after();
                if (leader) {
                    const uint32_t sf_col = tmem + MT_SF_COL + sf.stage * 16u, slot = sf_ring + sf.stage * scale_slot_bytes<MT>();
                    if ((k & 3) == 0) {
                        tmem_copy_scales(sf_col, smem_desc_rows16(slot));
                        tmem_copy_scales(sf_col + 4, smem_desc_rows16(slot + 512));
                    }
                    // K-major, 128-byte swizzle: 32 elements further along K = 32 bytes = 2 units of the descriptor's address
                    const uint64_t dA = desc0 + ((smem_base + ps.stage * MT_STAGE_BYTES) >> 4), dB = dA + ((MT * 128) >> 4);
                    const uint32_t idesc = idesc_mxf8(MT, MT, (uint32_t)k & 3u);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_mxf8(tmem + buf * MT, dA + 2 * kk, dB + 2 * kk, idesc, sf_col, sf_col + 4, (k == 0 && kk == 0) ? 0u : 1u);
                    mma_commit(empty_bar(ps.stage));
                    if ((k & 3) == 3 || k == a.kb - 1) mma_commit(sf_empty(sf.stage));
                }
                __syncwarp();
                ps.advance(MT_STAGES);
                if ((k & 3) == 3 || k == a.kb - 1) sf.advance(kScaleSlots);
            }
            if (ok && leader) mma_commit(acc_full(buf));
            __syncwarp();
        }
        if (!ok && leader) {
            mma_commit(drain_bar);
            int never = 0;
            mbar_wait(drain_bar, 0, &never, kLeaveLimitNs);
        }
        __syncwarp();
    } else if (warp < 6) {
        // ---------------- scales ----------------
        fetch_scales<MT, MT>(a, sf_ring, walk, 0, sf_full(0), sf_empty(0), abortp);
    } else {
        // ---------------- epilogue ----------------
        const uint32_t q = warp & 3;
        uint32_t n = 0;
        for (; walk.more(); walk.next(), ++n) {
            const int m0 = walk.m * MT, n0 = walk.n * MT;
            const uint32_t buf = n & 1u;
            if (!__all_sync(0xffffffffu, mbar_wait(acc_full(buf), (n >> 1) & 1u, abortp, a.wait_ns))) break;
            tc_fence_after();
            const uint32_t box = boxes + q * kBoxBytes;
            const int row0 = m0 + (int)q * 32, wide = a.out_bf16 ? 64 : 32;      // columns of a box
#pragma unroll 1
            for (int c = 0; c < MT; c += 16) {
                uint32_t r[16];
                tmem_ld16(tmem + ((q * 32u) << 16) + buf * MT + c, r);
                tmem_ld_wait();
                if (row0 >= a.M || n0 + (c & -wide) >= a.N) continue;            // uniform across the warp
                fill_box(a, box, lane, c & (wide - 1), n0 + c, r);
                if (((c + 16) & (wide - 1)) == 0) flush_box(a, box, lane, row0, n0 + (c & -wide));
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

// ---- 256 x 192 tiles shared by a CTA pair ---------------------------------------------------------
// One MMA over the two CTAs of a cluster (cta_group::2): CTA r holds rows 128 r .. + 127 of the tile in its tensor
// memory and loads those rows of A and one half of the rows of B.  192 columns leave room in tensor memory for two
// accumulators and the scale slots, so the tensor pipe never waits for the epilogue: with one accumulator of 256
// columns a tile's hand-over (last MMA, signal, read-out, signal, first MMA) cost about 1.3 us beside the 1.8 us of
// a tile's MMAs at K = 768.
// What bounds the rest is shared memory: a stage's MMAs read 28 KB of it and the copies write as much, 448 of its clocks
// against 384 of the tensor pipe (measured at long K: 447).  RESIDENT: where a panel of B (96 rows a CTA, up to 768 of K)
// fits, a worker keeps one panel, loaded once, and only A is streamed, 16 KB a stage instead of 28.
constexpr int MP_N = 192;
constexpr int MP_STAGES = 6;
constexpr int MP_A_BYTES = MT * 128, MP_B_BYTES = (MP_N / 2) * 128;
constexpr int MP_RESIDENT_KB = 6;                             // largest K of a resident panel, in blocks of 128
constexpr int MP_EPI_WARPS = 4 * MP_N / 64;                   // each 32 rows x 64 columns of a CTA's 128 x 192
constexpr int MP_SF_COL = 2 * MP_N;
constexpr int MP_SMEM = MP_STAGES * (MP_A_BYTES + MP_B_BYTES) + MP_EPI_WARPS * kBoxBytes + 1024 + 512 + kScaleSlots * scale_slot_bytes<MP_N>();
constexpr int MP_THREADS = 32 * (6 + MP_EPI_WARPS);           // warp 0 TMA, warp 1 MMA, warps 2-5 scales, the rest epilogue
static_assert(MP_RESIDENT_KB <= MP_STAGES, "a resident panel takes the B parts of the ring");

template <bool RESIDENT>
__global__ void __launch_bounds__(MP_THREADS, 1)
blockscale_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                       const __grid_constant__ CUtensorMap tmO, const MatArgs a) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t panel = smem_base + MP_STAGES * MP_A_BYTES;         // the B part of stage s, or block k of a resident panel
    const uint32_t boxes = panel + MP_STAGES * MP_B_BYTES;
    const uint32_t bars = boxes + MP_EPI_WARPS * kBoxBytes, sf_ring = bars + 512;
    auto full_bar = [&](uint32_t s) { return bars + 8u * s; };
    auto empty_bar = [&](uint32_t s) { return bars + 8u * (MP_STAGES + s); };
    auto sf_full = [&](uint32_t s) { return bars + 8u * (2 * MP_STAGES + s); };
    auto sf_empty = [&](uint32_t s) { return bars + 8u * (2 * MP_STAGES + kScaleSlots + s); };
    auto acc_full = [&](uint32_t s) { return bars + 8u * (2 * MP_STAGES + 2 * kScaleSlots + s); };
    auto acc_empty = [&](uint32_t s) { return bars + 8u * (2 * MP_STAGES + 2 * kScaleSlots + 2 + s); };
    auto panel_full = [&](uint32_t k) { return bars + 8u * (2 * MP_STAGES + 2 * kScaleSlots + 4 + k); };
    const uint32_t drain_bar = bars + 8u * (2 * MP_STAGES + 2 * kScaleSlots + 4 + MP_RESIDENT_KB);
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // warp: known to be uniform
    const uint32_t rank = cluster_cta_rank();                  // 0: the CTA that issues the MMAs
    TileWalk walk(a, (int)(blockIdx.x >> 1), (int)(gridDim.x >> 1));
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (uint32_t s = 0; s < MP_STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        // the even CTA's four scale warps and word from the odd CTA that its four are done
        for (uint32_t s = 0; s < kScaleSlots; ++s) { mbar_init(sf_full(s), rank == 0 ? 5 : 4); mbar_init(sf_empty(s), 1); }
        for (uint32_t s = 0; s < 2; ++s) { mbar_init(acc_full(s), 1); mbar_init(acc_empty(s), 2 * MP_EPI_WARPS); }
        for (uint32_t k = 0; k < MP_RESIDENT_KB; ++k) mbar_init(panel_full(k), 1);
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
    after_predecessor();
    const uint32_t tmem = tmem_slot;
    volatile int* abortp = &abort_flag;

    if (warp == 0) {
        // ---------------- TMA producer, one per CTA ----------------
        if (lane == 0) {
            Ring ps;
            bool ok = true;
            bool fresh = RESIDENT;                             // the panel comes along with the first tile
            for (; ok && walk.more(); walk.next()) {
                const int m0 = walk.m * 256 + (int)rank * MT, n0 = walk.n * MP_N + (int)rank * (MP_N / 2);
                for (int k = 0; k < a.kb; ++k) {
                    if (!mbar_wait(empty_bar(ps.stage), ps.phase ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
                    const uint32_t bar = map_to_cta(full_bar(ps.stage), 0);
                    if (rank == 0) mbar_arrive_expect_tx(full_bar(ps.stage), 2 * (MP_A_BYTES + (RESIDENT ? 0 : MP_B_BYTES)));
                    tma_load_2d_pair(smem_base + ps.stage * MP_A_BYTES, &tmA, bar, k * 128, m0);
                    if (!RESIDENT) {
                        tma_load_2d_pair(panel + ps.stage * MP_B_BYTES, &tmB, bar, k * 128, n0);
                    } else if (fresh) {
                        if (rank == 0) mbar_arrive_expect_tx(panel_full(k), 2 * MP_B_BYTES);
                        tma_load_2d_pair(panel + k * MP_B_BYTES, &tmB, map_to_cta(panel_full(k), 0), k * 128, n0);
                    }
                    ps.advance(MP_STAGES);
                }
                fresh = false;
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
        // ---------------- MMA issuer (even CTA only; the whole warp keeps step, one lane issues) ----------------
        if (rank == 0) {
            const bool leader = elect_one();
            const uint64_t desc0 = smem_desc_sw128(0, 16, 1024);
            Ring ps, sf;
            uint32_t n = 0;
            bool ok = true;
            for (; ok && walk.more(); walk.next(), ++n) {
                const uint32_t buf = n & 1u;
                if (!wait_warp<true>(acc_empty(buf), ((n >> 1) & 1u) ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
                for (int k = 0; k < a.kb; ++k) {
                    if ((k & 3) == 0 && !wait_warp<true>(sf_full(sf.stage), sf.phase, abortp, a.wait_ns)) { ok = false; break; }
                    if (RESIDENT && n == 0 && !wait_warp<false>(panel_full(k), 0, abortp, a.wait_ns)) { ok = false; break; }
                    if (!wait_warp<false>(full_bar(ps.stage), ps.phase, abortp, a.wait_ns)) { ok = false; break; }
                    tc_fence_after();
                    if (leader) {
                        // 32 elements further along K = 32 bytes = 2 units of the descriptor's address
                        const uint64_t dA = desc0 + ((smem_base + ps.stage * MP_A_BYTES) >> 4);
                        const uint64_t dB = desc0 + ((panel + (RESIDENT ? (uint32_t)k : ps.stage) * MP_B_BYTES) >> 4);
                        const uint32_t sf_col = tmem + MP_SF_COL + sf.stage * 16u, slot = sf_ring + sf.stage * scale_slot_bytes<MP_N>();
                        if ((k & 3) == 0) {
                            tmem_copy_scales_pair(sf_col, smem_desc_rows16(slot));
                            tmem_copy_scales_pair(sf_col + 4, smem_desc_rows16(slot + 512));
                            tmem_copy_scales_pair(sf_col + 8, smem_desc_rows16(slot + 1024));
                        }
                        const uint32_t idesc = idesc_mxf8(256, MP_N, (uint32_t)k & 3u);
#pragma unroll
                        for (int kk = 0; kk < 4; ++kk)
                            mma_mxf8_pair(tmem + buf * MP_N, dA + 2 * kk, dB + 2 * kk, idesc, sf_col, sf_col + 4, (k == 0 && kk == 0) ? 0u : 1u);
                        mma_commit_pair(empty_bar(ps.stage), 3);
                        if ((k & 3) == 3 || k == a.kb - 1) mma_commit_pair(sf_empty(sf.stage), 3);
                    }
                    __syncwarp();
                    ps.advance(MP_STAGES);
                    if ((k & 3) == 3 || k == a.kb - 1) sf.advance(kScaleSlots);
                }
                if (ok && leader) mma_commit_pair(acc_full(buf), 3);
                __syncwarp();
            }
            if (!ok && leader) {
                st_cluster_u32(map_to_cta(smem_u32(&abort_flag), 1u), 1u);
                mma_commit_pair(drain_bar, 1);
                int never = 0;
                mbar_wait(drain_bar, 0, &never, kLeaveLimitNs);
            }
            __syncwarp();
        } else {
            // the odd CTA's: passes its scale warps' signals on to the even CTA.  A release at cluster scope waits for every
            // load that its thread has in flight, and the scale warps always have some: signalled by them directly, a turn
            // took 2700 clocks.
            const uint32_t there = map_to_cta(sf_full(0), 0);
            Ring sf;
            bool ok = true;
            for (; ok && walk.more(); walk.next()) {
                for (int k = 0; k < a.kb; k += 4) {
                    if (!wait_warp<false>(sf_full(sf.stage), sf.phase, abortp, a.wait_ns)) { ok = false; break; }
                    if (lane == 0) mbar_arrive_cluster(there + 8u * sf.stage);
                    sf.advance(kScaleSlots);
                }
            }
        }
    } else if (warp < 6) {
        // ---------------- this CTA's scales ----------------
        fetch_scales<256, MP_N>(a, sf_ring, walk, (int)rank * MT, sf_full(0), sf_empty(0), abortp);
    } else {
        // ---------------- epilogue ----------------
        const uint32_t q = warp & 3, slice = (uint32_t)(warp - 6) >> 2;
        const uint32_t acc_empty_0 = map_to_cta(acc_empty(0), 0);
        const uint32_t box = boxes + (uint32_t)(warp - 6) * kBoxBytes;
        uint32_t n = 0;
        for (; walk.more(); walk.next(), ++n) {
            const uint32_t buf = n & 1u;
            const uint32_t taddr = tmem + ((q * 32u) << 16) + buf * MP_N + slice * 64u;
            const int row0 = walk.m * 256 + (int)rank * MT + (int)q * 32;
            const int col0 = walk.n * MP_N + (int)slice * 64;
            const bool some = row0 < a.M && col0 < a.N;                      // uniform across the warp
            if (!__all_sync(0xffffffffu, mbar_wait(acc_full(buf), (n >> 1) & 1u, abortp, a.wait_ns))) break;
            tc_fence_after();
            if (some && a.out_vec) {
                if (lane == 0) bulk_wait_read_all();                         // the last store has read the box
                __syncwarp();
            }
#pragma unroll 1
            for (int c = 0; c < 64; c += 16) {
                uint32_t r[16];
                tmem_ld16(taddr + c, r);
                tmem_ld_wait();
                if (c == 48) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster_relaxed(acc_empty_0 + 8u * buf);
                }
                if (!some) continue;
                fill_box(a, box, lane, a.out_bf16 ? c : c & 31, col0 + c, r);
                const bool full = a.out_bf16 ? c == 48 : (c & 16) != 0;      // 64 columns of bf16, 32 of fp32
                const int col = a.out_bf16 ? col0 : col0 + (c & 32);
                if (!full || col >= a.N) continue;
                if (!a.out_vec) {
                    flush_box(a, box, lane, row0, col);
                    continue;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    tma_store_2d(&tmO, box, col, row0);
                    bulk_commit_group();
                    if (c < 48) bulk_wait_read_all();
                }
                __syncwarp();
            }
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

// ---- few rows of A -----------------------------------------------------------------------------------
// Up to 16 tokens (8 tokens of 4096 x 4096: 5.4 us against 10.7 us in 128 x 128 tiles; with 17 to 32 the tiles win, 10.7 us
// against 14): the time is B's bytes from memory.  A block takes 16 rows of B, its warps the blocks of 128 of K in
// turn; a lane loads 16 bytes of two rows of B and of a row of each eight of A straight into the fragments of the warp's
// own matrix instruction (m16n8k32, B's rows as its M): the order of K within 64 is the same for both and does not
// matter.  A block of 128's sum is scaled in fp32 and added up; the warps' sums meet in shared memory in a fixed order.
constexpr int FR_ROWS = 16, FR_MAX_WARPS = 16, FR_MAX_M = 16;
__device__ __forceinline__ uint4 bytes16(const uint8_t* row, int k, int K) {      // zeros beyond K
    if (k + 16 <= K) return *reinterpret_cast<const uint4*>(row + k);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (k + i < K) w[i >> 2] |= (uint32_t)row[k + i] << (8 * (i & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
struct FewArgs {
    MatArgs a;
    const uint8_t *A, *B;
    int64_t a_stride, b_stride;
};
template <int TILES>                                                                // of eight rows of A
__global__ void __launch_bounds__(32 * FR_MAX_WARPS) blockscale_few_kernel(const __grid_constant__ FewArgs p) {
    extern __shared__ float sums[];                                                 // [warps][TILES * 8][FR_ROWS + 1]
    after_predecessor();
    const MatArgs& a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, g = lane >> 2, t = lane & 3;
    const int n0 = (int)blockIdx.x * FR_ROWS;
    const bool r0 = n0 + g < a.N, r1 = n0 + g + 8 < a.N;
    const uint8_t* b0 = p.B + (int64_t)(n0 + g) * p.b_stride;
    const uint8_t* b1 = b0 + 8 * p.b_stride;
    const uint8_t* sb = a.sb + (n0 >> 7) * a.sb_n;
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    float acc[TILES][4];
#pragma unroll
    for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
#pragma unroll 2
    for (int kb = warp; kb < a.kb; kb += warps) {
        uint4 w0[2], w1[2], x[TILES][2];
        uint32_t sa[TILES][2];
        const uint32_t sbyte = sb[kb * a.sb_k];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = kb * 128 + h * 64 + t * 16;
            w0[h] = r0 && k < a.K ? bytes16(b0, k, a.K) : none;
            w1[h] = r1 && k < a.K ? bytes16(b1, k, a.K) : none;
#pragma unroll
            for (int j = 0; j < TILES; ++j) {
                const int m = j * 8 + g;
                x[j][h] = m < a.M && k < a.K ? bytes16(p.A + (int64_t)m * p.a_stride, k, a.K) : none;
            }
        }
#pragma unroll
        for (int j = 0; j < TILES; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int m = j * 8 + 2 * t + i;
                sa[j][i] = m < a.M ? (uint32_t)a.sa[(int64_t)m * a.sa_stride + kb] : 127u;
            }
        const float fb = scale_of(sbyte);
#pragma unroll
        for (int j = 0; j < TILES; ++j) {
            float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                mma_e4m3(d, w0[h].x, w1[h].x, w0[h].y, w1[h].y, x[j][h].x, x[j][h].y);
                mma_e4m3(d, w0[h].z, w1[h].z, w0[h].w, w1[h].w, x[j][h].z, x[j][h].w);
            }
            // the two scales one after the other: their product may leave the range of fp32 where the result does not
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] = fmaf(d[i] * scale_of(sa[j][i & 1]), fb, acc[j][i]);
        }
    }
    float* mine = sums + warp * (TILES * 8) * (FR_ROWS + 1);
#pragma unroll
    for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[(j * 8 + 2 * t + (i & 1)) * (FR_ROWS + 1) + g + 8 * (i >> 1)] = acc[j][i];
    __syncthreads();
    for (int i = threadIdx.x; i < TILES * 8 * FR_ROWS; i += blockDim.x) {
        const int m = i / FR_ROWS, r = i % FR_ROWS, n = n0 + r;
        if (m >= a.M || n >= a.N) continue;
        float v = 0.f;
        for (int w = 0; w < warps; ++w) v += sums[(w * TILES * 8 + m) * (FR_ROWS + 1) + r];
        if (a.bias) v += a.bias[n];
        const int64_t at = (int64_t)m * a.out_stride + n;
        if (a.out_bf16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(a.out)[at] = v;
    }
}

}  // namespace

int launch_blockscale_matmul(adloco_ctx* ctx, const adloco_blockscale_matmul_args& p, cudaStream_t st) {
    MatArgs a;
    a.M = (int)p.M; a.N = (int)p.N; a.K = (int)p.K; a.kb = (int)((p.K + 127) / 128);
    a.sa = p.a_scale; a.sa_stride = p.a_scale_stride;
    a.sb = p.b_scale; a.sb_n = p.b_scale_stride_n; a.sb_k = p.b_scale_stride_k;
    a.bias = p.bias; a.out = p.out; a.out_stride = p.out_stride;
    a.out_bf16 = p.out_dtype == ADLOCO_BF16;
    // whole 16-byte pieces of every row (a TMA store writes a row's last piece in full, beyond the matrix too)
    const int64_t piece = a.out_bf16 ? 8 : 4;
    a.out_vec = aligned16(p.out) && p.out_stride % piece == 0 && p.N % piece == 0;
    a.status = ctx->gemm_status; a.wait_ns = ctx->wait_limit_ns;
    a.tiles_n = a.tiles = 0;
    if (p.M <= FR_MAX_M) {
        FewArgs f;
        f.a = a;
        f.A = static_cast<const uint8_t*>(p.a); f.a_stride = p.a_stride;
        f.B = static_cast<const uint8_t*>(p.b); f.b_stride = p.b_stride;
        const int warps = a.kb < FR_MAX_WARPS ? a.kb : FR_MAX_WARPS;
        const dim3 grid((unsigned)((p.N + FR_ROWS - 1) / FR_ROWS));
        const int tiles = p.M <= 8 ? 1 : 2;
        const size_t smem = (size_t)warps * tiles * 8 * (FR_ROWS + 1) * sizeof(float);
        const cudaError_t e = tiles == 1 ? launch_early(blockscale_few_kernel<1>, grid, 32 * warps, smem, st, 1, f)
                                         : launch_early(blockscale_few_kernel<2>, grid, 32 * warps, smem, st, 1, f);
        ADLOCO_CUDA_TRY(ctx, e);
        ctx->launches++;
        return ADLOCO_OK;
    }
    const int64_t pair_tiles = ((p.M + 255) / 256) * ((p.N + MP_N - 1) / MP_N);
    const bool pair = pair_tiles >= ctx->sm_count / 2 && cta_pairs_possible(ctx);
    const int64_t tm = (p.M + (pair ? 255 : MT - 1)) / (pair ? 256 : MT), tn = (p.N + (pair ? MP_N : MT) - 1) / (pair ? MP_N : MT);
    if (tm * tn > 0x7fffffff) return ADLOCO_ERR_UNSUPPORTED;
    a.tiles_n = (int)tn; a.tiles = (int)(tm * tn);
    CUtensorMap tmA, tmB, tmO;
    int rc = make_map(ctx, &tmA, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.a, p.M, p.K, p.a_stride, 128, MT);
    if (rc == ADLOCO_OK) rc = make_map(ctx, &tmB, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p.b, p.N, p.K, p.b_stride, 128, pair ? MP_N / 2 : MT);
    if (rc != ADLOCO_OK) return rc;
    static std::atomic<bool> attr_set[64];   // the attributes are per device
    if (!attr_set[ctx->device & 63].load()) {
        ADLOCO_CUDA_TRY(ctx, cudaFuncSetAttribute(blockscale_tile_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MT_SMEM));
        ADLOCO_CUDA_TRY(ctx, cudaFuncSetAttribute(blockscale_pair_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, MP_SMEM));
        ADLOCO_CUDA_TRY(ctx, cudaFuncSetAttribute(blockscale_pair_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, MP_SMEM));
        attr_set[ctx->device & 63].store(true);
    }
    if (pair) {
        tmO = tmA;                           // not looked at when the output takes no TMA stores
        if (a.out_vec) {
            rc = a.out_bf16 ? make_map(ctx, &tmO, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.out, p.M, p.N, p.out_stride, 64, 32)
                            : make_map(ctx, &tmO, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, p.out, p.M, p.N, p.out_stride, 32, 32);
            if (rc != ADLOCO_OK) return rc;
        }
        const int most = ctx->sm_count / 2;
        // a worker keeps its panel when the workers in use are a multiple of the panels; that may leave some idle and take more
        // rounds, against stages of 475 clocks of shared memory instead of 571 (K = 768, with the epilogue): 54.8 us against 56.1 at
        // 32768 x 2304 x 768 with 22 rounds against 21, 24.8 against 23.3 at 32768 x 768 x 768 with 8 against 7
        const int groups = most / a.tiles_n, kept = groups * a.tiles_n;
        const int64_t rounds = (a.tiles + most - 1) / most, rounds_kept = groups ? (tm + groups - 1) / groups : 0;
        const bool resident = a.kb <= MP_RESIDENT_KB && groups > 0 && rounds_kept * 10 <= rounds * 11;
        const int workers = resident ? kept : a.tiles < most ? a.tiles : most;
        if (resident) ADLOCO_CUDA_TRY(ctx, launch_early(blockscale_pair_kernel<true>, dim3(2 * workers), MP_THREADS, MP_SMEM, st, 2, tmA, tmB, tmO, a));
        else ADLOCO_CUDA_TRY(ctx, launch_early(blockscale_pair_kernel<false>, dim3(2 * workers), MP_THREADS, MP_SMEM, st, 2, tmA, tmB, tmO, a));
    } else {
        ADLOCO_CUDA_TRY(ctx, launch_early(blockscale_tile_kernel, dim3(a.tiles < ctx->sm_count ? a.tiles : ctx->sm_count), MT_THREADS, MT_SMEM,
                                          st, 1, tmA, tmB, a));
    }
    ctx->launches++;
    return ADLOCO_OK;
}

}  // namespace adloco

// Linear layers in bf16 with what follows them in the product's epilogue: bias, activation and residual; the gated pair
// of projections act(x Wg^T) * (x Wu^T); and the way back through either,
//   dx = (dy W) act'(z)      d_gate = (dy Wd) up act'(gate),  d_up = (dy Wd) act(gate).
// What the backward pass needs (z, or gate and up) is kept in bf16 or in 8 bits with a power-of-two scale for each block
// of 128 of a row, written by the forward epilogue and read by the backward one; the layer's input is recomputed there.
#include <algorithm>
#include <atomic>
#include <cuda_fp8.h>

#include "common.cuh"
#include "e4m3.cuh"
#include "f32x2.cuh"
#include "gemm_parts.cuh"
#include "ptx.cuh"

namespace adloco {

using namespace ptx;

namespace {

enum Kind { LINEAR, LINEAR_BACK, GATED, GATED_BACK };
enum Form { kNone, kBf16, kF32, kBytes };
// What the epilogue takes for a product: the tensor cores' sum as it is, or the parts of K added up in registers, for outputs
// in fp32 or ones whose sums go to 8 bits.
enum Sum { kPlain, kSummed, kSummedF32 };
enum { IN0, IN1, OUT0, OUT1, OUT2, SIDES };

// An elementwise operand or output of the epilogue.  Its box: 32 rows x 32 columns in shared memory, one for the even
// chunks of 32 columns and one for the odd ones (the same one where the epilogue does not fetch ahead).
struct Side {
    void* p = nullptr;
    int64_t pitch = 0;                // elements
    uint8_t* scale = nullptr;
    int64_t scale_pitch = 0;
    int form = kNone;
    int tma = 0;                      // 1: boxes go by TMA; 0: by the warp's own accesses, whole 16-byte pieces where `pieces`
    int pieces = 0;
    uint32_t box[2] = {0, 0};
};

struct GemmArgs {
    int M, N, K;                      // output rows, output columns (of each projection), contraction
    int kb;                           // stages along K
    int tiles_n, tiles;
    int act;
    int stages;
    int split;                        // 2: two CTAs of a cluster share a tile's K; 1: none do
    int a_bytes;                      // of A in a stage: of all its 128 rows, or of those that exist
    uint32_t warp_bytes;              // boxes of one epilogue warp
    uint32_t in_bytes;                // that arrive by TMA for one chunk
    int twice;                        // outputs have two boxes each, for even and odd chunks
    const float* bias;
    Side side[SIDES];
    int* status;
    uint64_t wait_ns;
};
struct Maps { CUtensorMap a, b[2], side[SIDES]; };

// ---- activations ------------------------------------------------------------------------------
// Value and derivative of two numbers in fp32, from the fast exponential and reciprocal.  The error function is formula
// 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical Functions (1964): with t = 1 / (1 + 0.3275911 x), x >= 0,
//   1 - erf(x) = (a1 t + a2 t^2 + ... + a5 t^5) exp(-x^2), off by less than 1.5e-7,
// whose exponential is the one that the derivative needs too.  (With CUDA's erff, a branch for each group of eight and the
// bias loaded number by number, 32768 x 768 -> 2048 took 208 us; 109 so.)
template <int ACT> struct Act {};
__device__ __forceinline__ F2 logistic(F2 z) {
    const F2 e = exp2_fast(mul2(z, both(-1.44269504f)));
    return rcp_fast(add2(e, both(1.f)));
}
// the normal distribution's tail beyond |z|, and exp(-z^2 / 2)
__device__ __forceinline__ F2 tail_of(F2 z, F2& e) {
    e = exp2_fast(mul2(mul2(z, z), both(-0.72134752f)));
    const F2 t = rcp_fast(F2{fmaf(fabsf(z.x), 0.23164189f, 1.f), fmaf(fabsf(z.y), 0.23164189f, 1.f)});
    F2 q = fma2(t, both(0.5307027145f), both(-0.7265760135f));       // half of 7.1.26's coefficients
    q = fma2(q, t, both(0.7107068705f));
    q = fma2(q, t, both(-0.142248368f));
    q = fma2(q, t, both(0.127414796f));
    return mul2(mul2(q, t), e);
}
// Of an infinity the limits: factors that meet one that is 0 there are kept finite, by a bound beyond which value and slope
// are z or 0 and 1 or 0 to the last bit.  A NaN stays one.
__device__ __forceinline__ float no_less(float z, float low) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(z), "f"(low));
    return r;
}
__device__ __forceinline__ float no_more(float z, float high) {
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(z), "f"(high));
    return r;
}
__device__ __forceinline__ F2 no_less(F2 z, float low) { return F2{no_less(z.x, low), no_less(z.y, low)}; }
__device__ __forceinline__ F2 no_more(F2 z, float high) { return F2{no_more(z.x, high), no_more(z.y, high)}; }
constexpr float kFar = 200.f;
__device__ __forceinline__ float relu(float z) { return z < 0.f ? 0.f : z; }                 // a NaN stays one
// (1 + tanh(v)) / 2 is the logistic function of 2 v, v = sqrt(2 / pi) (z + 0.044715 z^3)
constexpr float kTanhSlope = 1.5957691216f;
__device__ __forceinline__ F2 tanh_gate(F2 z) {
    return logistic(mul2(z, fma2(mul2(z, z), both(kTanhSlope * 0.044715f), both(kTanhSlope))));
}

__device__ __forceinline__ F2 value(Act<ADLOCO_ACT_NONE>, F2 z) { return z; }
__device__ __forceinline__ F2 value(Act<ADLOCO_ACT_RELU>, F2 z) { return F2{relu(z.x), relu(z.y)}; }
__device__ __forceinline__ F2 value(Act<ADLOCO_ACT_GELU>, F2 z) {
    F2 e;
    const F2 q = tail_of(z, e);
    // z where the tail is below all numbers; an infinity times its 0 would be none
    return F2{fmaf(-fminf(fabsf(z.x), 1e30f), q.x, fmaxf(z.x, 0.f)), fmaf(-fminf(fabsf(z.y), 1e30f), q.y, fmaxf(z.y, 0.f))};
}
__device__ __forceinline__ F2 value(Act<ADLOCO_ACT_GELU_TANH>, F2 z) { return mul2(no_less(z, -kFar), tanh_gate(z)); }
__device__ __forceinline__ F2 value(Act<ADLOCO_ACT_SILU>, F2 z) { return mul2(no_less(z, -kFar), logistic(z)); }

__device__ __forceinline__ F2 slope(Act<ADLOCO_ACT_NONE>, F2 z, F2& a) { a = z; return both(1.f); }
__device__ __forceinline__ F2 slope(Act<ADLOCO_ACT_RELU>, F2 z, F2& a) {
    a = F2{relu(z.x), relu(z.y)};
    return F2{z.x > 0.f ? 1.f : a.x, z.y > 0.f ? 1.f : a.y};                                // 0, or the NaN
}
__device__ __forceinline__ F2 slope(Act<ADLOCO_ACT_GELU>, F2 z, F2& a) {
    F2 e;
    const F2 q = tail_of(z, e), low = no_less(z, -kFar);
    const F2 h = {z.x < 0.f ? q.x : 1.f - q.x, z.y < 0.f ? q.y : 1.f - q.y};
    a = mul2(low, h);
    return fma2(mul2(no_more(low, kFar), e), both(0.39894228f), h);
}
__device__ __forceinline__ F2 slope(Act<ADLOCO_ACT_GELU_TANH>, F2 z, F2& a) {
    const F2 low = no_less(z, -kFar), near = no_more(low, kFar), h = tanh_gate(near);
    a = mul2(low, h);
    return fma2(mul2(mul2(near, h), fma2(h, both(-1.f), both(1.f))), fma2(mul2(near, near), both(kTanhSlope * 0.134145f), both(kTanhSlope)), h);
}
__device__ __forceinline__ F2 slope(Act<ADLOCO_ACT_SILU>, F2 z, F2& a) {
    const F2 h = logistic(z);
    a = mul2(no_less(z, -kFar), h);
    return fma2(no_more(a, kFar), fma2(h, both(-1.f), both(1.f)), h);
}
// f with the activation as a type: one branch for all that it does
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
    switch (act) {
        case ADLOCO_ACT_RELU: f(Act<ADLOCO_ACT_RELU>{}); break;
        case ADLOCO_ACT_GELU: f(Act<ADLOCO_ACT_GELU>{}); break;
        case ADLOCO_ACT_GELU_TANH: f(Act<ADLOCO_ACT_GELU_TANH>{}); break;
        case ADLOCO_ACT_SILU: f(Act<ADLOCO_ACT_SILU>{}); break;
        default: f(Act<ADLOCO_ACT_NONE>{});
    }
}

// ---- boxes --------------------------------------------------------------------------------------
// A row of a box is P pieces of 16 bytes (2 of bytes, 4 of bf16, 8 of fp32), swizzled as the tensor map of that width does
// it, so that neighbouring rows' equal pieces fall on different banks.
__device__ __forceinline__ int pieces_of(int form) { return form == kF32 ? 8 : form == kBf16 ? 4 : 2; }
template <int P>
__device__ __forceinline__ uint32_t piece_at(uint32_t box, int row, int piece) {
    return box + (uint32_t)row * (16u * P) + ((uint32_t)(piece ^ ((row * P >> 3) & (P - 1))) << 4);
}
__device__ __forceinline__ uint32_t piece_at(int form, uint32_t box, int row, int piece) {
    return form == kF32 ? piece_at<8>(box, row, piece) : form == kBf16 ? piece_at<4>(box, row, piece) : piece_at<2>(box, row, piece);
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ F2 pair_of(uint32_t w) { return F2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)}; }
__device__ __forceinline__ void bytes_to_pairs(uint32_t w, float s, F2* v) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * h)), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r));
        v[h] = mul2(F2{f.x, f.y}, both(s));
    }
}
// A chunk's operand of this lane's row as it lies in its box: read in one go, ahead of all that is computed from it (reads
// and writes of shared memory keep their order, so that reads between writes would each wait for what is computed before).
template <int FORM> struct Raw32 { uint4 w[FORM == kF32 ? 8 : FORM == kBf16 ? 4 : 2]; };
template <int FORM>
__device__ __forceinline__ void read32(uint32_t box, int row, Raw32<FORM>& r) {
    constexpr int P = FORM == kF32 ? 8 : FORM == kBf16 ? 4 : 2;
#pragma unroll
    for (int i = 0; i < P; ++i) r.w[i] = lds16(piece_at<P>(box, row, i));
}
// its columns 8 g .. 8 g + 7; s: the scale of bytes
template <int FORM>
__device__ __forceinline__ void numbers8(const Raw32<FORM>& r, int g, float s, F2 (&v)[4]) {
    if constexpr (FORM == kF32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 w = r.w[2 * g + h];
            v[2 * h] = F2{__uint_as_float(w.x), __uint_as_float(w.y)};
            v[2 * h + 1] = F2{__uint_as_float(w.z), __uint_as_float(w.w)};
        }
    } else if constexpr (FORM == kBf16) {
        const uint4 w = r.w[g];
        v[0] = pair_of(w.x); v[1] = pair_of(w.y); v[2] = pair_of(w.z); v[3] = pair_of(w.w);
    } else {
        const uint4 w = r.w[g >> 1];
        bytes_to_pairs((g & 1) ? w.z : w.x, s, v);
        bytes_to_pairs((g & 1) ? w.w : w.y, s, v + 2);
    }
}
__device__ __forceinline__ uint32_t pack(F2 v) { return pack_bf16(__float_as_uint(v.x), __float_as_uint(v.y)); }
__device__ __forceinline__ void write8(int form, uint32_t box, int row, int g, float inv, const F2 (&v)[4]) {
    if (form == kBf16) {
        st_shared_v4(piece_at<4>(box, row, g), pack(v[0]), pack(v[1]), pack(v[2]), pack(v[3]));
    } else if (form == kF32) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            st_shared_v4(piece_at<8>(box, row, 2 * g + h), __float_as_uint(v[2 * h].x), __float_as_uint(v[2 * h].y),
                         __float_as_uint(v[2 * h + 1].x), __float_as_uint(v[2 * h + 1].y));
    } else {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const F2 u = mul2(v[i], both(inv));
            h[i] = __nv_cvt_float2_to_fp8x2(make_float2(u.x, u.y), __NV_SATFINITE, __NV_E4M3);
        }
        asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(piece_at<2>(box, row, g >> 1) + 8u * (g & 1)), "r"(h[0] | (h[1] << 16)),
                     "r"(h[2] | (h[3] << 16)) : "memory");
    }
}
// all 32 columns of a chunk, the branch on the form taken once
__device__ __forceinline__ void write32(int form, uint32_t box, int row, float inv, const F2 (&v)[4][4]) {
    if (form == kBf16) {
#pragma unroll
        for (int g = 0; g < 4; ++g) write8(kBf16, box, row, g, inv, v[g]);
    } else if (form == kBytes) {
#pragma unroll
        for (int g = 0; g < 4; ++g) write8(kBytes, box, row, g, inv, v[g]);
    }
}
// A box by the warp's own accesses: where rows do not start on 16-byte boundaries (element by element along rows), or
// where a row's last 16-byte piece is not whole, which a TMA store would write in full.
template <typename W>
__device__ __forceinline__ void box_in_of(const Side& s, uint32_t box, int lane, int row0, int col, int M, int N) {
    constexpr int P = sizeof(W) == 4 ? 8 : 4, EACH = 16 / sizeof(W);
    const W* from = static_cast<const W*>(s.p) + (int64_t)row0 * s.pitch + col + lane;
    const int rows = col + lane < N ? M - row0 : 0;
    W v[32];                                           // all rows' loads in flight
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = i < rows ? from[i * s.pitch] : W(0);
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        const uint32_t to = piece_at<P>(box, i, lane / EACH) + (uint32_t)(lane % EACH * sizeof(W));
        if (sizeof(W) == 4) asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"((uint32_t)v[i]) : "memory");
        else asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"((unsigned short)v[i]) : "memory");
    }
}
__device__ __noinline__ void box_in(const Side& s, uint32_t box, int lane, int row0, int col, int M, int N) {
    if (s.form == kF32) box_in_of<uint32_t>(s, box, lane, row0, col, M, N);
    else box_in_of<unsigned short>(s, box, lane, row0, col, M, N);
    __syncwarp();
}
__device__ __noinline__ void box_out(const Side& s, uint32_t box, int lane, int row0, int col, int M, int N) {
    __syncwarp();
    const int es = s.form == kF32 ? 4 : s.form == kBf16 ? 2 : 1, P = pieces_of(s.form), each = 16 / es;
    char* out = static_cast<char*>(s.p) + ((int64_t)row0 * s.pitch + col) * es;
    const int64_t pitch = s.pitch * es;
    if (s.pieces) {
        const int piece = lane & (P - 1), c = piece * each;
        for (int row = lane / P; row < 32; row += 32 / P) {
            if (row0 + row >= M || col + c >= N) continue;
            const uint4 v = lds16(piece_at(s.form, box, row, piece));
            char* to = out + row * pitch + piece * 16;
            if (col + c + each <= N) {
                *reinterpret_cast<uint4*>(to) = v;
            } else {
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                for (int b = 0; b < (N - col - c) * es; ++b) to[b] = (char)(w[b >> 2] >> (8 * (b & 3)));
            }
        }
    } else {
        const int rows = min(32, M - row0);
        for (int row = 0; row < rows && col + lane < N; ++row) {
            const uint32_t from = piece_at(s.form, box, row, lane / each) + (uint32_t)((lane & (each - 1)) * es);
            if (es == 4) {
                uint32_t v;
                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(from) : "memory");
                reinterpret_cast<uint32_t*>(out + row * pitch)[lane] = v;
            } else {
                unsigned short v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(from) : "memory");
                reinterpret_cast<unsigned short*>(out + row * pitch)[lane] = v;
            }
        }
    }
    fence_proxy_async_smem();                          // a fetch may write the box next
    __syncwarp();
}

// the largest magnitude, a NaN included
__device__ __forceinline__ float larger(float m, float v) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(m), "f"(fabsf(v)));
    return r;
}

// ---- the tile kernel ------------------------------------------------------------------------------
// Persistent, 320 threads: warp 0 brings tiles by TMA, warp 1 issues the MMAs, warps 2-9 are the epilogue.  PAIR: 256 x BN
// tiles shared by the two CTAs of a cluster (cta_group::2): CTA r holds rows 128 r .. + 127 of the tile in its tensor memory
// and loads those rows of A and half of B's; otherwise 128 x BN tiles of one CTA.  A stage is 64 of K, 128 in small tiles.  Two accumulators
// take turns, so that a tile's epilogue runs beside the next tile's MMAs.  B is a weight [N, K] forward, its rows along the
// tensor cores' K; backward the same weight is read as it lies, its rows along the contraction (MN-major).
// GATED: the tile's columns are BN / 2 of each projection (in a pair, CTA r brings projection r), so a thread of the epilogue
// has both numbers of an output.
// SUMMED: the tensor cores cut off each sum's low bits (relative error 1e-6 after 1000 terms, growing with their number); the
// sum of every 512 of K is added up in registers instead, rounded to nearest: for fp32 outputs (F32), and where sums go to 8 bits,
// whose steps are so wide (2^-4) that each number on the other side of a border shows (4096 x 2048 -> 2 x 5632, both kept, and the way
// back: 7.0e-4 of the norm away from the fp32 form with the accumulator as it is, 3.4e-4 so, 2.4e-4 with a sum of every 256; 131, 132
// and 139 us forward).
// SPLIT K: where few tiles of 64 columns leave most SMs idle, two CTAs of a cluster take half of K each.  The second one writes its
// sums into the first one's shared memory, which adds them to its own and goes on alone.
// The epilogue's eight warps each own 32 rows and half the columns, in chunks of 32: the operands of the next chunk arrive by
// TMA while this one is computed, the results leave by TMA.  IN8: what the forward pass kept is in 8 bits.
// What bounds it: at long K the tensor pipe and the power cap (8192 x 4096 -> 4096: 176 us, 1.56 PFLOP/s); at K = 768 a tile's MMAs take
// 6.1 thousand clocks and its operands as many of L2's, and the epilogue's matrices go through the same L2 and copy engine
// beside them: 32768 x 768 -> 2048 takes 75 us with one bf16 output, 105 with gelu and z kept, 151 on the way back through the gate with
// five matrices (4.8 TB/s), as graph replays of some ms; in a long row of calls, at the power cap, 120 with gelu and z and 172 back through the gate.  Sixteen epilogue warps, operands and results without TMA, and prefetches into L2 gained nothing or lost.
constexpr int DG_THREADS = 320, DG_EPI = 8;
constexpr int DG_A_BYTES = 128 * 128;
constexpr int DG_MAX_STAGES = 8;
constexpr int DG_SEGMENT = 8;                              // blocks of K in one sum of a SUMMED tile
constexpr int DG_BAR_BYTES = 512 + DG_EPI * 512;            // and 128 columns of the bias for each warp of the epilogue
constexpr int DG_SMEM = 232448 - 256;                      // what a block can have, less the kernel's own few words
template <bool PAIR, int BN>
__host__ __device__ constexpr int dg_block_bytes() { return DG_A_BYTES + (PAIR ? BN / 2 : BN) * 128; }      // of 64 of K
// Blocks of K in a stage: waits, signals and issue take a thread about 370 clocks a stage, more than a small tile's operands and
// MMAs (256 x 4096 x 4096, operands in L2: 16.7 us with one block a stage, 12.9 with two).
template <bool PAIR, int BN>
__host__ __device__ constexpr int dg_stage_blocks() { return BN == 64 || (PAIR && BN == 128) ? 2 : 1; }
template <bool PAIR, int BN>
__host__ __device__ constexpr int dg_stage_bytes() { return dg_block_bytes<PAIR, BN>() * dg_stage_blocks<PAIR, BN>(); }

// The tiles of one worker: dealt round, the tiles along N fastest, so that all workers sit on the same rows of A at a time.
struct Walk {
    int left, m, n, step_m, step_n, line;
    __device__ __forceinline__ Walk(const GemmArgs& a, int worker, int workers) : line(a.tiles_n) {
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

template <int KIND, bool PAIR, int BN>
__host__ __device__ constexpr bool dg_can_split() { return !PAIR && KIND != GATED && BN == 64; }

template <int KIND, bool PAIR, int BN, int SUM, bool IN8>
__global__ void __launch_bounds__(DG_THREADS, 1) dense_tile_kernel(const __grid_constant__ Maps maps, const __grid_constant__ GemmArgs a) {
    constexpr bool TWO = KIND == GATED, BACK = KIND == LINEAR_BACK || KIND == GATED_BACK, FORWARD = !BACK;
    constexpr bool SUMMED = SUM != kPlain, F32 = SUM == kSummedF32, SPLIT = dg_can_split<KIND, PAIR, BN>();
    constexpr int COLS = TWO ? BN / 2 : BN;                // output columns of a tile
    constexpr int TM = PAIR ? 256 : 128;
    constexpr int CHUNKS = COLS / 64;                      // of an epilogue warp
    constexpr int STAGE = dg_stage_bytes<PAIR, BN>(), BLOCK = dg_block_bytes<PAIR, BN>(), BLOCKS = dg_stage_blocks<PAIR, BN>();
    constexpr int SEGMENT = DG_SEGMENT / BLOCKS;           // stages in one sum of a SUMMED tile
    constexpr int B_ROWS = PAIR ? BN / 2 : BN;             // of the weight (or of its columns, backward) in a CTA's stage
    static_assert(CHUNKS >= 1 && (!BACK || B_ROWS % 64 == 0), "a chunk is 32 columns, a box of the weight's columns 64");

    extern __shared__ uint8_t smem_raw[];
    const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t boxes = smem_base + (uint32_t)a.stages * STAGE;
    const uint32_t bars = boxes + DG_EPI * a.warp_bytes;
    auto full_bar = [&](uint32_t s) { return bars + 8u * s; };
    auto empty_bar = [&](uint32_t s) { return bars + 8u * (DG_MAX_STAGES + s); };
    auto acc_full = [&](uint32_t s) { return bars + 8u * (2 * DG_MAX_STAGES + s); };
    auto acc_empty = [&](uint32_t s) { return bars + 8u * (2 * DG_MAX_STAGES + 2 + s); };
    auto in_bar = [&](uint32_t w, uint32_t s) { return bars + 8u * (2 * DG_MAX_STAGES + 4 + 2 * w + s); };
    const uint32_t drain_bar = bars + 8u * (2 * DG_MAX_STAGES + 4 + 2 * DG_EPI), join_bar = drain_bar + 8u;
    auto swap_bar = [&](uint32_t w, uint32_t s) { return bars + 8u * (2 * DG_MAX_STAGES + 6 + 2 * DG_EPI + 2 * w + s); };
    const uint32_t join = bars + DG_BAR_BYTES;                 // the other half's sums, or the maxima that warps tell one another
    static_assert(8 * (2 * DG_MAX_STAGES + 6 + 4 * DG_EPI) <= 512, "barriers");
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;      // warp: known to be uniform
    const uint32_t rank = PAIR ? cluster_cta_rank() : 0;       // 0: the CTA that issues the MMAs
    const uint32_t split = SPLIT ? (uint32_t)a.split : 1u, part = split == 1 ? 0u : cluster_cta_rank();
    Walk walk(a, PAIR ? (int)(blockIdx.x >> 1) : (int)(blockIdx.x / split), PAIR ? (int)(gridDim.x >> 1) : (int)(gridDim.x / split));
    const int k_first = (int)(a.kb * part / split), k_end = (int)(a.kb * (part + 1) / split);      // this CTA's blocks of K
    const uint32_t stages = (uint32_t)a.stages;
    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (uint32_t s = 0; s < stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (uint32_t s = 0; s < 2; ++s) { mbar_init(acc_full(s), 1); mbar_init(acc_empty(s), (PAIR ? 2 : 1) * DG_EPI); }
        for (uint32_t w = 0; w < DG_EPI; ++w) {
            for (uint32_t s = 0; s < 2; ++s) { mbar_init(in_bar(w, s), 1); mbar_init(swap_bar(w, s), 1); }
        }
        mbar_init(drain_bar, 1);
        if (SPLIT) mbar_init(join_bar, DG_EPI + 1);
        fence_barrier_init();
        prefetch_tmap(&maps.a);
        prefetch_tmap(&maps.b[0]);
        if (TWO) prefetch_tmap(&maps.b[1]);
        for (int i = 0; i < SIDES; ++i)
            if (a.side[i].tma) prefetch_tmap(&maps.side[i]);
    }
    if (warp == 1) {
        if (PAIR) { tmem_alloc_pair(smem_u32(&tmem_slot), 512); tmem_relinquish_pair(); }
        else { tmem_alloc(smem_u32(&tmem_slot), 512); tmem_relinquish(); }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR || split > 1) cluster_sync_all();                 // the peers' barriers exist before anything is signalled on them
    tc_fence_after();
    after_predecessor();
    const uint32_t tmem = tmem_slot;
    volatile int* abortp = &abort_flag;
    const int segments = SUMMED ? (k_end - k_first + SEGMENT - 1) / SEGMENT : 1;

    if (warp == 0) {
        // ---------------- TMA producer, one per CTA ----------------
        {
            const bool leader = elect_one();
            Ring ps;
            uint32_t issued = 0;
            bool ok = true;
            for (; ok && walk.more(); walk.next()) {
                const int m0 = walk.m * TM + (int)rank * 128, n0 = walk.n * COLS;
                for (int k = k_first; k < k_end; ++k) {
                    if (!wait_warp<false>(empty_bar(ps.stage), ps.phase ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
                    if (leader) {
                        const uint32_t bar = PAIR ? map_to_cta(full_bar(ps.stage), 0) : full_bar(ps.stage);
                        if (rank == 0) mbar_arrive_expect_tx(full_bar(ps.stage), (PAIR ? 2 : 1) * BLOCKS * (BLOCK - DG_A_BYTES + a.a_bytes));
                        auto load = [&](uint32_t dst, const CUtensorMap* m, int c0, int c1) {
                            if (PAIR) tma_load_2d_pair(dst, m, bar, c0, c1);
                            else tma_load_2d(dst, m, bar, c0, c1);
                        };
#pragma unroll
                        for (int s = 0; s < BLOCKS; ++s) {
                            const uint32_t sA = smem_base + ps.stage * STAGE + s * BLOCK, sB = sA + DG_A_BYTES;
                            const int at = (k * BLOCKS + s) * 64;      // beyond K: zeros
                            load(sA, &maps.a, at, m0);
                            if (TWO) {
                                if (PAIR) {
                                    load(sB, &maps.b[rank], at, n0);
                                } else {
                                    load(sB, &maps.b[0], at, n0);
                                    load(sB + COLS * 128, &maps.b[1], at, n0);
                                }
                            } else if (!BACK) {
                                load(sB, &maps.b[0], at, n0 + (int)rank * B_ROWS);
                            } else {
#pragma unroll
                                for (int c = 0; c < B_ROWS; c += 64) load(sB + c * 128, &maps.b[0], n0 + (int)rank * B_ROWS + c, at);
                            }
                        }
                    }
                    __syncwarp();
                    ++issued;
                    ps.advance(stages);
                }
            }
            if (!ok && leader) {
                if (PAIR) {
                    // leaving after a time-out: the byte counts of copies in flight complete on the even CTA's barriers, which
                    // the odd CTA cannot wait on: both sit out a grace period far beyond the flight time of a copy
                    st_cluster_u32(map_to_cta(smem_u32(&abort_flag), rank ^ 1u), 1u);
                    const uint64_t t0 = globaltimer_ns();
                    while (globaltimer_ns() - t0 < kPairLeaveNs) { }
                } else {
                    Ring q = ps;                               // the copies still in flight land first
                    const uint32_t back = issued < stages ? issued : stages;
                    for (uint32_t r = 0; r < back; ++r) {
                        if (q.stage == 0) { q.stage = stages - 1; q.phase ^= 1u; } else { --q.stage; }
                        int never = 0;
                        mbar_wait(full_bar(q.stage), q.phase, &never, kLeaveLimitNs);
                    }
                }
            }
            __syncwarp();
        }
    } else if (warp == 1) {
        // ---------------- MMA issuer (of a pair the even CTA's; the whole warp keeps step, one lane issues) ----------------
        if (rank == 0) {
            const bool leader = elect_one();
            constexpr uint32_t idesc = idesc_bf16_f32(TM, BN, 0, BACK ? 1 : 0);
            const uint64_t descA = smem_desc_sw128(0, 16, 1024);
            const uint64_t descB = BACK ? smem_desc_sw128(0, 64 * 128, 1024) : descA;
            Ring ps;
            uint32_t n = 0;
            bool ok = true;
            for (; ok && walk.more(); walk.next()) {
                for (int k0 = k_first; ok && k0 < k_end; ++n) {
                    const uint32_t buf = n & 1u;
                    const int k1 = SUMMED ? min(k_end, k0 + SEGMENT) : k_end;
                    if (!wait_warp<PAIR>(acc_empty(buf), ((n >> 1) & 1u) ^ 1u, abortp, a.wait_ns)) { ok = false; break; }
                    for (int k = k0; k < k1; ++k) {
                        if (!wait_warp<false>(full_bar(ps.stage), ps.phase, abortp, a.wait_ns)) { ok = false; break; }
                        tc_fence_after();
                        if (leader) {
                            const uint32_t at = smem_base + ps.stage * STAGE;
                            const uint64_t dA = descA + (at >> 4), dB = descB + ((at + DG_A_BYTES) >> 4);
#pragma unroll
                            for (int kk = 0; kk < 4 * BLOCKS; ++kk) {
                                // 16 of K further: 32 bytes along a row, or 16 rows of 128 bytes
                                const uint64_t da = dA + (BLOCK >> 4) * (kk / 4) + 2 * (kk % 4), db = dB + (BLOCK >> 4) * (kk / 4) + (BACK ? 128 : 2) * (kk % 4);
                                if (PAIR) mma_bf16_pair(tmem + buf * BN, da, db, idesc, (k == k0 && kk == 0) ? 0u : 1u);
                                else mma_bf16(tmem + buf * BN, da, db, idesc, (k == k0 && kk == 0) ? 0u : 1u);
                            }
                            if (PAIR) mma_commit_pair(empty_bar(ps.stage), 3);
                            else mma_commit(empty_bar(ps.stage));
                        }
                        __syncwarp();
                        ps.advance(stages);
                    }
                    if (ok && leader) {
                        if (PAIR) mma_commit_pair(acc_full(buf), 3);
                        else mma_commit(acc_full(buf));
                    }
                    __syncwarp();
                    k0 = k1;
                }
            }
            if (!ok && leader) {
                if (PAIR) {
                    st_cluster_u32(map_to_cta(smem_u32(&abort_flag), 1u), 1u);
                    mma_commit_pair(drain_bar, 1);
                } else {
                    mma_commit(drain_bar);
                }
                int never = 0;
                mbar_wait(drain_bar, 0, &never, kLeaveLimitNs);
            }
            __syncwarp();
        }
    } else {
        // ---------------- epilogue ----------------
        const uint32_t q = warp & 3, half = (uint32_t)(warp - 2) >> 2, w = (uint32_t)(warp - 2);
        const uint32_t acc_empty_0 = PAIR ? map_to_cta(acc_empty(0), 0) : acc_empty(0);
        const uint32_t mine = boxes + w * a.warp_bytes;
        const uint32_t lane_tmem = tmem + ((q * 32u) << 16);
        const int first = (int)half * (COLS / 2);              // of the tile's columns
        const bool fetches = a.in_bytes != 0 && part == 0;
        uint32_t n = 0, chunk = 0;                             // accumulators and chunks so far
        uint32_t fetched = 0;                                  // chunks whose operands have been asked for
        uint32_t swaps = 0;                                    // maxima told to the other warp of these rows
        auto row_of = [&](const Walk& t) { return t.m * TM + (int)rank * 128 + (int)q * 32; };
        auto col_of = [&](const Walk& t, int i) { return t.n * COLS + first + 32 * i; };
        auto stored = [&]() {                                  // this warp's stores so far have read their boxes
            if (lane == 0) bulk_wait_read_all();
            __syncwarp();
        };
        auto fetch = [&](uint32_t c, int row, int col) {       // chunk c's operands; all lanes, boxes free
            if (lane == 0) {
                mbar_arrive_expect_tx(in_bar(w, c & 1u), a.in_bytes);
                for (int i = IN0; i <= IN1; ++i)
                    if (a.side[i].tma) tma_load_2d(mine + a.side[i].box[c & 1u], &maps.side[i], in_bar(w, c & 1u), col, row);
            }
            fetched = c + 1;
        };
        auto release = [&](uint32_t buf) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR) mbar_arrive_cluster_relaxed(acc_empty_0 + 8u * buf);
                else mbar_arrive(acc_empty_0 + 8u * buf);
            }
        };
        const uint32_t bias_at = bars + 512 + w * 512;
        const bool twice = a.twice != 0;
        const bool by_hand = KIND != GATED && KIND != GATED_BACK && a.side[IN0].form != kNone && !a.side[IN0].tma && part == 0;
        constexpr int OUT = F32 ? kF32 : kBf16, KEPT = IN8 ? kBytes : kBf16, FORM0 = KIND == GATED_BACK ? KEPT : OUT;
        const int form0 = a.side[OUT0].form, form1 = a.side[OUT1].form;
        const int in0 = a.side[IN0].form, in1 = a.side[IN1].form;
        constexpr int AROUND = COLS < 128 ? COLS : 128;
        float bias_next[AROUND / 32];
        auto load_bias = [&](const Walk& t) {
#pragma unroll
            for (int c = 0; c < AROUND / 32; ++c) {
                const int at = t.n * COLS + (first & ~127) + 32 * c + lane;
                bias_next[c] = at < a.N ? a.bias[at] : 0.f;
            }
        };
        if (KIND == LINEAR && a.bias && walk.more()) load_bias(walk);
        bool ok = true;
        for (; ok && walk.more(); walk.next()) {
            const int row0 = row_of(walk), row = row0 + lane;
            const int valid = row0 < a.M ? min(CHUNKS, max(0, (a.N - col_of(walk, 0) + 31) / 32)) : 0;
            if (fetches && fetched == chunk && valid > 0) {
                stored();
                fetch(chunk, row0, col_of(walk, 0));
            }
            if (by_hand && valid > 0) {                        // a residual whose rows lie anywhere: two chunks before the accumulator
                stored();
                for (int i = 0; i < min(2, valid); ++i)
                    box_in(a.side[IN0], mine + a.side[IN0].box[(chunk + i) & 1u], lane, row0, col_of(walk, i), a.M, a.N);
            }
            // the bias of the tile's 128 columns around this warp's, one copy a warp; the next tile's is on its way meanwhile
            const int block = first & ~127, col0 = walk.n * COLS + block;
            if (KIND == LINEAR && a.bias) {
                __syncwarp();
#pragma unroll
                for (int c = 0; c < AROUND / 32; ++c)
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(bias_at + 4u * (32 * c + lane)), "f"(bias_next[c]) : "memory");
                __syncwarp();
                if (walk.left > 1) {
                    Walk t = walk;
                    t.next();
                    load_bias(t);
                }
            }
            auto add_bias = [&](int c, F2 (&v)[4]) {           // to the eight columns from c of that block on
                if (KIND != LINEAR || !a.bias) return;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 w = lds16(bias_at + 4u * c + 16u * h);
                    v[2 * h] = add2(v[2 * h], F2{__uint_as_float(w.x), __uint_as_float(w.y)});
                    v[2 * h + 1] = add2(v[2 * h + 1], F2{__uint_as_float(w.z), __uint_as_float(w.w)});
                }
            };
            F2 sum[SUMMED ? CHUNKS : 1][4][4], sum2[SUMMED ? CHUNKS : 1][TWO ? 4 : 1][4];      // TWO: sum2 of the other projection
            uint32_t buf = n & 1u;
            if constexpr (SUMMED) {
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        sum[i][e >> 2][e & 3] = both(0.f);
                        if constexpr (TWO) sum2[i][e >> 2][e & 3] = both(0.f);
                    }
                for (int s = 0; s < segments; ++s, ++n) {
                    buf = n & 1u;
                    if (!wait_warp<false>(acc_full(buf), (n >> 1) & 1u, abortp, a.wait_ns)) { ok = false; break; }
                    tc_fence_after();
#pragma unroll
                    for (int i = 0; i < CHUNKS; ++i) {
                        uint32_t r[32];
                        tmem_ld32(lane_tmem + buf * BN + first + 32 * i, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            sum[i][e >> 2][e & 3] = add2(sum[i][e >> 2][e & 3], F2{__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])});
                        if constexpr (TWO) {
                            tmem_ld32(lane_tmem + buf * BN + COLS + first + 32 * i, r);
                            tmem_ld_wait();
#pragma unroll
                            for (int e = 0; e < 16; ++e)
                                sum2[i][e >> 2][e & 3] = add2(sum2[i][e >> 2][e & 3], F2{__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])});
                        }
                    }
                    release(buf);
                }
                if (!ok) break;
            } else {
                if (!wait_warp<false>(acc_full(buf), (n >> 1) & 1u, abortp, a.wait_ns)) { ok = false; break; }
                tc_fence_after();
                ++n;
            }
            const uint32_t acc = lane_tmem + buf * BN;
            // the second half's number of this lane's row: 16-byte pieces of a row swapped so that neighbouring rows fall on all banks
            auto joint = [&](uint32_t base, int c) { return base + (q * 32 + lane) * (BN * 4u) + (uint32_t)(((c >> 2) ^ (lane & 7)) << 4); };
            if (SPLIT && part > 0) {                           // the launch has one tile a cluster: this is all that it does
                const uint32_t there = map_to_cta(join, 0);
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) {
                    const int c = first + 32 * i;
                    uint32_t r[32];
                    if constexpr (SUMMED) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            r[2 * e] = __float_as_uint(sum[i][e >> 2][e & 3].x);
                            r[2 * e + 1] = __float_as_uint(sum[i][e >> 2][e & 3].y);
                        }
                    } else {
                        tmem_ld32(acc + c, r);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 4) st_cluster_v4(joint(there, c + e), r[e], r[e + 1], r[e + 2], r[e + 3]);
                }
                if (!SUMMED) release(buf);
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_cta(join_bar, 0));
                continue;
            }
            if (SPLIT && split > 1) {
                if (w == 0 && lane == 0) mbar_arrive(join_bar);
                if (!wait_warp<true>(join_bar, 0, abortp, a.wait_ns)) { ok = false; break; }
            }
            auto add_half = [&](int c, F2 (&v)[4]) {           // to the eight columns from c on of the accumulator
                if (!SPLIT || split == 1) return;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint4 o = lds16(joint(join, c + 4 * h));
                    v[2 * h] = add2(v[2 * h], F2{__uint_as_float(o.x), __uint_as_float(o.y)});
                    v[2 * h + 1] = add2(v[2 * h + 1], F2{__uint_as_float(o.z), __uint_as_float(o.w)});
                }
            };
            if constexpr (SUMMED) {
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        add_half(first + 32 * i + 8 * g, sum[i][g]);
                        add_bias(first - block + 32 * i + 8 * g, sum[i][g]);
                    }
            }
            // the scales of what is kept in 8 bits.  A warp whose sums are half of the block's 128 columns tells the other warp of
            // these rows their maxima: through one of two places and barriers in turn, since a warp may be a tile ahead, but is not
            // two before the other has been told of this one and has read it.
            float inv1 = 0.f, inv2 = 0.f;
            if (FORWARD && form1 == kBytes && row0 < a.M) {
                float m1 = 0.f, m2 = 0.f;
                if constexpr (SUMMED) {
#pragma unroll
                    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            m1 = larger(larger(m1, sum[i][e >> 2][e & 3].x), sum[i][e >> 2][e & 3].y);
                            if constexpr (TWO) m2 = larger(larger(m2, sum2[i][e >> 2][e & 3].x), sum2[i][e >> 2][e & 3].y);
                        }
                    if constexpr (CHUNKS < 4) {
                        const uint32_t turn = swaps & 1u, place = turn * 256u + (uint32_t)lane * 8u;
                        asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(join + w * 512u + place), "f"(m1), "f"(m2) : "memory");
                        __syncwarp();
                        if (lane == 0) mbar_arrive(swap_bar(w ^ 4u, turn));
                        if (!wait_warp<false>(swap_bar(w, turn), (swaps >> 1) & 1u, abortp, a.wait_ns)) { ok = false; break; }
                        ++swaps;
                        float o1, o2;
                        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(o1), "=f"(o2) : "r"(join + (w ^ 4u) * 512u + place) : "memory");
                        m1 = larger(m1, o1);
                        m2 = larger(m2, o2);
                    }
                }
                const uint32_t s1 = scale_byte(__float_as_uint(m1)), s2 = scale_byte(__float_as_uint(m2));
                inv1 = inv_scale(s1);
                inv2 = inv_scale(s2);
                if (first == block && row < a.M && valid > 0) {        // (a tile's second block may lie beyond the matrix)
                    a.side[OUT1].scale[(int64_t)row * a.side[OUT1].scale_pitch + (col0 >> 7)] = (uint8_t)s1;
                    if (TWO) a.side[OUT2].scale[(int64_t)row * a.side[OUT2].scale_pitch + (col0 >> 7)] = (uint8_t)s2;
                }
            }
            // the scales of what was kept
            float scale0 = 1.f, scale1 = 1.f;
            if (IN8 && valid > 0 && row < a.M) {
                const int at = col_of(walk, 0) >> 7;
                if (KIND == GATED_BACK) scale0 = scale_of(a.side[IN0].scale[(int64_t)row * a.side[IN0].scale_pitch + at]);
                scale1 = scale_of(a.side[IN1].scale[(int64_t)row * a.side[IN1].scale_pitch + at]);
            }

            auto one_chunk = [&](int i, F2 (&v)[4][4], F2 (&x)[TWO ? 4 : 1][4]) -> bool {
                const int col = col_of(walk, i);
                const uint32_t b = chunk & 1u;
                uint32_t r[SUMMED ? 1 : 32], u[TWO && !SUMMED ? 32 : 1];
                if constexpr (!SUMMED) tmem_ld32(acc + first + 32 * i, r);
                if constexpr (TWO && !SUMMED) tmem_ld32(acc + COLS + first + 32 * i, u);
                if (fetches) {
                    stored();                                  // the next chunk's boxes are free
                    const uint32_t now = chunk;
                    if (i + 1 < valid) {
                        fetch(now + 1, row0, col + 32);
                    } else if (walk.left > 1) {
                        Walk t = walk;
                        t.next();
                        if (row_of(t) < a.M && col_of(t, 0) < a.N) fetch(now + 1, row_of(t), col_of(t, 0));
                    }
                    if (!wait_warp<false>(in_bar(w, b), (now >> 1) & 1u, abortp, a.wait_ns)) return false;
                } else {
                    if (lane == 0) {
                        if (twice) bulk_wait_read_but_one();
                        else bulk_wait_read_all();
                    }
                    __syncwarp();
                }
                if constexpr (!SUMMED) {
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e >> 2][e & 3] = F2{__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])};
                    if constexpr (TWO) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) x[e >> 2][e & 3] = F2{__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1])};
                    }
                    if (i == CHUNKS - 1) release(buf);
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        add_half(first + 32 * i + 8 * g, v[g]);
                        add_bias(first - block + 32 * i + 8 * g, v[g]);
                    }
                }
                const uint32_t box_in0 = mine + a.side[IN0].box[b], box_in1 = mine + a.side[IN1].box[b];
                const uint32_t box0 = mine + a.side[OUT0].box[b], box1 = mine + a.side[OUT1].box[b], box2 = mine + a.side[OUT2].box[b];
                if constexpr (FORWARD) {
                    write32(form1, box1, lane, inv1, v);
                    if constexpr (TWO) write32(form1, box2, lane, inv2, x);
                }
                Raw32<FORM0> raw0;                             // the residual, or gate
                Raw32<KEPT> raw1;                              // z, or up
                if constexpr (KIND != GATED && FORM0 != kF32)  // (an fp32 one would take the registers of the sums)
                    if (in0 != kNone) read32<FORM0>(box_in0, lane, raw0);
                if constexpr (BACK)
                    if (in1 != kNone) read32<KEPT>(box_in1, lane, raw1);
                with_act(a.act, [&](auto t) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        F2 p[4], q[4];
                        if constexpr (KIND == LINEAR) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[g][e] = value(t, v[g][e]);
                        } else if constexpr (KIND == GATED) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[g][e] = mul2(value(t, v[g][e]), x[g][e]);
                        } else if constexpr (KIND == LINEAR_BACK) {
                            if (in1 != kNone) {
                                numbers8<KEPT>(raw1, g, scale1, p);
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[g][e] = mul2(v[g][e], slope(t, p[e], q[e]));
                                if (form1 != kNone) write8(kBf16, box1, lane, g, 1.f, q);
                            }
                        } else {
                            numbers8<KEPT>(raw0, g, scale0, p);
                            numbers8<KEPT>(raw1, g, scale1, q);
                            F2 up[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                F2 h;
                                const F2 s = slope(t, p[e], h);
                                p[e] = mul2(mul2(v[g][e], q[e]), s);
                                up[e] = mul2(v[g][e], h);
                                q[e] = mul2(q[e], h);
                            }
                            if (form0 != kNone) write8(kBf16, box0, lane, g, 1.f, q);
                            write8(kBf16, box1, lane, g, 1.f, p);
                            write8(kBf16, box2, lane, g, 1.f, up);
                        }
                        if constexpr (KIND == LINEAR || KIND == LINEAR_BACK) {
                            if (in0 != kNone) {
                                if constexpr (FORM0 == kF32) {
                                    raw0.w[2 * g] = lds16(piece_at<8>(box_in0, lane, 2 * g));
                                    raw0.w[2 * g + 1] = lds16(piece_at<8>(box_in0, lane, 2 * g + 1));
                                }
                                numbers8<FORM0>(raw0, g, 1.f, p);
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[g][e] = add2(v[g][e], p[e]);
                            }
                        }
                        if constexpr (KIND != GATED_BACK) write8(F32 ? kF32 : kBf16, box0, lane, g, 1.f, v[g]);
                    }
                });
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    for (int k = OUT0; k <= OUT2; ++k)
                        if (a.side[k].tma) tma_store_2d(&maps.side[k], mine + a.side[k].box[b], col, row0);
                    bulk_commit_group();
                }
                for (int k = OUT0; k <= OUT2; ++k)
                    if (a.side[k].form != kNone && !a.side[k].tma) box_out(a.side[k], mine + a.side[k].box[b], lane, row0, col, a.M, a.N);
                if (by_hand && i + 2 < valid) {
                    stored();
                    box_in(a.side[IN0], mine + a.side[IN0].box[b], lane, row0, col + 64, a.M, a.N);
                }
                ++chunk;
                return true;
            };
            if constexpr (SUMMED) {
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i)
                    if (ok && i < valid) ok = one_chunk(i, sum[i], sum2[i]);
            } else {
#pragma unroll 1
                for (int i = 0; ok && i < valid; ++i) ok = one_chunk(i, sum[0], sum2[0]);
                if (ok && valid < CHUNKS) release(buf);
            }
        }
        if (!ok && fetches && lane == 0) {                     // leaving after a time-out: operands on their way land first
            int never = 0;
            for (uint32_t c = chunk; c < fetched; ++c) mbar_wait(in_bar(w, c & 1u), (c >> 1) & 1u, &never, kLeaveLimitNs);
        }
        if (lane == 0) bulk_wait_all();                        // this warp's stores are complete
        __syncwarp();
    }

    // ---------------- teardown ----------------
    tc_fence_before();
    __syncthreads();
    if (PAIR || split > 1) cluster_sync_all();                 // no CTA frees tensor memory or leaves while a peer still works
    if (warp == 1) {
        tc_fence_after();
        if (PAIR) tmem_dealloc_pair(tmem, 512);
        else tmem_dealloc(tmem, 512);
    }
    if (threadIdx.x == 0 && abort_flag) atomicExch(a.status, (int)ADLOCO_ERR_TIMEOUT);
}

// ---- few rows ---------------------------------------------------------------------------------------
// Up to 16 tokens forward: the time is the weight's bytes from memory.  A block takes 16 rows of the weight (or eight of
// either projection), its warps the blocks of 64 of K in turn; a lane loads 16 bytes of two of those rows and of a row of
// each eight of x straight into the fragments of the warp's own matrix instruction (m16n8k16, the weight's rows as its M):
// the order of K within 32 is the same for both and does not matter.  The warps' sums meet in shared memory, in a fixed order.
// Blocks are small enough for four an SM, so that one wave of them covers the usual widths (with 16 warps and 74 registers a
// thread one block fitted: 13.1 us against 7.8 for one token through 2048 -> 8192).
constexpr int FEW_ROWS = 16, FEW_MAX_WARPS = 8, FEW_MAX_M = 16;
struct FewArgs {
    int M, N, K, act;
    const __nv_bfloat16 *x, *w[2];
    int64_t x_stride, w_stride[2];
    const float* bias;
    Side residual, out0, out1, out2;
};
__device__ __noinline__ uint4 last_of(const __nv_bfloat16* row, int n) {                // fewer than eight, zeros behind
    uint32_t w[4] = {0u, 0u, 0u, 0u};
    const unsigned short* h = reinterpret_cast<const unsigned short*>(row);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) w[i >> 1] |= (uint32_t)h[i] << (16 * (i & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float load_one(const Side& s, int64_t at) {
    return s.form == kF32 ? static_cast<const float*>(s.p)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(s.p)[at]);
}
__device__ __forceinline__ void store_one(const Side& s, int64_t at, float v) {
    if (s.form == kF32) static_cast<float*>(s.p)[at] = v;
    else static_cast<__nv_bfloat16*>(s.p)[at] = __float2bfloat16_rn(v);
}
// F32 outputs take a warp's sums out of the tensor cores every 512 terms, as the tile kernel's do.
template <int TILES, bool TWO, bool F32>                                            // TILES: of eight rows of x
__global__ void __launch_bounds__(32 * FEW_MAX_WARPS, TILES == 1 ? 4 : 3) dense_few_kernel(const __grid_constant__ FewArgs a) {
    extern __shared__ float sums[];                                                 // [warps][TILES * 8][FEW_ROWS + 1]
    after_predecessor();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5, g = lane >> 2, t = lane & 3;
    const int n0 = (int)blockIdx.x * (TWO ? FEW_ROWS / 2 : FEW_ROWS);
    const bool r0 = n0 + g < a.N, r1 = TWO ? r0 : n0 + g + 8 < a.N;
    const __nv_bfloat16* w0 = a.w[0] + (int64_t)(n0 + g) * a.w_stride[0];
    const __nv_bfloat16* w1 = TWO ? a.w[1] + (int64_t)(n0 + g) * a.w_stride[1] : w0 + 8 * a.w_stride[0];
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    float acc[TILES][4], total[F32 ? TILES : 1][4];
#pragma unroll
    for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            acc[j][i] = 0.f;
            if (F32) total[j][i] = 0.f;
        }
    auto add_up = [&]() {
#pragma unroll
        for (int j = 0; j < (F32 ? TILES : 0); ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) { total[j][i] += acc[j][i]; acc[j][i] = 0.f; }
    };
    const int whole = a.K / 64;                                                     // blocks that no row ends in
    int terms = 0;                                                                  // blocks in the sums
#pragma unroll 2
    for (int kb = warp; kb < whole; kb += warps) {
        if (F32 && terms++ == DG_SEGMENT) { add_up(); terms = 1; }
        uint4 p[2], q[2], x[TILES][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = kb * 64 + h * 32 + t * 8;
            p[h] = r0 ? *reinterpret_cast<const uint4*>(w0 + k) : none;
            q[h] = r1 ? *reinterpret_cast<const uint4*>(w1 + k) : none;
#pragma unroll
            for (int j = 0; j < TILES; ++j) {
                const int m = j * 8 + g;
                x[j][h] = m < a.M ? *reinterpret_cast<const uint4*>(a.x + (int64_t)m * a.x_stride + k) : none;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < TILES; ++j) {
                mma_16816(acc[j], p[h].x, q[h].x, p[h].y, q[h].y, x[j][h].x, x[j][h].y);
                mma_16816(acc[j], p[h].z, q[h].z, p[h].w, q[h].w, x[j][h].z, x[j][h].w);
            }
    }
    if (whole * 64 < a.K && whole % warps == warp) {                                // the last one, by the warp whose turn it is
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
            const int k = whole * 64 + h * 32 + t * 8, n = a.K - k;
            auto some = [&](const __nv_bfloat16* row, bool there) {
                return !there || n <= 0 ? none : n >= 8 ? *reinterpret_cast<const uint4*>(row + k) : last_of(row + k, n);
            };
            const uint4 p = some(w0, r0), q = some(w1, r1);
#pragma unroll
            for (int j = 0; j < TILES; ++j) {
                const int m = j * 8 + g;
                const uint4 x = some(a.x + (int64_t)m * a.x_stride, m < a.M);
                mma_16816(acc[j], p.x, q.x, p.y, q.y, x.x, x.y);
                mma_16816(acc[j], p.z, q.z, p.w, q.w, x.z, x.w);
            }
        }
    }
    add_up();
    float* mine = sums + warp * (TILES * 8) * (FEW_ROWS + 1);
#pragma unroll
    for (int j = 0; j < TILES; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) mine[(j * 8 + 2 * t + (i & 1)) * (FEW_ROWS + 1) + g + 8 * (i >> 1)] = F32 ? total[F32 ? j : 0][i] : acc[j][i];
    __syncthreads();
    constexpr int OUT = TWO ? FEW_ROWS / 2 : FEW_ROWS;
    for (int i = threadIdx.x; i < TILES * 8 * OUT; i += blockDim.x) {
        const int m = i / OUT, r = i % OUT, n = n0 + r;
        if (m >= a.M || n >= a.N) continue;
        float v = 0.f, u = 0.f;
        for (int w = 0; w < warps; ++w) {
            const float* at = sums + (w * TILES * 8 + m) * (FEW_ROWS + 1);
            v += at[r];
            if (TWO) u += at[r + 8];
        }
        if (!TWO && a.bias) v += a.bias[n];
        const float res = !TWO && a.residual.form != kNone ? load_one(a.residual, (int64_t)m * a.residual.pitch + n) : 0.f;      // before any output
        if (a.out1.form != kNone) store_one(a.out1, (int64_t)m * a.out1.pitch + n, v);
        if (TWO && a.out2.form != kNone) store_one(a.out2, (int64_t)m * a.out2.pitch + n, u);
        with_act(a.act, [&](auto t) { v = value(t, both(v)).x; });
        if (TWO) v *= u;
        else if (a.residual.form != kNone) v += res;
        store_one(a.out0, (int64_t)m * a.out0.pitch + n, v);
    }
}

// ---- host ---------------------------------------------------------------------------------------------
int64_t elem(int form) { return form == kF32 ? 4 : form == kBf16 ? 2 : 1; }
Side side_of(const void* p, int64_t pitch, int form) {
    Side s;
    if (!p) return s;
    s.p = const_cast<void*>(p);
    s.pitch = pitch;
    s.form = form;
    return s;
}
Side kept_side(const adloco_kept& k) {
    Side s = side_of(k.p, k.stride, k.scale ? kBytes : kBf16);
    s.scale = k.scale;
    s.scale_pitch = k.scale_stride;
    return s;
}

// What a call is, before tiles are chosen.
struct Product {
    int64_t M, N, K;
    int act;
    const void* a;
    int64_t a_stride;
    const void* b[2];
    int64_t b_stride[2];
    const float* bias;
    Side side[SIDES];
    uint32_t warp_bytes, in_bytes;    // what lay_out makes of the sides
    int twice;
};

// How the sides reach their boxes, and where these lie in an epilogue warp's memory: largest first so that each starts on a
// multiple of its swizzle's span; operands twice (they are fetched a chunk ahead), outputs twice where nothing is fetched and
// that takes no more than 8 KB, an output over the operand of its form that is read at the same place.
template <int KIND>
void lay_out(Product& p) {
    p.in_bytes = 0;
    int64_t outputs = 0;
    for (int i = 0; i < SIDES; ++i) {
        Side& s = p.side[i];
        if (s.form == kNone) continue;
        const int64_t es = elem(s.form);
        s.pieces = aligned16(s.p) && s.pitch * es % 16 == 0;
        // a store writes a row's last 16 bytes in full, beyond the matrix too
        s.tma = s.pieces && (i <= IN1 || p.N * es % 16 == 0);
        if (s.tma && i <= IN1) p.in_bytes += (uint32_t)(1024 * es);
        if (i >= OUT0) outputs += 1024 * es;
    }
    p.twice = p.in_bytes == 0 && 2 * outputs <= 8192;
    constexpr int over[SIDES] = {-1, -1, KIND == GATED_BACK ? -1 : IN0, KIND == GATED_BACK ? IN0 : KIND == LINEAR_BACK ? IN1 : -1,
                                 KIND == GATED_BACK ? IN1 : -1};
    uint32_t used = 0;
    for (int form : {(int)kF32, (int)kBf16, (int)kBytes})
        for (int i = 0; i < SIDES; ++i) {
            Side& s = p.side[i];
            if (s.form != form || (over[i] >= 0 && p.side[over[i]].form == form)) continue;
            const uint32_t bytes = (uint32_t)(1024 * elem(form));
            s.box[0] = used;
            s.box[1] = i <= IN1 || p.twice ? used + bytes : used;
            used = s.box[1] + bytes;
        }
    for (int i = OUT0; i < SIDES; ++i)
        if (over[i] >= 0 && p.side[i].form != kNone && p.side[over[i]].form == p.side[i].form)
            for (int b = 0; b < 2; ++b) p.side[i].box[b] = p.side[over[i]].box[b];
    p.warp_bytes = (used + 1023u) & ~1023u;
}

// Shared memory beside the ring and the boxes: barriers, the bias, and the sums of K's other half or the maxima of what goes to 8 bits.
int64_t words_of(const Product& p, int split) { return DG_BAR_BYTES + (split > 1 ? 128 * 64 * 4 : p.side[OUT1].form == kBytes ? DG_EPI * 512 : 0); }
template <bool PAIR, int BN>
int stages_of(const Product& p, int split) {
    const int64_t n = (DG_SMEM - 1024 - words_of(p, split) - (int64_t)DG_EPI * p.warp_bytes) / dg_stage_bytes<PAIR, BN>();
    return (int)(n < DG_MAX_STAGES ? n : DG_MAX_STAGES);
}

template <int KIND, bool PAIR, int BN, int SUM, bool IN8>
int launch_tiles(adloco_ctx* ctx, const Product& p, cudaStream_t st, int split = 1) {
    constexpr bool TWO = KIND == GATED, BACK = KIND == LINEAR_BACK || KIND == GATED_BACK;
    constexpr int COLS = TWO ? BN / 2 : BN, TM = PAIR ? 256 : 128, STAGE = dg_stage_bytes<PAIR, BN>();
    GemmArgs a;
    a.M = (int)p.M; a.N = (int)p.N; a.K = (int)p.K;
    constexpr int BLOCKS = dg_stage_blocks<PAIR, BN>();
    a.kb = (int)((p.K + 64 * BLOCKS - 1) / (64 * BLOCKS));
    const int64_t tm = (p.M + TM - 1) / TM, tn = (p.N + COLS - 1) / COLS;
    if (tm * tn > 0x7fffffff) return ADLOCO_ERR_UNSUPPORTED;
    a.tiles_n = (int)tn; a.tiles = (int)(tm * tn);
    a.act = p.act; a.bias = p.bias;
    a.status = ctx->gemm_status; a.wait_ns = ctx->wait_limit_ns;
    a.in_bytes = p.in_bytes; a.twice = p.twice; a.warp_bytes = p.warp_bytes;
    a.split = split;
    a.stages = stages_of<PAIR, BN>(p, split);
    if (a.stages < 2) return ADLOCO_ERR_UNSUPPORTED;
    Maps maps;
    // (what lies in the rest of A's 128 rows only reaches rows of the result that do not exist)
    const uint32_t a_rows = p.M < 128 ? (uint32_t)(p.M + 7) / 8 * 8 : 128;
    a.a_bytes = (int)a_rows * 128;
    int rc = make_map(ctx, &maps.a, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.a, p.M, p.K, p.a_stride, 64, a_rows);
    for (int i = 0; i < (TWO ? 2 : 1) && rc == ADLOCO_OK; ++i)
        rc = BACK ? make_map(ctx, &maps.b[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.b[i], p.K, p.N, p.b_stride[i], 64, 64)
                  : make_map(ctx, &maps.b[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p.b[i], p.N, p.K, p.b_stride[i], 64, TWO ? COLS : PAIR ? BN / 2 : BN);
    if (!TWO) maps.b[1] = maps.b[0];
    for (int i = 0; i < SIDES && rc == ADLOCO_OK; ++i) {
        const Side& s = a.side[i] = p.side[i];
        maps.side[i] = maps.a;                        // not looked at where no box goes by TMA
        if (!s.tma) continue;
        rc = s.form == kBf16 ? make_map(ctx, &maps.side[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, s.p, p.M, p.N, s.pitch, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B)
           : s.form == kF32 ? make_map(ctx, &maps.side[i], CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, s.p, p.M, p.N, s.pitch, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B)
                            : make_map(ctx, &maps.side[i], CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, s.p, p.M, p.N, s.pitch, 32, 32, CU_TENSOR_MAP_SWIZZLE_32B);
    }
    if (rc != ADLOCO_OK) return rc;
    auto* kernel = dense_tile_kernel<KIND, PAIR, BN, SUM, IN8>;
    static std::atomic<bool> attr_set[64];            // the attribute is per device
    if (!attr_set[ctx->device & 63].load()) {
        ADLOCO_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, DG_SMEM));
        attr_set[ctx->device & 63].store(true);
    }
    const size_t smem = (size_t)a.stages * STAGE + DG_EPI * (size_t)a.warp_bytes + (size_t)words_of(p, split) + 1024;
    const int most = PAIR ? ctx->sm_count / 2 : ctx->sm_count, workers = a.tiles < most ? a.tiles : most;
    ADLOCO_CUDA_TRY(ctx, launch_early(kernel, dim3((PAIR ? 2 : split) * workers), DG_THREADS, smem, st, PAIR ? 2 : split, maps, a));
    ctx->launches++;
    return ADLOCO_OK;
}

// Which tiles: those that take the least time in rounds of all SMs.  A stage of 64 of K takes a CTA as long as L2 needs to
// deliver its operands, 64 bytes a clock: 512 clocks for a pair's 256 x 256 (as long as its MMAs) and for one CTA's 128 x 128,
// 384 for a pair's 256 x 128 and one CTA's 128 x 64, less where A has fewer rows; a tile's epilogue as much as four (two, one) stages
// that nothing hides when there is one round.
template <int KIND, int SUM, bool IN8 = false>
int choose_tiles(adloco_ctx* ctx, Product& p, cudaStream_t st) {
    lay_out<KIND>(p);
    constexpr int SHARE = KIND == GATED ? 2 : 1;      // of a tile's columns a projection's are
    const bool bytes = p.side[OUT1].form == kBytes;   // 8-bit outputs: a block of 128 columns in one tile
    const bool pairs = cta_pairs_possible(ctx);
    const int64_t kb = (p.K + 63) / 64, a_rows = p.M < 128 ? p.M : 128;
    auto clocks = [&](int64_t tile_m, int64_t tile_n, int64_t workers, int64_t bytes_a_stage, int64_t epilogue) {
        const int64_t tiles = ((p.M + tile_m - 1) / tile_m) * ((p.N + tile_n / SHARE - 1) / (tile_n / SHARE)), rounds = (tiles + workers - 1) / workers;
        return rounds * kb * (bytes_a_stage / 64) + epilogue * 512 * (rounds > 1 ? 1 : 2);
    };
    const int64_t never = int64_t(1) << 62, sms = ctx->sm_count;
    // (z in 8 bits beside a bf16 output: the sums of 128 columns spill beside all else in registers: 32768 x 768 -> 2048 131 us,
    // 117 with tiles of 128 columns, whose warps have 64 each)
    const int64_t pair256 = pairs && !(KIND == LINEAR && SUM == kSummed) ? clocks(256, 256, sms / 2, a_rows * 128 + 16384, 4) : never;
    const int64_t pair128 = pairs && !(bytes && SHARE == 2) ? clocks(256, 128, sms / 2, a_rows * 128 + 8192, 2) : never;
    const int64_t solo128 = bytes && SHARE == 2 ? never : clocks(128, 128, sms, a_rows * 128 + 16384, 2);
    const int64_t least = std::min(std::min(pair256, pair128), solo128);
    if constexpr (KIND == GATED && SUM == kSummed) {  // 128 columns of each projection in any case
        return clocks(128, 256, sms, a_rows * 128 + 32768, 4) < pair256 ? launch_tiles<KIND, false, 256, SUM, IN8>(ctx, p, st)
                                                                        : launch_tiles<KIND, true, 256, SUM, IN8>(ctx, p, st);
    } else {
        if constexpr (KIND != GATED && SUM != kSummed) {
            if (!bytes) {
                // tiles of 64 columns, and half of K for each of two CTAs where all clusters run at once, there is work for both, and their
                // join leaves the ring two stages beside the boxes: the join takes as long as four stages
                const int64_t alone = clocks(128, 64, sms, a_rows * 128 + 8192, 1), tiles = ((p.M + 127) / 128) * ((p.N + 63) / 64);
                const bool split = pairs && tiles * 2 <= sms && kb >= 16 && stages_of<false, 64>(p, 2) >= 2;
                const int64_t both = split ? (kb + 1) / 2 * ((a_rows * 128 + 8192) / 64) + 3 * 1024 : never;
                if (std::min(alone, both) < least) return launch_tiles<KIND, false, 64, SUM, IN8>(ctx, p, st, both < alone ? 2 : 1);
            }
        }
        if constexpr (SUM != kSummed)
            if (least == pair256) return launch_tiles<KIND, true, 256, SUM, IN8>(ctx, p, st);
        if (least == pair128) return launch_tiles<KIND, true, 128, SUM, IN8>(ctx, p, st);
        return launch_tiles<KIND, false, 128, SUM, IN8>(ctx, p, st);
    }
}

template <bool TWO, bool F32>
int launch_few(adloco_ctx* ctx, const Product& p, cudaStream_t st) {
    FewArgs a;
    a.M = (int)p.M; a.N = (int)p.N; a.K = (int)p.K; a.act = p.act;
    a.x = static_cast<const __nv_bfloat16*>(p.a); a.x_stride = p.a_stride;
    for (int i = 0; i < 2; ++i) { a.w[i] = static_cast<const __nv_bfloat16*>(p.b[i]); a.w_stride[i] = p.b_stride[i]; }
    a.bias = p.bias;
    a.residual = p.side[IN0]; a.out0 = p.side[OUT0]; a.out1 = p.side[OUT1]; a.out2 = p.side[OUT2];
    const int each = TWO ? FEW_ROWS / 2 : FEW_ROWS, blocks = (int)((p.K + 63) / 64);
    const int tiles = p.M <= 8 ? 1 : 2;
    const dim3 grid((unsigned)((p.N + each - 1) / each));
    // as many warps a block as leave room for all blocks at once (64 registers a thread: 32 warps an SM), where that is no fewer than two
    const int an_sm = (int)((grid.x + ctx->sm_count - 1) / ctx->sm_count), fit = an_sm <= 16 ? 32 / an_sm : FEW_MAX_WARPS;
    const int warps = std::min(std::min(blocks, fit), FEW_MAX_WARPS);
    const size_t smem = (size_t)warps * tiles * 8 * (FEW_ROWS + 1) * sizeof(float);
    const cudaError_t e = tiles == 1 ? launch_early(dense_few_kernel<1, TWO, F32>, grid, 32 * warps, smem, st, 1, a)
                                     : launch_early(dense_few_kernel<2, TWO, F32>, grid, 32 * warps, smem, st, 1, a);
    ADLOCO_CUDA_TRY(ctx, e);
    ctx->launches++;
    return ADLOCO_OK;
}

}  // namespace

int launch_linear(adloco_ctx* ctx, const adloco_linear_args& c, cudaStream_t st) {
    Product p = {c.M, c.N, c.K, c.activation, c.x, c.x_stride, {c.w, c.w}, {c.w_stride, c.w_stride}, c.bias, {}};
    const int form = c.out_dtype == ADLOCO_BF16 ? kBf16 : kF32;
    p.side[IN0] = side_of(c.residual, c.residual_stride, form);
    p.side[OUT0] = side_of(c.y, c.y_stride, form);
    p.side[OUT1] = kept_side(c.z);
    if (c.M <= FEW_MAX_M && p.side[OUT1].form != kBytes) return form == kF32 ? launch_few<false, true>(ctx, p, st) : launch_few<false, false>(ctx, p, st);
    if (form == kF32) return choose_tiles<LINEAR, kSummedF32>(ctx, p, st);
    return p.side[OUT1].form == kBytes ? choose_tiles<LINEAR, kSummed>(ctx, p, st) : choose_tiles<LINEAR, kPlain>(ctx, p, st);
}

int launch_linear_backward(adloco_ctx* ctx, const adloco_linear_backward_args& c, cudaStream_t st) {
    Product p = {c.M, c.K, c.N, c.activation, c.dy, c.dy_stride, {c.w, c.w}, {c.w_stride, c.w_stride}, nullptr, {}};
    const int form = c.out_dtype == ADLOCO_BF16 ? kBf16 : kF32;
    p.side[IN0] = side_of(c.residual, c.residual_stride, form);
    p.side[IN1] = kept_side(c.z);
    p.side[OUT0] = side_of(c.dx, c.dx_stride, form);
    p.side[OUT1] = side_of(c.a, c.a_stride, kBf16);
    if (c.z.scale) return form == kF32 ? choose_tiles<LINEAR_BACK, kSummedF32, true>(ctx, p, st) : choose_tiles<LINEAR_BACK, kPlain, true>(ctx, p, st);
    return form == kF32 ? choose_tiles<LINEAR_BACK, kSummedF32>(ctx, p, st) : choose_tiles<LINEAR_BACK, kPlain>(ctx, p, st);
}

int launch_gated_linear(adloco_ctx* ctx, const adloco_gated_linear_args& c, cudaStream_t st) {
    Product p = {c.M, c.f, c.d, c.activation, c.x, c.x_stride, {c.w_gate, c.w_up}, {c.w_gate_stride, c.w_up_stride}, nullptr, {}};
    p.side[OUT0] = side_of(c.a, c.a_stride, kBf16);
    p.side[OUT1] = kept_side(c.gate);
    p.side[OUT2] = kept_side(c.up);
    if (c.M <= FEW_MAX_M && p.side[OUT1].form != kBytes) return launch_few<true, false>(ctx, p, st);
    return p.side[OUT1].form == kBytes ? choose_tiles<GATED, kSummed>(ctx, p, st) : choose_tiles<GATED, kPlain>(ctx, p, st);
}

int launch_gated_linear_backward(adloco_ctx* ctx, const adloco_gated_linear_backward_args& c, cudaStream_t st) {
    Product p = {c.M, c.f, c.d, c.activation, c.dy, c.dy_stride, {c.w_down, c.w_down}, {c.w_down_stride, c.w_down_stride}, nullptr, {}};
    p.side[IN0] = kept_side(c.gate);
    p.side[IN1] = kept_side(c.up);
    p.side[OUT0] = side_of(c.a, c.a_stride, kBf16);
    p.side[OUT1] = side_of(c.d_gate, c.d_gate_stride, kBf16);
    p.side[OUT2] = side_of(c.d_up, c.d_up_stride, kBf16);
    return c.gate.scale ? choose_tiles<GATED_BACK, kPlain, true>(ctx, p, st) : choose_tiles<GATED_BACK, kPlain>(ctx, p, st);
}

}  // namespace adloco

// Operators of a decoder block between its linear layers: norm with the residual's addition and
// dropout, its backward pass with the gain's per-sample norms, dropout alone, rotary positions,
// and quantisation to 8 bits with power-of-two scales.  All are bound by HBM: each input is read
// once, each output written once, everything between stays in registers.
#include <cuda_fp8.h>

#include "common.cuh"

namespace adloco {

namespace {

// ---- eight adjacent elements of a row ---------------------------------------------------
// The vector form is one 16-byte access (two for float); the guarded form takes rows that do not
// start on 16-byte boundaries and a row's last, incomplete group.
template <bool VEC>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int n, float (&v)[8]) {
    if (VEC) {
        const uint4 w = __ldcs(reinterpret_cast<const uint4*>(p));
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? __bfloat162float(p[i]) : 0.f;
    }
}
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
    if (VEC) {
        const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
    }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <bool VEC>
__device__ __forceinline__ void store8(__nv_bfloat16* p, int n, const float (&v)[8]) {
    if (VEC) {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = __float2bfloat16_rn(v[i]);
    }
}
template <bool VEC>
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
    if (VEC) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
        __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i];
    }
}
// the gain is read by every row: it stays in L1
__device__ __forceinline__ void load_gain8(const void* gain, int bf16, int col, int n, float (&g)[8]) {
    if (n == 8 && (reinterpret_cast<uintptr_t>(gain) & 15u) == 0) {
        if (bf16) {
            const uint4 w = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(gain) + col));
            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                g[2 * i] = __uint_as_float(u[i] << 16);
                g[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
            }
        } else {
            const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(gain) + col);
            const float4 a = __ldg(p), b = __ldg(p + 1);
            g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w;
            g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= n) g[i] = 0.f;
        else g[i] = bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(gain)[col + i]) : __ldg(static_cast<const float*>(gain) + col + i);
    }
}

// ---- Philox-4x32-10 ---------------------------------------------------------------------
// Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3" (2011): ten rounds of two
// 32 x 32 -> 64-bit products on a 128-bit counter.  One call serves eight elements, 16 bits each: with
// 32 bits an element the integer work, not HBM, would set the time of dropout on bf16.
__device__ __forceinline__ uint4 philox(uint64_t group, const DropoutKey& k) {
    uint32_t c0 = (uint32_t)group, c1 = (uint32_t)(group >> 32), c2 = k.off_lo, c3 = k.off_hi;
    uint32_t k0 = k.seed_lo, k1 = k.seed_hi;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}
// drop() of the eight elements from flat index e on; a dropped element is 0 whatever it held.  Rows whose length
// is not a multiple of eight start inside a group: such eight elements span two groups.
__device__ __forceinline__ void drop8(float (&v)[8], uint64_t e, const DropoutKey& k) {
    const uint4 w = philox(e >> 3, k);
    uint32_t u[8] = {w.x, w.y, w.z, w.w, 0u, 0u, 0u, 0u};
    const uint32_t sh = (uint32_t)e & 7u;
    if (sh) {
        const uint4 w2 = philox((e >> 3) + 1, k);
        u[4] = w2.x; u[5] = w2.y; u[6] = w2.z; u[7] = w2.w;
        // shift the 16 halves down by sh
        if (sh & 4u) { u[0] = u[2]; u[1] = u[3]; u[2] = u[4]; u[3] = u[5]; u[4] = u[6]; u[5] = u[7]; }
        if (sh & 2u) { u[0] = u[1]; u[1] = u[2]; u[2] = u[3]; u[3] = u[4]; u[4] = u[5]; }
        if (sh & 1u) {
#pragma unroll
            for (int i = 0; i < 4; ++i) u[i] = __funnelshift_r(u[i], u[i + 1], 16);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t h = (i & 1) ? u[i >> 1] >> 16 : u[i >> 1] & 0xffffu;
        v[i] = h >= k.drop ? v[i] * k.scale : 0.f;
    }
}

// ---- 8-bit blocks -------------------------------------------------------------------------
// The scale's byte from the bits of the block's largest magnitude: with that magnitude m 2^k, 1 <= m < 2, and
// 448 = 1.75 2^8, the smallest whole e with m 2^k <= 448 2^e is k - 8, or k - 7 where m > 1.75; adding
// 0x1fffff to the fraction carries into the exponent exactly when m > 1.75.  An Inf or NaN (compared as whole
// numbers, so that a NaN is not lost in a maximum) gives 255.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return 255u;
    if (amax_bits == 0u) return 127u;
    const int b = (int)((amax_bits + 0x1fffffu) >> 23) - 8;
    return b < 0 ? 0u : (uint32_t)b;
}
// 1 / scale: a power of two, so multiplying by it is exact (byte 0..247 of a finite block)
__device__ __forceinline__ float inv_scale(uint32_t byte) { return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ uint32_t abs_max8(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}
__device__ __forceinline__ uint2 to_e4m3x8(const float (&v)[8], float inv) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * i] * inv, v[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}
// The 16 lanes that hold one block of a row (8 adjacent elements each) agree on its scale; the lane of the
// block's first elements writes it.  Every lane of the warp takes part; n = 0 for lanes beyond the row.
__device__ __forceinline__ void quantise_block(const float (&v)[8], int n, uint8_t* q_row, uint8_t* scale_row, int col) {
    uint32_t m = n > 0 ? abs_max8(v) : 0u;          // elements beyond n are zero
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (n <= 0) return;
    const uint32_t s = scale_byte(m);
    const uint2 w = to_e4m3x8(v, inv_scale(s));
    if (n == 8) *reinterpret_cast<uint2*>(q_row + col) = w;          // pitch and base are multiples of 16
    else
        for (int i = 0; i < n; ++i) q_row[col + i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
    if ((col & 127) == 0) scale_row[col >> 7] = (uint8_t)s;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// sum over the TPR threads of a row; smem: one float per warp of the block.  `turn` alternates between two
// halves of smem, so one barrier a call is enough
template <int TPR, int THREADS>
__device__ __forceinline__ float row_sum(float v, float* smem, int turn) {
    v = warp_sum(v);
    if (TPR == 32) return v;
    constexpr int W = TPR / 32;
    float* half = smem + (turn & 1) * (THREADS / 32);
    if ((threadIdx.x & 31) == 0) half[threadIdx.x >> 5] = v;
    __syncthreads();
    const float* mine = half + (threadIdx.x / TPR) * W;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) s += mine[i];
    return s;
}

__host__ __device__ constexpr int row_threads(int tpr) { return tpr > 256 ? tpr : 256; }

// ---- norm, forward --------------------------------------------------------------------------
// TPR threads hold a row of up to TPR * C * 8 elements in registers: one read of x and of the residual, the
// sum of squares in fp32, then every output from the registers.
template <typename XT, typename ST, int TPR, int C, bool VEC>
__global__ void __launch_bounds__(row_threads(TPR)) add_rmsnorm_kernel(const __grid_constant__ adloco_rmsnorm_args a,
                                                                        const __grid_constant__ DropoutKey key) {
    constexpr int THREADS = row_threads(TPR), ROWS = THREADS / TPR;
    __shared__ float smem[2 * THREADS / 32];
    const int t = threadIdx.x % TPR;
    const int64_t row_asked = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    const bool there = row_asked < a.rows;
    if (TPR == 32 && !there) return;                       // whole warps leave; wider rows meet at a barrier
    const int64_t row = there ? row_asked : a.rows - 1;
    const int d = (int)a.d;
    const XT* x = static_cast<const XT*>(a.x) + row * a.x_stride;
    const ST* r = a.residual ? static_cast<const ST*>(a.residual) + row * a.residual_stride : nullptr;
    float h[C][8], e[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8, n = min(8, d - col);
        if (n > 0) load8<VEC>(x + col, n, h[c]);
        else for (int i = 0; i < 8; ++i) h[c][i] = 0.f;
    }
    if (r) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * 8, n = min(8, d - col);
            if (n > 0) load8<VEC>(r + col, n, e[c]);
            else for (int i = 0; i < 8; ++i) e[c][i] = 0.f;
        }
    }
    if (key.drop) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * 8;
            if (col < d) drop8(h[c], (uint64_t)(row * d + col), key);
        }
    }
    const float inv_d = 1.0f / (float)d;
    float ss = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8, n = min(8, d - col);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r) h[c][i] += e[c][i];
            if (!VEC && i >= n) h[c][i] = 0.f;
            ss = fmaf(h[c][i] * inv_d, h[c][i], ss);      // the mean: the sum of squares that fit fp32 may not fit
        }
        if (a.h && there && n > 0) store8<VEC>(static_cast<ST*>(a.h) + row * a.h_stride + col, n, h[c]);
    }
    ss = row_sum<TPR, THREADS>(ss, smem, 0);
    const float rstd = rsqrtf(ss + a.eps);
    if (a.rstd && there && t == 0) a.rstd[row] = rstd;
    uint8_t* q_row = static_cast<uint8_t*>(a.q) + row * a.q_stride;
    uint8_t* s_row = a.q_scale + row * a.q_scale_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8, n = there ? min(8, d - col) : 0;
        float y[8], g[8];
        if (n > 0) load_gain8(a.gain, a.gain_dtype == ADLOCO_BF16, col, n, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = n > i ? h[c][i] * rstd * g[i] : 0.f;
        if (a.y && n > 0) store8<VEC>(static_cast<XT*>(a.y) + row * a.y_stride + col, n, y);
        if (a.q) quantise_block(y, n, q_row, s_row, col);
    }
}

// ---- norm, backward ---------------------------------------------------------------------------
// A block takes `rows_per_chunk` consecutive rows of one sample, ROWS at a time.  With the row in registers the
// two row sums of the formula collapse into one (gain dy . xhat), and the gain's gradient dy xhat is added up in
// registers over the block's rows; blocks leave it in the workspace [B, chunks, d] for rmsnorm_gain_kernel, so
// h and dy are read once for both gradients and no sum depends on the order of atomics.
struct RmsBackArgs {
    adloco_rmsnorm_backward_args a;
    int64_t chunks, rows_per_chunk;
};
template <typename XT, typename ST, int TPR, int C, bool VEC, bool GAIN>
__global__ void __launch_bounds__(row_threads(TPR)) rmsnorm_backward_kernel(const __grid_constant__ RmsBackArgs p,
                                                                            const __grid_constant__ DropoutKey key) {
    constexpr int THREADS = row_threads(TPR), ROWS = THREADS / TPR;
    const adloco_rmsnorm_backward_args& a = p.a;
    extern __shared__ float columns[];                     // [ROWS][d] when GAIN and ROWS > 1
    __shared__ float smem[2 * THREADS / 32];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR, d = (int)a.d;
    const int64_t sample = (int64_t)blockIdx.x / p.chunks, chunk = (int64_t)blockIdx.x % p.chunks;
    const int64_t first = chunk * p.rows_per_chunk, last = min(a.T, first + p.rows_per_chunk);
    const float inv_d = 1.0f / (float)d;
    float acc[GAIN ? C : 1][8];
    if (GAIN) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[c][i] = 0.f;
    }
    int turn = 0;
    for (int64_t at = first; at < last; at += ROWS, ++turn) {
        const bool there = at + sub < last;
        if (TPR == 32 && !there) break;
        const int64_t row = sample * a.T + (there ? at + sub : last - 1);
        const XT* dy = static_cast<const XT*>(a.dy) + row * a.dy_stride;
        const ST* h = static_cast<const ST*>(a.h) + row * a.h_stride;
        float u[C][8], v[C][8], r[C][8];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * 8, n = min(8, d - col);
            if (n > 0) { load8<VEC>(dy + col, n, u[c]); load8<VEC>(h + col, n, v[c]); }
            else for (int i = 0; i < 8; ++i) { u[c][i] = 0.f; v[c][i] = 0.f; }
        }
        if (a.dh_residual) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * 8, n = min(8, d - col);
                if (n > 0) load8<VEC>(static_cast<const ST*>(a.dh_residual) + row * a.dh_residual_stride + col, n, r[c]);
            }
        }
        const float rstd = a.rstd[row];
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * 8, n = min(8, d - col);
            if (n <= 0) continue;
            float g[8];
            load_gain8(a.gain, a.gain_dtype == ADLOCO_BF16, col, n, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] *= rstd;                                               // xhat
                if (GAIN && there) acc[c][i] = fmaf(u[c][i], v[c][i], acc[c][i]);
                u[c][i] *= g[i];
                dot = fmaf(u[c][i], v[c][i], dot);
            }
        }
        const float m = row_sum<TPR, THREADS>(dot, smem, turn) * inv_d;
        if (!there) continue;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * 8, n = min(8, d - col);
            if (n <= 0) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                o[i] = rstd * (u[c][i] - v[c][i] * m);
                if (a.dh_residual) o[i] += r[c][i];
            }
            store8<VEC>(static_cast<ST*>(a.dh) + row * a.dh_stride + col, n, o);
            if (a.dx) {
                if (key.drop) drop8(o, (uint64_t)(row * d + col), key);
                store8<VEC>(static_cast<XT*>(a.dx) + row * a.dx_stride + col, n, o);
            }
        }
    }
    if (!GAIN) return;
    float* part = static_cast<float*>(a.workspace) + (int64_t)blockIdx.x * d;
    if (ROWS == 1) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int col = (c * TPR + t) * 8 + i;
                if (col < d) part[col] = acc[c][i];
            }
        return;
    }
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int col = (c * TPR + t) * 8 + i;
            if (col < d) columns[sub * d + col] = acc[c][i];
        }
    __syncthreads();
    for (int col = threadIdx.x; col < d; col += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < ROWS; ++k) s += columns[k * d + col];
        part[col] = s;
    }
}

// Adds up the workspace in a fixed order.  Blocks [0, B) (when norms are asked for): one sample's gradient over
// all columns, squared and summed.  The rest: 32 columns each of the sum over all samples.
constexpr int kGainThreads = 512;
__global__ void __launch_bounds__(kGainThreads) rmsnorm_gain_kernel(const float* part, int64_t B, int64_t chunks, int d,
                                                                    float* norms, int accumulate_norms, float* sum,
                                                                    int accumulate_sum) {
    constexpr int G = kGainThreads / 32;
    __shared__ float smem[G][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t norm_blocks = norms ? B : 0;
    if ((int64_t)blockIdx.x < norm_blocks) {
        const float* mine = part + (int64_t)blockIdx.x * chunks * d;
        float ss = 0.f;
        for (int col = threadIdx.x; col < d; col += kGainThreads) {
            float g = 0.f;
#pragma unroll 8
            for (int64_t k = 0; k < chunks; ++k) g += mine[k * d + col];
            ss = fmaf(g, g, ss);
        }
        ss = warp_sum(ss);
        if (lane == 0) smem[0][warp] = ss;
        __syncthreads();
        if (threadIdx.x == 0) {
            float n = 0.f;
            for (int w = 0; w < G; ++w) n += smem[0][w];
            if (accumulate_norms) atomicAdd(norms + blockIdx.x, n);      // layers on other streams add here too
            else norms[blockIdx.x] = n;
        }
        return;
    }
    const int col = (int)(blockIdx.x - norm_blocks) * 32 + lane;
    float s = 0.f;
    if (col < d) {
        const int64_t rows = B * chunks;
#pragma unroll 8
        for (int64_t k = warp; k < rows; k += G) s += part[k * d + col];
    }
    smem[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < d) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < G; ++w) t += smem[w][lane];
        sum[col] = accumulate_sum ? sum[col] + t : t;
    }
}

// ---- dropout ------------------------------------------------------------------------------------
// A thread takes the eight elements of one call of the generator.  They are adjacent in memory unless a row ends
// among them; the vector form needs rows of a multiple of eight elements, or no gaps between rows.
struct DropArgs {
    const void *x, *r;
    void* y;
    int64_t rows, cols, x_stride, r_stride, y_stride, groups;
};
template <typename T, bool VEC, bool FLAT>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropArgs a, const __grid_constant__ DropoutKey key) {
    const T* x = static_cast<const T*>(a.x);
    const T* r = static_cast<const T*>(a.r);
    T* y = static_cast<T*>(a.y);
    const int64_t total = a.rows * a.cols;
    for (int64_t g = (int64_t)blockIdx.x * 256 + threadIdx.x; g < a.groups; g += (int64_t)gridDim.x * 256) {
        const int64_t e = g * 8;
        const int n = (int)min((int64_t)8, total - e);
        float v[8], s[8];
        if (FLAT) {
            if (VEC && n == 8) {
                load8<true>(x + e, 8, v);
                if (r) load8<true>(r + e, 8, s);
            } else {
                load8<false>(x + e, n, v);
                if (r) load8<false>(r + e, n, s);
            }
        } else {
            const int64_t row = e / a.cols, col = e - row * a.cols;
            if (VEC) {
                load8<true>(x + row * a.x_stride + col, 8, v);
                if (r) load8<true>(r + row * a.r_stride + col, 8, s);
            } else {
                int64_t i = row, j = col;
                for (int k = 0; k < 8; ++k) {
                    v[k] = s[k] = 0.f;
                    if (k < n) {
                        v[k] = (float)x[i * a.x_stride + j];
                        if (r) s[k] = (float)r[i * a.r_stride + j];
                        if (++j == a.cols) { j = 0; ++i; }
                    }
                }
            }
        }
        drop8(v, (uint64_t)e, key);
        if (r) {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += s[k];
        }
        if (FLAT) {
            if (VEC && n == 8) store8<true>(y + e, 8, v);
            else store8<false>(y + e, n, v);
        } else {
            const int64_t row = e / a.cols, col = e - row * a.cols;
            if (VEC) {
                store8<true>(y + row * a.y_stride + col, 8, v);
            } else {
                int64_t i = row, j = col;
                for (int k = 0; k < n; ++k) {
                    y[i * a.y_stride + j] = (T)v[k];
                    if (++j == a.cols) { j = 0; ++i; }
                }
            }
        }
    }
}

// ---- rotary positions -----------------------------------------------------------------------------
// A block takes a few tokens: it first forms the cosines and sines of their positions in shared memory (one
// sincospi for each pair, shared by all heads of all tensors), then goes through the tokens' heads in units of P
// pairs, neighbouring threads on neighbouring memory.
struct RopeArgs {
    adloco_rope_tensor t[4];
    int n;
    int heads_before[5];
    int64_t B, T, tokens;
    int D, R, rot_units, units;        // units of P pairs a head: rotated, and with the copied rest
    int tokens_per_block;
    const uint64_t* turns;
    const int32_t* positions;
    int64_t positions_stride, first;
    float magnitude;
    int inverse;
};
template <typename T, int P>
struct alignas(sizeof(T) * P) Pack { T v[P]; };

template <typename T, int P, bool INTERLEAVED>
__global__ void __launch_bounds__(256) rope_kernel(const __grid_constant__ RopeArgs a) {
    extern __shared__ float2 turn_cs[];                // [tokens_per_block][R / 2]
    const int half = a.R / 2;
    const int64_t token0 = (int64_t)blockIdx.x * a.tokens_per_block;
    const int here = (int)min((int64_t)a.tokens_per_block, a.tokens - token0);
    for (int i = threadIdx.x; i < here * half; i += 256) {
        const int tok = i / half, j = i - tok * half;
        const int64_t b = (token0 + tok) / a.T, s = (token0 + tok) - b * a.T;
        const int64_t pos = a.positions ? (int64_t)a.positions[b * a.positions_stride + s] : a.first + s;
        // the phase in units of 2^-64 turns is exact; its top 32 bits, as a signed number, are half turns in [-1, 1)
        const int32_t top = (int32_t)(((uint64_t)pos * a.turns[j]) >> 32);
        float sn, cs;
        sincospif((float)top * 4.656612873077392578125e-10f, &sn, &cs);
        if (a.inverse) sn = -sn;
        turn_cs[i] = make_float2(a.magnitude * cs, a.magnitude * sn);
    }
    __syncthreads();
    const int per_token = a.heads_before[a.n] * a.units;
    for (int i = threadIdx.x; i < here * per_token; i += 256) {
        const int tok = i / per_token, rem = i - tok * per_token;
        int head = rem / a.units;
        const int unit = rem - head * a.units;
        int k = 0;
        while (k + 1 < a.n && head >= a.heads_before[k + 1]) ++k;
        head -= a.heads_before[k];
        const adloco_rope_tensor& t = a.t[k];
        const int64_t b = (token0 + tok) / a.T, s = (token0 + tok) - b * a.T;
        const T* in = static_cast<const T*>(t.in) + b * t.in_batch + s * t.in_token + head * t.in_head;
        T* out = static_cast<T*>(t.out) + b * t.out_batch + s * t.out_token + head * t.out_head;
        using V = Pack<T, P>;
        if (unit >= a.rot_units) {                     // the part of the head that is not rotated
            const int at = a.R + (unit - a.rot_units) * P;
            *reinterpret_cast<V*>(out + at) = *reinterpret_cast<const V*>(in + at);
            continue;
        }
        const int j0 = unit * P;                       // first pair
        const int at0 = INTERLEAVED ? 2 * j0 : j0, at1 = INTERLEAVED ? 2 * j0 + P : j0 + half;
        V x0 = *reinterpret_cast<const V*>(in + at0), x1 = *reinterpret_cast<const V*>(in + at1);
        const float2* cs = turn_cs + tok * half + j0;
        float f[2 * P];                                // pair p: f[2p], f[2p + 1] interleaved, else f[p], f[P + p]
#pragma unroll
        for (int p = 0; p < P; ++p) { f[p] = (float)x0.v[p]; f[P + p] = (float)x1.v[p]; }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float& lo = f[INTERLEAVED ? 2 * p : p];
            float& hi = f[INTERLEAVED ? 2 * p + 1 : P + p];
            const float u = lo, w = hi;
            lo = u * cs[p].x - w * cs[p].y;
            hi = u * cs[p].y + w * cs[p].x;
        }
#pragma unroll
        for (int p = 0; p < P; ++p) { x0.v[p] = (T)f[p]; x1.v[p] = (T)f[P + p]; }
        *reinterpret_cast<V*>(out + at0) = x0;
        *reinterpret_cast<V*>(out + at1) = x1;
    }
}

// ---- quantisation -----------------------------------------------------------------------------------
// Rows: 16 lanes hold a block of 128.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) quantise_rows_kernel(const T* x, int64_t x_stride, uint8_t* q, int64_t q_stride,
                                                            uint8_t* scale, int64_t scale_stride, int64_t rows, int64_t cols,
                                                            int64_t blocks_per_row) {
    const int64_t block = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    const bool there = block < rows * blocks_per_row;
    const int64_t row = there ? block / blocks_per_row : 0;
    const int64_t col = (block - row * blocks_per_row) * 128 + (threadIdx.x & 15) * 8;
    const int n = there ? (int)min((int64_t)8, cols - col) : 0;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (n > 0) {
        if (VEC && n == 8) load8<true>(x + row * x_stride + col, 8, v);
        else load8<false>(x + row * x_stride + col, n, v);
    }
    // columns relative to the block: its scale is element 0 of what is passed
    quantise_block(v, n, q + row * q_stride + (col & ~(int64_t)127), scale + row * scale_stride + (col >> 7), (int)(col & 127));
}

// Weights: a block of threads holds a 128 x 128 block (64 elements a thread), agrees on its scale, writes its
// rows and, through shared memory, its columns.
template <typename T>
__global__ void __launch_bounds__(256) quantise_weight_kernel(const T* W, int64_t W_stride, uint8_t* q, int64_t q_stride, uint8_t* q_t,
                                                              int64_t q_t_stride, uint8_t* scale, int64_t scale_stride, int64_t rows,
                                                              int64_t cols, int vec) {
    __shared__ uint32_t amax[8];
    alignas(16) __shared__ uint8_t tile[128][132];                   // [column][row]; rows of 33 words: threads of a warp fall on different banks
    const int64_t r0 = (int64_t)blockIdx.y * 128, c0 = (int64_t)blockIdx.x * 128;
    const int cl = (threadIdx.x & 15) * 8, rl = threadIdx.x >> 4;
    const int n = (int)max((int64_t)0, min((int64_t)8, cols - (c0 + cl)));
    float v[8][8];
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t r = r0 + rl + 16 * k;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = 0.f;
        if (r < rows && n > 0) {
            if (vec && n == 8) load8<true>(W + r * W_stride + c0 + cl, 8, v[k]);
            else load8<false>(W + r * W_stride + c0 + cl, n, v[k]);
        }
        m = max(m, abs_max8(v[k]));
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) amax[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 8; ++w) m = max(m, amax[w]);
    const uint32_t s = scale_byte(m);
    const float inv = inv_scale(s);
    if (threadIdx.x == 0) scale[blockIdx.y * scale_stride + blockIdx.x] = (uint8_t)s;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t r = r0 + rl + 16 * k;
        const uint2 w = to_e4m3x8(v[k], inv);
        if (r < rows && n > 0) {
            uint8_t* to = q + r * q_stride + c0 + cl;
            if (n == 8) *reinterpret_cast<uint2*>(to) = w;
            else
                for (int i = 0; i < n; ++i) to[i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
        }
        if (q_t) {
#pragma unroll
            for (int i = 0; i < 8; ++i) tile[cl + i][rl + 16 * k] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
        }
    }
    if (!q_t) return;
    __syncthreads();
    for (int i = threadIdx.x; i < 128 * 32; i += 256) {
        const int c = i >> 5, w = (i & 31) * 4;
        if (c0 + c >= cols || r0 + w >= rows) continue;
        uint8_t* to = q_t + (c0 + c) * q_t_stride + r0 + w;
        if (r0 + w + 4 <= rows) *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(&tile[c][w]);
        else
            for (int j = 0; r0 + w + j < rows; ++j) to[j] = tile[c][w + j];
    }
}

bool vec_rows(const void* p, int64_t stride, bool bf16) {
    return p == nullptr || (aligned16(p) && (stride & (bf16 ? 7 : 3)) == 0);
}

}  // namespace

// Threads a row and groups of eight a thread: a warp up to 1024 elements, four warps up to 4096, sixteen beyond.
#define ADLOCO_ROW_CASES(LAUNCH)                                                      \
    const int64_t groups = (d + 7) / 8;                                               \
    if (groups <= 32) { LAUNCH(32, 1); }                                              \
    else if (groups <= 64) { LAUNCH(32, 2); }                                         \
    else if (groups <= 96) { LAUNCH(32, 3); }                                         \
    else if (groups <= 128) { LAUNCH(32, 4); }                                        \
    else if (groups <= 256) { LAUNCH(128, 2); }                                       \
    else if (groups <= 384) { LAUNCH(128, 3); }                                       \
    else if (groups <= 512) { LAUNCH(128, 4); }                                       \
    else if (groups <= 1024) { LAUNCH(512, 2); }                                      \
    else { LAUNCH(512, 4); }

template <typename XT, typename ST, bool VEC>
static void add_rmsnorm_sized(const adloco_rmsnorm_args& a, const DropoutKey& key, cudaStream_t st) {
    const int64_t d = a.d;
#define ADLOCO_LAUNCH(TPR, C)                                                                                      \
    add_rmsnorm_kernel<XT, ST, TPR, C, VEC>                                                                        \
        <<<(unsigned)((a.rows + row_threads(TPR) / TPR - 1) / (row_threads(TPR) / TPR)), row_threads(TPR), 0, st>>>(a, key)
    ADLOCO_ROW_CASES(ADLOCO_LAUNCH)
#undef ADLOCO_LAUNCH
}

int launch_add_rmsnorm(adloco_ctx* ctx, const adloco_rmsnorm_args& a, const DropoutKey& key, cudaStream_t st) {
    const bool xb = a.dtype == ADLOCO_BF16, sb = a.stream_dtype == ADLOCO_BF16;
    const bool vec = (a.d & 7) == 0 && vec_rows(a.x, a.x_stride, xb) && vec_rows(a.residual, a.residual_stride, sb) &&
                     vec_rows(a.h, a.h_stride, sb) && vec_rows(a.y, a.y_stride, xb);
#define ADLOCO_TYPES(XT, ST)                                              \
    if (vec) add_rmsnorm_sized<XT, ST, true>(a, key, st);                 \
    else add_rmsnorm_sized<XT, ST, false>(a, key, st)
    if (xb && sb) { ADLOCO_TYPES(__nv_bfloat16, __nv_bfloat16); }
    else if (xb) { ADLOCO_TYPES(__nv_bfloat16, float); }
    else { ADLOCO_TYPES(float, float); }
#undef ADLOCO_TYPES
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    return ADLOCO_OK;
}

// Blocks a sample's rows are cut into: about two blocks an SM over all samples, at least a row for every group of
// threads in a block.
static int64_t rmsnorm_chunks(const adloco_ctx* ctx, int64_t B, int64_t T, int64_t d) {
    const int64_t rows_at_once = d <= 1024 ? 8 : d <= 4096 ? 2 : 1;
    const int64_t most = (T + rows_at_once - 1) / rows_at_once;
    const int64_t want = 2 * (int64_t)ctx->sm_count / B;
    return want < 1 ? 1 : want > most ? most : want;
}
int64_t rmsnorm_backward_workspace(const adloco_ctx* ctx, int64_t B, int64_t T, int64_t d) {
    return B * rmsnorm_chunks(ctx, B, T, d) * d * (int64_t)sizeof(float);
}

template <typename XT, typename ST, bool VEC, bool GAIN>
static void rmsnorm_backward_sized(const RmsBackArgs& p, const DropoutKey& key, cudaStream_t st) {
    const int64_t d = p.a.d;
    const unsigned grid = (unsigned)(p.a.B * p.chunks);
#define ADLOCO_LAUNCH(TPR, C)                                                                                                 \
    rmsnorm_backward_kernel<XT, ST, TPR, C, VEC, GAIN>                                                                        \
        <<<grid, row_threads(TPR), GAIN && row_threads(TPR) > TPR ? (size_t)(row_threads(TPR) / TPR) * d * sizeof(float) : 0, st>>>(p, key)
    ADLOCO_ROW_CASES(ADLOCO_LAUNCH)
#undef ADLOCO_LAUNCH
}

int launch_add_rmsnorm_backward(adloco_ctx* ctx, const adloco_rmsnorm_backward_args& a, const DropoutKey& key, cudaStream_t st) {
    const bool xb = a.dtype == ADLOCO_BF16, sb = a.stream_dtype == ADLOCO_BF16;
    const bool vec = (a.d & 7) == 0 && vec_rows(a.dy, a.dy_stride, xb) && vec_rows(a.h, a.h_stride, sb) &&
                     vec_rows(a.dh_residual, a.dh_residual_stride, sb) && vec_rows(a.dh, a.dh_stride, sb) && vec_rows(a.dx, a.dx_stride, xb);
    const bool gain = a.per_sample_sqnorm || a.grad_sum;
    RmsBackArgs p;
    p.a = a;
    p.chunks = rmsnorm_chunks(ctx, a.B, a.T, a.d);
    p.rows_per_chunk = (a.T + p.chunks - 1) / p.chunks;
#define ADLOCO_TYPES(XT, ST)                                                          \
    if (vec && gain) rmsnorm_backward_sized<XT, ST, true, true>(p, key, st);          \
    else if (vec) rmsnorm_backward_sized<XT, ST, true, false>(p, key, st);            \
    else if (gain) rmsnorm_backward_sized<XT, ST, false, true>(p, key, st);           \
    else rmsnorm_backward_sized<XT, ST, false, false>(p, key, st)
    if (xb && sb) { ADLOCO_TYPES(__nv_bfloat16, __nv_bfloat16); }
    else if (xb) { ADLOCO_TYPES(__nv_bfloat16, float); }
    else { ADLOCO_TYPES(float, float); }
#undef ADLOCO_TYPES
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    if (gain) {
        const int64_t grid = (a.per_sample_sqnorm ? a.B : 0) + (a.grad_sum ? (a.d + 31) / 32 : 0);
        rmsnorm_gain_kernel<<<(unsigned)grid, kGainThreads, 0, st>>>(static_cast<const float*>(a.workspace), a.B, p.chunks, (int)a.d,
                                                                     a.per_sample_sqnorm, a.accumulate_norms, a.grad_sum,
                                                                     a.accumulate_sum);
        ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
        ctx->launches++;
    }
    return ADLOCO_OK;
}

int launch_dropout(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* x, int64_t x_stride, const void* r,
                   int64_t r_stride, void* y, int64_t y_stride, const DropoutKey& key, cudaStream_t st) {
    DropArgs a;
    a.x = x; a.r = r; a.y = y;
    a.rows = rows; a.cols = cols; a.x_stride = x_stride; a.r_stride = r_stride; a.y_stride = y_stride;
    a.groups = (rows * cols + 7) / 8;
    const bool flat = rows == 1 || (x_stride == cols && y_stride == cols && (!r || r_stride == cols));
    bool vec = aligned16(x) && aligned16(y) && aligned16(r);
    if (!flat) vec = vec && (cols & 7) == 0 && vec_rows(x, x_stride, bf16) && vec_rows(y, y_stride, bf16) && vec_rows(r, r_stride, bf16);
    const int64_t want = (a.groups + 255) / 256, most = (int64_t)ctx->sm_count * 64;
    const unsigned grid = (unsigned)(want < most ? want : most);
#define ADLOCO_TYPES(T)                                                                          \
    if (flat && vec) dropout_kernel<T, true, true><<<grid, 256, 0, st>>>(a, key);                \
    else if (flat) dropout_kernel<T, false, true><<<grid, 256, 0, st>>>(a, key);                 \
    else if (vec) dropout_kernel<T, true, false><<<grid, 256, 0, st>>>(a, key);                  \
    else dropout_kernel<T, false, false><<<grid, 256, 0, st>>>(a, key)
    if (bf16) { ADLOCO_TYPES(__nv_bfloat16); }
    else { ADLOCO_TYPES(float); }
#undef ADLOCO_TYPES
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    return ADLOCO_OK;
}

int launch_rope(adloco_ctx* ctx, int bf16, const adloco_rope_tensor* t, int n, int64_t B, int64_t T, int64_t D, int64_t R,
                const uint64_t* turns, float magnitude, const int32_t* pos, int64_t pos_stride, int64_t first, int interleaved,
                int inverse, cudaStream_t st) {
    RopeArgs a;
    memset(&a, 0, sizeof(a));
    a.n = n;
    const int64_t es = bf16 ? 2 : 4;
    bool copies = false;                                 // in place the part that is not rotated is there already
    int64_t P = 16 / es;                                 // pairs a unit: up to 16 bytes on either side of the pairs
    for (int i = 0; i < n; ++i) {
        a.t[i] = t[i];
        if (B == 1) a.t[i].in_batch = a.t[i].out_batch = 0;      // strides of extents of one are not looked at
        if (T == 1) a.t[i].in_token = a.t[i].out_token = 0;
        if (t[i].heads == 1) a.t[i].in_head = a.t[i].out_head = 0;
        a.heads_before[i + 1] = a.heads_before[i] + (int)t[i].heads;
        copies = copies || t[i].in != t[i].out;
    }
    auto fits = [&](int64_t p) {
        if ((R / 2) % p || (copies && (D - R) % p)) return false;
        for (int i = 0; i < n; ++i) {
            if ((reinterpret_cast<uintptr_t>(t[i].in) | reinterpret_cast<uintptr_t>(t[i].out)) % (uintptr_t)(p * es)) return false;
            const adloco_rope_tensor& u = a.t[i];
            if ((u.in_batch | u.in_token | u.in_head | u.out_batch | u.out_token | u.out_head) % p) return false;
        }
        return true;
    };
    while (P > 1 && !fits(P)) P >>= 1;
    a.B = B; a.T = T; a.tokens = B * T;
    a.D = (int)D; a.R = (int)R;
    a.rot_units = (int)(R / 2 / P);
    a.units = a.rot_units + (copies ? (int)((D - R) / P) : 0);
    a.turns = turns; a.positions = pos; a.positions_stride = pos_stride; a.first = first;
    a.magnitude = magnitude; a.inverse = inverse;
    // about four units a thread, as long as every SM has several blocks
    const int64_t per_token = (int64_t)a.heads_before[n] * a.units;
    int64_t tpb = 1024 / per_token;
    const int64_t spread = a.tokens / (4 * (int64_t)ctx->sm_count);
    if (tpb > spread) tpb = spread;
    if (tpb > 16) tpb = 16;
    if (tpb < 1) tpb = 1;
    a.tokens_per_block = (int)tpb;
    const unsigned grid = (unsigned)((a.tokens + tpb - 1) / tpb);
    const size_t smem = (size_t)tpb * (size_t)(R / 2) * sizeof(float2);
    if (smem > 48 * 1024) return ADLOCO_ERR_UNSUPPORTED;
#define ADLOCO_LAUNCH(TY, PP)                                                             \
    if (interleaved) rope_kernel<TY, PP, true><<<grid, 256, smem, st>>>(a);               \
    else rope_kernel<TY, PP, false><<<grid, 256, smem, st>>>(a)
    if (bf16) {
        if (P == 8) { ADLOCO_LAUNCH(__nv_bfloat16, 8); }
        else if (P == 4) { ADLOCO_LAUNCH(__nv_bfloat16, 4); }
        else if (P == 2) { ADLOCO_LAUNCH(__nv_bfloat16, 2); }
        else { ADLOCO_LAUNCH(__nv_bfloat16, 1); }
    } else {
        if (P == 4) { ADLOCO_LAUNCH(float, 4); }
        else if (P == 2) { ADLOCO_LAUNCH(float, 2); }
        else { ADLOCO_LAUNCH(float, 1); }
    }
#undef ADLOCO_LAUNCH
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    return ADLOCO_OK;
}

int launch_blockscale_quantize(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* x, int64_t x_stride, void* q,
                               int64_t q_stride, uint8_t* scale, int64_t scale_stride, cudaStream_t st) {
    const int64_t per_row = (cols + 127) / 128, grid = (rows * per_row + 15) / 16;
    if (grid > 0x7fffffff) return ADLOCO_ERR_UNSUPPORTED;
    const bool vec = vec_rows(x, x_stride, bf16);
#define ADLOCO_LAUNCH(T, V)                                                                                                  \
    quantise_rows_kernel<T, V><<<(unsigned)grid, 256, 0, st>>>(static_cast<const T*>(x), x_stride, static_cast<uint8_t*>(q), \
                                                               q_stride, scale, scale_stride, rows, cols, per_row)
    if (bf16 && vec) ADLOCO_LAUNCH(__nv_bfloat16, true);
    else if (bf16) ADLOCO_LAUNCH(__nv_bfloat16, false);
    else if (vec) ADLOCO_LAUNCH(float, true);
    else ADLOCO_LAUNCH(float, false);
#undef ADLOCO_LAUNCH
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    return ADLOCO_OK;
}

int launch_blockscale_quantize_weight(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* W, int64_t W_stride,
                                      void* q, int64_t q_stride, void* q_t, int64_t q_t_stride, uint8_t* scale,
                                      int64_t scale_stride, cudaStream_t st) {
    const int64_t gx = (cols + 127) / 128, gy = (rows + 127) / 128;
    if (gx > 0x7fffffff || gy > 65535) return ADLOCO_ERR_UNSUPPORTED;
    const int vec = vec_rows(W, W_stride, bf16);
    const dim3 grid((unsigned)gx, (unsigned)gy);
    uint8_t *qb = static_cast<uint8_t*>(q), *qtb = static_cast<uint8_t*>(q_t);
    if (bf16)
        quantise_weight_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(W), W_stride, qb, q_stride, qtb,
                                                                    q_t_stride, scale, scale_stride, rows, cols, vec);
    else
        quantise_weight_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float*>(W), W_stride, qb, q_stride, qtb, q_t_stride,
                                                            scale, scale_stride, rows, cols, vec);
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    return ADLOCO_OK;
}

}  // namespace adloco

// Operators of a decoder block between its linear layers: norm with the residual's addition and
// dropout, its backward pass with the gain's per-sample norms, dropout alone, rotary positions,
// and quantisation to 8 bits with power-of-two scales.  All are bound by HBM: each input is read
// once, each output written once, everything between stays in registers.
#include <algorithm>
#include <cuda_fp8.h>
#include <atomic>

#include "common.cuh"
#include "ptx.cuh"

namespace adloco {

namespace {

// ---- two fp32 operations an instruction ----------------------------------------------------
struct F2 { float x, y; };
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 d;
    asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\n"
        "fma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
    F2 d;
    asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ F2 both(float v) { return F2{v, v}; }

// ---- eight adjacent elements of a row ---------------------------------------------------
// As they lie in memory (four or eight words), so that what waits for use takes half the registers in bf16.  The
// vector form is one 16-byte access (two for float); the guarded form takes rows that do not start on 16-byte
// boundaries and a row's last, incomplete group, and reads what is missing as zero.
template <typename T>
struct Raw { uint32_t w[sizeof(T) * 2]; };

template <bool VEC>
__device__ __forceinline__ Raw<__nv_bfloat16> load_raw(const __nv_bfloat16* p, int n) {
    Raw<__nv_bfloat16> r;
    if (VEC) {
        const uint4 v = __ldcs(reinterpret_cast<const uint4*>(p));
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
    } else {
        const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r.w[i] = (2 * i < n ? (uint32_t)h[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)h[2 * i + 1] << 16 : 0u);
    }
    return r;
}
template <bool VEC>
__device__ __forceinline__ Raw<float> load_raw(const float* p, int n) {
    Raw<float> r;
    if (VEC) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p)), b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
        r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
        r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = i < n ? __float_as_uint(p[i]) : 0u;
    }
    return r;
}
template <typename T>
__device__ __forceinline__ Raw<T> zero_raw() {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * 2); ++i) r.w[i] = 0u;
    return r;
}
// elements 2 i and 2 i + 1
__device__ __forceinline__ F2 pair_of(const Raw<__nv_bfloat16>& r, int i) {
    return F2{__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xffff0000u)};
}
__device__ __forceinline__ F2 pair_of(const Raw<float>& r, int i) {
    return F2{__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1])};
}
__device__ __forceinline__ uint32_t pack2(F2 v) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void set_pair(Raw<__nv_bfloat16>& r, int i, F2 v) { r.w[i] = pack2(v); }
__device__ __forceinline__ void set_pair(Raw<float>& r, int i, F2 v) {
    r.w[2 * i] = __float_as_uint(v.x);
    r.w[2 * i + 1] = __float_as_uint(v.y);
}
template <bool VEC>
__device__ __forceinline__ void store_raw(__nv_bfloat16* p, int n, const Raw<__nv_bfloat16>& r) {
    if (VEC) {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]));
    } else {
        unsigned short* h = reinterpret_cast<unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) h[i] = (unsigned short)(r.w[i >> 1] >> (16 * (i & 1)));
    }
}
template <bool VEC>
__device__ __forceinline__ void store_raw(float* p, int n, const Raw<float>& r) {
    if (VEC) {
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]));
        __stcs(reinterpret_cast<uint4*>(p) + 1, make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = __uint_as_float(r.w[i]);
    }
}
// The gain is read by every row: it stays in L1.  FREE loads may move across the memory clobbers of the copies and stores
// around them, down to the next settled(); others stay in their place.  Kernels on an fp32 stream take the first, whose one or
// two blocks an SM hide little (norm backward of 32768 x 768, bf16 on fp32: 107 us, 126 in their place), those on a bf16
// stream the second, which leave the registers for one block more (98304 x 64: 17.7 us, 20.2 with free ones; 1216 x 5120:
// 32 and 35).
template <bool FREE>
__device__ __forceinline__ uint4 gain16(const void* p) {
    if (!FREE) return *static_cast<const uint4*>(p);
    uint4 v;
    asm("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(__cvta_generic_to_global(p)));
    return v;
}
template <bool FREE>
__device__ __forceinline__ void load_gain(const void* gain, int bf16, int col, int n, F2 (&g)[4]) {
    const __nv_bfloat16* half = static_cast<const __nv_bfloat16*>(gain) + col;
    const float* full = static_cast<const float*>(gain) + col;
    if (n == 8 && (reinterpret_cast<uintptr_t>(gain) & 15u) == 0) {
        if (bf16) {
            const uint4 v = gain16<FREE>(half);
            const Raw<__nv_bfloat16> r = {{v.x, v.y, v.z, v.w}};
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = pair_of(r, i);
        } else {
            const uint4 a = gain16<FREE>(full), b = gain16<FREE>(full + 4);
            const Raw<float> r = {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}};
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = pair_of(r, i);
        }
        return;
    }
    auto one = [&](int i) { return i >= n ? 0.f : bf16 ? __bfloat162float(half[i]) : full[i]; };
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = F2{one(2 * i), one(2 * i + 1)};
}

// ---- Philox-4x32-10 and the mask -----------------------------------------------------------
// Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3" (2011): ten rounds of two
// 32 x 32 -> 64-bit products on a 128-bit counter.  One call serves eight elements, 16 bits each: with
// 32 bits an element the integer work, not HBM, would set the time of dropout on bf16.
__device__ __forceinline__ uint4 philox(uint64_t group, const DropoutKey& k) {
    uint32_t c0 = (uint32_t)group, c1 = (uint32_t)(group >> 32), c2 = k.off_lo, c3 = k.off_hi;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k.round[2 * r];
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k.round[2 * r + 1];
        c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}
// What stays of the eight elements from flat index e on: word i has the answer for elements 2 i and 2 i + 1 in bits
// 15 and 31.  Rows whose length is not a multiple of eight start inside a group (ALIGNED false): their eight
// elements span two groups.
struct Kept { uint32_t w[4]; };
template <bool ALIGNED>
__device__ __forceinline__ Kept kept_of(uint64_t e, const DropoutKey& k) {
    const uint4 w = philox(e >> 3, k);
    uint32_t u[8] = {w.x, w.y, w.z, w.w, 0u, 0u, 0u, 0u};
    const uint32_t sh = ALIGNED ? 0u : (uint32_t)e & 7u;
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
    Kept r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // half >= limit in both halves at once: z's top bits compare the lower 15 bits, the top bits decide where they differ
        const uint32_t z = (u[i] | 0x80008000u) - (k.limit & 0x7fff7fffu);
        r.w[i] = (u[i] & ~k.limit) | ((u[i] | ~k.limit) & z);
    }
    return r;
}
// bytes of v by the selector's nibbles: with a nibble's top bit set, the byte's sign in all its bits; 4..7 give zero
__device__ __forceinline__ uint32_t spread(uint32_t v, uint32_t selector) {
    uint32_t r;
    asm("prmt.b32 %0, %1, 0, %2;" : "=r"(r) : "r"(v), "r"(selector));
    return r;
}
// a dropped element is 0 whatever it held
__device__ __forceinline__ void drop_raw(Raw<__nv_bfloat16>& v, const Kept& m, const DropoutKey& k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v.w[i] &= spread(m.w[i], k.of_pair);
}
__device__ __forceinline__ void drop_raw(Raw<float>& v, const Kept& m, const DropoutKey& k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v.w[2 * i] &= spread(m.w[i], k.of_low);
        v.w[2 * i + 1] &= spread(m.w[i], k.of_high);
    }
}

// r + x scale by two fused operations, the scale's high part first: exactly r where x was dropped, and as good as its inputs
// where the residual cancels the branch, since what is rounded is then small already.  (The low part first would be lost in
// r; r + x scale with a rounded scale loses as much.)  low = 0 is left out: times an Inf it would give NaN.
__device__ __forceinline__ F2 scaled(F2 x, const DropoutKey& k, F2 r) {
    F2 v = fma2(x, both(k.high), r);
    if (k.low != 0.f) v = fma2(x, both(k.low), v);
    return v;
}

// n / d for n < 2^31 by a multiplication: with s = ceil(log2 d) and m = ceil(2^(31 + s) / d), the error of m d is
// below d <= 2^s, and n times it below 2^(31 + s)
struct FastDiv {
    uint32_t d, m, s;
    FastDiv() = default;
    explicit FastDiv(uint32_t div) : d(div), m(0), s(0) {
        while ((uint64_t(1) << s) < div) ++s;
        m = (uint32_t)(((uint64_t(1) << (31 + s)) + div - 1) / div);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> (31 + s)); }
};

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
__device__ __forceinline__ uint32_t abs_max8(const F2 (&v)[4]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max(m, max(__float_as_uint(v[i].x) & 0x7fffffffu, __float_as_uint(v[i].y) & 0x7fffffffu));
    return m;
}
__device__ __forceinline__ uint2 to_e4m3x8(const F2 (&v)[4], float inv) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 u = mul2(v[i], both(inv));
        h[i] = __nv_cvt_float2_to_fp8x2(make_float2(u.x, u.y), __NV_SATFINITE, __NV_E4M3);
    }
    return make_uint2(h[0] | (h[1] << 16), h[2] | (h[3] << 16));
}
// The LANES lanes that hold one block of a row (8 adjacent elements each; fewer than 16 where the row ends) agree on its scale; the lane of the
// block's first elements writes it.  Every lane of the warp takes part; n = 0 for lanes beyond the row.
template <int LANES>
__device__ __forceinline__ void quantise_block(const F2 (&v)[4], int n, uint8_t* q_row, uint8_t* scale_row, int col) {
    uint32_t m = n > 0 ? abs_max8(v) : 0u;          // elements beyond n are zero
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
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
    if (TPR <= 32) {
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        return v;
    }
    v = warp_sum(v);
    constexpr int W = TPR > 32 ? TPR / 32 : 1;
    float* half = smem + (turn & 1) * (THREADS / 32);
    if ((threadIdx.x & 31) == 0) half[threadIdx.x >> 5] = v;
    __syncthreads();
    const float* mine = half + (threadIdx.x / TPR) * W;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) s += mine[i];
    return s;
}

// ---- rows that do not start on 16-byte boundaries ------------------------------------------------
// They pass through shared memory at the alignment they have in global memory (a row's element j at byte skew + j es of its
// buffer, skew = the row's address modulo 16): whole 16-byte pieces go by cp.async, the ends one by one, and a group of eight
// elements is put together from the aligned pieces around it.  (Norm of 6272 x 1001 bf16 out of L2: 18.7 us, its backward pass 45.9;
// with element-wise copies 31 and 78; eight guarded scalar accesses a thread were slower still.)  Rows of fp32 go element by
// element into an aligned buffer instead (skew 0): four bytes a lane are whole cache lines already, and a group written back
// to a skewed buffer would be eight stores that meet in four banks (norm backward of 1665 x 1001 fp32, when it was cut into
// 145 blocks: 22.2 us so, 18.3 us this way).
__host__ __device__ constexpr int pad8(int d) { return (d + 7) / 8 * 8; }
// bytes of a row's buffer: the skew before it, and the piece read beyond its last group
__host__ __device__ constexpr int buffer_bytes(int d, int es) { return (pad8(d) * es + 15) / 16 * 16 + 32; }

// 16 bytes from byte `off` (a multiple of the element size) of a 16-byte aligned buffer; the shift is the same for all of a row
__device__ __forceinline__ uint4 unaligned16(const uint8_t* buf, int off) {
    const uint4* p = reinterpret_cast<const uint4*>(buf + (off & ~15));
    uint4 a = p[0];
    const int sh = off & 15;
    if (sh == 0) return a;
    const uint4 b = p[1];
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (sh & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (sh & 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    if (sh & 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// A row into its buffer, zeros up to a multiple of eight elements; returns the skew.  The ends that are not copied
// asynchronously wait in registers (`ends`) for finish_in, so that a row can be on its way during the one before it.
// Complete after start_in, copies_done (or a wait for its group) and finish_in.
template <int TPR>
__host__ __device__ constexpr int row_ends() { return TPR >= 32 ? 1 : 32 / TPR; }      // up to 7 before, 7 after, 7 zeros
template <int TPR>
__device__ __forceinline__ int start_in(uint8_t* buf, const float* row, int d, int t, float (&)[row_ends<TPR>()]) {
    const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(buf));
#pragma unroll 8
    for (int j = t; j < d; j += TPR) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to + 4u * j), "l"(row + j) : "memory");
    if (t < pad8(d) - d) reinterpret_cast<float*>(buf)[d + t] = 0.f;
    return 0;
}
template <int TPR>
__device__ __forceinline__ void finish_in(uint8_t*, int, int, int, const float (&)[row_ends<TPR>()]) {}
template <int TPR>
__device__ __forceinline__ int start_in(uint8_t* buf, const __nv_bfloat16* row, int d, int t, __nv_bfloat16 (&ends)[row_ends<TPR>()]) {
    const int skew = (int)(reinterpret_cast<uintptr_t>(row) & 15);
    const int head = min(d, ((16 - skew) & 15) / 2), pieces = (d - head) / 8, rest = head + pieces * 8;
    const uint32_t to = static_cast<uint32_t>(__cvta_generic_to_shared(buf)) + skew + head * 2;
    const uint8_t* from = reinterpret_cast<const uint8_t*>(row + head);
#pragma unroll 4
    for (int c = t; c < pieces; c += TPR) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + 16u * c), "l"(from + 16 * (int64_t)c) : "memory");
#pragma unroll
    for (int k = 0; k < row_ends<TPR>(); ++k) {
        const int i = t + k * TPR, j = i < head ? i : rest + i - head;
        ends[k] = j < d ? row[j] : __nv_bfloat16(0.f);
    }
    return skew;
}
template <int TPR>
__device__ __forceinline__ void finish_in(uint8_t* buf, int skew, int d, int t, const __nv_bfloat16 (&ends)[row_ends<TPR>()]) {
    const int head = min(d, ((16 - skew) & 15) / 2), rest = head + (d - head) / 8 * 8;
#pragma unroll
    for (int k = 0; k < row_ends<TPR>(); ++k) {
        const int i = t + k * TPR, j = i < head ? i : rest + i - head;
        if (j < pad8(d)) reinterpret_cast<__nv_bfloat16*>(buf + skew)[j] = ends[k];
    }
}
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <int TPR, typename T>
__device__ __forceinline__ int copy_in(uint8_t* buf, const T* row, int d, int t) {
    T ends[row_ends<TPR>()];
    const int skew = start_in<TPR>(buf, row, d, t, ends);
    finish_in<TPR>(buf, skew, d, t, ends);
    return skew;
}
// A buffer's row (at its skew) to global memory
template <int TPR>
__device__ __forceinline__ void copy_out(float* row, const uint8_t* buf, int, int d, int t) {
    const float* at = reinterpret_cast<const float*>(buf);
#pragma unroll 8
    for (int j = t; j < d; j += TPR) row[j] = at[j];
}
template <int TPR>
__device__ __forceinline__ void copy_out(__nv_bfloat16* row, const uint8_t* buf, int skew, int d, int t) {
    using T = __nv_bfloat16;
    constexpr int ES = (int)sizeof(T), PER = 16 / ES;
    const int head = min(d, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / ES), pieces = (d - head) / PER, rest = head + pieces * PER;
    uint4* to = reinterpret_cast<uint4*>(row + head);
#pragma unroll 4
    for (int c = t; c < pieces; c += TPR) __stcs(to + c, unaligned16(buf, skew + head * ES + 16 * c));
    const T* at = reinterpret_cast<const T*>(buf + skew);
    for (int i = t; i < head + d - rest; i += TPR) {
        const int j = i < head ? i : rest + i - head;
        row[j] = at[j];
    }
}
// the threads of a row (and, where a row is wider than a warp, of all rows of the block)
template <int TPR>
__device__ __forceinline__ void row_barrier() {
    if (TPR <= 32) __syncwarp();
    else __syncthreads();
}
// eight elements from 16-byte aligned shared memory
template <typename T>
__device__ __forceinline__ Raw<T> from_aligned(const T* p) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint4 v = reinterpret_cast<const uint4*>(p)[i];
        r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
    }
    return r;
}
// eight elements of a row's buffer from column col on
template <typename T>
__device__ __forceinline__ Raw<T> from_buffer(const uint8_t* buf, int skew, int col) {
    if constexpr (sizeof(T) == 4) {
        return from_aligned(reinterpret_cast<const T*>(buf) + col);
    } else {
        const uint4 v = unaligned16(buf, skew + col * (int)sizeof(T));
        Raw<T> r;
        r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
        return r;
    }
}
// ... and back to where they were, which no other thread reads
__device__ __forceinline__ void to_buffer(uint8_t* buf, int, int col, const Raw<float>& r) {
    uint4* p = reinterpret_cast<uint4*>(buf + col * 4);
    p[0] = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]);
    p[1] = make_uint4(r.w[4], r.w[5], r.w[6], r.w[7]);
}
__device__ __forceinline__ void to_buffer(uint8_t* buf, int skew, int col, const Raw<__nv_bfloat16>& r) {
    uint8_t* p = buf + skew + col * 2;
    if (skew & 2) {
        *reinterpret_cast<unsigned short*>(p) = (unsigned short)r.w[0];
#pragma unroll
        for (int i = 0; i < 3; ++i) *reinterpret_cast<uint32_t*>(p + 2 + 4 * i) = __funnelshift_r(r.w[i], r.w[i + 1], 16);
        *reinterpret_cast<unsigned short*>(p + 14) = (unsigned short)(r.w[3] >> 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<uint32_t*>(p + 4 * i) = r.w[i];
    }
}
__host__ __device__ constexpr int row_threads(int tpr) { return tpr > 256 ? tpr : 256; }

// ---- norm, forward --------------------------------------------------------------------------
// TPR threads hold a row of up to TPR * C * 8 elements in registers: one read of x and of the residual, the
// mean square in fp32, then every output from the registers.
template <typename XT, typename ST, int TPR, int C, bool VEC>
__global__ void __launch_bounds__(row_threads(TPR)) add_rmsnorm_kernel(const __grid_constant__ adloco_rmsnorm_args a,
                                                                        const __grid_constant__ DropoutKey key) {
    after_predecessor();
    constexpr bool FREE = sizeof(ST) == 4;
    const void* gain = FREE ? settled(a.gain) : a.gain;
    constexpr int THREADS = row_threads(TPR), ROWS = THREADS / TPR;
    extern __shared__ __align__(16) uint8_t row_buffers[];                  // !VEC: x, then the residual, of ROWS rows
    __shared__ float smem[2 * THREADS / 32];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const int64_t row_asked = (int64_t)blockIdx.x * ROWS + sub;
    const bool there = row_asked < a.rows;
    if (TPR <= 32 && __all_sync(0xffffffffu, !there)) return;            // whole warps leave; wider rows meet at a barrier
    const int64_t row = there ? row_asked : a.rows - 1;
    const int d = (int)a.d;
    const XT* x = static_cast<const XT*>(a.x) + row * a.x_stride;
    const ST* r = static_cast<const ST*>(a.residual) + row * a.residual_stride;
    uint8_t* x_buf = row_buffers + sub * buffer_bytes(d, sizeof(XT));
    uint8_t* r_buf = row_buffers + ROWS * buffer_bytes(d, sizeof(XT)) + sub * buffer_bytes(d, sizeof(ST));
    int x_skew = 0, r_skew = 0;
    if (!VEC) {
        x_skew = copy_in<TPR>(x_buf, x, d, t);
        if (a.residual) r_skew = copy_in<TPR>(r_buf, r, d, t);
        copies_done();
        row_barrier<TPR>();
    }
    Raw<XT> xr[C];
    Raw<ST> rr[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8;
        xr[c] = zero_raw<XT>();
        if (col < d) xr[c] = VEC ? load_raw<true>(x + col, 8) : from_buffer<XT>(x_buf, x_skew, col);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8;
        rr[c] = zero_raw<ST>();
        if (a.residual && col < d) rr[c] = VEC ? load_raw<true>(r + col, 8) : from_buffer<ST>(r_buf, r_skew, col);
    }
    if (key.on) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * 8;
            if (col < d) drop_raw(xr[c], kept_of<VEC>((uint64_t)(row * d + col), key), key);
        }
    }
    const float inv_d = 1.0f / (float)d;
    F2 h[C][4], ss = both(0.f);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8;
        Raw<ST> out;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[c][i] = scaled(pair_of(xr[c], i), key, pair_of(rr[c], i));
            ss = fma2(mul2(h[c][i], both(inv_d)), h[c][i], ss);      // the mean: a sum of squares that fit fp32 may not fit
            set_pair(out, i, h[c][i]);
        }
        if (a.h && there && col < d) {
            if (VEC) store_raw<true>(static_cast<ST*>(a.h) + row * a.h_stride + col, 8, out);
            else to_buffer(r_buf, r_skew, col, out);
        }
    }
    const float mean = row_sum<TPR, THREADS>(ss.x + ss.y, smem, 0);
    const float rstd = rsqrtf(mean + a.eps);
    if (a.rstd && there && t == 0) a.rstd[row] = rstd;
    uint8_t* q_row = static_cast<uint8_t*>(a.q) + row * a.q_stride;
    uint8_t* s_row = a.q_scale + row * a.q_scale_stride;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int col = (c * TPR + t) * 8, n = there ? min(8, d - col) : 0;
        F2 g[4];
        Raw<XT> out;
        if (n > 0) {
            load_gain<FREE>(gain, a.gain_dtype == ADLOCO_BF16, col, n, g);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                g[i] = mul2(mul2(h[c][i], both(rstd)), g[i]);
                set_pair(out, i, g[i]);
            }
            if (!VEC && n < 8) {                                     // elements beyond the row: 0, also where rstd is not finite
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (2 * i >= n) g[i].x = 0.f;
                    if (2 * i + 1 >= n) g[i].y = 0.f;
                }
            }
            if (a.y) {
                if (VEC) store_raw<true>(static_cast<XT*>(a.y) + row * a.y_stride + col, 8, out);
                else to_buffer(x_buf, x_skew, col, out);
            }
        }
        if (a.q) quantise_block<(TPR < 16 ? TPR : 16)>(g, n, q_row, s_row, col);
    }
    if (!VEC) {
        row_barrier<TPR>();
        if (a.h && there) copy_out<TPR>(static_cast<ST*>(a.h) + row * a.h_stride, r_buf, r_skew, d, t);
        if (a.y && there) copy_out<TPR>(static_cast<XT*>(a.y) + row * a.y_stride, x_buf, x_skew, d, t);
    }
}

// ---- norm, backward ---------------------------------------------------------------------------
// A block takes `rows_per_chunk` consecutive rows of one sample, ROWS at a time.  With the row in registers the
// two row sums of the formula collapse into one (gain dy . xhat), and the gain's gradient dy xhat is added up in
// registers over the block's rows; blocks leave it in the workspace [B, chunks, d] for rmsnorm_gain_kernel, so
// h and dy are read once for both gradients and no sum depends on the order of atomics.
// A thread's own elements of the next rows travel ahead through shared memory (cp.async, each thread reads only
// what it copied, so no barrier): registers for three operands of one row leave 16 warps an SM, too few loads in
// flight without it.
constexpr size_t kTwoRows = 120 * 1024;          // above what two rows' buffers of a block take off the 16-byte grid
struct RmsBackArgs {
    adloco_rmsnorm_backward_args a;
    int64_t chunks, rows_per_chunk;
    int buffers;                                            // rows in shared memory off the 16-byte grid: one, or one ahead
};
__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
template <typename T>
__device__ __forceinline__ void stage_async(uint32_t dst, uint32_t step, const T* src) {       // step: from one 16-byte piece to the next
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) copy16_async(dst + i * step, reinterpret_cast<const uint4*>(src) + i);
}
template <typename T>
__device__ __forceinline__ Raw<T> staged(uint32_t at, uint32_t step) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint4 v = lds128(at + i * step);
        r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
    }
    return r;
}
// 16-byte pieces a thread stages for one row: dy, h, and the stream's gradient
template <typename XT, typename ST, int C>
__host__ __device__ constexpr int stage_pieces() { return C * ((int)sizeof(XT) / 2 + 2 * ((int)sizeof(ST) / 2)); }
// rows on their way or in use: two (with three blocks an SM at widths up to 768 in bf16; on an fp32 stream one block is left at
// 768, and 32768 x 768 takes 108 us with a bf16 branch, 143 in fp32, against floors of 62 and 77; three rows deep and two blocks
// measured slower), or one -- no staging, loads straight into registers -- where two do not fit
template <typename XT, typename ST, int C, int THREADS>
__host__ __device__ constexpr int stage_depth() {
    const int row = stage_pieces<XT, ST, C>() * 16 * THREADS;
    return 2 * row <= 224 * 1024 ? 2 : 1;
}
template <typename XT, typename ST, int C, int THREADS>
__host__ __device__ constexpr int stage_smem() { return stage_depth<XT, ST, C, THREADS>() < 2 ? 0 : stage_depth<XT, ST, C, THREADS>() * stage_pieces<XT, ST, C>() * 16 * THREADS; }

template <typename XT, typename ST, int TPR, int C, bool VEC, bool GAIN>
__global__ void __launch_bounds__(row_threads(TPR)) rmsnorm_backward_kernel(const __grid_constant__ RmsBackArgs p,
                                                                            const __grid_constant__ DropoutKey key) {
    after_predecessor();
    constexpr int THREADS = row_threads(TPR), ROWS = THREADS / TPR;
    constexpr uint32_t STEP = THREADS * 16;                 // piece i of thread t at i * STEP + 16 t: free of bank conflicts
    constexpr int XP = (int)sizeof(XT) / 2, SP = (int)sizeof(ST) / 2, PIECES = C * (XP + 2 * SP);
    constexpr int DEPTH = stage_depth<XT, ST, C, THREADS>();
    constexpr bool STAGED = VEC && DEPTH > 1, FREE = sizeof(ST) == 4;
    const adloco_rmsnorm_backward_args& a = p.a;
    extern __shared__ __align__(16) float columns[];        // staged rows, or (!VEC) dy, h and the stream's gradient of ROWS rows;
                                                            // at the end [ROWS][d] (GAIN and ROWS > 1)
    __shared__ float smem[2 * THREADS / 32];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR, d = (int)a.d;
    const int64_t sample = (int64_t)blockIdx.x / p.chunks, chunk = (int64_t)blockIdx.x % p.chunks;
    const int64_t first = chunk * p.rows_per_chunk, last = min(a.T, first + p.rows_per_chunk);
    const float inv_d = 1.0f / (float)d;
    const uint32_t mine = static_cast<uint32_t>(__cvta_generic_to_shared(columns)) + threadIdx.x * 16;
    const int wide_x = buffer_bytes(d, sizeof(XT)), wide_s = buffer_bytes(d, sizeof(ST));
    uint8_t* u_buf = reinterpret_cast<uint8_t*>(columns) + sub * wide_x;
    uint8_t* v_buf = reinterpret_cast<uint8_t*>(columns) + ROWS * wide_x + sub * wide_s;
    uint8_t* r_buf = v_buf + ROWS * wide_s;
    const int other = p.buffers > 1 ? ROWS * (wide_x + 2 * wide_s) : 0;     // from a row's buffers to the next row's
    int u_skew = 0, v_skew = 0, r_skew = 0, u_next = 0, v_next = 0, r_next = 0;
    XT u_ends[row_ends<TPR>()] = {};
    ST v_ends[row_ends<TPR>()] = {}, r_ends[row_ends<TPR>()] = {};
    // !VEC: starts the copies of row at + sub into its buffers, one group a call, empty beyond the last row
    auto start = [&](int64_t at, int offset) {
        if (at + sub < last) {
            const int64_t row = sample * a.T + at + sub;
            u_next = start_in<TPR>(u_buf + offset, static_cast<const XT*>(a.dy) + row * a.dy_stride, d, t, u_ends);
            v_next = start_in<TPR>(v_buf + offset, static_cast<const ST*>(a.h) + row * a.h_stride, d, t, v_ends);
            if (a.dh_residual) r_next = start_in<TPR>(r_buf + offset, static_cast<const ST*>(a.dh_residual) + row * a.dh_residual_stride, d, t, r_ends);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (!VEC && other) start(first, 0);
    F2 acc[GAIN ? C : 1][4];
    if (GAIN) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[c][i] = both(0.f);
    }
    // copies of this thread's part of row at + sub into a stage; one group a call, empty beyond the last row
    auto fetch = [&](int64_t at, int stage) {
        if (at + sub < last) {
            const int64_t row = sample * a.T + at + sub;
            const uint32_t to = mine + (uint32_t)(stage * PIECES) * STEP;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * 8;
                if (col >= d) continue;
                stage_async(to + (c * XP) * STEP, STEP, static_cast<const XT*>(a.dy) + row * a.dy_stride + col);
                stage_async(to + (C * XP + c * SP) * STEP, STEP, static_cast<const ST*>(a.h) + row * a.h_stride + col);
                if (a.dh_residual)
                    stage_async(to + (C * XP + C * SP + c * SP) * STEP, STEP,
                                static_cast<const ST*>(a.dh_residual) + row * a.dh_residual_stride + col);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (STAGED) {
#pragma unroll
        for (int k = 0; k < DEPTH - 1; ++k) fetch(first + k * ROWS, k);
    }
    int turn = 0, stage = 0;
    const float* rstds = a.rstd + sample * a.T;
    float rstd_next = rstds[min(first + sub, last - 1)];     // a row ahead of its use
    for (int64_t at = first; at < last; at += ROWS, ++turn) {
        const bool there = at + sub < last;
        if (TPR <= 32 && __all_sync(0xffffffffu, !there)) break;
        const int64_t row = sample * a.T + (there ? at + sub : last - 1);
        const float rstd = rstd_next;
        rstd_next = rstds[min(at + ROWS + sub, last - 1)];
        const XT* dy = static_cast<const XT*>(a.dy) + row * a.dy_stride;
        const ST* h = static_cast<const ST*>(a.h) + row * a.h_stride;
        const ST* res = static_cast<const ST*>(a.dh_residual) + row * a.dh_residual_stride;
        const uint32_t from = mine + (uint32_t)(stage * PIECES) * STEP;
        if (STAGED) {
            // the stage freed by the row before (its values are in registers or stored) takes the next fetch
            fetch(at + (DEPTH - 1) * ROWS, stage == 0 ? DEPTH - 1 : stage - 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
        } else if (!VEC) {
            if (!other) {
                row_barrier<TPR>();                          // the buffers' last rows are stored
                start(at, 0);
            }
            u_skew = u_next; v_skew = v_next; r_skew = r_next;
            if (there) {
                finish_in<TPR>(u_buf, u_skew, d, t, u_ends);
                finish_in<TPR>(v_buf, v_skew, d, t, v_ends);
                if (a.dh_residual) finish_in<TPR>(r_buf, r_skew, d, t, r_ends);
            }
            copies_done();
            row_barrier<TPR>();                              // this row is there, and the row before it stored
            if (other) start(at + ROWS, turn & 1 ? -other : other);
        }
        auto dy_of = [&](int c, int col) {
            return STAGED ? staged<XT>(from + (c * XP) * STEP, STEP) : VEC ? load_raw<true>(dy + col, 8) : from_buffer<XT>(u_buf, u_skew, col);
        };
        auto h_of = [&](int c, int col) {
            return STAGED ? staged<ST>(from + (C * XP + c * SP) * STEP, STEP) : VEC ? load_raw<true>(h + col, 8) : from_buffer<ST>(v_buf, v_skew, col);
        };
        // The row is gone through twice, before and after its sum, from shared memory: holding gain dy and xhat in registers in
        // between left two blocks an SM instead of three.  (Rows too wide for two stages are read from global memory twice.)
        const void* gain = FREE ? settled(a.gain) : a.gain;
        F2 dot = both(0.f);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int col = (c * TPR + t) * 8;
            if (!there || col >= d) continue;
            const Raw<XT> ur = dy_of(c, col);
            const Raw<ST> vr = h_of(c, col);
            F2 g[4];
            load_gain<FREE>(gain, a.gain_dtype == ADLOCO_BF16, col, min(8, d - col), g);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const F2 u = pair_of(ur, i), v = mul2(pair_of(vr, i), both(rstd));      // dy, xhat
                if (GAIN) acc[c][i] = fma2(u, v, acc[c][i]);
                dot = fma2(mul2(u, g[i]), v, dot);
            }
        }
        const float m = row_sum<TPR, THREADS>(dot.x + dot.y, smem, turn) * inv_d;
        const float m_rstd = -m * rstd;
        if (FREE) gain = settled(a.gain);
        if (there) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int col = (c * TPR + t) * 8;
                if (col >= d) continue;
                const Raw<XT> ur = dy_of(c, col);
                const Raw<ST> vr = h_of(c, col);
                Raw<ST> r = zero_raw<ST>(), out;
                if (a.dh_residual)
                    r = STAGED ? staged<ST>(from + (C * XP + C * SP + c * SP) * STEP, STEP) : VEC ? load_raw<true>(res + col, 8) : from_buffer<ST>(r_buf, r_skew, col);
                F2 g[4], o[4];
                load_gain<FREE>(gain, a.gain_dtype == ADLOCO_BF16, col, min(8, d - col), g);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    o[i] = fma2(fma2(pair_of(vr, i), both(m_rstd), mul2(pair_of(ur, i), g[i])), both(rstd), pair_of(r, i));
                    set_pair(out, i, o[i]);
                }
                if (VEC) store_raw<true>(static_cast<ST*>(a.dh) + row * a.dh_stride + col, 8, out);
                else to_buffer(v_buf, v_skew, col, out);
                if (a.dx) {
                    Raw<XT> x;
#pragma unroll
                    for (int i = 0; i < 4; ++i) set_pair(x, i, mul2(o[i], both(key.scale)));
                    if (key.on) drop_raw(x, kept_of<VEC>((uint64_t)(row * d + col), key), key);
                    if (VEC) store_raw<true>(static_cast<XT*>(a.dx) + row * a.dx_stride + col, 8, x);
                    else to_buffer(u_buf, u_skew, col, x);
                }
            }
        }
        if (!VEC) {
            row_barrier<TPR>();
            if (there) copy_out<TPR>(static_cast<ST*>(a.dh) + row * a.dh_stride, v_buf, v_skew, d, t);
            if (there && a.dx) copy_out<TPR>(static_cast<XT*>(a.dx) + row * a.dx_stride, u_buf, u_skew, d, t);
            const int step = turn & 1 ? -other : other;
            u_buf += step; v_buf += step; r_buf += step;
        }
        stage = stage == DEPTH - 1 ? 0 : stage + 1;
    }
    if (!GAIN) return;
    asm volatile("cp.async.wait_all;" ::: "memory");
    float* part = static_cast<float*>(a.workspace) + (int64_t)blockIdx.x * d;
    if (ROWS == 1) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = (c * TPR + t) * 8 + 2 * i;
                if (col < d) part[col] = acc[c][i].x;
                if (col + 1 < d) part[col + 1] = acc[c][i].y;
            }
        return;
    }
    __syncthreads();                                        // every thread is done with its rows
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = (c * TPR + t) * 8 + 2 * i;
            if (col < d) columns[sub * d + col] = acc[c][i].x;
            if (col + 1 < d) columns[sub * d + col + 1] = acc[c][i].y;
        }
    __syncthreads();
    for (int col = threadIdx.x; col < d; col += THREADS) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < ROWS; ++k) s += columns[k * d + col];
        part[col] = s;
    }
}

// Adds up the workspace [B][chunks][d] in a fixed order, two kinds of blocks side by side.  Blocks [0, sums): eight columns
// of the sum over all samples; a warp reads eight columns of four rows at a time.  The others, SPAN for each sample's norm:
// a lane has one column in a quarter of the sample's chunks, a warp every 16 SPANth eight columns.  With few samples, whose
// chunks are many, SPAN is a cluster of eight whose sums of squares meet in the first one's shared memory (one sample of
// 8192 x 768: 47 us with one block, 30 with eight; 64 samples of 256 x 768: 29.7 against 34.2).  Both kinds read the workspace
// once each from L2, with nothing to wait for in between: a chain from columns to squares to norms, by a counter, took 3 us
// more.  Loads leave in groups, short last groups included (an unrolled loop's remainder would go one by one).
constexpr int kGainThreads = 512, kGainCols = 8, kGainCluster = 8;
constexpr int64_t kGainSpread = 131072;          // elements of a sample's chunks from which on its norm takes a cluster
template <int SPAN>
__global__ void __launch_bounds__(kGainThreads) rmsnorm_gain_kernel(const float* part, int64_t B, int64_t chunks, int d, int sums, float* sum,
                                                                    int accumulate_sum, float* norms, int accumulate_norms) {
    constexpr int WARPS = kGainThreads / 32;
    __shared__ float smem[WARPS][kGainCols];
    __shared__ float squares[kGainCluster];
    after_predecessor();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quarter = lane >> 3;
    if ((int)blockIdx.x < sums) {                       // whole clusters
        const int col = (int)blockIdx.x * kGainCols + (lane & 7);
        const int64_t rows = B * chunks;
        float s = 0.f;
        for (int64_t k0 = warp * 4 + quarter; k0 < rows; k0 += WARPS * 4 * 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = k0 + u * WARPS * 4 < rows && col < d ? part[(k0 + u * WARPS * 4) * d + col] : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) s += v[u];
        }
        s += __shfl_xor_sync(0xffffffffu, s, 8);
        s += __shfl_xor_sync(0xffffffffu, s, 16);
        if (lane < kGainCols) smem[warp][lane] = s;
        __syncthreads();
        if (warp == 0 && lane < kGainCols && col < d) {
            s = 0.f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) s += smem[w][lane];
            sum[col] = accumulate_sum ? sum[col] + s : s;
        }
        return;
    }
    if (SPAN > 1) ptx::cluster_started();
    constexpr int COLS = SPAN > 1 ? 1 : 3, ROWS = SPAN > 1 ? 16 : 6;      // loads of a group: of so many eights of columns, and chunks
    constexpr int STEP = SPAN * WARPS * kGainCols;
    const int64_t b = ((int64_t)blockIdx.x - sums) / SPAN;
    const int rank = SPAN > 1 ? (int)ptx::cluster_cta_rank() : 0;
    const float* mine = part + b * chunks * d;
    float q = 0.f;
    for (int c0 = (rank * WARPS + warp) * kGainCols; c0 < d; c0 += COLS * STEP) {
        float g[COLS];
#pragma unroll
        for (int j = 0; j < COLS; ++j) g[j] = 0.f;
        for (int64_t k0 = quarter; k0 < chunks; k0 += 4 * ROWS) {
            float v[ROWS][COLS];
#pragma unroll
            for (int u = 0; u < ROWS; ++u)
#pragma unroll
                for (int j = 0; j < COLS; ++j) {
                    const int col = c0 + j * STEP + (lane & 7);
                    v[u][j] = k0 + 4 * u < chunks && col < d ? mine[(k0 + 4 * u) * d + col] : 0.f;
                }
#pragma unroll
            for (int u = 0; u < ROWS; ++u)
#pragma unroll
                for (int j = 0; j < COLS; ++j) g[j] += v[u][j];
        }
#pragma unroll
        for (int j = 0; j < COLS; ++j) {
            g[j] += __shfl_xor_sync(0xffffffffu, g[j], 8);
            g[j] += __shfl_xor_sync(0xffffffffu, g[j], 16);
            q = fmaf(g[j], g[j], q);
        }
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);       // the four quarters hold the same
    if (lane == 0) smem[warp][0] = q;
    __syncthreads();
    if (SPAN > 1) ptx::cluster_all_started();            // a block without columns comes here before the first one may have started
    if (threadIdx.x == 0) {
        q = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) q += smem[w][0];
        if (SPAN > 1) ptx::st_cluster_u32(ptx::map_to_cta(ptx::smem_u32(&squares[rank]), 0), __float_as_uint(q));
    }
    if (SPAN > 1) ptx::cluster_sync_all();
    if (rank == 0 && threadIdx.x == 0) {
        if (SPAN > 1) {
            q = 0.f;
#pragma unroll
            for (int r = 0; r < kGainCluster; ++r) q += squares[r];
        }
        if (accumulate_norms) atomicAdd(norms + b, q);      // layers on other streams add here too
        else norms[b] = q;
    }
}

// ---- dropout ------------------------------------------------------------------------------------
// A thread takes the eight elements of one call of the generator, two such groups at a time so that enough loads
// are in flight.  The eight are adjacent in memory unless a row ends among them; the vector form needs rows of a
// multiple of eight elements, or no gaps between rows (FLAT), and takes whole groups only.
struct DropArgs {
    const void *x, *r;
    void* y;
    int64_t rows, cols, x_stride, r_stride, y_stride;
    int64_t groups, whole;           // groups, and those of eight elements
    int small;                       // group indices are below 2^31
    FastDiv groups_per_row;          // VEC rows
};
// the elements of a group that has fewer than eight, or that a row's end or the alignment cuts
template <typename T>
__device__ __noinline__ void drop_elements(const DropArgs& a, const DropoutKey& key, int64_t g) {
    const T* x = static_cast<const T*>(a.x);
    const T* r = static_cast<const T*>(a.r);
    T* y = static_cast<T*>(a.y);
    const int64_t e = g * 8;
    const int n = (int)min((int64_t)8, a.rows * a.cols - e);
    int64_t row = e / a.cols, col = e - row * a.cols;
    Raw<float> v = zero_raw<float>(), s = zero_raw<float>();
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        if (q >= n) continue;
        v.w[q] = __float_as_uint((float)x[row * a.x_stride + col]);
        if (r) s.w[q] = __float_as_uint((float)r[row * a.r_stride + col]);
        if (++col == a.cols) { col = 0; ++row; }
    }
    if (key.on) drop_raw(v, kept_of<true>((uint64_t)e, key), key);
    row = e / a.cols;
    col = e - row * a.cols;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 o = scaled(pair_of(v, i), key, pair_of(s, i));
#pragma unroll
        for (int q = 2 * i; q < 2 * i + 2; ++q) {
            if (q >= n) continue;
            y[row * a.y_stride + col] = (T)(q & 1 ? o.y : o.x);
            if (++col == a.cols) { col = 0; ++row; }
        }
    }
}
template <typename T, bool VEC, bool FLAT, bool RES>
__global__ void __launch_bounds__(256) dropout_kernel(const __grid_constant__ DropArgs a, const __grid_constant__ DropoutKey key) {
    constexpr int U = 2;
    after_predecessor();
    const T* x = static_cast<const T*>(a.x);
    const T* r = static_cast<const T*>(a.r);
    T* y = static_cast<T*>(a.y);
    for (int64_t g0 = (int64_t)blockIdx.x * (256 * U) + threadIdx.x; g0 < a.groups; g0 += (int64_t)gridDim.x * (256 * U)) {
        if constexpr (!VEC) {
            drop_elements<T>(a, key, g0);
            if (g0 + 256 < a.groups) drop_elements<T>(a, key, g0 + 256);
            continue;
        } else {
        Raw<T> v[U], s[U];
        int64_t out[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t g = g0 + k * 256;
            if (g >= a.whole) continue;
            int64_t at = g * 8, at_r = at;
            out[k] = at;
            if (!FLAT) {
                const int64_t row = a.small ? (int64_t)a.groups_per_row((uint32_t)g) : g / (int64_t)a.groups_per_row.d;
                const int64_t col = at - row * a.cols;
                at = row * a.x_stride + col;
                at_r = row * a.r_stride + col;
                out[k] = row * a.y_stride + col;
            }
            v[k] = load_raw<true>(x + at, 8);
            if (RES) s[k] = load_raw<true>(r + at_r, 8);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int64_t g = g0 + k * 256;
            if (g >= a.whole) continue;
            if (key.on) drop_raw(v[k], kept_of<true>((uint64_t)g * 8, key), key);
            Raw<T> o;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                set_pair(o, i, RES ? scaled(pair_of(v[k], i), key, pair_of(s[k], i)) : mul2(pair_of(v[k], i), both(key.scale)));
            store_raw<true>(y + out[k], 8, o);
        }
        }
    }
    if (VEC && blockIdx.x == 0 && threadIdx.x == 0 && a.whole < a.groups) drop_elements<T>(a, key, a.whole);
}

// ---- rotary positions -----------------------------------------------------------------------------
// A thread takes one token and one unit of a head -- P pairs to rotate (two pieces of P elements: of either half, or
// adjacent when interleaved), or two pieces of the part that is only copied -- in kRopeHeads heads of one tensor, whose
// loads it issues together before it forms its P sines and cosines, once for all of them.  Neighbouring threads take
// neighbouring units, then heads, then tokens; a grid row takes a tensor, so that its pointers and strides are uniform.
// What costs here is instructions and loads in flight (three heads a thread: 36 us, two at twice the warps: 39 us, six: 34 us): a thread that looked its heads' tensors up and converted element by element needed
// 790 of them for 48 elements and took 69 us for the queries and keys of 32768 tokens of 12 heads of 64 in bf16.
struct RopeArgs {
    adloco_rope_tensor t[4];
    int at_once[4], tokens_per_block[4];       // of a tensor: threads along its heads, tokens of a block
    FastDiv by_heads[4];
    int64_t B, T, tokens;
    int D, R, rot_units, units;                // units a head: rotated, and with the copied rest
    int lanes;                                 // threads along a head's units
    FastDiv by_lanes, by_T;
    const uint64_t* turns;
    const int32_t* positions;
    int64_t positions_stride, first;
    float magnitude;
    int inverse;
};
// P adjacent elements as they lie in memory
template <typename T, int P>
struct alignas(sizeof(T) * P) Piece;
template <int P>
struct alignas(4 * P) Piece<float, P> {
    float v[P];
    __device__ __forceinline__ void get(float* y) const {
#pragma unroll
        for (int p = 0; p < P; ++p) y[p] = v[p];
    }
    __device__ __forceinline__ void set(const float* y) {
#pragma unroll
        for (int p = 0; p < P; ++p) v[p] = y[p];
    }
};
template <int P>
struct alignas(2 * P) Piece<__nv_bfloat16, P> {
    uint32_t w[P / 2];
    __device__ __forceinline__ void get(float* y) const {
#pragma unroll
        for (int i = 0; i < P / 2; ++i) { y[2 * i] = __uint_as_float(w[i] << 16); y[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    __device__ __forceinline__ void set(const float* y) {
#pragma unroll
        for (int i = 0; i < P / 2; ++i) w[i] = pack2(F2{y[2 * i], y[2 * i + 1]});
    }
};
template <>
struct alignas(2) Piece<__nv_bfloat16, 1> {
    __nv_bfloat16 v;
    __device__ __forceinline__ void get(float* y) const { y[0] = __bfloat162float(v); }
    __device__ __forceinline__ void set(const float* y) { v = __float2bfloat16_rn(y[0]); }
};

template <typename T, int P, bool INTERLEAVED>
__device__ __forceinline__ void rotate(Piece<T, P>& x0, Piece<T, P>& x1, const float (&cs)[P], const float (&sn)[P]) {
    float y[2 * P];                                    // pair p: y[2p], y[2p + 1] interleaved, else y[p], y[P + p]
    x0.get(y);
    x1.get(y + P);
    if (P == 1) {
        const float lo = y[0], hi = y[P];
        y[0] = lo * cs[0] - hi * sn[0];
        y[P] = lo * sn[0] + hi * cs[0];
    }
#pragma unroll
    for (int p = 0; p + 1 < P; p += 2) {               // two pairs an instruction
        float &l0 = y[INTERLEAVED ? 2 * p : p], &l1 = y[INTERLEAVED ? 2 * p + 2 : p + 1];
        float &h0 = y[INTERLEAVED ? 2 * p + 1 : P + p], &h1 = y[INTERLEAVED ? 2 * p + 3 : P + p + 1];
        const F2 lo = {l0, l1}, hi = {h0, h1}, c = {cs[p], cs[p + 1]}, s = {sn[p], sn[p + 1]};
        const F2 a = mul2(hi, s), b = fma2(lo, s, mul2(hi, c));
        const F2 d = fma2(lo, c, F2{-a.x, -a.y});
        l0 = d.x; l1 = d.y;
        h0 = b.x; h1 = b.y;
    }
    x0.set(y);
    x1.set(y + P);
}
// Sine and cosine of top 2^-31 half turns.  For fp32 outputs to fp32; for bf16 ones by the fast instructions, whose error of
// 2^-21 is far below the outputs' rounding.
__device__ __forceinline__ void sine_cosine(int32_t top, float& sn, float& cs, float) { sincospif((float)top * 0x1p-31f, &sn, &cs); }
__device__ __forceinline__ void sine_cosine(int32_t top, float& sn, float& cs, __nv_bfloat16) {
    const float angle = (float)top * (3.14159265358979f * 0x1p-31f);      // in [-pi, pi]
    sn = __sinf(angle);
    cs = __cosf(angle);
}

constexpr int kRopeHeads = 6;

template <typename T, int P, bool INTERLEAVED>
__global__ void __launch_bounds__(256, 2) rope_kernel(const __grid_constant__ RopeArgs a) {
    after_predecessor();
    using V = Piece<T, P>;
    const adloco_rope_tensor& t = a.t[blockIdx.y];
    const int heads = (int)t.heads, at_once = a.at_once[blockIdx.y], tokens_per_block = a.tokens_per_block[blockIdx.y];
    const uint32_t slot = a.by_lanes(threadIdx.x), lane = threadIdx.x - slot * a.lanes;
    const uint32_t tok = a.by_heads[blockIdx.y](slot);
    const int head0 = (int)slot - (int)tok * at_once;
    const int64_t token = (int64_t)blockIdx.x * tokens_per_block + tok;
    if ((int)tok >= tokens_per_block || token >= a.tokens) return;
    const uint32_t b = a.by_T((uint32_t)token), s = (uint32_t)token - b * (uint32_t)a.T;
    const int64_t in_step = at_once * t.in_head, out_step = at_once * t.out_head;
    for (int unit = (int)lane; unit < a.units; unit += a.lanes) {
        const bool rotates = unit < a.rot_units;
        // the two pieces; of the copied part the second may lie beyond the head
        const int at = rotates ? (INTERLEAVED ? 2 * unit * P : unit * P) : a.R + (unit - a.rot_units) * 2 * P;
        const int apart = rotates && !INTERLEAVED ? a.R / 2 : P;
        const bool second = at + apart < a.D;
        const T* in = static_cast<const T*>(t.in) + b * t.in_batch + s * t.in_token + head0 * t.in_head + at;
        T* out = static_cast<T*>(t.out) + b * t.out_batch + s * t.out_token + head0 * t.out_head + at;
        float cs[P], sn[P];
        for (int h0 = head0; h0 < heads; h0 += kRopeHeads * at_once) {
            V x0[kRopeHeads], x1[kRopeHeads];
#pragma unroll
            for (int i = 0; i < kRopeHeads; ++i) {
                if (h0 + i * at_once >= heads) continue;
                x0[i] = *reinterpret_cast<const V*>(in + i * in_step);
                if (second) x1[i] = *reinterpret_cast<const V*>(in + i * in_step + apart);
            }
            if (rotates && h0 == head0) {
                const int64_t pos = a.positions ? (int64_t)a.positions[b * a.positions_stride + s] : a.first + (int64_t)s;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    // the phase in units of 2^-64 turns is exact; its top 32 bits, as a signed number, are half turns in [-1, 1)
                    sine_cosine((int32_t)(((uint64_t)pos * a.turns[unit * P + p]) >> 32), sn[p], cs[p], T());
                    cs[p] *= a.magnitude;
                    sn[p] *= a.inverse ? -a.magnitude : a.magnitude;
                }
            }
#pragma unroll
            for (int i = 0; i < kRopeHeads; ++i) {
                if (h0 + i * at_once >= heads) continue;
                if (rotates) rotate<T, P, INTERLEAVED>(x0[i], x1[i], cs, sn);
                *reinterpret_cast<V*>(out + i * out_step) = x0[i];
                if (second) *reinterpret_cast<V*>(out + i * out_step + apart) = x1[i];
            }
            in += kRopeHeads * in_step;
            out += kRopeHeads * out_step;
        }
    }
}

// ---- quantisation -----------------------------------------------------------------------------------
// the largest magnitude's bits of eight elements; bf16 in pairs, as bits of the same number in fp32
__device__ __forceinline__ uint32_t abs_max(const Raw<__nv_bfloat16>& r) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __vmaxu2(m, r.w[i] & 0x7fff7fffu);
    return max(m << 16, m & 0xffff0000u);
}
__device__ __forceinline__ uint32_t abs_max(const Raw<float>& r) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, r.w[i] & 0x7fffffffu);
    return m;
}
template <typename T>
__device__ __forceinline__ uint2 raw_to_e4m3(const Raw<T>& r, float inv) {
    F2 f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pair_of(r, i);
    return to_e4m3x8(f, inv);
}
// Rows: 8 lanes hold a block of 128, 16 adjacent elements each; two blocks one after the other with their loads issued
// together.  (With 8 elements a lane the exchange of the maximum and the scale's arithmetic, which every lane does,
// took more issue slots than the elements: 19.7 us for 32768 x 768 bf16.)
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) quantise_rows_kernel(const T* x, int64_t x_stride, uint8_t* q, int64_t q_stride,
                                                            uint8_t* scale, int64_t scale_stride, uint32_t blocks, int64_t cols,
                                                            const __grid_constant__ FastDiv blocks_per_row) {
    after_predecessor();
    constexpr int U = 2;
    const uint32_t b0 = blockIdx.x * (32 * U) + (threadIdx.x >> 3);
    const int lane_col = (threadIdx.x & 7) * 16;
    Raw<T> v[U][2];
    uint32_t row[U], kb[U];
    int n[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const uint32_t b = b0 + 32 * k;
        const bool there = b < blocks;
        row[k] = there ? blocks_per_row(b) : 0u;
        kb[k] = there ? b - row[k] * blocks_per_row.d : 0u;
        const int64_t col = (int64_t)kb[k] * 128 + lane_col;
        n[k] = there ? (int)min((int64_t)16, cols - col) : 0;
        if (!VEC) continue;
        const T* at = x + row[k] * x_stride + col;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            v[k][j] = zero_raw<T>();
            if (n[k] <= 8 * j) continue;
            if (n[k] >= 8 * j + 8) v[k][j] = load_raw<true>(at + 8 * j, 8);
            else v[k][j] = load_raw<false>(at + 8 * j, n[k] - 8 * j);
        }
    }
    if constexpr (!VEC) {
        // rows off the 16-byte grid: the warp loads its blocks one after the other, 32 adjacent elements an instruction, and hands
        // them out through shared memory
        __shared__ alignas(16) T stage[8][U][4][128];
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t b = blockIdx.x * (32 * U) + 32 * k + warp * 4 + g;
                const bool there = b < blocks;
                const uint32_t br = there ? blocks_per_row(b) : 0u;
                const int64_t c0 = there ? (int64_t)(b - br * blocks_per_row.d) * 128 : cols;
                const T* from = x + br * x_stride + c0;
#pragma unroll
                for (int i = 0; i < 4; ++i) stage[warp][k][g][32 * i + lane] = c0 + 32 * i + lane < cols ? from[32 * i + lane] : T(0.f);
            }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < U; ++k)
#pragma unroll
            for (int j = 0; j < 2; ++j) v[k][j] = from_aligned(&stage[warp][k][(lane >> 3)][lane_col + 8 * j]);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        uint32_t m = max(abs_max(v[k][0]), abs_max(v[k][1]));           // what is missing reads as zero
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (n[k] <= 0) continue;
        const uint32_t s = scale_byte(m);
        const float inv = inv_scale(s);
        const uint2 lo = raw_to_e4m3(v[k][0], inv), hi = raw_to_e4m3(v[k][1], inv);
        uint8_t* to = q + row[k] * q_stride + (int64_t)kb[k] * 128 + lane_col;
        const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
        if (n[k] == 16) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);     // pitch and base are multiples of 16
        else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < n[k]) to[i] = (uint8_t)(w[i >> 2] >> (8 * (i & 3)));
        }
        if (lane_col == 0) scale[row[k] * scale_stride + kb[k]] = (uint8_t)s;
    }
}

// Weights: a block of threads holds a 128 x 128 block (64 elements a thread), agrees on its scale, writes its
// rows and, through shared memory, its columns.
template <typename T>
__global__ void __launch_bounds__(256) quantise_weight_kernel(const T* W, int64_t W_stride, uint8_t* q, int64_t q_stride, uint8_t* q_t,
                                                              int64_t q_t_stride, uint8_t* scale, int64_t scale_stride, int64_t rows,
                                                              int64_t cols, int vec) {
    after_predecessor();
    __shared__ uint32_t amax[8];
    alignas(16) __shared__ uint8_t tile[128][132];                   // [column][row]; 33 words a row: the 16 columns a warp writes, eight apart, meet four on a bank (128 words: all on one)
    const int64_t r0 = (int64_t)blockIdx.y * 128, c0 = (int64_t)blockIdx.x * 128;
    const int cl = (threadIdx.x & 15) * 8, rl = threadIdx.x >> 4;
    const int n = (int)max((int64_t)0, min((int64_t)8, cols - (c0 + cl)));
    Raw<T> raw[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int64_t r = r0 + rl + 16 * k;
        raw[k] = zero_raw<T>();
        if (r < rows && n > 0) {
            if (vec && n == 8) raw[k] = load_raw<true>(W + r * W_stride + c0 + cl, 8);
            else raw[k] = load_raw<false>(W + r * W_stride + c0 + cl, n);
        }
    }
    F2 v[4];
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair_of(raw[k], i);
        m = max(m, abs_max8(v));
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
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair_of(raw[k], i);
        const uint2 w = to_e4m3x8(v, inv);
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

// Threads a row and groups of eight a thread: a quarter of a warp up to 64 elements, a half up to 128, a warp up to 1024, four
// warps up to 4096, sixteen beyond.
#define ADLOCO_ROW_CASES(LAUNCH)                                                      \
    const int64_t groups = (d + 7) / 8;                                               \
    if (groups <= 8) { LAUNCH(8, 1); }                                                \
    else if (groups <= 16) { LAUNCH(16, 1); }                                         \
    else if (groups <= 32) { LAUNCH(32, 1); }                                         \
    else if (groups <= 64) { LAUNCH(32, 2); }                                         \
    else if (groups <= 96) { LAUNCH(32, 3); }                                         \
    else if (groups <= 128) { LAUNCH(32, 4); }                                        \
    else if (groups <= 256) { LAUNCH(128, 2); }                                       \
    else if (groups <= 384) { LAUNCH(128, 3); }                                       \
    else if (groups <= 512) { LAUNCH(128, 4); }                                       \
    else if (groups <= 1024) { LAUNCH(512, 2); }                                      \
    else { LAUNCH(512, 4); }

// more than 48 KB of shared memory a block, static arrays included, has to be asked for, once for each kernel and device
template <typename Kernel>
static int allow_smem(adloco_ctx* ctx, Kernel kernel, size_t most, std::atomic<bool> (&done)[64]) {
    if (done[ctx->device & 63].load()) return ADLOCO_OK;
    ADLOCO_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most));
    done[ctx->device & 63].store(true);
    return ADLOCO_OK;
}

template <typename XT, typename ST, int TPR, int C, bool VEC>
static int add_rmsnorm_launch(adloco_ctx* ctx, const adloco_rmsnorm_args& a, const DropoutKey& key, cudaStream_t st) {
    constexpr int THREADS = row_threads(TPR), ROWS = THREADS / TPR;
    auto kernel = add_rmsnorm_kernel<XT, ST, TPR, C, VEC>;
    const size_t smem = VEC ? 0 : (size_t)ROWS * (buffer_bytes((int)a.d, sizeof(XT)) + buffer_bytes((int)a.d, sizeof(ST)));
    if (smem > 40 * 1024) {
        static std::atomic<bool> done[64];
        const int rc = allow_smem(ctx, kernel, (size_t)ROWS * (buffer_bytes(TPR * C * 8, sizeof(XT)) + buffer_bytes(TPR * C * 8, sizeof(ST))), done);
        if (rc != ADLOCO_OK) return rc;
    }
    ADLOCO_CUDA_TRY(ctx, launch_early(kernel, dim3((unsigned)((a.rows + ROWS - 1) / ROWS)), THREADS, smem, st, 1, a, key));
    return ADLOCO_OK;
}
template <typename XT, typename ST, bool VEC>
static int add_rmsnorm_sized(adloco_ctx* ctx, const adloco_rmsnorm_args& a, const DropoutKey& key, cudaStream_t st) {
    const int64_t d = a.d;
    int rc = ADLOCO_OK;
#define ADLOCO_LAUNCH(TPR, C) rc = add_rmsnorm_launch<XT, ST, TPR, C, VEC>(ctx, a, key, st)
    ADLOCO_ROW_CASES(ADLOCO_LAUNCH)
#undef ADLOCO_LAUNCH
    return rc;
}

int launch_add_rmsnorm(adloco_ctx* ctx, const adloco_rmsnorm_args& a, const DropoutKey& key, cudaStream_t st) {
    const bool xb = a.dtype == ADLOCO_BF16, sb = a.stream_dtype == ADLOCO_BF16;
    const bool vec = (a.d & 7) == 0 && vec_rows(a.x, a.x_stride, xb) && vec_rows(a.residual, a.residual_stride, sb) &&
                     vec_rows(a.h, a.h_stride, sb) && vec_rows(a.y, a.y_stride, xb);
    int rc = ADLOCO_OK;
#define ADLOCO_TYPES(XT, ST)                                              \
    if (vec) rc = add_rmsnorm_sized<XT, ST, true>(ctx, a, key, st);       \
    else rc = add_rmsnorm_sized<XT, ST, false>(ctx, a, key, st)
    if (xb && sb) { ADLOCO_TYPES(__nv_bfloat16, __nv_bfloat16); }
    else if (xb) { ADLOCO_TYPES(__nv_bfloat16, float); }
    else { ADLOCO_TYPES(float, float); }
#undef ADLOCO_TYPES
    if (rc != ADLOCO_OK) return rc;
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    return ADLOCO_OK;
}

// Blocks a sample's rows are cut into: about as many over all samples as are resident at once, counted in whole turns of a row
// for every group of a block's threads (4 samples of 1024 x 300 bf16 by ten rows a block, eight and two: 24.4 us; by
// sixteen: 15.7).  The rows are then spread evenly over the blocks, which gives none of them more turns.  Blocks an SM by
// width: of 2, 3, 4 and 6 these measured best at 256, 768, 1024, 2048, 3000 and 4096 in bf16, where registers set them; five
// for narrow rows off the 16-byte grid.  `fit` is what shared memory allows beside that, and what decides on the grid from 257
// on where the stream is fp32; off the grid the registers of 512 threads leave one block, however little memory it takes
// (counted as two, 64 samples of 12 x 8191 bf16 took 100 us instead of 72).
static int64_t rmsnorm_blocks(int64_t d, bool vec) {
    return d <= 256 ? (vec ? 4 : 5) : d <= 768 ? 3 : d <= 1024 ? 2 : d <= 2048 ? 4 : d <= 3072 ? 3 : 2;
}
static int64_t rows_of_block(int64_t d) { return d <= 64 ? 32 : d <= 128 ? 16 : d <= 1024 ? 8 : d <= 4096 ? 2 : 1; }
static int64_t rmsnorm_chunks(const adloco_ctx* ctx, int64_t B, int64_t T, int64_t d, bool vec, int64_t fit) {
    const int64_t rows_at_once = rows_of_block(d);
    int64_t blocks = rmsnorm_blocks(d, vec);
    if (blocks > fit) blocks = fit < 1 ? 1 : fit;
    const int64_t want = blocks * (int64_t)ctx->sm_count / B;
    if (want <= 1 || T <= rows_at_once) return 1;
    const int64_t rows = ((T + want - 1) / want + rows_at_once - 1) / rows_at_once * rows_at_once;
    return (T + rows - 1) / rows;
}
int64_t rmsnorm_backward_workspace(const adloco_ctx* ctx, int64_t B, int64_t T, int64_t d) {
    const int64_t one = rmsnorm_chunks(ctx, B, T, d, true, 8), other = rmsnorm_chunks(ctx, B, T, d, false, 8);
    return B * (one > other ? one : other) * d * (int64_t)sizeof(float);
}

template <typename XT, typename ST, int TPR, int C, bool VEC, bool GAIN>
static int rmsnorm_backward_launch(adloco_ctx* ctx, const RmsBackArgs& p, const DropoutKey& key, unsigned grid, cudaStream_t st) {
    constexpr int THREADS = row_threads(TPR), ROWS = THREADS / TPR;
    auto kernel = rmsnorm_backward_kernel<XT, ST, TPR, C, VEC, GAIN>;
    auto buffers = [](int d) { return (size_t)ROWS * (buffer_bytes(d, sizeof(XT)) + 2 * buffer_bytes(d, sizeof(ST))); };
    size_t smem = VEC ? stage_smem<XT, ST, C, THREADS>() : p.buffers * buffers((int)p.a.d);
    if (GAIN && ROWS > 1 && smem < (size_t)ROWS * p.a.d * sizeof(float)) smem = (size_t)ROWS * p.a.d * sizeof(float);
    if (smem > 40 * 1024) {
        static std::atomic<bool> done[64];
        const int rc = allow_smem(ctx, kernel, VEC ? stage_smem<XT, ST, C, THREADS>() : std::max(buffers(TPR * C * 8), std::min(2 * buffers(TPR * C * 8), kTwoRows)), done);
        if (rc != ADLOCO_OK) return rc;
    }
    ADLOCO_CUDA_TRY(ctx, launch_early(kernel, dim3(grid), THREADS, smem, st, 1, p, key));
    return ADLOCO_OK;
}

template <typename XT, typename ST, bool VEC, bool GAIN>
static int rmsnorm_backward_sized(adloco_ctx* ctx, const RmsBackArgs& p, const DropoutKey& key, cudaStream_t st) {
    const int64_t d = p.a.d;
    const unsigned grid = (unsigned)(p.a.B * p.chunks);
#define ADLOCO_LAUNCH(TPR, C) rc = rmsnorm_backward_launch<XT, ST, TPR, C, VEC, GAIN>(ctx, p, key, grid, st)
    int rc = ADLOCO_OK;
    ADLOCO_ROW_CASES(ADLOCO_LAUNCH)
#undef ADLOCO_LAUNCH
    return rc;
}

int launch_add_rmsnorm_backward(adloco_ctx* ctx, const adloco_rmsnorm_backward_args& a, const DropoutKey& key, cudaStream_t st) {
    const bool xb = a.dtype == ADLOCO_BF16, sb = a.stream_dtype == ADLOCO_BF16;
    const bool vec = (a.d & 7) == 0 && vec_rows(a.dy, a.dy_stride, xb) && vec_rows(a.h, a.h_stride, sb) &&
                     vec_rows(a.dh_residual, a.dh_residual_stride, sb) && vec_rows(a.dh, a.dh_stride, sb) && vec_rows(a.dx, a.dx_stride, xb);
    const bool gain = a.per_sample_sqnorm || a.grad_sum;
    RmsBackArgs p;
    p.a = a;
    const int64_t row_bytes = (xb ? 2 : 4) + 2 * (sb ? 2 : 4), threads = a.d > 4096 ? 512 : 256;
    const int64_t groups = a.d <= 1024 ? (a.d + 255) / 256 : a.d <= 4096 ? (a.d + 1023) / 1024 : (a.d + 4095) / 4096;     // of eight a thread
    const int64_t one = vec ? threads * groups * 8 * row_bytes
                            : rows_of_block(a.d) * (buffer_bytes((int)a.d, xb ? 2 : 4) + 2 * buffer_bytes((int)a.d, sb ? 2 : 4));
    constexpr int64_t most = 227 * 1024, beside = 1024 + 128;      // of an SM; what a block takes beside its rows
    // a row ahead where it takes no block from an SM
    p.buffers = !vec && (2 * one + beside) * rmsnorm_blocks(a.d, vec) <= most ? 2 : 1;
    const int64_t smem = (vec ? 2 : p.buffers) * one;
    p.chunks = rmsnorm_chunks(ctx, a.B, a.T, a.d, vec, !vec && threads > 256 ? 1 : most / (smem + beside));
    p.rows_per_chunk = (a.T + p.chunks - 1) / p.chunks;
    int rc = ADLOCO_OK;
#define ADLOCO_TYPES(XT, ST)                                                               \
    if (vec && gain) rc = rmsnorm_backward_sized<XT, ST, true, true>(ctx, p, key, st);     \
    else if (vec) rc = rmsnorm_backward_sized<XT, ST, true, false>(ctx, p, key, st);       \
    else if (gain) rc = rmsnorm_backward_sized<XT, ST, false, true>(ctx, p, key, st);      \
    else rc = rmsnorm_backward_sized<XT, ST, false, false>(ctx, p, key, st)
    if (xb && sb) { ADLOCO_TYPES(__nv_bfloat16, __nv_bfloat16); }
    else if (xb) { ADLOCO_TYPES(__nv_bfloat16, float); }
    else { ADLOCO_TYPES(float, float); }
#undef ADLOCO_TYPES
    if (rc != ADLOCO_OK) return rc;
    ADLOCO_CUDA_TRY(ctx, cudaGetLastError());
    ctx->launches++;
    if (gain) {
        const bool spread = a.per_sample_sqnorm && p.chunks * a.d > kGainSpread;
        const int64_t span = spread ? kGainCluster : 1, cols = kGainCols * span;     // the sum's blocks in whole clusters
        const int sums = a.grad_sum ? (int)((a.d + cols - 1) / cols * span) : 0;
        const dim3 blocks((unsigned)(sums + (a.per_sample_sqnorm ? a.B * span : 0)));
        ADLOCO_CUDA_TRY(ctx, launch_early(spread ? rmsnorm_gain_kernel<kGainCluster> : rmsnorm_gain_kernel<1>, blocks, kGainThreads, 0, st,
                                          (unsigned)span, static_cast<const float*>(a.workspace), a.B, p.chunks, (int)a.d, sums, a.grad_sum,
                                          (int)a.accumulate_sum, a.per_sample_sqnorm, (int)a.accumulate_norms));
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
    a.whole = rows * cols / 8;
    const bool flat = rows == 1 || (x_stride == cols && y_stride == cols && (!r || r_stride == cols));
    bool vec = aligned16(x) && aligned16(y) && aligned16(r);
    if (!flat) vec = vec && (cols & 7) == 0 && cols < 0x7fffffff && vec_rows(x, x_stride, bf16) && vec_rows(y, y_stride, bf16) && vec_rows(r, r_stride, bf16);
    a.small = a.groups <= 0x7fffffff;
    a.groups_per_row = FastDiv((uint32_t)(cols < 0x7fffffff ? (cols + 7) / 8 : 1));
    const int64_t want = (a.groups + 511) / 512, most = (int64_t)ctx->sm_count * 64;
    const unsigned grid = (unsigned)(want < most ? want : most);
    cudaError_t e = cudaSuccess;
#define ADLOCO_LAUNCH(T, V, F, R) e = launch_early(dropout_kernel<T, V, F, R>, dim3(grid), 256, 0, st, 1, a, key)
#define ADLOCO_TYPES(T)                                                       \
    if (!vec) ADLOCO_LAUNCH(T, false, false, false);                          \
    else if (flat && r) ADLOCO_LAUNCH(T, true, true, true);                   \
    else if (flat) ADLOCO_LAUNCH(T, true, true, false);                       \
    else if (r) ADLOCO_LAUNCH(T, true, false, true);                          \
    else ADLOCO_LAUNCH(T, true, false, false)
    if (bf16) { ADLOCO_TYPES(__nv_bfloat16); }
    else { ADLOCO_TYPES(float); }
#undef ADLOCO_LAUNCH
#undef ADLOCO_TYPES
    ADLOCO_CUDA_TRY(ctx, e);
    ctx->launches++;
    return ADLOCO_OK;
}

int launch_rope(adloco_ctx* ctx, int bf16, const adloco_rope_tensor* t, int n, int64_t B, int64_t T, int64_t D, int64_t R,
                const uint64_t* turns, float magnitude, const int32_t* pos, int64_t pos_stride, int64_t first, int interleaved,
                int inverse, cudaStream_t st) {
    RopeArgs a;
    memset(&a, 0, sizeof(a));
    const int64_t es = bf16 ? 2 : 4;
    bool copies = false;                                 // in place the part that is not rotated is there already
    int64_t P = 16 / es;                                 // pairs a unit: up to 16 bytes on either side of the pairs
    for (int i = 0; i < n; ++i) {
        a.t[i] = t[i];
        if (B == 1) a.t[i].in_batch = a.t[i].out_batch = 0;      // strides of extents of one are not looked at
        if (T == 1) a.t[i].in_token = a.t[i].out_token = 0;
        if (t[i].heads == 1) a.t[i].in_head = a.t[i].out_head = 0;
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
    a.units = a.rot_units + (copies ? (int)((D - R + 2 * P - 1) / (2 * P)) : 0);
    a.turns = turns; a.positions = pos; a.positions_stride = pos_stride; a.first = first;
    a.magnitude = magnitude; a.inverse = inverse;
    // a block's 256 threads: the units of a head, so many heads of the tensor that a thread comes to kRopeHeads of them, and
    // tokens with what is left; where that gives an SM fewer than four blocks, more threads along the heads
    a.lanes = a.units < 256 ? a.units : 256;
    a.by_lanes = FastDiv((uint32_t)a.lanes);
    a.by_T = FastDiv((uint32_t)T);
    const int64_t slots = 256 / a.lanes;
    int64_t blocks = 0;
    for (int i = 0; i < n; ++i) {
        int64_t at_once = (t[i].heads + kRopeHeads - 1) / kRopeHeads;
        while (at_once < t[i].heads && a.tokens * at_once < slots * 4 * ctx->sm_count) ++at_once;
        if (at_once > slots) at_once = slots;
        a.at_once[i] = (int)at_once;
        a.tokens_per_block[i] = (int)(slots / at_once);
        a.by_heads[i] = FastDiv((uint32_t)at_once);
        const int64_t need = (a.tokens + a.tokens_per_block[i] - 1) / a.tokens_per_block[i];
        if (need > blocks) blocks = need;
    }
    const dim3 grid((unsigned)blocks, (unsigned)n);
    cudaError_t e = cudaSuccess;
#define ADLOCO_LAUNCH(TY, PP)                                                             \
    if (interleaved) e = launch_early(rope_kernel<TY, PP, true>, grid, 256, 0, st, 1, a);               \
    else e = launch_early(rope_kernel<TY, PP, false>, grid, 256, 0, st, 1, a)
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
    ADLOCO_CUDA_TRY(ctx, e);
    ctx->launches++;
    return ADLOCO_OK;
}

int launch_blockscale_quantize(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* x, int64_t x_stride, void* q,
                               int64_t q_stride, uint8_t* scale, int64_t scale_stride, cudaStream_t st) {
    const int64_t per_row = (cols + 127) / 128;
    if (rows > 0x7fffffff / per_row) return ADLOCO_ERR_UNSUPPORTED;
    const uint32_t blocks = (uint32_t)(rows * per_row), grid = (blocks + 63) / 64;
    const bool vec = vec_rows(x, x_stride, bf16);
    cudaError_t e = cudaSuccess;
#define ADLOCO_LAUNCH(T, V)                                                                                                      \
    e = launch_early(quantise_rows_kernel<T, V>, dim3(grid), 256, 0, st, 1, static_cast<const T*>(x), x_stride, static_cast<uint8_t*>(q), \
                     q_stride, scale, scale_stride, blocks, cols, FastDiv((uint32_t)per_row))
    if (bf16 && vec) ADLOCO_LAUNCH(__nv_bfloat16, true);
    else if (bf16) ADLOCO_LAUNCH(__nv_bfloat16, false);
    else if (vec) ADLOCO_LAUNCH(float, true);
    else ADLOCO_LAUNCH(float, false);
#undef ADLOCO_LAUNCH
    ADLOCO_CUDA_TRY(ctx, e);
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
    cudaError_t e;
    if (bf16)
        e = launch_early(quantise_weight_kernel<__nv_bfloat16>, grid, 256, 0, st, 1, static_cast<const __nv_bfloat16*>(W), W_stride, qb,
                         q_stride, qtb, q_t_stride, scale, scale_stride, rows, cols, vec);
    else
        e = launch_early(quantise_weight_kernel<float>, grid, 256, 0, st, 1, static_cast<const float*>(W), W_stride, qb, q_stride, qtb,
                         q_t_stride, scale, scale_stride, rows, cols, vec);
    ADLOCO_CUDA_TRY(ctx, e);
    ctx->launches++;
    return ADLOCO_OK;
}

}  // namespace adloco

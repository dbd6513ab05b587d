// The loss of a decoder and the way back from 8 bits: log-probabilities of given tokens with entropy and the best
// alternatives, their gradient, and the values that rows in 8 bits stand for.  All are bound by HBM.
#include <atomic>
#include <cuda_fp8.h>

#include "common.cuh"
#include "e4m3.cuh"
#include "f32x2.cuh"
#include "ptx.cuh"

namespace adloco {

using namespace ptx;

namespace {

constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// ---- 16 bytes of a row as numbers -----------------------------------------------------------
template <typename T> struct Piece { static constexpr int N = 16 / sizeof(T); };
__device__ __forceinline__ float number(const float* p) { return *p; }
__device__ __forceinline__ float number(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void unpack(const uint4& w, float (&v)[4]) {
    v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ void unpack(const uint4& w, float (&v)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(u[i] << 16);
        v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 repack(const float (&v)[4]) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 repack(const float (&v)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// A run of n numbers that starts anywhere: `head` of them before the first 16-byte boundary, `body` whole pieces of 16
// bytes, `tail` behind.
template <typename T>
struct Run {
    const T* p;
    int head, body, tail;
    __device__ __forceinline__ Run(const T* at, int n) : p(at) {
        const int skew = (int)((reinterpret_cast<uintptr_t>(at) & 15u) / sizeof(T));
        head = skew ? min(n, Piece<T>::N - skew) : 0;
        body = (n - head) / Piece<T>::N;
        tail = n - head - body * Piece<T>::N;
    }
    __device__ __forceinline__ const uint4* pieces() const { return reinterpret_cast<const uint4*>(p + head); }
    __device__ __forceinline__ int index(int piece) const { return head + piece * Piece<T>::N; }
};

// ---- log-probabilities -----------------------------------------------------------------------
// One pass with the running maximum m and the sums S = sum e^(l - m), E = sum (l - m) e^(l - m) of each thread's share:
//   lse = m + log S,   entropy = log S - E / S.
// A row is shared by TPR threads (a warp, or a block), a long row of few by the blocks of a cluster.  m starts at the
// lowest finite number, so that l - m is a number for every finite l, and -Inf gives the 0 that it should.  Shares are
// brought to the row's maximum once and then only added (joined two by two, each pair with its own maximum, they cost
// half as much as the pass itself).
//
// The best tokens: the top-th largest of the maxima of G groups of threads is a lower bound of the top-th largest
// logit.  Only the few threads whose own maximum reaches it have anything that counts: the row's threads look at those
// threads' shares once more together, collect what reaches the bound, and sort that by counting.  Where too much
// reaches it (long runs of equal logits), they take the best one by one instead, a pass over the row for each.
constexpr int kMaxTop = 64;
constexpr int kTopThreads = 256, kClusterThreads = 512;
constexpr int kCluster = 8;
// 64 registers a thread: more blocks with fewer spill (8192 x 50257 bf16: 170 us, with 5 and 6 blocks an SM 235 and 312)
template <int TPR, bool CLUSTER> constexpr int kBlocks = TPR == 32 ? 8 : CLUSTER ? 2 : 4;
template <int TPR> __host__ __device__ constexpr int groups_of() { return TPR < 128 ? TPR : 128; }
constexpr int kCandidates = 512;                                // of a row
static_assert(kCluster * kMaxTop <= kCandidates, "what a cluster's blocks bring");

// a number's place among numbers as an unsigned one, NaN lowest, -0 as 0; then the lower index first
__device__ __forceinline__ uint32_t place_of(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);
    return v != v ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float number_at(uint32_t place) {
    return place == 0u ? __uint_as_float(0x7fffffffu) : __uint_as_float((place & 0x80000000u) ? place & 0x7fffffffu : ~place);
}
__device__ __forceinline__ uint64_t key_of(float v, int index) { return ((uint64_t)place_of(v) << 32) | (uint32_t)~index; }
__device__ __forceinline__ float value_of(uint64_t key) { return number_at((uint32_t)(key >> 32)); }

struct Sums { float m, s, e; };
// sums to a maximum m that is no smaller.  A share without numbers has s = 0; the distance may be beyond all bounds.
__device__ __forceinline__ Sums brought_to(const Sums& a, float m) {
    const float d = a.m - m, f = exp2_fast(d * kLog2e);
    return Sums{m, a.s * f, f == 0.f && a.s == a.s ? 0.f : fmaf(d, a.s, a.e) * f};
}

template <int TPR>
struct RowShared {
    float m[TPR / 32], s[TPR / 32], e[TPR / 32];
    Sums sums;
    alignas(16) uint32_t group_max[groups_of<TPR>()];
    uint32_t bound;
    int hot, found;
    unsigned short hot_thread[TPR];
    uint64_t best[kMaxTop];
    uint64_t wave[TPR / 32];
    uint64_t candidate[kCandidates];
};

struct LogprobArgs {
    int64_t rows, stride;
    int V, top;
    const void* logits;
    const int32_t* targets;
    float *logp, *entropy, *lse, *top_values;
    int32_t* top_ids;
};

template <bool V> struct Is { static constexpr bool value = V; };
template <int TPR>
__device__ __forceinline__ void row_sync() {
    if (TPR == 32) __syncwarp();
    else __syncthreads();
}

// The extremes of U pieces.  A NaN counts as neither; bf16 takes two numbers an instruction.
template <int U>
__device__ __forceinline__ void extremes(const uint4 (&w)[U], float& low, float& high, float) {
    high = -INFINITY;
    low = -INFINITY;                                            // not looked for: as dear as what knowing it saves
#pragma unroll
    for (int u = 0; u < U; ++u)
        high = fmaxf(high, fmaxf(fmaxf(__uint_as_float(w[u].x), __uint_as_float(w[u].y)), fmaxf(__uint_as_float(w[u].z), __uint_as_float(w[u].w))));
}
template <int U>
__device__ __forceinline__ void extremes(const uint4 (&w)[U], float& low, float& high, __nv_bfloat16) {
    const __nv_bfloat162* v = reinterpret_cast<const __nv_bfloat162*>(&w[0]);
    __nv_bfloat162 h = v[0], l = v[0];
#pragma unroll
    for (int i = 1; i < 4 * U; ++i) { h = __hmax2(h, v[i]); l = __hmin2(l, v[i]); }
    high = fmaxf(__low2float(h), __high2float(h));
    low = fminf(__low2float(l), __high2float(l));
}
template <typename T, bool ENTROPY, int U>
__device__ __forceinline__ void add_pieces(const uint4 (&w)[U], Sums& a, float& top) {
    constexpr int N = Piece<T>::N;
    float low, m;
    extremes(w, low, m, T());
    top = fmaxf(top, m);
    if (m > a.m) a = brought_to(a, m);
    const F2 minus = both(-a.m);
    F2 s = both(0.f), e = both(0.f);
    auto add = [&](auto some_infinite) {                        // a logit of -Inf adds 0, which its distance would make a NaN of
        constexpr bool CLAMP = decltype(some_infinite)::value;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[N];
            unpack(w[u], v);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const F2 d = add2(F2{v[i], v[i + 1]}, minus), x = exp2_fast(mul2(d, both(kLog2e)));
                s = add2(s, x);
                if (ENTROPY) e = fma2(x, CLAMP ? F2{max_or_nan(d.x, -1e4f), max_or_nan(d.y, -1e4f)} : d, e);
            }
        }
    };
    // (of the distances to the running maximum, which may be far above these pieces' own)
    if (sizeof(T) == 2 && ENTROPY && low > -INFINITY && a.m - low < 1e30f) add(Is<false>{});
    else add(Is<true>{});
    a.s += s.x + s.y;
    if (ENTROPY) a.e += e.x + e.y;
}
__device__ __forceinline__ void add_two(float u, float v, Sums& a, float& top) {      // -Inf adds nothing
    top = fmaxf(top, fmaxf(u, v));
    a = brought_to(a, fmaxf(a.m, fmaxf(u, v)));
    const F2 d = {u - a.m, v - a.m}, x = exp2_fast(mul2(d, both(kLog2e)));
    a.s += x.x + x.y;
    a.e += fmaf(x.x, max_or_nan(d.x, -1e4f), x.y * max_or_nan(d.y, -1e4f));
}

// The largest `top` keys of a run of n numbers whose first has index `base`, in order, into sh.best; all threads of the row.
template <typename T, int TPR>
__device__ __noinline__ void best_one_by_one(RowShared<TPR>& sh, const T* p, int n, int base, int top) {
    const int t = threadIdx.x & (TPR - 1), lane = t & 31;
    uint64_t last = ~0ull;
    for (int k = 0; k < top; ++k) {
        uint64_t most = 0;
        for (int i = t; i < n; i += TPR) {
            const uint64_t key = key_of(number(p + i), base + i);
            if (key < last && key > most) most = key;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) { const uint64_t other = __shfl_xor_sync(0xffffffffu, most, o); most = other > most ? other : most; }
        if (lane == 0) sh.wave[t >> 5] = most;
        row_sync<TPR>();
        most = 0;
        for (int i = 0; i < TPR / 32; ++i) most = sh.wave[i] > most ? sh.wave[i] : most;
        row_sync<TPR>();
        if (t == 0) sh.best[k] = most;
        last = most;
        if (most == 0) {                                        // fewer numbers than asked for
            for (int i = k + t; i < top; i += TPR) sh.best[i] = 0;
            break;
        }
    }
    row_sync<TPR>();
}

template <typename T, int TPR, bool CLUSTER, bool ENTROPY>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, kBlocks<TPR, CLUSTER>) logprob_kernel(const __grid_constant__ LogprobArgs a) {
    constexpr int ROWS = TPR < 128 ? 128 / TPR : 1;             // of a block
    constexpr int U = TPR > 32 && sizeof(T) == 4 ? 8 : 4, N = Piece<T>::N;      // pieces a thread has on their way
    constexpr bool PRE = TPR > 32 && sizeof(T) == 2;            // the next U while U are added up: where these take the longer time
    __shared__ RowShared<TPR> shared_rows[ROWS];
    RowShared<TPR>& sh = shared_rows[threadIdx.x / TPR];
    const int t = threadIdx.x & (TPR - 1), lane = t & 31;
    const uint32_t rank = CLUSTER ? cluster_cta_rank() : 0;
    if (CLUSTER) cluster_started();
    after_predecessor();
    const int64_t row = CLUSTER ? blockIdx.x / kCluster : (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (!CLUSTER && row >= a.rows) return;                      // whole warps
    // this block's part of the row
    const int part = CLUSTER ? ((a.V + kCluster - 1) / kCluster + 7) / 8 * 8 : a.V;
    const int from = min(a.V, (int)rank * part), n = min(a.V - from, part);
    const T* p = static_cast<const T*>(a.logits) + row * a.stride;
    const Run<T> run(p + from, n);
    const int32_t target = a.logp && t == 0 && rank == 0 ? a.targets[row] : -1;
    const bool given = target >= 0 && target < a.V;
    const float at_target = given ? number(p + target) : 0.f;
    Sums sums = {-3.402823466e38f, 0.f, 0.f};
    float own_max = -INFINITY;
    {
        // the ends of the row come first and are added last
        const float first = t < run.head ? number(run.p + t) : -INFINITY, last = t < run.tail ? number(run.p + n - run.tail + t) : -INFINITY;
        const uint4* pieces = run.pieces();
        uint4 next[U];
        auto load = [&](int i) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * TPR < run.body) next[u] = pieces[i + u * TPR];
        };
        load(t);
        for (int i = t; i < run.body; i += U * TPR) {
            uint4 w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = next[u];
            if (PRE) load(i + U * TPR);
            if (i + (U - 1) * TPR < run.body) {
                add_pieces<T, ENTROPY, U>(w, sums, own_max);
            } else {
#pragma unroll
                for (int u = 0; u < U - 1; ++u) {
                    const uint4 one[1] = {w[u]};
                    if (i + u * TPR < run.body) add_pieces<T, ENTROPY, 1>(one, sums, own_max);
                }
            }
            if (!PRE) load(i + U * TPR);
        }
        add_two(first, last, sums, own_max);
    }
    // the row's maximum, and the maxima of groups of threads, each with its number in the low bits so that no two are alike
    // (which lowers a bound made of them, if anything)
    const int G = TPR < 128 ? TPR : a.top <= 16 ? 64 : 128;
    float m = sums.m, g = own_max;
    for (int o = 1; o < TPR / G; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
    if (a.top && t % (TPR / G) == 0) sh.group_max[t / (TPR / G)] = (place_of(g) & ~127u) | (uint32_t)(t / (TPR / G));
    if (t == 0) { sh.hot = 0; sh.found = 0; sh.bound = 0; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (TPR > 32) {
        if (lane == 0) sh.m[t >> 5] = m;
        row_sync<TPR>();
#pragma unroll
        for (int i = 0; i < TPR / 32; ++i) m = fmaxf(m, sh.m[i]);
    } else {
        row_sync<TPR>();
    }
    Sums all = brought_to(sums, m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        all.s += __shfl_xor_sync(0xffffffffu, all.s, o);
        if (ENTROPY) all.e += __shfl_xor_sync(0xffffffffu, all.e, o);
    }
    if (TPR > 32 && lane == 0) { sh.s[t >> 5] = all.s; sh.e[t >> 5] = all.e; }
    if (a.top && a.top <= G && t < G) {
        const uint32_t mine = sh.group_max[t];
        const uint4* others = reinterpret_cast<const uint4*>(sh.group_max);
        int above = 0;
#pragma unroll 4
        for (int i = 0; i < G / 4; ++i) {
            const uint4 o = others[i];
            above += (o.x > mine) + (o.y > mine) + (o.z > mine) + (o.w > mine);
        }
        if (above == a.top - 1) sh.bound = mine & ~127u;
    }
    row_sync<TPR>();
    if (TPR > 32) {
        all.s = all.e = 0.f;
#pragma unroll
        for (int i = 0; i < TPR / 32; ++i) { all.s += sh.s[i]; all.e += sh.e[i]; }
    }
    if (a.top) {
        const uint32_t bound = sh.bound;                        // below -Inf's place (too few groups): everything counts
        const float least = bound < 0x007fffffu ? -INFINITY : number_at(bound);
        if (own_max >= least) sh.hot_thread[atomicAdd(&sh.hot, 1)] = (unsigned short)t;
        row_sync<TPR>();
        const int hot = sh.hot;
        auto offer = [&](float v, int i) {
            const int at = atomicAdd(&sh.found, 1);
            if (at < kCandidates) sh.candidate[at] = key_of(v, from + i);
        };
        // pieces of a thread, and its one of the head and of the tail: a power of two or less
        const int bits = 32 - __clz((run.body + TPR - 1) / TPR);
        for (int i = t; i < hot << bits; i += TPR) {
            const int who = sh.hot_thread[i >> bits], k = (i & ((1 << bits) - 1)) - 1;
            if (k < 0) {
                const int last = n - run.tail + who;
                if (who < run.head && number(run.p + who) >= least) offer(number(run.p + who), who);
                if (who < run.tail && number(run.p + last) >= least) offer(number(run.p + last), last);
            } else if (who + k * TPR < run.body) {
                const int piece = who + k * TPR;
                float v[N];
                unpack(run.pieces()[piece], v);
                uint32_t hits = 0;                              // few: one after the other, lanes together
#pragma unroll
                for (int e = 0; e < N; ++e) hits |= v[e] >= least ? 1u << e : 0u;
                for (; hits; hits &= hits - 1) {
                    const int at = run.index(piece) + __ffs(hits) - 1;
                    offer(number(run.p + at), at);
                }
            }
        }
        row_sync<TPR>();
        const int found = sh.found;
        if (found > kCandidates || found < min(a.top, n)) {     // too much reaches the bound, or NaN in the way
            best_one_by_one<T, TPR>(sh, run.p, n, from, a.top);
        } else {
            for (int i = t; i < found; i += TPR) {
                const uint64_t key = sh.candidate[i];
                int above = 0;
#pragma unroll 4
                for (int j = 0; j < found; ++j) above += sh.candidate[j] > key;
                if (above < a.top) sh.best[above] = key;
            }
            for (int i = found + t; i < a.top; i += TPR) sh.best[i] = 0;
            row_sync<TPR>();
        }
    }
    all.m = m;
    if (CLUSTER) {                                              // the first block takes all blocks' sums and best
        if (t == 0) sh.sums = all;
        __syncthreads();
        cluster_all_started();
        cluster_sync_all();
        if (rank == 0) {
            const uint32_t at = smem_u32(&sh.sums), list = smem_u32(&sh.best[0]);
            auto far = [](uint32_t addr, uint32_t r) {
                uint32_t v;
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(map_to_cta(addr, r)) : "memory");
                return v;
            };
            Sums each[kCluster];
#pragma unroll
            for (int r = 0; r < kCluster; ++r) {
                each[r] = Sums{__uint_as_float(far(at, r)), __uint_as_float(far(at + 4, r)), __uint_as_float(far(at + 8, r))};
                all.m = fmaxf(all.m, each[r].m);
            }
            all.s = all.e = 0.f;
#pragma unroll
            for (int r = 0; r < kCluster; ++r) {
                const Sums s = brought_to(each[r], all.m);
                all.s += s.s;
                all.e += s.e;
            }
            for (int i = t; i < kCluster * a.top; i += TPR) {
                const uint32_t r = (uint32_t)(i / a.top), k = (uint32_t)(i % a.top);
                sh.candidate[i] = (uint64_t)far(list + 8 * k, r) | ((uint64_t)far(list + 8 * k + 4, r) << 32);
            }
        }
        cluster_sync_all();                                     // nobody leaves while its memory is read
        if (rank != 0) return;
        if (a.top) {
            // keys are of different tokens, or 0; each block's are in order: a key's place is the sum of its places in them
            for (int i = t; i < kCluster * a.top; i += TPR) {
                const uint64_t key = sh.candidate[i];
                int place[kCluster] = {};
#pragma unroll
                for (int step = kMaxTop; step > 0; step >>= 1)
#pragma unroll
                    for (int r = 0; r < kCluster; ++r) {
                        const int next = place[r] + step;
                        if (next <= a.top && sh.candidate[r * a.top + next - 1] > key) place[r] = next;
                    }
                int above = 0;
#pragma unroll
                for (int r = 0; r < kCluster; ++r) above += place[r];
                if (key != 0 && above < a.top) sh.best[above] = key;
            }
            __syncthreads();
        }
    }
    const bool none = all.s == 0.f;                             // every logit is -Inf
    const float log_s = logf(all.s);
    const float lse = none ? -INFINITY : all.m + log_s;
    // log-probabilities from the distance to the maximum: lse is rounded to its own size, which says nothing about theirs
    auto logp_of = [&](float l) { return none ? -INFINITY : (l - all.m) - log_s; };
    if (t == 0) {
        if (a.logp) a.logp[row] = given ? logp_of(at_target) : 0.f;
        if (ENTROPY) a.entropy[row] = none ? 0.f : log_s - __fdiv_rn(all.e, all.s);
        if (a.lse) a.lse[row] = lse;
    }
    for (int i = t; i < a.top; i += TPR) {
        const uint64_t key = sh.best[i];
        a.top_values[row * a.top + i] = logp_of(value_of(key));
        a.top_ids[row * a.top + i] = (int32_t)~(uint32_t)key;
    }
}

// ---- their gradient ----------------------------------------------------------------------------
// d_j = s (delta_jt - p_j) - c p_j (log p_j + H): every logit read once, every gradient written once.  A warp or a block a
// row, long rows in parts.
struct LogprobBackArgs {
    int64_t rows, stride, out_stride, items;
    int V, parts, span;                                         // parts of a row, logits in one
    const void* logits;
    const int32_t* targets;
    const float *lse, *d_logp, *entropy, *d_entropy;
    void* d_logits;
};
template <typename T, int TPR>
__global__ void __launch_bounds__(256) logprob_back_kernel(const __grid_constant__ LogprobBackArgs a) {
    constexpr int N = Piece<T>::N, U = TPR == 32 ? 2 : 4, ROWS = 256 / TPR;
    after_predecessor();
    const int t = threadIdx.x & (TPR - 1);
    for (int64_t item = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; item < a.items; item += (int64_t)gridDim.x * ROWS) {
        const int64_t row = item / a.parts;
        const int from = (int)(item % a.parts) * a.span, n = min(a.V - from, a.span);
        const T* p = static_cast<const T*>(a.logits) + row * a.stride + from;
        T* out = static_cast<T*>(a.d_logits) + row * a.out_stride + from;
        const int target = a.targets[row];
        const float lse = a.lse[row], weight = a.d_logp[row], s = target >= 0 && target < a.V ? weight : 0.f;
        const float c = a.d_entropy ? a.d_entropy[row] : 0.f, H = a.d_entropy ? a.entropy[row] : 0.f;
        const bool zero = (s == 0.f && c == 0.f) || lse == -INFINITY;
        const int at = target - from;
        // -p (c (log p + H) + s); where p is 0 the logarithm is kept finite
        const F2 minus = both(-lse), slope = both(-c), offset = both(-fmaf(c, H, s));
        auto two = [&](F2 l) {
            const F2 d = add2(l, minus), x = {max_or_nan(d.x, -1e4f), max_or_nan(d.y, -1e4f)};
            return mul2(exp2_fast(mul2(x, both(kLog2e))), fma2(x, slope, offset));
        };
        auto one = [&](float l, int i) {
            if (zero) return 0.f;
            const float d = two(both(l)).x;
            return i == at ? d + s : d;
        };
        Run<T> run(p, n);
        if ((reinterpret_cast<uintptr_t>(p) & 15u) != (reinterpret_cast<uintptr_t>(out) & 15u)) {
            for (int i = t; i < n; i += TPR) put(out + i, one(number(p + i), i));
            continue;
        }
        const uint4* pieces = run.pieces();
        uint4* to = reinterpret_cast<uint4*>(out + run.head);
        for (int i0 = t; i0 < run.body; i0 += U * TPR) {
            uint4 w[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i0 + u * TPR < run.body) w[u] = __ldcs(pieces + i0 + u * TPR);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u * TPR >= run.body) continue;
                float v[N];
                unpack(w[u], v);
                const int mine = at - run.index(i0 + u * TPR);  // the target's place among these
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const F2 d = two(F2{v[e], v[e + 1]});
                    v[e] = d.x;
                    v[e + 1] = d.y;
                }
                if (mine >= 0 && mine < N) {
#pragma unroll
                    for (int e = 0; e < N; ++e) v[e] += e == mine ? s : 0.f;
                }
                __stcs(to + i0 + u * TPR, zero ? make_uint4(0u, 0u, 0u, 0u) : repack(v));
            }
        }
        if (t < run.head) put(out + t, one(number(p + t), t));
        if (t < run.tail) put(out + n - run.tail + t, one(number(p + n - run.tail + t), n - run.tail + t));
    }
}

// ---- values of 8 bits ----------------------------------------------------------------------------
__device__ __forceinline__ float2 two_of(uint32_t w) {
    const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2*>(&r));
}
__device__ __forceinline__ uint32_t two_bf16(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
constexpr int kDequantEach = 4;                                 // (2: 14.6 us for 32768 x 768 to bf16, 8: 15.6, 4: 14.1)
struct DequantArgs {
    int64_t rows, q_stride, scale_stride, x_stride;
    int cols;
    const uint8_t *q, *scale;
    void* x;
};
// VEC: rows of x on the 16-byte grid, whose 16 bytes are a lane's each time, so that a warp writes 512 in a row.  Otherwise a
// warp takes a block of 128, lanes side by side.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dequantise_kernel(const __grid_constant__ DequantArgs a) {
    constexpr int EACH = VEC ? kDequantEach : 4, N = Piece<T>::N;      // pieces of x, or blocks of a warp, a thread
    after_predecessor();
    const uint32_t per_row = VEC ? (uint32_t)(a.cols + N - 1) / N : (uint32_t)(a.cols + 127) / 128;
    const int64_t base = (int64_t)blockIdx.x * (VEC ? 256 * EACH : 8 * EACH);
    const int64_t row0 = base / per_row;
    const uint32_t skip = (uint32_t)(base - row0 * per_row);
    if (VEC) {
        uint32_t w[EACH][N / 4], byte[EACH], col[EACH];
        int64_t row[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const uint32_t at = skip + threadIdx.x + 256 * i, r = at / per_row;
            row[i] = row0 + r;
            col[i] = (at - r * per_row) * N;
            if (row[i] >= a.rows) continue;
            const uint8_t* q = a.q + row[i] * a.q_stride + col[i];
            if ((int)col[i] + N <= a.cols) {
#pragma unroll
                for (int j = 0; j < N / 4; ++j) w[i][j] = 0u;
                if (N == 8) {
                    const uint2 v = *reinterpret_cast<const uint2*>(q);
                    w[i][0] = v.x;
                    w[i][N / 4 - 1] = v.y;
                } else {
                    w[i][0] = *reinterpret_cast<const uint32_t*>(q);
                }
            } else {                                            // a row's last, incomplete piece
#pragma unroll
                for (int j = 0; j < N / 4; ++j) {
                    w[i][j] = 0u;
#pragma unroll
                    for (int b = 0; b < 4; ++b)
                        if ((int)col[i] + 4 * j + b < a.cols) w[i][j] |= (uint32_t)q[4 * j + b] << (8 * b);
                }
            }
            byte[i] = a.scale[row[i] * a.scale_stride + (col[i] >> 7)];
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (row[i] >= a.rows) continue;
            const float s = scale_of(byte[i]);
            T* to = static_cast<T*>(a.x) + row[i] * a.x_stride + col[i];
            float v[N];
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const float2 f = two_of(w[i][e >> 2] >> (16 * ((e >> 1) & 1)));
                v[e] = f.x * s;
                v[e + 1] = f.y * s;
            }
            if ((int)col[i] + N <= a.cols) {
                __stcs(reinterpret_cast<uint4*>(to), repack(v));
            } else {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if ((int)col[i] + e < a.cols) put(to + e, v[e]);
            }
        }
    } else {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const uint32_t at = skip + (threadIdx.x >> 5) + 8 * i, r = at / per_row;
            const int64_t row = row0 + r;
            const int block = (int)(at - r * per_row), n = min(128, a.cols - block * 128);
            if (row >= a.rows) continue;
            const float s = scale_of(a.scale[row * a.scale_stride + block]);
            const uint8_t* q = a.q + row * a.q_stride + block * 128;
            T* to = static_cast<T*>(a.x) + row * a.x_stride + block * 128;
            if (sizeof(T) == 2 && n == 128) {
                // four in a row a lane; where a row starts between two words, its words take the next lane's first number
                const uint32_t w = *reinterpret_cast<const uint32_t*>(q + 4 * lane);
                const float2 u = two_of(w), v = two_of(w >> 16);
                const float first = u.x * s, second = u.y * s, third = v.x * s, fourth = v.y * s;
                uint32_t* words = reinterpret_cast<uint32_t*>((reinterpret_cast<uintptr_t>(to + 4 * lane) + 3) & ~uintptr_t(3));
                if ((reinterpret_cast<uintptr_t>(to) & 3u) == 0) {
                    words[0] = two_bf16(first, second);
                    words[1] = two_bf16(third, fourth);
                } else {
                    const float beyond = __shfl_down_sync(0xffffffffu, first, 1);
                    if (lane == 0) put(to, first);
                    words[0] = two_bf16(second, third);
                    if (lane < 31) words[1] = two_bf16(fourth, beyond);
                    else put(to + 127, fourth);
                }
                continue;
            }
            uint32_t v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = e * 32 + lane < n ? q[e * 32 + lane] : 0u;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e * 32 + lane < n) put(to + e * 32 + lane, two_of(v[e]).x * s);
        }
    }
}

template <typename T, int TPR, bool CLUSTER>
int launch_logprob_rows(adloco_ctx* ctx, const LogprobArgs& a, cudaStream_t st) {
    constexpr int ROWS = TPR < 128 ? 128 / TPR : 1, THREADS = TPR < 128 ? 128 : TPR;
    const int64_t blocks = CLUSTER ? a.rows * kCluster : (a.rows + ROWS - 1) / ROWS;
    if (blocks > 0x7fffffff) return ADLOCO_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)blocks);
    const cudaError_t e = a.entropy ? launch_early(logprob_kernel<T, TPR, CLUSTER, true>, grid, THREADS, 0, st, CLUSTER ? kCluster : 1, a)
                                    : launch_early(logprob_kernel<T, TPR, CLUSTER, false>, grid, THREADS, 0, st, CLUSTER ? kCluster : 1, a);
    ADLOCO_CUDA_TRY(ctx, e);
    ctx->launches++;
    return ADLOCO_OK;
}
constexpr int kWarpV = 12288;
template <typename T>
int launch_logprob(adloco_ctx* ctx, const LogprobArgs& a, cudaStream_t st) {
    // a cluster a row where there are fewer rows than would fill the machine and each is long
    if (a.rows * 4 <= ctx->sm_count && a.V >= 16384 && cta_pairs_possible(ctx)) return launch_logprob_rows<T, kClusterThreads, true>(ctx, a, st);
    // a warp a row while its 32 maxima bound the best tokens and there are rows for many warps, or where all of the row are candidates
    if (a.V <= kCandidates || (a.V <= kWarpV && a.top <= 24 && a.rows >= 8 * ctx->sm_count)) return launch_logprob_rows<T, 32, false>(ctx, a, st);
    return launch_logprob_rows<T, kTopThreads, false>(ctx, a, st);
}
template <typename T>
int launch_logprob_back(adloco_ctx* ctx, LogprobBackArgs a, cudaStream_t st) {
    const bool narrow = a.V <= 2048;
    // Long parts, whose blocks spend their time in the loop (8192 x 50257 bf16: 260 us with 16 pieces a thread, 315 with four, 269 with
    // 32), as far as they leave eight blocks an SM.
    for (int each = 16;; each /= 2) {
        a.span = narrow ? a.V : 256 * each * Piece<T>::N;
        a.parts = (a.V + a.span - 1) / a.span;
        a.items = a.rows * a.parts;
        if (narrow || each == 2 || a.items >= 8 * ctx->sm_count) break;
    }
    const int64_t blocks = narrow ? (a.items + 7) / 8 : a.items, most = int64_t(1) << 30;
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    ADLOCO_CUDA_TRY(ctx, narrow ? launch_early(logprob_back_kernel<T, 32>, grid, 256, 0, st, 1, a) : launch_early(logprob_back_kernel<T, 256>, grid, 256, 0, st, 1, a));
    ctx->launches++;
    return ADLOCO_OK;
}
template <typename T>
int launch_dequantise(adloco_ctx* ctx, const DequantArgs& a, cudaStream_t st) {
    const bool vec = aligned16(a.x) && a.x_stride % Piece<T>::N == 0;
    const int64_t units = a.rows * (vec ? (a.cols + Piece<T>::N - 1) / Piece<T>::N : (a.cols + 127) / 128), each = vec ? 256 * kDequantEach : 32;
    if ((units + each - 1) / each > 0x7fffffff) return ADLOCO_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((units + each - 1) / each));
    ADLOCO_CUDA_TRY(ctx, vec ? launch_early(dequantise_kernel<T, true>, grid, 256, 0, st, 1, a) : launch_early(dequantise_kernel<T, false>, grid, 256, 0, st, 1, a));
    ctx->launches++;
    return ADLOCO_OK;
}

}  // namespace

int launch_blockscale_dequantize(adloco_ctx* ctx, int bf16, int64_t rows, int64_t cols, const void* q, int64_t q_stride,
                                 const uint8_t* scale, int64_t scale_stride, void* x, int64_t x_stride, cudaStream_t st) {
    const DequantArgs a = {rows, q_stride, scale_stride, x_stride, (int)cols, static_cast<const uint8_t*>(q), scale, x};
    return bf16 ? launch_dequantise<__nv_bfloat16>(ctx, a, st) : launch_dequantise<float>(ctx, a, st);
}

int launch_token_logprobs(adloco_ctx* ctx, const adloco_token_logprobs_args& c, cudaStream_t st) {
    const LogprobArgs a = {c.rows, c.logits_stride, (int)c.V, c.top, c.logits, c.targets, c.logp, c.entropy, c.lse, c.top_values, c.top_ids};
    return c.dtype == ADLOCO_BF16 ? launch_logprob<__nv_bfloat16>(ctx, a, st) : launch_logprob<float>(ctx, a, st);
}

int launch_token_logprobs_backward(adloco_ctx* ctx, const adloco_token_logprobs_backward_args& c, cudaStream_t st) {
    LogprobBackArgs a = {c.rows, c.logits_stride, c.d_logits_stride, 0, (int)c.V, 0, 0, c.logits, c.targets, c.lse, c.d_logp, c.entropy, c.d_entropy, c.d_logits};
    return c.dtype == ADLOCO_BF16 ? launch_logprob_back<__nv_bfloat16>(ctx, a, st) : launch_logprob_back<float>(ctx, a, st);
}

}  // namespace adloco

// C ABI of the operators between the linear layers: argument checks and dispatch.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "common.cuh"

using namespace adloco;

namespace {

constexpr int64_t kMaxExtent = int64_t(1) << 30;      // rows, columns, tokens, heads

bool known(adloco_dtype t) { return t == ADLOCO_F32 || t == ADLOCO_BF16; }
uintptr_t elem_bytes(adloco_dtype t) { return t == ADLOCO_BF16 ? 2 : 4; }
bool elem_aligned(const void* p, adloco_dtype t) { return (reinterpret_cast<uintptr_t>(p) & (elem_bytes(t) - 1)) == 0; }

int make_key(double p, uint64_t seed, uint64_t offset, bool residual, DropoutKey* key) {
    if (!(p >= 0.0) || !(p <= 1.0)) return ADLOCO_ERR_INVALID_ARG;
    const uint32_t drop = (uint32_t)std::nearbyint(p * 65536.0);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
    for (int r = 0; r < 10; ++r, k0 += 0x9E3779B9u, k1 += 0xBB67AE85u) {      // Weyl sequence of the generator's key
        key->round[2 * r] = k0;
        key->round[2 * r + 1] = k1;
    }
    key->off_lo = (uint32_t)offset; key->off_hi = (uint32_t)(offset >> 32);
    key->on = drop != 0;
    if (drop < 65536u) {
        const double scale = 65536.0 / (65536.0 - (double)drop);
        key->scale = key->high = (float)scale;
        if (residual) {
            if ((double)key->high > scale) key->high = std::nextafterf(key->high, 0.f);
            key->low = (float)(scale - (double)key->high);
        }
    }
    key->limit = (drop & 0xffffu) | (drop << 16);
    if (drop == 65536u) key->of_pair = key->of_low = key->of_high = 0x4444u;
    return ADLOCO_OK;
}

// An output at the address of an input is that input, row for row: with another pitch its rows are other rows' inputs.
bool in_step(const void* out, int64_t out_stride, const void* in, int64_t in_stride, int64_t rows) {
    return out == nullptr || out != in || rows == 1 || out_stride == in_stride;
}

// the pair of types an operator with a residual stream takes
int check_types(adloco_dtype t, adloco_dtype stream, adloco_dtype gain) {
    if (!known(t) || !known(stream) || !known(gain)) return ADLOCO_ERR_UNSUPPORTED;
    if (t == ADLOCO_F32 && stream == ADLOCO_BF16) return ADLOCO_ERR_UNSUPPORTED;
    return ADLOCO_OK;
}

// an 8-bit matrix and its scales, as the tensor cores' copies need them
int check_bytes(const void* q, int64_t q_stride, int64_t cols) {
    if (q_stride < cols) return ADLOCO_ERR_INVALID_ARG;
    if (!aligned16(q) || (q_stride & 15) != 0) return ADLOCO_ERR_ALIGNMENT;
    return ADLOCO_OK;
}
int check_row_scales(const void* s, int64_t stride, int64_t cols) {
    if (stride < (cols + 127) / 128) return ADLOCO_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(s) & 3u) != 0 || (stride & 3) != 0) return ADLOCO_ERR_ALIGNMENT;
    return ADLOCO_OK;
}

// Do runs of `width` elements at i s[0] + j s[1] + k s[2], i < n[0], j < n[1], k < n[2], fall on one another?  Strides that
// nest (each one spans what the smaller ones reach) do not.  Otherwise two runs meet exactly when a difference
// i s[0] + j s[1] + k s[2], not all of i, j, k zero, is less than the width; the smallest stride's k follows from i and j.  A
// layout that takes more than kSteps of them to decide counts as falling on itself.
bool fall_on_one_another(const int64_t (&extents)[3], const int64_t (&strides)[3], int64_t width) {
    constexpr int64_t kSteps = 1 << 20;
    typedef __int128 wide;
    struct Dim { int64_t n; wide s; } d[3];
    for (int i = 0; i < 3; ++i) d[i] = Dim{extents[i], extents[i] > 1 ? (wide)strides[i] : 0};
    std::sort(d, d + 3, [](const Dim& a, const Dim& b) { return a.s > b.s; });
    bool nested = true;
    wide reach = width;
    for (int i = 2; i >= 0; --i) {
        if (d[i].n > 1 && d[i].s < reach) nested = false;
        reach += d[i].s * (d[i].n - 1);
    }
    if (nested) return false;
    const wide most_k = d[2].s * (d[2].n - 1), most_j = d[1].s * (d[1].n - 1);
    int64_t steps = 0;
    for (int64_t i = 0; i < d[0].n && i * d[0].s < most_j + most_k + width; ++i) {
        if (++steps > kSteps) return true;
        const wide at = i * d[0].s;
        // j with |at + j s| < most_k + width, both signs of j where i is zero being the same
        int64_t j = 0, last = d[1].n - 1;
        if (d[1].s > 0) {
            const wide low = -((at + most_k + width) / d[1].s), high = (most_k + width - at) / d[1].s;
            j = (int64_t)std::max<wide>(i ? low : 0, -(wide)(d[1].n - 1));
            last = (int64_t)std::min<wide>(high, d[1].n - 1);
        } else if (d[1].n > 1) {
            return true;                                     // a stride of zero
        }
        for (; j <= last; ++j) {
            if (++steps > kSteps) return true;
            const wide off = at + j * d[1].s, far = off < 0 ? -off : off;
            int64_t k = 0;
            if (d[2].n > 1) {
                if (d[2].s == 0) return true;
                k = (int64_t)std::min<wide>(far / d[2].s, d[2].n - 1);
            }
            const wide here = far - k * d[2].s, next = k + 1 < d[2].n ? (k + 1) * d[2].s - far : (wide)width;
            const bool same = i == 0 && j == 0;              // k = 0 is the run itself
            if ((!(same && k == 0) && here < width) || (next >= 0 && next < width)) return true;
        }
    }
    return false;
}

// an operand of a bf16 product: rows that the tensor cores' copies can take
int check_operand(const void* p, int64_t stride, int64_t cols) {
    if (!p || stride < cols) return ADLOCO_ERR_INVALID_ARG;
    if (!aligned16(p) || (stride & 7) != 0) return ADLOCO_ERR_ALIGNMENT;
    return ADLOCO_OK;
}
int check_kept(const adloco_kept& k, int64_t cols) {
    if (!k.p) return k.scale ? ADLOCO_ERR_INVALID_ARG : ADLOCO_OK;
    if (!k.scale) return check_operand(k.p, k.stride, cols);
    const int rc = check_bytes(k.p, k.stride, cols);
    return rc != ADLOCO_OK ? rc : check_row_scales(k.scale, k.scale_stride, cols);
}
// Where a matrix lies: rows of `width` bytes, `pitch` bytes apart.
struct Area {
    const void* p;
    int64_t pitch, width, rows;
};
Area area(const void* p, int64_t stride, int64_t cols, int64_t rows, int64_t bytes) { return Area{p, stride * bytes, cols * bytes, rows}; }
Area line(const void* p, int64_t n, int64_t bytes = 4) { return Area{p, n * bytes, n * bytes, 1}; }
Area values_of(const adloco_kept& k, int64_t rows, int64_t cols) { return area(k.p, k.stride, cols, rows, k.scale ? 1 : 2); }
Area scales_of(const adloco_kept& k, int64_t rows, int64_t cols) { return area(k.scale, k.scale_stride, (cols + 127) / 128, rows, 1); }
bool same_place(const Area& a, const Area& b) {
    return a.p == b.p && a.width == b.width && a.rows == b.rows && (a.rows == 1 || a.pitch == b.pitch);
}
// Do two matrices share a byte?  Exact where the pitches are alike (columns of one matrix) or one of them is a single row no
// longer than the other's pitch; what else lies within one another's span counts as sharing.
bool touch(const Area& a, const Area& b) {
    typedef __int128 wide;
    if (!a.p || !b.p) return false;
    const wide at = (wide)reinterpret_cast<uintptr_t>(a.p), bt = (wide)reinterpret_cast<uintptr_t>(b.p);
    if (at + (wide)(a.rows - 1) * a.pitch + a.width <= bt || bt + (wide)(b.rows - 1) * b.pitch + b.width <= at) return false;
    if (a.rows == 1 && b.rows == 1) return true;
    const int64_t pitch = a.rows > 1 ? a.pitch : b.pitch;
    if ((b.rows > 1 && b.pitch != pitch) || a.width > pitch || b.width > pitch) return true;
    // row j of b begins d bytes behind the beginning of a's row j + k, and reaches into its next one where it passes the pitch
    wide k = (bt - at) / pitch, d = (bt - at) % pitch;
    if (d < 0) { d += pitch; --k; }
    const auto some = [&](wide shift) { return shift < a.rows && -shift < b.rows; };
    return (d < a.width && some(k)) || (d + b.width > pitch && some(k + 1));
}
// An output may be one of the operands that are read at the place that is written (the same elements, row for row), but may
// share nothing else with them, nor anything with another output or with what is read elsewhere.
bool apart(std::initializer_list<Area> outs, std::initializer_list<Area> elementwise, std::initializer_list<Area> others) {
    for (const Area* o = outs.begin(); o != outs.end(); ++o) {
        for (const Area* other = outs.begin(); other != o; ++other)
            if (touch(*o, *other)) return false;
        for (const Area& e : elementwise)
            if (touch(*o, e) && !same_place(*o, e)) return false;
        for (const Area& x : others)
            if (touch(*o, x)) return false;
    }
    return true;
}
bool known_act(int32_t a) { return a >= ADLOCO_ACT_NONE && a <= ADLOCO_ACT_SILU; }
bool too_large(std::initializer_list<int64_t> extents) {
    for (int64_t e : extents)
        if (e > kMaxExtent) return true;
    return false;
}

}  // namespace

extern "C" {

int adloco_add_rmsnorm(adloco_ctx* ctx, const adloco_rmsnorm_args* a, void* stream) {
    if (!ctx || !a || !a->x || !a->gain || (!a->y && !a->q) || (!a->q) != (!a->q_scale)) return ADLOCO_ERR_INVALID_ARG;
    int rc = check_types(a->dtype, a->stream_dtype, a->gain_dtype);
    if (rc != ADLOCO_OK) return rc;
    if (a->rows < 1 || a->d < 1 || !(a->eps >= 0.f) || !std::isfinite(a->eps)) return ADLOCO_ERR_INVALID_ARG;
    if (a->rows > kMaxExtent || a->d > 16384) return ADLOCO_ERR_UNSUPPORTED;
    if (a->x_stride < a->d || (a->residual && a->residual_stride < a->d) || (a->h && a->h_stride < a->d) ||
        (a->y && a->y_stride < a->d) || !in_step(a->h, a->h_stride, a->residual, a->residual_stride, a->rows))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(a->x, a->dtype) || !elem_aligned(a->y, a->dtype) || !elem_aligned(a->residual, a->stream_dtype) ||
        !elem_aligned(a->h, a->stream_dtype) || !elem_aligned(a->gain, a->gain_dtype) || !elem_aligned(a->rstd, ADLOCO_F32))
        return ADLOCO_ERR_ALIGNMENT;
    if (a->q) {
        rc = check_bytes(a->q, a->q_stride, a->d);
        if (rc == ADLOCO_OK) rc = check_row_scales(a->q_scale, a->q_scale_stride, a->d);
        if (rc != ADLOCO_OK) return rc;
    }
    DropoutKey key;
    rc = make_key(a->dropout_p, a->seed, a->offset, a->residual != nullptr, &key);
    if (rc != ADLOCO_OK) return rc;
    DeviceGuard g(ctx->device);
    return launch_add_rmsnorm(ctx, *a, key, static_cast<cudaStream_t>(stream));
}

int64_t adloco_add_rmsnorm_backward_workspace(const adloco_ctx* ctx, int64_t B, int64_t T, int64_t d) {
    if (!ctx || B < 1 || T < 1 || d < 1 || B > (kMaxExtent >> 3) || T > kMaxExtent || d > 16384) return 0;
    return rmsnorm_backward_workspace(ctx, B, T, d);
}

int adloco_add_rmsnorm_backward(adloco_ctx* ctx, const adloco_rmsnorm_backward_args* a, void* stream) {
    if (!ctx || !a || !a->dy || !a->h || !a->rstd || !a->gain || !a->dh) return ADLOCO_ERR_INVALID_ARG;
    int rc = check_types(a->dtype, a->stream_dtype, a->gain_dtype);
    if (rc != ADLOCO_OK) return rc;
    if (a->B < 1 || a->T < 1 || a->d < 1) return ADLOCO_ERR_INVALID_ARG;
    // samples: a cluster of eight blocks each forms their norms
    if (a->B > (kMaxExtent >> 3) || a->T > kMaxExtent || a->B * a->T > kMaxExtent || a->d > 16384) return ADLOCO_ERR_UNSUPPORTED;
    if (a->dy_stride < a->d || a->h_stride < a->d || a->dh_stride < a->d ||
        (a->dh_residual && a->dh_residual_stride < a->d) || (a->dx && a->dx_stride < a->d) ||
        !in_step(a->dh, a->dh_stride, a->dh_residual, a->dh_residual_stride, a->B * a->T) ||
        !in_step(a->dx, a->dx_stride, a->dy, a->dy_stride, a->B * a->T))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(a->dy, a->dtype) || !elem_aligned(a->dx, a->dtype) || !elem_aligned(a->h, a->stream_dtype) ||
        !elem_aligned(a->dh, a->stream_dtype) || !elem_aligned(a->dh_residual, a->stream_dtype) ||
        !elem_aligned(a->gain, a->gain_dtype) || !elem_aligned(a->rstd, ADLOCO_F32) ||
        !elem_aligned(a->per_sample_sqnorm, ADLOCO_F32) || !elem_aligned(a->grad_sum, ADLOCO_F32))
        return ADLOCO_ERR_ALIGNMENT;
    if (a->per_sample_sqnorm || a->grad_sum) {
        if (!a->workspace) return ADLOCO_ERR_INVALID_ARG;
        if (!aligned16(a->workspace)) return ADLOCO_ERR_ALIGNMENT;
        if (a->workspace_bytes < rmsnorm_backward_workspace(ctx, a->B, a->T, a->d)) return ADLOCO_ERR_WORKSPACE;
    }
    DropoutKey key;
    rc = make_key(a->dropout_p, a->seed, a->offset, false, &key);
    if (rc != ADLOCO_OK) return rc;
    DeviceGuard g(ctx->device);
    return launch_add_rmsnorm_backward(ctx, *a, key, static_cast<cudaStream_t>(stream));
}

int adloco_dropout(adloco_ctx* ctx, adloco_dtype dtype, int64_t rows, int64_t cols, const void* x, int64_t x_stride,
                   const void* residual, int64_t residual_stride, void* y, int64_t y_stride, double p, uint64_t seed,
                   uint64_t offset, void* stream) {
    if (!ctx || !x || !y || rows < 1 || cols < 1) return ADLOCO_ERR_INVALID_ARG;
    if (!known(dtype)) return ADLOCO_ERR_UNSUPPORTED;
    if (rows > kMaxExtent || cols > (int64_t(1) << 40) || rows > (int64_t(1) << 50) / cols) return ADLOCO_ERR_UNSUPPORTED;
    if (x_stride < cols || y_stride < cols || (residual && residual_stride < cols) || !in_step(y, y_stride, x, x_stride, rows) ||
        !in_step(y, y_stride, residual, residual_stride, rows))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(x, dtype) || !elem_aligned(y, dtype) || !elem_aligned(residual, dtype)) return ADLOCO_ERR_ALIGNMENT;
    DropoutKey key;
    const int rc = make_key(p, seed, offset, residual != nullptr, &key);
    if (rc != ADLOCO_OK) return rc;
    DeviceGuard g(ctx->device);
    return launch_dropout(ctx, dtype == ADLOCO_BF16, rows, cols, x, x_stride, residual, residual_stride, y, y_stride, key,
                          static_cast<cudaStream_t>(stream));
}

int adloco_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double context, double low,
                            double high, uint64_t* turns_host) {
    if (!turns_host || rot_dim < 2 || (rot_dim & 1) || !(base > 0.0) || !std::isfinite(base)) return ADLOCO_ERR_INVALID_ARG;
    if (scaling < ADLOCO_ROPE_NONE || scaling > ADLOCO_ROPE_BY_PARTS) return ADLOCO_ERR_INVALID_ARG;
    if (scaling != ADLOCO_ROPE_NONE && (!(factor > 0.0) || !std::isfinite(factor))) return ADLOCO_ERR_INVALID_ARG;
    if (scaling == ADLOCO_ROPE_BY_PARTS && (!(high > low) || !(context > 0.0) || !std::isfinite(high - low) || !std::isfinite(context)))
        return ADLOCO_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    if (scaling == ADLOCO_ROPE_NTK && rot_dim > 2) base *= std::pow(factor, (double)rot_dim / (double)(rot_dim - 2));
    for (int32_t j = 0; j < rot_dim / 2; ++j) {
        double w = std::pow(base, -2.0 * j / rot_dim);
        if (scaling == ADLOCO_ROPE_LINEAR) w /= factor;
        if (scaling == ADLOCO_ROPE_BY_PARTS) {
            double u = (w * context / two_pi - low) / (high - low);
            u = u < 0.0 ? 0.0 : u > 1.0 ? 1.0 : u;
            w = u * w + (1.0 - u) * w / factor;
        }
        double t = w / two_pi;                                  // whole turns a position do not matter
        t -= std::floor(t);
        if (!std::isfinite(t)) return ADLOCO_ERR_INVALID_ARG;   // a base or a factor that takes the frequency out of range
        const double units = std::nearbyint(t * 18446744073709551616.0);
        turns_host[j] = units >= 18446744073709551616.0 ? 0u : (uint64_t)units;
    }
    return ADLOCO_OK;
}

int adloco_rope(adloco_ctx* ctx, adloco_dtype dtype, const adloco_rope_tensor* tensors, int32_t n_tensors, int64_t B,
                int64_t T, int64_t head_dim, int64_t rot_dim, const uint64_t* turns_dev, float magnitude,
                const int32_t* positions, int64_t positions_stride, int64_t first_position, int interleaved, int inverse,
                void* stream) {
    if (!ctx || !tensors || n_tensors < 1 || !turns_dev || B < 1 || T < 1 || head_dim < 1) return ADLOCO_ERR_INVALID_ARG;
    if (rot_dim < 2 || (rot_dim & 1) || rot_dim > head_dim || !std::isfinite(magnitude)) return ADLOCO_ERR_INVALID_ARG;
    if (!known(dtype) || n_tensors > 4) return ADLOCO_ERR_UNSUPPORTED;
    if (B > kMaxExtent || T > kMaxExtent || B * T > kMaxExtent || head_dim > 4096) return ADLOCO_ERR_UNSUPPORTED;
    if (positions && (positions_stride < T || (reinterpret_cast<uintptr_t>(positions) & 3u) != 0))
        return positions_stride < T ? ADLOCO_ERR_INVALID_ARG : ADLOCO_ERR_ALIGNMENT;
    if ((reinterpret_cast<uintptr_t>(turns_dev) & 7u) != 0) return ADLOCO_ERR_ALIGNMENT;
    int64_t heads = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const adloco_rope_tensor& t = tensors[i];
        if (!t.in || !t.out || t.heads < 1) return ADLOCO_ERR_INVALID_ARG;
        if (t.in_batch < 0 || t.in_token < 0 || t.in_head < 0 || t.out_batch < 0 || t.out_token < 0 || t.out_head < 0)
            return ADLOCO_ERR_INVALID_ARG;
        if (t.heads > 65536) return ADLOCO_ERR_UNSUPPORTED;
        // in place: the same strides, those of extents of one aside
        if (t.in == t.out && ((B > 1 && t.in_batch != t.out_batch) || (T > 1 && t.in_token != t.out_token) ||
                              (t.heads > 1 && t.in_head != t.out_head)))
            return ADLOCO_ERR_INVALID_ARG;
        if (fall_on_one_another({B, T, t.heads}, {t.out_batch, t.out_token, t.out_head}, head_dim)) return ADLOCO_ERR_INVALID_ARG;
        if (!elem_aligned(t.in, dtype) || !elem_aligned(t.out, dtype)) return ADLOCO_ERR_ALIGNMENT;
        heads += t.heads;
    }
    if (heads * head_dim > kMaxExtent) return ADLOCO_ERR_UNSUPPORTED;
    DeviceGuard g(ctx->device);
    return launch_rope(ctx, dtype == ADLOCO_BF16, tensors, n_tensors, B, T, head_dim, rot_dim, turns_dev, magnitude, positions,
                       positions_stride, first_position, interleaved, inverse, static_cast<cudaStream_t>(stream));
}

int adloco_blockscale_quantize(adloco_ctx* ctx, adloco_dtype dtype, int64_t rows, int64_t cols, const void* x,
                               int64_t x_stride, void* q, int64_t q_stride, uint8_t* scale, int64_t scale_stride,
                               void* stream) {
    if (!ctx || !x || !q || !scale || rows < 1 || cols < 1 || x_stride < cols) return ADLOCO_ERR_INVALID_ARG;
    if (!known(dtype) || rows > kMaxExtent || cols > kMaxExtent) return ADLOCO_ERR_UNSUPPORTED;
    if (!elem_aligned(x, dtype)) return ADLOCO_ERR_ALIGNMENT;
    int rc = check_bytes(q, q_stride, cols);
    if (rc == ADLOCO_OK) rc = check_row_scales(scale, scale_stride, cols);
    if (rc != ADLOCO_OK) return rc;
    DeviceGuard g(ctx->device);
    return launch_blockscale_quantize(ctx, dtype == ADLOCO_BF16, rows, cols, x, x_stride, q, q_stride, scale, scale_stride,
                                      static_cast<cudaStream_t>(stream));
}

int adloco_blockscale_quantize_weight(adloco_ctx* ctx, adloco_dtype dtype, int64_t rows, int64_t cols, const void* W,
                                      int64_t W_stride, void* q, int64_t q_stride, void* q_t, int64_t q_t_stride,
                                      uint8_t* scale, int64_t scale_stride, void* stream) {
    if (!ctx || !W || !q || !scale || rows < 1 || cols < 1 || W_stride < cols) return ADLOCO_ERR_INVALID_ARG;
    if (scale_stride < (cols + 127) / 128) return ADLOCO_ERR_INVALID_ARG;
    if (!known(dtype) || rows > kMaxExtent || cols > kMaxExtent) return ADLOCO_ERR_UNSUPPORTED;
    if (!elem_aligned(W, dtype)) return ADLOCO_ERR_ALIGNMENT;
    int rc = check_bytes(q, q_stride, cols);
    if (rc == ADLOCO_OK && q_t) rc = check_bytes(q_t, q_t_stride, rows);
    if (rc != ADLOCO_OK) return rc;
    DeviceGuard g(ctx->device);
    return launch_blockscale_quantize_weight(ctx, dtype == ADLOCO_BF16, rows, cols, W, W_stride, q, q_stride, q_t, q_t_stride,
                                             scale, scale_stride, static_cast<cudaStream_t>(stream));
}

int adloco_blockscale_matmul(adloco_ctx* ctx, const adloco_blockscale_matmul_args* a, void* stream) {
    if (!ctx || !a || !a->a || !a->a_scale || !a->b || !a->b_scale || !a->out) return ADLOCO_ERR_INVALID_ARG;
    if (a->M < 1 || a->N < 1 || a->K < 1 || a->out_stride < a->N) return ADLOCO_ERR_INVALID_ARG;
    if (!known(a->out_dtype) || a->M > kMaxExtent || a->N > kMaxExtent || a->K > kMaxExtent) return ADLOCO_ERR_UNSUPPORTED;
    const int64_t kb = (a->K + 127) / 128, nb = (a->N + 127) / 128;
    if (a->b_scale_stride_n < 0 || a->b_scale_stride_k < 0 || (nb > 1 && a->b_scale_stride_n < 1) ||
        (kb > 1 && a->b_scale_stride_k < 1))
        return ADLOCO_ERR_INVALID_ARG;
    int rc = check_bytes(a->a, a->a_stride, a->K);
    if (rc == ADLOCO_OK) rc = check_row_scales(a->a_scale, a->a_scale_stride, a->K);
    if (rc == ADLOCO_OK) rc = check_bytes(a->b, a->b_stride, a->K);
    if (rc != ADLOCO_OK) return rc;
    if (!elem_aligned(a->out, a->out_dtype) || !elem_aligned(a->bias, ADLOCO_F32)) return ADLOCO_ERR_ALIGNMENT;
    DeviceGuard g(ctx->device);
    return launch_blockscale_matmul(ctx, *a, static_cast<cudaStream_t>(stream));
}

int adloco_blockscale_dequantize(adloco_ctx* ctx, adloco_dtype dtype, int64_t rows, int64_t cols, const void* q,
                                 int64_t q_stride, const uint8_t* scale, int64_t scale_stride, void* x, int64_t x_stride,
                                 void* stream) {
    if (!ctx || !q || !scale || !x || rows < 1 || cols < 1 || x_stride < cols) return ADLOCO_ERR_INVALID_ARG;
    if (!known(dtype) || too_large({rows, cols})) return ADLOCO_ERR_UNSUPPORTED;
    if (!elem_aligned(x, dtype)) return ADLOCO_ERR_ALIGNMENT;
    int rc = check_bytes(q, q_stride, cols);
    if (rc == ADLOCO_OK) rc = check_row_scales(scale, scale_stride, cols);
    if (rc != ADLOCO_OK) return rc;
    if (!apart({area(x, x_stride, cols, rows, (int64_t)elem_bytes(dtype))}, {},
               {area(q, q_stride, cols, rows, 1), area(scale, scale_stride, (cols + 127) / 128, rows, 1)}))
        return ADLOCO_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    return launch_blockscale_dequantize(ctx, dtype == ADLOCO_BF16, rows, cols, q, q_stride, scale, scale_stride, x, x_stride,
                                        static_cast<cudaStream_t>(stream));
}

int adloco_linear(adloco_ctx* ctx, const adloco_linear_args* a, void* stream) {
    if (!ctx || !a || !a->y || a->M < 1 || a->N < 1 || a->K < 1 || !known_act(a->activation)) return ADLOCO_ERR_INVALID_ARG;
    if (!known(a->out_dtype) || too_large({a->M, a->N, a->K})) return ADLOCO_ERR_UNSUPPORTED;
    if (a->y_stride < a->N || (a->residual && a->residual_stride < a->N)) return ADLOCO_ERR_INVALID_ARG;
    int rc = check_operand(a->x, a->x_stride, a->K);
    if (rc == ADLOCO_OK) rc = check_operand(a->w, a->w_stride, a->K);
    if (rc == ADLOCO_OK) rc = check_kept(a->z, a->N);
    if (rc != ADLOCO_OK) return rc;
    const int64_t es = (int64_t)elem_bytes(a->out_dtype);
    if (!apart({area(a->y, a->y_stride, a->N, a->M, es), values_of(a->z, a->M, a->N), scales_of(a->z, a->M, a->N)},
               {area(a->residual, a->residual_stride, a->N, a->M, es)},
               {area(a->x, a->x_stride, a->K, a->M, 2), area(a->w, a->w_stride, a->K, a->N, 2), line(a->bias, a->N)}))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(a->y, a->out_dtype) || !elem_aligned(a->residual, a->out_dtype) || !elem_aligned(a->bias, ADLOCO_F32)) return ADLOCO_ERR_ALIGNMENT;
    DeviceGuard g(ctx->device);
    return launch_linear(ctx, *a, static_cast<cudaStream_t>(stream));
}

int adloco_linear_backward(adloco_ctx* ctx, const adloco_linear_backward_args* a, void* stream) {
    if (!ctx || !a || !a->dx || a->M < 1 || a->N < 1 || a->K < 1 || !known_act(a->activation)) return ADLOCO_ERR_INVALID_ARG;
    if (!known(a->out_dtype) || too_large({a->M, a->N, a->K})) return ADLOCO_ERR_UNSUPPORTED;
    if (a->dx_stride < a->K || (a->residual && a->residual_stride < a->K) || (a->a && a->a_stride < a->K)) return ADLOCO_ERR_INVALID_ARG;
    if (!a->z.p && (a->activation != ADLOCO_ACT_NONE || a->a)) return ADLOCO_ERR_INVALID_ARG;
    int rc = check_operand(a->dy, a->dy_stride, a->N);
    if (rc == ADLOCO_OK) rc = check_operand(a->w, a->w_stride, a->K);
    if (rc == ADLOCO_OK) rc = check_kept(a->z, a->K);
    if (rc != ADLOCO_OK) return rc;
    const int64_t es = (int64_t)elem_bytes(a->out_dtype);
    if (!apart({area(a->dx, a->dx_stride, a->K, a->M, es), area(a->a, a->a_stride, a->K, a->M, 2)},
               {area(a->residual, a->residual_stride, a->K, a->M, es), values_of(a->z, a->M, a->K)},
               {area(a->dy, a->dy_stride, a->N, a->M, 2), area(a->w, a->w_stride, a->K, a->N, 2), scales_of(a->z, a->M, a->K)}))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(a->dx, a->out_dtype) || !elem_aligned(a->residual, a->out_dtype) || !elem_aligned(a->a, ADLOCO_BF16)) return ADLOCO_ERR_ALIGNMENT;
    DeviceGuard g(ctx->device);
    return launch_linear_backward(ctx, *a, static_cast<cudaStream_t>(stream));
}

int adloco_gated_linear(adloco_ctx* ctx, const adloco_gated_linear_args* a, void* stream) {
    if (!ctx || !a || !a->a || a->M < 1 || a->d < 1 || a->f < 1 || !known_act(a->activation) || a->a_stride < a->f) return ADLOCO_ERR_INVALID_ARG;
    if (too_large({a->M, a->d, a->f})) return ADLOCO_ERR_UNSUPPORTED;
    if (!a->gate.p != !a->up.p || !a->gate.scale != !a->up.scale) return ADLOCO_ERR_INVALID_ARG;
    int rc = check_operand(a->x, a->x_stride, a->d);
    if (rc == ADLOCO_OK) rc = check_operand(a->w_gate, a->w_gate_stride, a->d);
    if (rc == ADLOCO_OK) rc = check_operand(a->w_up, a->w_up_stride, a->d);
    if (rc == ADLOCO_OK) rc = check_kept(a->gate, a->f);
    if (rc == ADLOCO_OK) rc = check_kept(a->up, a->f);
    if (rc != ADLOCO_OK) return rc;
    if (!apart({area(a->a, a->a_stride, a->f, a->M, 2), values_of(a->gate, a->M, a->f), values_of(a->up, a->M, a->f), scales_of(a->gate, a->M, a->f),
                scales_of(a->up, a->M, a->f)},
               {}, {area(a->x, a->x_stride, a->d, a->M, 2), area(a->w_gate, a->w_gate_stride, a->d, a->f, 2), area(a->w_up, a->w_up_stride, a->d, a->f, 2)}))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(a->a, ADLOCO_BF16)) return ADLOCO_ERR_ALIGNMENT;
    DeviceGuard g(ctx->device);
    return launch_gated_linear(ctx, *a, static_cast<cudaStream_t>(stream));
}

int adloco_gated_linear_backward(adloco_ctx* ctx, const adloco_gated_linear_backward_args* a, void* stream) {
    if (!ctx || !a || !a->gate.p || !a->up.p || !a->d_gate || !a->d_up || a->M < 1 || a->d < 1 || a->f < 1 || !known_act(a->activation))
        return ADLOCO_ERR_INVALID_ARG;
    if (too_large({a->M, a->d, a->f})) return ADLOCO_ERR_UNSUPPORTED;
    if (!a->gate.scale != !a->up.scale || a->d_gate_stride < a->f || a->d_up_stride < a->f || (a->a && a->a_stride < a->f)) return ADLOCO_ERR_INVALID_ARG;
    int rc = check_operand(a->dy, a->dy_stride, a->d);
    if (rc == ADLOCO_OK) rc = check_operand(a->w_down, a->w_down_stride, a->f);
    if (rc == ADLOCO_OK) rc = check_kept(a->gate, a->f);
    if (rc == ADLOCO_OK) rc = check_kept(a->up, a->f);
    if (rc != ADLOCO_OK) return rc;
    if (!apart({area(a->d_gate, a->d_gate_stride, a->f, a->M, 2), area(a->d_up, a->d_up_stride, a->f, a->M, 2), area(a->a, a->a_stride, a->f, a->M, 2)},
               {values_of(a->gate, a->M, a->f), values_of(a->up, a->M, a->f)},
               {area(a->dy, a->dy_stride, a->d, a->M, 2), area(a->w_down, a->w_down_stride, a->f, a->d, 2), scales_of(a->gate, a->M, a->f),
                scales_of(a->up, a->M, a->f)}))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(a->d_gate, ADLOCO_BF16) || !elem_aligned(a->d_up, ADLOCO_BF16) || !elem_aligned(a->a, ADLOCO_BF16)) return ADLOCO_ERR_ALIGNMENT;
    DeviceGuard g(ctx->device);
    return launch_gated_linear_backward(ctx, *a, static_cast<cudaStream_t>(stream));
}

int adloco_token_logprobs(adloco_ctx* ctx, const adloco_token_logprobs_args* a, void* stream) {
    if (!ctx || !a || !a->logits || a->rows < 1 || a->V < 1 || a->logits_stride < a->V) return ADLOCO_ERR_INVALID_ARG;
    if (!known(a->dtype) || too_large({a->rows, a->V}) || a->top > 64) return ADLOCO_ERR_UNSUPPORTED;
    if (a->top < 0 || a->top > a->V || (a->top > 0) != (a->top_values != nullptr) || (a->top > 0) != (a->top_ids != nullptr)) return ADLOCO_ERR_INVALID_ARG;
    if (a->logp && !a->targets) return ADLOCO_ERR_INVALID_ARG;
    if (!a->logp && !a->entropy && !a->lse && a->top == 0) return ADLOCO_ERR_INVALID_ARG;
    if (!apart({line(a->logp, a->rows), line(a->entropy, a->rows), line(a->lse, a->rows), line(a->top_values, a->rows * a->top),
                line(a->top_ids, a->rows * a->top)},
               {}, {area(a->logits, a->logits_stride, a->V, a->rows, (int64_t)elem_bytes(a->dtype)), line(a->targets, a->rows)}))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(a->logits, a->dtype) || !elem_aligned(a->targets, ADLOCO_F32) || !elem_aligned(a->logp, ADLOCO_F32) ||
        !elem_aligned(a->entropy, ADLOCO_F32) || !elem_aligned(a->lse, ADLOCO_F32) || !elem_aligned(a->top_values, ADLOCO_F32) ||
        !elem_aligned(a->top_ids, ADLOCO_F32))
        return ADLOCO_ERR_ALIGNMENT;
    DeviceGuard g(ctx->device);
    return launch_token_logprobs(ctx, *a, static_cast<cudaStream_t>(stream));
}

int adloco_token_logprobs_backward(adloco_ctx* ctx, const adloco_token_logprobs_backward_args* a, void* stream) {
    if (!ctx || !a || !a->logits || !a->targets || !a->lse || !a->d_logp || !a->d_logits || a->rows < 1 || a->V < 1) return ADLOCO_ERR_INVALID_ARG;
    if (!known(a->dtype) || too_large({a->rows, a->V})) return ADLOCO_ERR_UNSUPPORTED;
    if (a->logits_stride < a->V || a->d_logits_stride < a->V || !a->entropy != !a->d_entropy) return ADLOCO_ERR_INVALID_ARG;
    const int64_t es = (int64_t)elem_bytes(a->dtype);
    if (!apart({area(a->d_logits, a->d_logits_stride, a->V, a->rows, es)}, {area(a->logits, a->logits_stride, a->V, a->rows, es)},
               {line(a->targets, a->rows), line(a->lse, a->rows), line(a->d_logp, a->rows), line(a->entropy, a->rows), line(a->d_entropy, a->rows)}))
        return ADLOCO_ERR_INVALID_ARG;
    if (!elem_aligned(a->logits, a->dtype) || !elem_aligned(a->d_logits, a->dtype) || !elem_aligned(a->targets, ADLOCO_F32) ||
        !elem_aligned(a->lse, ADLOCO_F32) || !elem_aligned(a->d_logp, ADLOCO_F32) || !elem_aligned(a->entropy, ADLOCO_F32) ||
        !elem_aligned(a->d_entropy, ADLOCO_F32))
        return ADLOCO_ERR_ALIGNMENT;
    DeviceGuard g(ctx->device);
    return launch_token_logprobs_backward(ctx, *a, static_cast<cudaStream_t>(stream));
}

}  // extern "C"

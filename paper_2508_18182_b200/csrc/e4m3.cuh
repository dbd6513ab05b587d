// Blocks of 128 numbers in 8 bits (e4m3) with a power-of-two scale, its biased exponent in a byte.
#pragma once

#include <stdint.h>

namespace adloco {
namespace {

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
__device__ __forceinline__ float scale_of(uint32_t byte) {                          // 2^(byte - 127); 255: NaN
    return byte == 255u ? __uint_as_float(0x7fffffffu) : byte == 0u ? 0x1p-127f : __uint_as_float(byte << 23);
}

}  // namespace
}  // namespace adloco

// The 8-bit caches' numbers: e4m3 values of a row (one token of one KV head) that all stand
// for themselves times a power of two, held as an e8m0 byte (the exponent + 127).  The power
// is the smallest 2^e, e in [-60, 119], with max |x| <= 448 * 2^e, so the largest value meets
// e4m3's largest number and no sum or product is needed to scale: x * 2^-e is exact, and the
// one rounding is that to e4m3 (half a step: 2^-4 of the value, 2^-10 of the power for values
// below 2^-6 of it).  A power per row costs one byte beside 64 or 128.  The exponents are
// kept where value * power and their bf16 forms are normal numbers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace atf {
namespace q8 {

constexpr uint32_t kMinByte = 127 - 60, kMaxByte = 127 + 119;
constexpr uint32_t kInfBits = 0x7F800000u;

// The byte of a row whose largest finite magnitude has these fp32 bits: 448 = 1.75 * 2^8, so
// a significand above 1.75 takes the next power.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
    const uint32_t e = (amax_bits + 0x1FFFFFu) >> 23;  // biased exponent, + 1 above 1.75
    return min(max(e, kMinByte + 8u) - 8u, kMaxByte);
}

// 2^-e of a byte e + 127, and 2^e (bytes 1 .. 254)
__device__ __forceinline__ float inverse_power(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float power(uint32_t byte) { return __uint_as_float(byte << 23); }

// Magnitudes whose largest has bits up to here are finite and meet 448 or less: nearly all
// rows, whose numbers need no more than the product (kPlain below).
constexpr uint32_t kPlainBits = (kMaxByte + 8) << 23 | 0x600000u;  // 448 * 2^119

// x scaled by 2^-e, ready to be rounded: in range (the clamp binds at the largest power only),
// and NaN where x is not finite
template <bool kPlain>
__device__ __forceinline__ float scaled(float x, float inv) {
    if constexpr (kPlain) return x * inv;
    const float y = __builtin_amdgcn_fmed3f(x * inv, -448.f, 448.f);
    return fabsf(x) < INFINITY ? y : __uint_as_float(0x7FC00000u);
}

// four e4m3 numbers, round to nearest even
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true));
}

// two of them into the low (0) or the high half of a word
template <int kHigh>
__device__ __forceinline__ uint32_t pack2(float a, float b, uint32_t word) {
    return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, int(word), kHigh != 0));
}

}  // namespace q8
}  // namespace atf

// Activations in 8 bits: e4m3 codes with one power of two for each 32 consecutive values of a row (8.25 bits a value).
//     scale = 2^e,  e the smallest integer with max |x| <= 448 * 2^e (at least -127),  code = e4m3(x / scale)
// Division by a power of two is exact, so a value is rounded once, to nearest even.  The group of 32 is what one thread
// of a matrix product's epilogue holds of a row: its maximum needs no exchange between threads, and e4m3's own exponent
// takes care of what varies inside it.  A power of two instead of an fp32 factor costs up to one bit of range, not of
// mantissa, and a byte instead of four.
#pragma once
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace dynbatch {
namespace ck8 {

constexpr int kGroup = 32;

// e + 127 of a group whose largest finite magnitude has these bits: 448 = 1.75 * 2^8, so a mantissa above 1.75 needs
// one power more.
__device__ __forceinline__ uint32_t scale_byte(float top) {
    const int e = static_cast<int>((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 8;
    return static_cast<uint32_t>(e < 0 ? 0 : e);
}
__device__ __forceinline__ float scale_value(uint32_t byte) {  // 2^(byte - 127); byte 0 is the subnormal 2^-127, 255 a NaN
    return __uint_as_float(byte == 0 ? 0x400000u : byte == 255 ? 0x7FFFFFFFu : byte << 23);
}
__device__ __forceinline__ float scale_inverse(uint32_t byte) {  // 2^(127 - byte), for byte <= 247
    return __uint_as_float((254u - byte) << 23);
}
// Codes of four scaled values; a NaN gets the code NaN.
__device__ __forceinline__ uint32_t codes_of_finite(float a, float b, float c, float d) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
__device__ __forceinline__ float finite_magnitude(float x) {  // 0 for what is not finite
    const float m = fabsf(x);
    return m < __uint_as_float(0x7F800000u) ? m : 0.f;
}
// The same for any values, not yet scaled: infinities get the code NaN too, and with the largest scale, 2^120, the codes
// from 256 on would stand for 2^128 and more, so finite values stop at 240 there.
constexpr uint32_t kTopByte = 247;
__device__ __forceinline__ float held(float x, float inverse, uint32_t byte) {
    const float m = fabsf(x), y = x * inverse;
    if (!(m < __uint_as_float(0x7F800000u))) return __uint_as_float(0x7FFFFFFFu);
    return byte >= kTopByte && fabsf(y) > 240.f ? copysignf(240.f, y) : y;
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float inverse, uint32_t byte) {
    return codes_of_finite(held(a, inverse, byte), held(b, inverse, byte), held(c, inverse, byte), held(d, inverse, byte));
}
__device__ __forceinline__ float2 values2(uint32_t two_codes) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two_codes & 0xFFFFu), __NV_E4M3);
    return __half22float2(__half2(h));
}

}  // namespace ck8
}  // namespace dynbatch

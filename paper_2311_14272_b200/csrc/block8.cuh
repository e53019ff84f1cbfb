// Device-side arithmetic of the 8-bit forms: largest magnitudes of bf16 pairs, exponents, codes.
#pragma once

#include <cuda_fp8.h>
#include <stdint.h>

namespace crisp {
namespace block8 {

__device__ __forceinline__ float2 floats(uint32_t pair) { return make_float2(__uint_as_float(pair << 16), __uint_as_float(pair & 0xFFFF0000u)); }
// The larger magnitudes of two pairs of bf16, as their bits (NaN if one is).
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t pair) {
    uint32_t r;
    asm("{\n\t.reg .b32 m;\n\tabs.bf16x2 m, %2;\n\tmax.NaN.bf16x2 %0, %1, m;\n\t}" : "=r"(r) : "r"(a), "r"(pair));
    return r;
}
__device__ __forceinline__ uint32_t larger_of(uint32_t a) { return max(a & 0xFFFFu, a >> 16); }
// What is not finite becomes NaN and leaves the block's largest value alone: the pair with zeros in its place.
__device__ __forceinline__ uint32_t finite(uint32_t pair) {
    if ((pair & 0x7F80u) == 0x7F80u) pair &= 0xFFFF0000u;
    if ((pair & 0x7F800000u) == 0x7F800000u) pair &= 0xFFFFu;
    return pair;
}
__device__ __forceinline__ uint32_t nan_for_infinity(uint32_t pair) {
    if ((pair & 0x7F80u) == 0x7F80u) pair |= 0x7FFFu;
    if ((pair & 0x7F800000u) == 0x7F800000u) pair |= 0x7FFF0000u;
    return pair;
}
// Biased exponent (E + 127) for a largest magnitude given as bf16 bits: its own exponent less 8, one more where its fraction is above 448's.
__device__ __forceinline__ uint32_t exponent_of(uint32_t bits) { return (uint32_t)max((int)((bits + (0x7Fu - 0x60u)) >> 7) - 8, 1); }
__device__ __forceinline__ uint32_t codes2(uint32_t pair, float down) {
    const float2 v = floats(pair);
    return __nv_cvt_float2_to_fp8x2(make_float2(v.x * down, v.y * down), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float power_of(uint32_t biased) { return __uint_as_float(biased << 23); }

}  // namespace block8
}  // namespace crisp

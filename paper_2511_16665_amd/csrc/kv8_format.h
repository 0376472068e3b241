// How rows become codes and exponent bytes of the 8-bit cache (kv8.hip states the format).
#pragma once
#include "dev_common.h"

namespace tlt {

// exponent byte of a row from the largest bit pattern of its magnitudes: 448 = 1.75 * 2^8
__device__ __forceinline__ uint32_t exponent_of(uint32_t amax_bits) {
    if (amax_bits >= 0x7f800000u) return 255u;
    const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return (uint32_t)max(e, 1);
}
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23); }          // 2^(e - 127)
// 2^(127 - e): e is 248 at most for finite rows, so this is a normal number, and 0 for e = 255 (rows that are not finite: see encode4)
__device__ __forceinline__ float inverse_scale_of(uint32_t e) { return __uint_as_float(e == 255u ? 0u : (254u - e) << 23); }
// four codes: round to nearest, ties to even
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv) {
    if (inv == 0.f) return 0u;
    uint32_t w = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, (int)w, true);
}

}  // namespace tlt

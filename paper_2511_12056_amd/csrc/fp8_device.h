// Device helpers for 8-bit floating point with power-of-two scales.
#pragma once
#include <hip/hip_runtime.h>
#include "train_device.h"

namespace pda {

// |x|, 0 for what is not finite: magnitudes that a scale goes by.
__device__ __forceinline__ float finite_magnitude(float x) {
    const unsigned u = __float_as_uint(x) & 0x7fffffffu;
    return __uint_as_float(u < 0x7f800000u ? u : 0u);
}
// The scale of a block whose largest finite magnitude is `top`, as 127 + e: the smallest e >= -127 with top <= 1.75 * 2^(LOG + e), where 1.75 * 2^LOG is
// the type's largest value; e = 0 for a block of zeros.  From the exponent and the mantissa (1.75 is 0x600000), so exact.
template <bool E5M2>
__device__ __forceinline__ unsigned scale_byte(float top) {
    const unsigned u = __float_as_uint(top);
    const int e = (int)(u >> 23) - (E5M2 ? 15 : 8) + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return u == 0u ? 127u : (unsigned)(e > 0 ? e : 0);         // at most 254 - 8 + 1
}
// 1 over the scale: 2^(127 - byte), a normal number for every byte that scale_byte gives.
__device__ __forceinline__ float inverse_scale(unsigned byte) { return __uint_as_float((254u - byte) << 23); }

// Four values, none beyond e4m3's largest but those that are not finite, to four bytes of it, nearest even.
__device__ __forceinline__ unsigned pack_e4m3(float a, float b, float c, float d) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    return (unsigned)r;
}

// Maximum over groups of 32 consecutive lanes, in every lane of the group.
__device__ __forceinline__ float lane_max32(float x) {
    x = fmaxf(x, lane_perm<0xB1>(x));
    x = fmaxf(x, lane_perm<0x4E>(x));
    x = fmaxf(x, lane_perm<0x141>(x));
    x = fmaxf(x, lane_perm<0x140>(x));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

}  // namespace pda

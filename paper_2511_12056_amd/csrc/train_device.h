// Device helpers of the training operators.
#pragma once
#include <hip/hip_runtime.h>
#include "attn_device.h"

namespace pda {

template <int CTRL>
__device__ __forceinline__ float lane_perm(float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
// Sum over groups of N consecutive lanes (N = 8, 16, 32, 64), in every lane of the group; registers only, a fixed order.
template <int N>
__device__ __forceinline__ float lane_sum(float x) {
    x += lane_perm<0xB1>(x);                  // quad_perm [1,0,3,2]: lane ^ 1
    x += lane_perm<0x4E>(x);                  // quad_perm [2,3,0,1]: lane ^ 2
    x += lane_perm<0x141>(x);                 // row_half_mirror: the other quad of each 8
    if constexpr (N >= 16) x += lane_perm<0x140>(x);        // row_mirror: the other half of each 16
    if constexpr (N >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (N >= 64) x = pair_sum(x);
    return x;
}

// The lane's index, formed anew where it is used: the compiler cannot trace two of them back to each other, so it keeps nothing
// derived from it in registers in between.
__device__ __forceinline__ int opaque_lane() {
    int lane;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(lane));
    return lane;
}

__device__ __forceinline__ float bf16_lo(unsigned x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(unsigned x) { return __uint_as_float(x & 0xffff0000u); }

}  // namespace pda

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

// Sum of the squares of a d-vector, four columns of it in each of its LPV lanes.
template <int LPV>
__device__ __forceinline__ float sum_of_squares(const float4& a) { return lane_sum<LPV>(a.x * a.x + a.y * a.y + a.z * a.z + a.w * a.w); }
// What a vector is to be multiplied by, before its squares are summed again and it is divided by their root, where the sum is not 0 but so small that single squares
// have lost bits, or past fp32's range; 1 elsewhere.  Exact (columns that this takes below the normal numbers are nothing beside the largest).
__device__ __forceinline__ float into_range(float ss) { return ss > 0.f && ss < 0x1p-100f ? 0x1p60f : ss == __builtin_huge_valf() ? 0x1p-80f : 1.f; }

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

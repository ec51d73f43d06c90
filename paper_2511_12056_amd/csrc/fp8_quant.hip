// Quantisation to 8 bits with power-of-two scales, bound by HBM: a workgroup holds a 128 x 128 tile in registers, finds the largest magnitude of its rows, of
// its columns or of all of it, and writes it in both orders, so that x is read once.
//
// A thread holds 4 consecutive columns of 16 rows: rows 32 i + 4 (thread / 32) + j, so that four rows of a column are one thread's and become one word of the
// transposed tile, which goes through LDS.  Rows lie 33 words apart there: 32 lanes that write one word each of every fourth row meet 16 of 64 banks.
//
// Workgroups go to the eight XCDs in turn, each with an L2 of its own; 4 x 4 tiles that share words of the scales (a byte a row and tile) are therefore given to
// workgroups of one XCD that run side by side.
#include <hip/hip_runtime.h>
#include "attn_internal.h"
#include "fp8_device.h"
#include "proj_internal.h"

namespace pda {

template <typename T, bool VEC>
__device__ __forceinline__ void load4(const T* p, int n, float (&x)[4]) {        // n <= 0: none
    if constexpr (VEC) {
        if (n > 0) {                                            // (a row's end lies behind whole groups)
            if constexpr (sizeof(T) == 4) {
                const f32x4 v = __builtin_nontemporal_load(reinterpret_cast<const f32x4*>(p));
                x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
            } else {
                const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(p));
                x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) x[e] = (float)p[e];
    }
}

template <typename T, bool VEC, bool E5M2>
__global__ __launch_bounds__(256) void fp8_quant_kernel(const QuantParams p, int64_t tiles_r, int64_t tiles_c) {
    constexpr int PITCH = 33;
    __shared__ unsigned turned[128 * PITCH];
    __shared__ float tops[8][128];
    // tile of this workgroup: blocks of 4 x 4 tiles, consecutive workgroups of one XCD (every eighth) side by side in a block
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, blocks_c = (tiles_c + 3) / 4;
    const int64_t blk = id / 128 * 8 + id % 8;
    const int in = (int)(id / 8 % 16);
    const int64_t tr = blk / blocks_c * 4 + in / 4, tc = blk % blocks_c * 4 + in % 4;
    if (tr >= tiles_r || tc >= tiles_c) return;
    const int t = threadIdx.x, l = t & 31, w = t >> 5;
    const int64_t r0 = tr * 128 + 4 * w, c0 = tc * 128 + 4 * l;
    const int n = c0 < p.cols ? (int)(p.cols - c0 < 4 ? p.cols - c0 : 4) : 0;
    float x[4][4][4];                                           // [i][j][column]
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t r = r0 + 32 * i + j;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][j][e] = 0.f;
            load4<T, VEC>(static_cast<const T*>(p.x) + r * p.ldx + c0, r < p.rows ? n : 0, x[i][j]);
        }
    const int64_t q_cols = fp8_cols(p.cols), qt_cols = fp8_cols(p.rows);
    const int64_t q_sc = fp8_scale_cols(p.cols), qt_sc = fp8_scale_cols(p.rows);
    unsigned square_byte = 127;
    if (p.square) {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, finite_magnitude(x[i][j][e]));
        top = lane_max<32>(top);
        if (l == 0) tops[0][w] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, tops[0][i]);
        square_byte = scale_byte<E5M2>(top);
        if (t == 0) {
            if (p.q) p.q_scales[tr * q_sc + tc] = (uint8_t)square_byte;
            if (p.qt) p.qt_scales[tc * qt_sc + tr] = (uint8_t)square_byte;
        }
    }
    if (p.q) {
        unsigned char* q = static_cast<unsigned char*>(p.q);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t r = r0 + 32 * i + j;
                float(&v)[4] = x[i][j];
                unsigned byte = square_byte;
                if (!p.square) byte = scale_byte<E5M2>(lane_max<32>(fmaxf(fmaxf(finite_magnitude(v[0]), finite_magnitude(v[1])), fmaxf(finite_magnitude(v[2]), finite_magnitude(v[3])))));
                const float f = inverse_scale(byte);
                if (r < p.rows) {
                    __builtin_nontemporal_store(pack_fp8<E5M2>(v[0] * f, v[1] * f, v[2] * f, v[3] * f), reinterpret_cast<unsigned*>(q + r * q_cols + c0));
                    if (!p.square && l == 0) p.q_scales[r * q_sc + tc] = (uint8_t)byte;
                }
            }
    }
    if (!p.qt) return;
    float f[4];
    if (p.square) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = inverse_scale(square_byte);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = fmaxf(top, finite_magnitude(x[i][j][e]));
            f[e] = top;
        }
        *reinterpret_cast<f32x4*>(&tops[w][4 * l]) = f32x4{f[0], f[1], f[2], f[3]};
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[e] = fmaxf(f[e], tops[i][4 * l + e]);
            const unsigned byte = scale_byte<E5M2>(f[e]);
            f[e] = inverse_scale(byte);
            if (w == 0 && c0 + e < p.cols) p.qt_scales[(c0 + e) * qt_sc + tr] = (uint8_t)byte;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            turned[(4 * l + e) * PITCH + 8 * i + w] = pack_fp8<E5M2>(x[i][0][e] * f[e], x[i][1][e] * f[e], x[i][2][e] * f[e], x[i][3][e] * f[e]);
    __syncthreads();
    unsigned char* qt = static_cast<unsigned char*>(p.qt) + tr * 128 + 4 * l;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int c = 8 * i + w;
        const int64_t col = tc * 128 + c;
        if (col < p.cols) __builtin_nontemporal_store(turned[c * PITCH + l], reinterpret_cast<unsigned*>(qt + col * qt_cols));
    }
}

template <typename T, bool VEC>
static hipError_t launch_quant(const QuantParams& p, hipStream_t st) {
    const int64_t tr = (p.rows + 127) / 128, tc = (p.cols + 127) / 128;
    const int64_t blocks = (tr + 3) / 4 * ((tc + 3) / 4), n = (blocks + 7) / 8 * 128;     // whole rounds of eight blocks of 16 tiles
    const int64_t gx = n < 1 << 23 ? n : 1 << 23;                                       // a launch has fewer than 2^32 threads along x
    const dim3 grid((unsigned)gx, (unsigned)((n + gx - 1) / gx));
    if (p.e5m2) hipLaunchKernelGGL((fp8_quant_kernel<T, VEC, true>), grid, dim3(256), 0, st, p, tr, tc);
    else hipLaunchKernelGGL((fp8_quant_kernel<T, VEC, false>), grid, dim3(256), 0, st, p, tr, tc);
    return hipGetLastError();
}

hipError_t launch_fp8_quant(const QuantParams& p, hipStream_t st) {
    const int64_t size = p.x_bf16 ? 2 : 4;
    const bool vec = p.cols % 4 == 0 && p.ldx % 4 == 0 && reinterpret_cast<uintptr_t>(p.x) % (4 * size) == 0;
    if (p.x_bf16) return vec ? launch_quant<__bf16, true>(p, st) : launch_quant<__bf16, false>(p, st);
    return vec ? launch_quant<float, true>(p, st) : launch_quant<float, false>(p, st);
}

}  // namespace pda

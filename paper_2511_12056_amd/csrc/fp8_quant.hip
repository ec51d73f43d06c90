// Quantisation to 8 bits with power-of-two scales, bound by HBM: a workgroup holds a 128 x 128 tile in registers, finds the largest magnitude of its rows, of
// its columns or of all of it, and writes it in both orders, so that x is read once.
//
// What takes time beside memory is the arithmetic on each value, so there is little of it.  bf16 stays in pairs: magnitudes are 16-bit integers (as such ordered like
// the values, with what is not finite above all of them, so only tiles that hold some look at each), and v_cvt_scalef32_pk divides by the scale and rounds two at
// once.  With each value widened, filtered, multiplied and packed by itself, 119 056 x 1 536 to both orders took 219 us instead of 138 (5.3 TB/s, what a copy reaches).
//
// A thread holds 8 consecutive columns of 8 consecutive rows: 8 values of a row are 8 bytes of q, and those of a column 8 bytes of the transposed tile, which goes
// through LDS, its granules of 16 bytes swizzled by the column's block of 8.
//
// Workgroups go to the eight XCDs in turn, each with an L2 of its own; 4 x 4 tiles that share words of the scales (a byte a row and tile) are therefore given to
// workgroups of one XCD that run side by side.
#include <hip/hip_runtime.h>
#include "attn_internal.h"
#include "fp8_device.h"
#include "proj_internal.h"

namespace pda {

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// Eight consecutive values of a row in W words, and magnitudes of all values of a word at once.
template <typename T> struct Held;
template <> struct Held<__bf16> {
    static constexpr int W = 4;
    typedef u32x4 Piece __attribute__((aligned(2)));
    static __device__ __forceinline__ unsigned magnitude(unsigned x) { return x & 0x7fff7fffu; }
    static __device__ __forceinline__ unsigned larger(unsigned a, unsigned b) {
        return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    }
    static __device__ __forceinline__ unsigned finite(unsigned m) { return ((m & 0xffffu) < 0x7f80u ? m & 0xffffu : 0u) | (m < 0x7f800000u ? m & 0xffff0000u : 0u); }
    static __device__ __forceinline__ unsigned one(unsigned m) { return (m > m << 16 ? m : m << 16) & 0xffff0000u; }      // the largest of a word, as fp32's bits
};
template <> struct Held<float> {
    static constexpr int W = 8;
    typedef u32x4 Piece __attribute__((aligned(4)));
    static __device__ __forceinline__ unsigned magnitude(unsigned x) { return x & 0x7fffffffu; }
    static __device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }
    static __device__ __forceinline__ unsigned finite(unsigned m) { return m < 0x7f800000u ? m : 0u; }
    static __device__ __forceinline__ unsigned one(unsigned m) { return m; }
};

// n < 8 at a row's end; n <= 0: none.  Rows of any length start at any element.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, unsigned (&x)[Held<T>::W]) {
    if (n == 8) {
#pragma unroll
        for (int i = 0; i < Held<T>::W / 4; ++i) {
            const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const typename Held<T>::Piece*>(p) + i);
            x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) {
                if constexpr (sizeof(T) == 4) x[e] = __float_as_uint(p[e]);
                else x[e / 2] |= (unsigned)__builtin_bit_cast(unsigned short, p[e]) << (16 * (e % 2));
            }
    }
}

// Four values over a scale (the exponent of `scale`), to four bytes, nearest even; none is beyond the type's largest but those that are not finite.
template <bool E5M2>
__device__ __forceinline__ unsigned to_fp8(unsigned ab, unsigned cd, float scale) {
    const bf16x2 x = __builtin_bit_cast(bf16x2, ab), y = __builtin_bit_cast(bf16x2, cd);
    s16x2 r = {0, 0};
    if constexpr (E5M2) {
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, x, scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(r, y, scale, true);
    } else {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, x, scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, y, scale, true);
    }
    return __builtin_bit_cast(unsigned, r);
}
template <bool E5M2>
__device__ __forceinline__ unsigned to_fp8(unsigned a, unsigned b, unsigned c, unsigned d, float scale) {
    s16x2 r = {0, 0};
    if constexpr (E5M2) {
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, __uint_as_float(a), __uint_as_float(b), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, __uint_as_float(c), __uint_as_float(d), scale, true);
    } else {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(a), __uint_as_float(b), scale, false);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(c), __uint_as_float(d), scale, true);
    }
    return __builtin_bit_cast(unsigned, r);
}

template <int CTRL>
__device__ __forceinline__ unsigned word_perm(unsigned x) { return __builtin_amdgcn_update_dpp(0u, x, CTRL, 0xF, 0xF, false); }

template <typename T, bool E5M2>
__global__ __launch_bounds__(256) void fp8_quant_kernel(const QuantParams p, int64_t tiles_r, int64_t tiles_c) {
    using H = Held<T>;
    constexpr int W = H::W;
    __shared__ __attribute__((aligned(16))) unsigned char turned[128 * 128];
    __shared__ __attribute__((aligned(16))) unsigned col_tops[4][128], row_scales[128], col_scales[128];      // scales as fp32 with the exponent alone
    // tile of this workgroup: blocks of 4 x 4 tiles, consecutive workgroups of one XCD (every eighth) side by side in a block
    const int64_t id = (int64_t)blockIdx.y * gridDim.x + blockIdx.x, blocks_c = (tiles_c + 3) / 4;
    const int64_t blk = id / 128 * 8 + id % 8;
    const int in = (int)(id / 8 % 16);
    const int64_t tr = blk / blocks_c * 4 + in / 4, tc = blk % blocks_c * 4 + in % 4;
    if (tr >= tiles_r || tc >= tiles_c) return;
    const int t = threadIdx.x, l = t & 15, rg = t >> 4, w = t >> 6;
    const int64_t r0 = tr * 128 + 8 * rg, c0 = tc * 128 + 8 * l;
    const int n = c0 < p.cols ? (int)(p.cols - c0 < 8 ? p.cols - c0 : 8) : 0, rows = (int)(p.rows - r0 < 8 ? p.rows - r0 : 8);
    unsigned x[8][W];
    const T* px = static_cast<const T*>(p.x) + r0 * p.ldx + c0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
#pragma unroll
        for (int k = 0; k < W; ++k) x[j][k] = 0u;
        load8<T>(px + j * p.ldx, j < rows ? n : 0, x[j]);
    }
    unsigned rt[8], ct[W];                                      // largest magnitudes of the thread's rows (two columns of bf16 a word) and columns
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const unsigned m = H::magnitude(x[j][k]);
            rt[j] = k ? H::larger(rt[j], m) : m;
            ct[k] = j ? H::larger(ct[k], m) : m;
        }
    unsigned most = ct[0];
#pragma unroll
    for (int k = 1; k < W; ++k) most = H::larger(most, ct[k]);
    if (__any(H::one(most) >= 0x7f800000u)) {                   // magnitudes of what is finite alone
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const unsigned m = H::finite(H::magnitude(x[j][k]));
                rt[j] = k ? H::larger(rt[j], m) : m;
                ct[k] = j ? H::larger(ct[k], m) : m;
            }
        most = ct[0];
#pragma unroll
        for (int k = 1; k < W; ++k) most = H::larger(most, ct[k]);
    }
    const int64_t q_cols = fp8_cols(p.cols), qt_cols = fp8_cols(p.rows);
    const int64_t q_sc = fp8_scale_cols(p.cols), qt_sc = fp8_scale_cols(p.rows);
    if (p.square) {
        const float top = pair_max(lane_max32(__uint_as_float(H::one(most))));
        if ((t & 63) == 0) col_tops[w][0] = __float_as_uint(top);
        __syncthreads();
        float all = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) all = fmaxf(all, __uint_as_float(col_tops[i][0]));
        const unsigned byte = scale_byte<E5M2>(all);
        if (t == 0) {
            if (p.q) p.q_scales[tr * q_sc + tc] = (uint8_t)byte;
            if (p.qt) p.qt_scales[tc * qt_sc + tr] = (uint8_t)byte;
        }
        if (t < 128) row_scales[t] = col_scales[t] = byte << 23;
    } else {
        // rows: three steps over the 16 lanes halve the number of rows a lane deals with, and the fourth joins the two lanes of a row, row lane / 2 of the eight
        const bool b3 = t & 8, b2 = t & 4, b1 = t & 2;
#pragma unroll
        for (int j = 0; j < 4; ++j) rt[j] = H::larger(b3 ? rt[j + 4] : rt[j], word_perm<0x140>(b3 ? rt[j] : rt[j + 4]));        // lane 15 - l
#pragma unroll
        for (int j = 0; j < 2; ++j) rt[j] = H::larger(b2 ? rt[j + 2] : rt[j], word_perm<0x141>(b2 ? rt[j] : rt[j + 2]));        // lane 7 - l of eight
        rt[0] = H::larger(b1 ? rt[1] : rt[0], word_perm<0x4E>(b1 ? rt[0] : rt[1]));                                             // lane ^ 2
        rt[0] = H::larger(rt[0], word_perm<0xB1>(rt[0]));                                                                       // lane ^ 1
        row_scales[8 * rg + l / 2] = scale_byte<E5M2>(__uint_as_float(H::one(rt[0]))) << 23;
        // columns: over the four lanes of a wavefront that share them, then over the wavefronts
#pragma unroll
        for (int k = 0; k < W; ++k) {
            const auto a = __builtin_amdgcn_permlane16_swap(ct[k], ct[k], false, false);
            ct[k] = H::larger(a[0], a[1]);
            const auto b = __builtin_amdgcn_permlane32_swap(ct[k], ct[k], false, false);
            ct[k] = H::larger(b[0], b[1]);
        }
        if ((t & 48) == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *reinterpret_cast<u32x4*>(&col_tops[w][8 * l + 4 * i]) = W == 4 ? u32x4{ct[2 * i % W] << 16, ct[2 * i % W] & 0xffff0000u, ct[(2 * i + 1) % W] << 16, ct[(2 * i + 1) % W] & 0xffff0000u}
                                                                               : u32x4{ct[4 * i % W], ct[(4 * i + 1) % W], ct[(4 * i + 2) % W], ct[(4 * i + 3) % W]};
        }
        __syncthreads();
        if (t < 128) {
            if (p.qt) {
                unsigned top = col_tops[0][t];
#pragma unroll
                for (int i = 1; i < 4; ++i) top = col_tops[i][t] > top ? col_tops[i][t] : top;
                const unsigned byte = scale_byte<E5M2>(__uint_as_float(top));
                col_scales[t] = byte << 23;
                if (tc * 128 + t < p.cols) p.qt_scales[(tc * 128 + t) * qt_sc + tr] = (uint8_t)byte;
            }
        } else if (p.q && tr * 128 + t - 128 < p.rows) {
            p.q_scales[(tr * 128 + t - 128) * q_sc + tc] = (uint8_t)(row_scales[t - 128] >> 23);
        }
    }
    __syncthreads();
    if (p.q) {
        unsigned char* q = static_cast<unsigned char*>(p.q) + r0 * q_cols + c0;
        float f[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(&row_scales[8 * rg + 4 * i]);
            f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            u32x2 v;
            if constexpr (W == 4) v = u32x2{to_fp8<E5M2>(x[j][0], x[j][1], f[j]), to_fp8<E5M2>(x[j][2], x[j][3], f[j])};
            else v = u32x2{to_fp8<E5M2>(x[j][0], x[j][1], x[j][2], x[j][3], f[j]), to_fp8<E5M2>(x[j][4], x[j][5], x[j][6], x[j][7], f[j])};
            if (j < rows) __builtin_nontemporal_store(v, reinterpret_cast<u32x2*>(q + j * q_cols));
        }
    }
    if (!p.qt) return;
    {
        float f[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(&col_scales[8 * l + 4 * i]);
            f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
        }
        unsigned char* to = turned + 8 * l * 128 + ((rg / 2) ^ (l & 7)) * 16 + rg % 2 * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u32x2 v;
            if constexpr (W == 4) {                             // rows 2i and 2i + 1 of column e: the lower or upper halves of two words
                constexpr unsigned lower = 0x05040100u, upper = 0x07060302u;
                unsigned pairs[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) pairs[i] = __builtin_amdgcn_perm(x[2 * i + 1][e / 2], x[2 * i][e / 2], e % 2 ? upper : lower);
                v = u32x2{to_fp8<E5M2>(pairs[0], pairs[1], f[e]), to_fp8<E5M2>(pairs[2], pairs[3], f[e])};
            } else {
                v = u32x2{to_fp8<E5M2>(x[0][e % W], x[1][e % W], x[2][e % W], x[3][e % W], f[e]), to_fp8<E5M2>(x[4][e % W], x[5][e % W], x[6][e % W], x[7][e % W], f[e])};
            }
            *reinterpret_cast<u32x2*>(to + e * 128) = v;
        }
    }
    __syncthreads();
    unsigned char* qt = static_cast<unsigned char*>(p.qt) + tr * 128 + (t & 7) * 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = 32 * i + t / 8;
        const int64_t col = tc * 128 + c;
        if (col < p.cols) __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(turned + c * 128 + ((t & 7) ^ (c / 8 & 7)) * 16), reinterpret_cast<u32x4*>(qt + col * qt_cols));
    }
}

template <typename T>
static hipError_t launch_quant(const QuantParams& p, hipStream_t st) {
    const int64_t tr = (p.rows + 127) / 128, tc = (p.cols + 127) / 128;
    const int64_t blocks = (tr + 3) / 4 * ((tc + 3) / 4), n = (blocks + 7) / 8 * 128;     // whole rounds of eight blocks of 16 tiles
    const int64_t gx = n < 1 << 23 ? n : 1 << 23;                                       // a launch has fewer than 2^32 threads along x
    const dim3 grid((unsigned)gx, (unsigned)((n + gx - 1) / gx));
    if (p.e5m2) hipLaunchKernelGGL((fp8_quant_kernel<T, true>), grid, dim3(256), 0, st, p, tr, tc);
    else hipLaunchKernelGGL((fp8_quant_kernel<T, false>), grid, dim3(256), 0, st, p, tr, tc);
    return hipGetLastError();
}

hipError_t launch_fp8_quant(const QuantParams& p, hipStream_t st) {
    return p.x_bf16 ? launch_quant<__bf16>(p, st) : launch_quant<float>(p, st);
}

}  // namespace pda

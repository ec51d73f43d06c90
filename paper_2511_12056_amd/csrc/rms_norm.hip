// Root-mean-square norm, forward (with the residual's addition in front and 8-bit results behind) and backward, bound by HBM: every element is
// read once, held in fp32 registers across the sum over its row, and written once.  Threads of a row, accesses and the backward pass's sums over
// rows as in layer_norm.hip, where the reasons stand.
//
// Forward, the types of x, the residual and y are branches that all threads take alike (36 combinations of them would otherwise be as many kernels
// a row length); an access by groups of four keeps a block of 128 columns in 32 consecutive lanes, whose largest magnitude five lane permutations find.
//
// 119 056 x 1 536: forward, bf16 x and fp32 stream to 8 bits, 347 us (5.8 TB/s); backward, bf16 dy, fp32 h and dres, 471 us (5.5 TB/s; 6 us of them the second kernel).
#include <hip/hip_runtime.h>
#include "attn_internal.h"
#include "fp8_device.h"
#include "proj_internal.h"
#include "row_io.h"

namespace pda {

template <bool VEC, int TPR, int NV>
__device__ __forceinline__ void load_row(const void* p, int type, int64_t at, int D, int t, float (&x)[NV][4]) {
    if (type == PDA_BF16) RowIO<__bf16, VEC, TPR, NV>::load(static_cast<const __bf16*>(p) + at, D, t, x);
    else RowIO<float, VEC, TPR, NV>::load(static_cast<const float*>(p) + at, D, t, x);
}
template <bool VEC, int TPR, int NV>
__device__ __forceinline__ void store_row(void* p, int type, int64_t at, int D, int t, const float (&x)[NV][4]) {
    if (type == PDA_BF16) RowIO<__bf16, VEC, TPR, NV>::store(static_cast<__bf16*>(p) + at, D, t, x);
    else RowIO<float, VEC, TPR, NV>::store(static_cast<float*>(p) + at, D, t, x);
}

// A block's largest value within 32 of its last bits of where the scale doubles (1.75 times a power of two, large enough that the byte is not held at 0).
__device__ __forceinline__ bool is_close(float top) {
    const unsigned u = __float_as_uint(top);
    return (u & 0x7fffffu) - 0x600000u + 32u <= 64u && u >> 23 >= 8;
}

// A largest value so near to where the scale doubles that fp32 may be on the wrong side: 64 bits decide.  fp32 is off by at most 25 half-steps of 2^-23 (38 of them in the
// sum: up to 32 additions in a thread and 6 across lanes, halved by the root; then the root, the quotient and two products), 22 of the steps looked at here, near 1.75.
// One row of 10 000 at 12 blocks a row: its results are written again, from memory and group by group, so that the others need no
// registers for it (119 056 x 1 536: 347 us with and without; 4 797 x 1 152: 12 instead of 10.6 us when there is such a row, for its own time).
template <bool VEC, int TPR>
__device__ __forceinline__ void settle_row(const RmsNormParams& p, int64_t r, int t, float rstd) {
    const int D = p.D;
    const int64_t cols = fp8_cols(D), scale_cols = fp8_scale_cols(D), g = p.groups == 1 ? 0 : (unsigned)r / (unsigned)p.group_rows;
    unsigned char* y = static_cast<unsigned char*>(p.y) + r * cols;
    constexpr int L = TPR < 64 ? TPR : 64;              // a wavefront by itself: what the row's others have stored lies ahead of the sum's barrier
    const auto stored = [&](int c, int lane, float (&x)[1][4]) __attribute__((always_inline)) {      // from column c on
        if (p.res) load_row<VEC, TPR, 1>(p.h, p.h_type, r * D + c, D - c, lane, x);
        else load_row<VEC, TPR, 1>(p.x, p.x_type, r * D + c, D - c, lane, x);
    };
    double square = 0.0;
#pragma unroll 3
    for (int c = 0; c < D; c += 4 * L) {
        float x[1][4];
        stored(c, t % L, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) square = __builtin_fma((double)x[0][e], (double)x[0][e], square);
    }
#pragma unroll
    for (int o = 1; o < L; o *= 2) square += __shfl_xor(square, o);
    square += (double)p.eps * D;                        // D over the square of rstd: no root and no quotient
#pragma unroll 1
    for (int at = 0; at < cols; at += 4 * TPR) {
        const int c = at + 4 * t;
        float x[1][4], w[1][4] = {{1.f, 1.f, 1.f, 1.f}}, top = 0.f;
        double exact = 0.0;
        stored(at, t, x);
        if (p.weight) RowIO<float, VEC, TPR, 1>::load(p.weight + g * D + at, D - at, t, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double product = fabs((double)x[0][e] * w[0][e]);
            x[0][e] = c + e < D ? x[0][e] * (p.weight ? rstd * w[0][e] : rstd) : 0.f;
            const float m = finite_magnitude(x[0][e]);
            top = fmaxf(top, m);
            if (m > 0.f && product > exact) exact = product;
        }
        top = lane_max32(top);
#pragma unroll
        for (int o = 1; o < 32; o *= 2) exact = fmax(exact, __shfl_xor(exact, o));
        unsigned byte = scale_byte<false>(top);
        if (is_close(top)) {
            const float border = __uint_as_float((__float_as_uint(top) & 0x7f800000u) | 0x600000u);
            byte = scale_byte<false>(border) + (exact * exact * D > (double)border * border * square ? 1u : 0u);
        }
        const float f = inverse_scale(byte);
        if (c < cols) {
            __builtin_nontemporal_store(pack_e4m3(x[0][0] * f, x[0][1] * f, x[0][2] * f, x[0][3] * f), reinterpret_cast<unsigned*>(y + c));
            if (t % 32 == 0) p.y_scales[r * scale_cols + c / 128] = (uint8_t)byte;
        }
    }
}

template <bool VEC, int TPR, int NV>
__global__ __launch_bounds__(ln_threads(TPR)) void rms_norm_fwd_kernel(const RmsNormParams p) {
    constexpr int RPW = ln_threads(TPR) / TPR;                  // rows of a workgroup
    __shared__ float lds[TPR > 64 ? 4 * (TPR / 64) : 1];
    const int t = threadIdx.x % TPR, D = p.D;
    const int64_t r = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * RPW + threadIdx.x / TPR;
    if (r >= p.rows) return;                                    // RPW > 1: no barrier follows
    float h[NV][4], ss = 0.f, zero = 0.f;
    load_row<VEC, TPR, NV>(p.x, p.x_type, r * D, D, t, h);
    if (p.res) {
        float a[NV][4];
        load_row<VEC, TPR, NV>(p.res, p.h_type, r * D, D, t, a);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) h[i][e] += a[i][e];
        if (p.h_type == PDA_BF16)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) h[i][e] = (float)(__bf16)h[i][e];      // the stream as it is stored is what is normalised
        store_row<VEC, TPR, NV>(p.h, p.h_type, r * D, D, t, h);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) ss = __builtin_fmaf(h[i][e], h[i][e], ss);
    row_sum<TPR>(ss, zero, lds);
    float rstd = 1.0f / sqrtf(ss / (float)D + p.eps);
    // Squares so small that they lose bits, and no eps that hides it: those of the row times a power of two.  The threads of a row take this alike.
    const float by = ss < 0x1p-100f && p.eps < 0x1p-90f ? 0x1p60f : 1.f;
    if (__any(by != 1.f)) {
        float again = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) again = __builtin_fmaf(h[i][e] * by, h[i][e] * by, again);
        row_sum<TPR>(again, zero, lds + 2 * (TPR / 64));
        if (by != 1.f) rstd = by / sqrtf(again / (float)D + p.eps * by * by);
    }
    const int64_t g = p.groups == 1 ? 0 : (unsigned)r / (unsigned)p.group_rows;       // rows < 2^31
    if (p.weight) {
        float w[NV][4];
        RowIO<float, VEC, TPR, NV>::load(p.weight + g * D, D, t, w);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) h[i][e] *= rstd * w[i][e];
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) h[i][e] *= rstd;
    }
    if (p.y_type == PDA_E4M3) {
        if constexpr (TPR >= 32) {
            const int64_t cols = fp8_cols(D), scale_cols = fp8_scale_cols(D);
            bool close = false;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (i * TPR + t) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e) h[i][e] = c + e < D ? h[i][e] : 0.f;       // (0 times a NaN or an infinity above)
                const float top = lane_max32(fmaxf(fmaxf(finite_magnitude(h[i][0]), finite_magnitude(h[i][1])), fmaxf(finite_magnitude(h[i][2]), finite_magnitude(h[i][3]))));
                const unsigned byte = scale_byte<false>(top);
                const float f = inverse_scale(byte);
                close = close || is_close(top);
                if (c < cols) {                                 // (a block of lanes alike)
                    const unsigned q = pack_e4m3(h[i][0] * f, h[i][1] * f, h[i][2] * f, h[i][3] * f);
                    __builtin_nontemporal_store(q, reinterpret_cast<unsigned*>(static_cast<unsigned char*>(p.y) + r * cols + c));
                    if (t % 32 == 0) p.y_scales[r * scale_cols + c / 128] = (uint8_t)byte;
                }
            }
            if (__any(close)) settle_row<VEC, TPR>(p, r, t, rstd);
        }
    } else {
        store_row<VEC, TPR, NV>(p.y, p.y_type, r * D, D, t, h);
    }
    if (t == 0 && p.rstd) p.rstd[r] = rstd;
}

template <typename TY, typename TH, bool VEC, int TPR, int NV>
__global__ __launch_bounds__(ln_threads(TPR)) void rms_norm_bwd_kernel(const RmsNormParams p) {
    constexpr int RPW = ln_threads(TPR) / TPR;
    using X = RowIO<TH, VEC, TPR, NV>;
    using Y = RowIO<TY, VEC, TPR, NV>;
    using W = RowIO<float, VEC, TPR, NV>;
    __shared__ float lds[TPR > 64 ? 4 * (TPR / 64) : 1];
    int par = 0;
    __shared__ float joined[RPW > 1 ? RPW * NV * 4 * TPR : 1];
    const int t = threadIdx.x % TPR, own = threadIdx.x / TPR, D = p.D;
    const int64_t g = blockIdx.y;
    const float inv_d = 1.0f / (float)D;
    float sw[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sw[i][e] = 0.f;
    const int64_t step = RPW * p.chunks, r0 = g * p.group_rows;
    const TH* hp = static_cast<const TH*>(p.h);
    const TY* yp = static_cast<const TY*>(p.x);
    const TH* rp = static_cast<const TH*>(p.res);
    int64_t n = (int64_t)blockIdx.x * RPW + own;
    typename X::Group hn[NV], rn[NV];
    typename Y::Group yn[NV];
    float rstd_n = 0.f;
    auto fetch = [&](int64_t r) __attribute__((always_inline)) {
        X::fetch(hp + r * D, D, t, hn);
        Y::fetch(yp + r * D, D, t, yn);
        if (rp) X::fetch(rp + r * D, D, t, rn);
        rstd_n = p.rstd[r];
    };
    if (n < p.group_rows) fetch(r0 + n);
    for (; n < p.group_rows; n += step) {                      // RPW == 1: all threads of the workgroup alike
        const int64_t r = r0 + n;
        float hh[NV][4], dy[NV][4], dr[NV][4], w[NV][4], a = 0.f, b = 0.f;
        const float rstd = rstd_n;
        if (p.weight) {
            typename W::Group wn[NV];
            W::fetch(p.weight + g * D, D, t, wn);
            W::settle(wn, D, t);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[i][e] = W::value(wn, i, e);
        }
        X::settle(hn, D, t);
        Y::settle(yn, D, t);
        if (rp) X::settle(rn, D, t);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                hh[i][e] = X::value(hn, i, e) * rstd;           // columns behind D: zeros
                dy[i][e] = Y::value(yn, i, e);
                dr[i][e] = rp ? X::value(rn, i, e) : 0.f;
            }
        if (n + step < p.group_rows) fetch(r + step);           // the next row travels under this one's arithmetic
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sw[i][e] = __builtin_fmaf(dy[i][e], hh[i][e], sw[i][e]);
                if (p.weight) dy[i][e] *= w[i][e];
                b = __builtin_fmaf(dy[i][e], hh[i][e], b);
            }
        if (p.y) {
            row_sum<TPR>(a, b, lds + par);
            par ^= 2 * (TPR / 64);
            b *= inv_d;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) hh[i][e] = __builtin_fmaf(rstd, dy[i][e] - hh[i][e] * b, dr[i][e]);
            X::store(static_cast<TH*>(p.y) + r * D, D, t, hh);
        }
    }
    if (!p.dweight) return;
    // the sums of the workgroup's rows: its own place in the workspace, or the result if it is alone in the group
    if constexpr (RPW > 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) joined[(own * NV * 4 + i * 4 + e) * TPR + t] = sw[i][e];
        __syncthreads();
        if (own != 0) return;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int o = 1; o < RPW; ++o) sw[i][e] += joined[(o * NV * 4 + i * 4 + e) * TPR + t];
    }
    W::store(p.chunks == 1 ? p.dweight + g * D : p.part + (g * p.chunks + blockIdx.x) * D, D, t, sw);
}

// 32 columns a workgroup, 32 threads a column, each with every 32nd of the chunks.
__global__ __launch_bounds__(1024) void rms_norm_join_kernel(const RmsNormParams p) {
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    const int64_t g = blockIdx.y;
    float s = 0.f;
    if (col < p.D) {
        const float* src = p.part + g * p.chunks * p.D + col;
        for (int64_t k = w; k < p.chunks; k += 32 * 16) {      // sixteen loads in flight
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = k + 32 * i < p.chunks ? src[(k + 32 * i) * p.D] : 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) s += x[i];
        }
    }
    lds[w][c] = s;
    __syncthreads();
    if (w == 0 && col < p.D) {
#pragma unroll
        for (int i = 1; i < 32; ++i) s += lds[i][c];
        p.dweight[g * p.D + col] = s;
    }
}

// rows == 0: no sums
__global__ __launch_bounds__(256) void rms_norm_zero_kernel(float* a, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) a[i] = 0.f;
}

template <bool VEC, int TPR, int NV>
static hipError_t launch_fwd(const RmsNormParams& p, hipStream_t st) {
    constexpr int rpw = ln_threads(TPR) / TPR;
    const int64_t n = (p.rows + rpw - 1) / rpw, x = n < 1 << 21 ? n : 1 << 21;           // a launch has fewer than 2^32 threads along x
    hipLaunchKernelGGL((rms_norm_fwd_kernel<VEC, TPR, NV>), dim3((unsigned)x, (unsigned)((n + x - 1) / x)), dim3(ln_threads(TPR)), 0, st, p);
    return hipGetLastError();
}

template <bool VEC>
static hipError_t launch_fwd(const RmsNormParams& p, hipStream_t st) {
    const int D = p.y_type == PDA_E4M3 ? (int)fp8_cols(p.D) : p.D;      // the padded columns are written too
    // Short rows of bf16 alone take two groups a thread, so that as many bytes are on their way as with fp32 (400 000 x 128, bf16 throughout: 71 us, with one group 102;
    // fp32 throughout, x 100: 122 and 107).  Up to 256 that is better for all types (199 076 x 164, fp32 + bf16 to e4m3: 67 us, with one 97).
    if (p.x_type == PDA_BF16 && (!p.res || p.h_type == PDA_BF16) && p.y_type == PDA_BF16) {
        if (D <= 64) return launch_fwd<VEC, 8, 2>(p, st);
        if (D <= 128) return launch_fwd<VEC, 16, 2>(p, st);
        if (D > 256 && D <= 384) return launch_fwd<VEC, 32, 3>(p, st);
    }
    if (D <= 64) return launch_fwd<VEC, 16, 1>(p, st);
    if (D <= 128) return launch_fwd<VEC, 32, 1>(p, st);
    if (D <= 256) return launch_fwd<VEC, 32, 2>(p, st);
    if (D <= 512) return launch_fwd<VEC, 64, 2>(p, st);
    if (D <= 1024) return launch_fwd<VEC, 64, 4>(p, st);
    if constexpr (VEC) {
        if (D <= 1536) return launch_fwd<VEC, 64, 6>(p, st);
        if (D <= 2048) return launch_fwd<VEC, 64, 8>(p, st);
    } else {
        if (D <= 2048) return launch_fwd<VEC, 256, 2>(p, st);
    }
    if (D <= 4096) return launch_fwd<VEC, 512, 2>(p, st);
    return launch_fwd<VEC, 512, 4>(p, st);                     // up to PDA_LAYER_NORM_MAX = 8192
}

hipError_t launch_rms_norm_fwd(const RmsNormParams& p, hipStream_t st) {
    return p.D % 4 == 0 ? launch_fwd<true>(p, st) : launch_fwd<false>(p, st);
}

template <typename TY, typename TH, bool VEC, int TPR, int NV>
static hipError_t launch_bwd(const RmsNormParams& p, hipStream_t st) {
    hipLaunchKernelGGL((rms_norm_bwd_kernel<TY, TH, VEC, TPR, NV>), dim3((unsigned)p.chunks, (unsigned)p.groups), dim3(ln_threads(TPR)), 0, st, p);
    return hipGetLastError();
}

template <typename TY, typename TH, bool VEC>
static hipError_t launch_bwd(const RmsNormParams& p, hipStream_t st) {
    if (p.D <= 64) return launch_bwd<TY, TH, VEC, 16, 1>(p, st);
    if (p.D <= 128) return launch_bwd<TY, TH, VEC, 32, 1>(p, st);
    if (p.D <= 256) return launch_bwd<TY, TH, VEC, 64, 1>(p, st);
    if (p.D <= 512) return launch_bwd<TY, TH, VEC, 64, 2>(p, st);
    if (p.D <= 1024) return launch_bwd<TY, TH, VEC, 256, 1>(p, st);
    if (p.D <= 2048) return launch_bwd<TY, TH, VEC, 256, 2>(p, st);
    if (p.D <= 4096) return launch_bwd<TY, TH, VEC, 512, 2>(p, st);
    return launch_bwd<TY, TH, VEC, 512, 4>(p, st);
}

hipError_t launch_rms_norm_bwd(const RmsNormParams& p, hipStream_t st) {
    if (p.rows == 0) {
        const int64_t n = p.groups * p.D;
        hipLaunchKernelGGL(rms_norm_zero_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, p.dweight, n);
        return hipGetLastError();
    }
    const bool vec = p.D % 4 == 0, y_bf16 = p.x_type == PDA_BF16;
    hipError_t e;
    if (p.h_type == PDA_BF16) {
        if (y_bf16) e = vec ? launch_bwd<__bf16, __bf16, true>(p, st) : launch_bwd<__bf16, __bf16, false>(p, st);
        else e = vec ? launch_bwd<float, __bf16, true>(p, st) : launch_bwd<float, __bf16, false>(p, st);
    } else {
        if (y_bf16) e = vec ? launch_bwd<__bf16, float, true>(p, st) : launch_bwd<__bf16, float, false>(p, st);
        else e = vec ? launch_bwd<float, float, true>(p, st) : launch_bwd<float, float, false>(p, st);
    }
    if (e != hipSuccess || p.chunks == 1 || !p.dweight) return e;
    hipLaunchKernelGGL(rms_norm_join_kernel, dim3((unsigned)((p.D + 31) / 32), (unsigned)p.groups), dim3(1024), 0, st, p);
    return hipGetLastError();
}

}  // namespace pda

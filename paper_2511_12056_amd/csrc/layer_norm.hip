// Layer norm forward and backward over the last axis, bound by HBM: every element is read once, held in fp32 registers
// across the sums over its row, and written once.
//
// A row belongs to TPR threads: a wavefront, up to D = 64 and 128 a quarter and half of one (sums over the row in registers, no barrier), or a whole workgroup (one
// barrier, the sums of two rows alternate between two places in LDS).  1 000 000 x 64, fp32 -> bf16, a wavefront each forward 219 us, a quarter 69, backward 228 and 125;
// x 128 298 and 167, 275 and 247.  Forward, a wavefront up to D = 2 048: rows x D fp32 -> bf16 with a workgroup
// each instead 119 056 x 1 536 191 -> 218 us.  Backward, a wavefront up to D = 512 only: there a thread also keeps the sums of its columns
// over the rows, and four times the columns are four times the registers (60 000 x 2 048 bf16 394 -> 152 us with a workgroup a row).
// A thread holds NV groups of four elements: 16 (fp32) or 8 bytes (bf16) an access, consecutive threads side by side.  Rows that are
// not a multiple of four elements long start at any address, and their accesses do too; the group that crosses the row's end is read element by element forward,
// and backward, where the next row must not be waited for, together with the elements before it (single elements throughout instead, us, bf16: 30 000 x 1 541
// forward 91 and now 49, backward 196 and 65; 20 000 x 4 999 backward 747 and 177; fp32 alone backward 111 and 121).  Forward, such rows of more than 1 024 elements
// go to a workgroup (a wavefront would hold too many registers: 20 000 x 1 101 53 and 32).
//
// Backward, the sums over the rows (dweight, dbias): workgroup i of a group takes rows i, i + chunks, ..., so that all of them stream through
// neighbouring rows (each through rows of its own: 5 to 25 % slower), and keeps its columns' sums in registers; they go to the workspace,
// where a second kernel adds those of a group in order.  The next row is requested before a row's arithmetic (60 000 x 2 048 172 -> 152 us).
// Stores are non-temporal (119 056 x 1 536 forward 191 -> 185, backward 333 -> 323 us; 100 000 x 1 024 forward, bf16, 82 -> 60).
// Measured: 119 056 x 1 536, fp32 x, bf16 y: forward 185 us = 5.9 TB/s, backward 323 us = 5.7 TB/s; 9 594 x 1 152 bf16 9.2 and 20 us.
#include <hip/hip_runtime.h>
#include <type_traits>
#include "attn_internal.h"
#include "train_device.h"
#include "train_internal.h"

namespace pda {

template <typename T, bool VEC, int TPR, int NV>
struct RowIO {
    // element e of group i of thread t
    static __device__ __forceinline__ int col(int i, int e, int t) { return (i * TPR + t) * 4 + e; }
    // A thread's part of a row as it lies in memory, zeros behind the row's end.
    using Group = std::conditional_t<sizeof(T) == 4, f32x4, u32x2>;
    typedef Group Loose __attribute__((aligned(sizeof(T))));   // rows of any length start at any element
    using Access = std::conditional_t<VEC, Group, Loose>;
    // Elements by which group i of thread t ends behind the row's end; such a group is read from that many elements before it (rows of four elements at least).
    static __device__ __forceinline__ int over(int c, int D) { return VEC || D < 4 || c + 4 <= D ? 0 : c + 4 - D; }
    static __device__ __forceinline__ void fetch(const T* row, int D, int t, Group (&g)[NV]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col(i, 0, t);
            g[i] = Group{};
            if (c < D && (VEC || D >= 4)) g[i] = *reinterpret_cast<const Access*>(row + c - over(c, D));
        }
        if (!VEC && D < 4 && t == 0)
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < D) {
                    if constexpr (sizeof(T) == 4) g[0][e] = row[e];
                    else g[0][e / 2] |= (unsigned)__builtin_bit_cast(unsigned short, row[e]) << (e % 2 * 16);
                }
    }
    // What fetch has read, each element in its place (apart from it: this waits for the loads).
    static __device__ __forceinline__ void settle(Group (&g)[NV], int D, int t) {
        if constexpr (!VEC) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = col(i, 0, t), n = c < D ? over(c, D) : 0;
                if constexpr (sizeof(T) == 4) {
                    if (n & 1) g[i] = Group{g[i][1], g[i][2], g[i][3], 0.f};
                    if (n & 2) g[i] = Group{g[i][2], g[i][3], 0.f, 0.f};
                } else {
                    g[i] = __builtin_bit_cast(Group, __builtin_bit_cast(uint64_t, g[i]) >> (16 * n));
                }
            }
        }
    }
    static __device__ __forceinline__ float value(const Group (&g)[NV], int i, int e) {
        if constexpr (sizeof(T) == 4) return g[i][e];
        else return e % 2 ? bf16_hi(g[i][e / 2]) : bf16_lo(g[i][e / 2]);
    }
    static __device__ __forceinline__ void load(const T* row, int D, int t, float (&x)[NV][4]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col(i, 0, t);
            Group g[1] = {Group{}};
            if (c + (VEC ? 0 : 3) < D) g[0] = *reinterpret_cast<const Access*>(row + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] = RowIO<T, VEC, TPR, 1>::value(g, 0, e);
            if (!VEC && c < D && c + 3 >= D)                   // the row's last one to three elements
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (c + e < D) x[i][e] = (float)row[c + e];
        }
    }
    static __device__ __forceinline__ void store(T* row, int D, int t, const float (&x)[NV][4]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = col(i, 0, t);
            if (c + (VEC ? 0 : 3) < D) {
                if constexpr (sizeof(T) == 4) __builtin_nontemporal_store(f32x4{x[i][0], x[i][1], x[i][2], x[i][3]}, reinterpret_cast<Access*>(row + c));
                else __builtin_nontemporal_store(u32x2{pack_bf16(x[i][0], x[i][1]), pack_bf16(x[i][2], x[i][3])}, reinterpret_cast<Access*>(row + c));
            } else if (!VEC && c < D) {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (c + e < D) row[c + e] = (T)x[i][e];
            }
        }
    }
};

// Sum of (a, b) over the TPR threads of a row, in every one of them.
template <int TPR>
__device__ __forceinline__ void row_sum(float& a, float& b, float* lds) {
    a = lane_sum<TPR < 64 ? TPR : 64>(a);
    b = lane_sum<TPR < 64 ? TPR : 64>(b);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) { lds[w] = a; lds[W + w] = b; }
        __syncthreads();
        a = lds[0];
        b = lds[W];
#pragma unroll
        for (int i = 1; i < W; ++i) { a += lds[i]; b += lds[W + i]; }
    }
}

constexpr int ln_threads(int tpr) { return tpr > 256 ? tpr : 256; }

template <typename TX, typename TY, bool VEC, int TPR, int NV>
__global__ __launch_bounds__(ln_threads(TPR)) void layer_norm_fwd_kernel(const LayerNormParams p) {
    constexpr int RPW = ln_threads(TPR) / TPR;                  // rows of a workgroup
    __shared__ float lds[TPR > 64 ? 4 * (TPR / 64) : 1];
    const int t = threadIdx.x % TPR, D = p.D;
    const int64_t r = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * RPW + threadIdx.x / TPR;
    if (r >= p.rows) return;                                    // RPW > 1: no barrier follows
    float x[NV][4], a = 0.f, zero = 0.f;
    RowIO<TX, VEC, TPR, NV>::load(static_cast<const TX*>(p.x) + r * D, D, t, x);
#pragma unroll
    for (int i = 0; i < NV; ++i) a += (x[i][0] + x[i][1]) + (x[i][2] + x[i][3]);
    row_sum<TPR>(a, zero, lds);
    const float mean = a / (float)D;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[i][e] = RowIO<TX, VEC, TPR, NV>::col(i, e, t) < D ? x[i][e] - mean : 0.f;
            ss = __builtin_fmaf(x[i][e], x[i][e], ss);
        }
    row_sum<TPR>(ss, zero, lds + 2 * (TPR / 64));
    const float rstd = 1.0f / sqrtf(ss / (float)D + p.eps);
    const int64_t g = p.groups == 1 ? 0 : (unsigned)r / (unsigned)p.group_rows;       // rows < 2^31
    if (p.weight) {
        float w[NV][4];
        RowIO<float, VEC, TPR, NV>::load(p.weight + g * D, D, t, w);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] *= rstd * w[i][e];
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] *= rstd;
    }
    if (p.bias) {
        float w[NV][4];
        RowIO<float, VEC, TPR, NV>::load(p.bias + g * D, D, t, w);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] += w[i][e];
    }
    RowIO<TY, VEC, TPR, NV>::store(static_cast<TY*>(p.y) + r * D, D, t, x);
    if (t == 0 && p.mean) {
        p.mean[r] = mean;
        p.rstd[r] = rstd;
    }
}

template <typename TX, typename TY, bool VEC, int TPR, int NV>
__global__ __launch_bounds__(ln_threads(TPR)) void layer_norm_bwd_kernel(const LayerNormParams p) {
    constexpr int RPW = ln_threads(TPR) / TPR;
    using X = RowIO<TX, VEC, TPR, NV>;
    using Y = RowIO<TY, VEC, TPR, NV>;
    using W = RowIO<float, VEC, TPR, NV>;
    __shared__ float lds[TPR > 64 ? 4 * (TPR / 64) : 1];
    int par = 0;
    __shared__ float joined[RPW > 1 ? RPW * NV * 4 * TPR : 1];
    const int t = threadIdx.x % TPR, own = threadIdx.x / TPR, D = p.D;
    const int64_t g = blockIdx.y;
    const float inv_d = 1.0f / (float)D;
    float sw[NV][4], sb[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sw[i][e] = sb[i][e] = 0.f;
    const int64_t step = RPW * p.chunks, r0 = g * p.group_rows;
    const TX* xp = static_cast<const TX*>(p.x);
    const TY* yp = static_cast<const TY*>(p.dy);
    int64_t n = (int64_t)blockIdx.x * RPW + own;
    typename X::Group xn[NV];
    typename Y::Group yn[NV];
    float mean_n = 0.f, rstd_n = 0.f;
    auto fetch = [&](int64_t r) __attribute__((always_inline)) {
        X::fetch(xp + r * D, D, t, xn);
        Y::fetch(yp + r * D, D, t, yn);
        mean_n = p.mean[r];
        rstd_n = p.rstd[r];
    };
    if (n < p.group_rows) fetch(r0 + n);
    for (; n < p.group_rows; n += step) {                      // RPW == 1: all threads of the workgroup alike
        const int64_t r = r0 + n;
        float x[NV][4], dy[NV][4], w[NV][4], a = 0.f, b = 0.f;
        const float mean = mean_n, rstd = rstd_n;
        if (p.weight) {
            typename W::Group wn[NV];
            W::fetch(p.weight + g * D, D, t, wn);
            W::settle(wn, D, t);
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) w[i][e] = W::value(wn, i, e);
        }
        X::settle(xn, D, t);
        Y::settle(yn, D, t);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[i][e] = (X::value(xn, i, e) - mean) * rstd;   // columns behind D: dy = 0 there
                dy[i][e] = Y::value(yn, i, e);
            }
        if (n + step < p.group_rows) fetch(r + step);           // the next row travels under this one's arithmetic
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sw[i][e] = __builtin_fmaf(dy[i][e], x[i][e], sw[i][e]);
                sb[i][e] += dy[i][e];
                if (p.weight) dy[i][e] *= w[i][e];
                a += dy[i][e];
                b = __builtin_fmaf(dy[i][e], x[i][e], b);
            }
        if (p.y) {
            row_sum<TPR>(a, b, lds + par);
            par ^= 2 * (TPR / 64);
            a *= inv_d;
            b *= inv_d;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i][e] = rstd * (dy[i][e] - a - x[i][e] * b);
            X::store(static_cast<TX*>(p.y) + r * D, D, t, x);
        }
    }
    // the sums of the workgroup's rows: its own place in the workspace, or the result if it is alone in the group
    auto finish = [&](float (&s)[NV][4], float* to) __attribute__((always_inline)) {
        if constexpr (RPW > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) joined[(own * NV * 4 + i * 4 + e) * TPR + t] = s[i][e];
            __syncthreads();
            if (own != 0) return;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int o = 1; o < RPW; ++o) s[i][e] += joined[(o * NV * 4 + i * 4 + e) * TPR + t];
        }
        RowIO<float, VEC, TPR, NV>::store(to, D, t, s);
    };
    const bool alone = p.chunks == 1;
    float* part = alone ? nullptr : p.part + ((g * p.chunks + blockIdx.x) * 2) * D;
    if (p.dweight) finish(sw, alone ? p.dweight + g * D : part);
    if (p.dbias) finish(sb, alone ? p.dbias + g * D : part + D);
}

// dweight (blockIdx.z = 0) or dbias: 32 columns a workgroup, 32 threads a column, each with every 32nd of the chunks.
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const LayerNormParams p) {
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    const int64_t g = blockIdx.y;
    float* to = blockIdx.z == 0 ? p.dweight : p.dbias;
    if (!to) return;
    float s = 0.f;
    if (col < p.D) {
        const float* src = p.part + (g * p.chunks * 2 + blockIdx.z) * p.D + col;
        for (int64_t k = w; k < p.chunks; k += 32 * 16) {      // sixteen loads in flight
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = k + 32 * i < p.chunks ? src[(k + 32 * i) * 2 * p.D] : 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) s += x[i];
        }
    }
    lds[w][c] = s;
    __syncthreads();
    if (w == 0 && col < p.D) {
#pragma unroll
        for (int i = 1; i < 32; ++i) s += lds[i][c];
        to[g * p.D + col] = s;
    }
}

// rows == 0: no sums
__global__ __launch_bounds__(256) void layer_norm_zero_kernel(float* a, float* b, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    if (a) a[i] = 0.f;
    if (b) b[i] = 0.f;
}

template <bool BWD, typename TX, typename TY, bool VEC, int TPR, int NV>
static hipError_t launch_ln(const LayerNormParams& p, hipStream_t st) {
    if constexpr (BWD) {
        hipLaunchKernelGGL((layer_norm_bwd_kernel<TX, TY, VEC, TPR, NV>), dim3((unsigned)p.chunks, (unsigned)p.groups), dim3(ln_threads(TPR)), 0, st, p);
    } else {
        constexpr int rpw = ln_threads(TPR) / TPR;
        const int64_t n = (p.rows + rpw - 1) / rpw, x = n < 1 << 21 ? n : 1 << 21;       // a launch has fewer than 2^32 threads along x
        hipLaunchKernelGGL((layer_norm_fwd_kernel<TX, TY, VEC, TPR, NV>), dim3((unsigned)x, (unsigned)((n + x - 1) / x)), dim3(ln_threads(TPR)), 0, st, p);
    }
    return hipGetLastError();
}

template <bool BWD, typename TX, typename TY, bool VEC>
static hipError_t launch_ln(const LayerNormParams& p, hipStream_t st) {
    if (p.D <= 64) return launch_ln<BWD, TX, TY, VEC, 16, 1>(p, st);
    if (p.D <= 128) return launch_ln<BWD, TX, TY, VEC, 32, 1>(p, st);
    if (p.D <= 256) return launch_ln<BWD, TX, TY, VEC, 64, 1>(p, st);
    if (p.D <= 512) return launch_ln<BWD, TX, TY, VEC, 64, 2>(p, st);
    if constexpr (BWD) {
        if (p.D <= 1024) return launch_ln<BWD, TX, TY, VEC, 256, 1>(p, st);
    } else {
        if (p.D <= 1024) return launch_ln<BWD, TX, TY, VEC, 64, 4>(p, st);
    }
    if constexpr (BWD || !VEC) {
        if (p.D <= 2048) return launch_ln<BWD, TX, TY, VEC, 256, 2>(p, st);
    } else {
        if (p.D <= 1536) return launch_ln<BWD, TX, TY, VEC, 64, 6>(p, st);
        if (p.D <= 2048) return launch_ln<BWD, TX, TY, VEC, 64, 8>(p, st);
    }
    if (p.D <= 4096) return launch_ln<BWD, TX, TY, VEC, 512, 2>(p, st);
    return launch_ln<BWD, TX, TY, VEC, 512, 4>(p, st);         // up to PDA_LAYER_NORM_MAX = 8192
}

template <bool BWD>
static hipError_t launch_ln(const LayerNormParams& p, bool x_bf16, bool y_bf16, hipStream_t st) {
    const bool vec = p.D % 4 == 0;
    if (x_bf16) {
        if (y_bf16) return vec ? launch_ln<BWD, __bf16, __bf16, true>(p, st) : launch_ln<BWD, __bf16, __bf16, false>(p, st);
        return vec ? launch_ln<BWD, __bf16, float, true>(p, st) : launch_ln<BWD, __bf16, float, false>(p, st);
    }
    if (y_bf16) return vec ? launch_ln<BWD, float, __bf16, true>(p, st) : launch_ln<BWD, float, __bf16, false>(p, st);
    return vec ? launch_ln<BWD, float, float, true>(p, st) : launch_ln<BWD, float, float, false>(p, st);
}

hipError_t launch_layer_norm_fwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, hipStream_t st) {
    return launch_ln<false>(p, x_bf16, y_bf16, st);
}

hipError_t launch_layer_norm_bwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, hipStream_t st) {
    if (p.rows == 0) {
        const int64_t n = p.groups * p.D;
        hipLaunchKernelGGL(layer_norm_zero_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, p.dweight, p.dbias, n);
        return hipGetLastError();
    }
    const hipError_t e = launch_ln<true>(p, x_bf16, y_bf16, st);
    if (e != hipSuccess || p.chunks == 1 || (!p.dweight && !p.dbias)) return e;
    hipLaunchKernelGGL(layer_norm_join_kernel, dim3((unsigned)((p.D + 31) / 32), (unsigned)p.groups, 2), dim3(1024), 0, st, p);
    return hipGetLastError();
}

}  // namespace pda

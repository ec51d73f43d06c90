// Layer norm forward and backward over the last axis, bound by HBM: every element is read once, held in fp32 registers
// across the sums over its row, and written once.
//
// A row belongs to TPR threads: a wavefront up to D = 2 048 (sums over the row in registers, no barrier), beyond that a whole
// workgroup.  A thread holds NV groups of four elements: 16 (fp32) or 8 bytes (bf16) an access, consecutive threads side by side.  Rows that are
// not a multiple of four elements long start at any address, so there a thread takes single elements, consecutive threads side by
// side again.
//
// Backward, the sums over the rows (dweight, dbias): a workgroup takes consecutive rows of one group and keeps its threads'
// columns in registers; its sums go to the workspace, where a second kernel adds those of a group in order.
#include <hip/hip_runtime.h>
#include "attn_internal.h"
#include "train_device.h"
#include "train_internal.h"

namespace pda {

template <typename T, bool VEC, int TPR, int NV>
struct RowIO {
    // element e of group i of thread t
    static __device__ __forceinline__ int col(int i, int e, int t) { return VEC ? (i * TPR + t) * 4 + e : (i * 4 + e) * TPR + t; }
    static __device__ __forceinline__ void load(const T* row, int D, int t, float (&x)[NV][4]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (VEC) {
                const int c = col(i, 0, t);
                if (c < D) {
                    if constexpr (sizeof(T) == 4) {
                        const f32x4 v = *reinterpret_cast<const f32x4*>(row + c);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[i][e] = v[e];
                    } else {
                        const u32x2 v = *reinterpret_cast<const u32x2*>(row + c);
                        x[i][0] = bf16_lo(v.x); x[i][1] = bf16_hi(v.x); x[i][2] = bf16_lo(v.y); x[i][3] = bf16_hi(v.y);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[i][e] = 0.f;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i][e] = col(i, e, t) < D ? (float)row[col(i, e, t)] : 0.f;
            }
        }
    }
    static __device__ __forceinline__ void store(T* row, int D, int t, const float (&x)[NV][4]) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (VEC) {
                const int c = col(i, 0, t);
                if (c < D) {
                    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4*>(row + c) = f32x4{x[i][0], x[i][1], x[i][2], x[i][3]};
                    else *reinterpret_cast<u32x2*>(row + c) = u32x2{pack_bf16(x[i][0], x[i][1]), pack_bf16(x[i][2], x[i][3])};
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col(i, e, t) < D) row[col(i, e, t)] = (T)x[i][e];
            }
        }
    }
};

// Sum of (a, b) over the TPR threads of a row, in every one of them.
template <int TPR>
__device__ __forceinline__ void row_sum(float& a, float& b, float* lds) {
    a = lane_sum<64>(a);
    b = lane_sum<64>(b);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        const int w = threadIdx.x >> 6;
        __syncthreads();                                        // the sums before these have been read
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
    __shared__ float lds[2 * (TPR / 64)];
    const int t = threadIdx.x % TPR, D = p.D;
    const int64_t r = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
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
    row_sum<TPR>(ss, zero, lds);
    const float rstd = 1.0f / sqrtf(ss / (float)D + p.eps);
    const int64_t g = p.groups == 1 ? 0 : r / p.group_rows;
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
    __shared__ float lds[2 * (TPR / 64)];
    __shared__ float joined[RPW > 1 ? RPW * NV * 4 * TPR : 1];
    const int t = threadIdx.x % TPR, own = threadIdx.x / TPR, D = p.D;
    const int64_t g = blockIdx.y, first = (int64_t)blockIdx.x * p.chunk_rows;
    const int64_t last = first + p.chunk_rows < p.group_rows ? first + p.chunk_rows : p.group_rows;
    const float inv_d = 1.0f / (float)D;
    float w[NV][4], sw[NV][4], sb[NV][4];
    if (p.weight) RowIO<float, VEC, TPR, NV>::load(p.weight + g * D, D, t, w);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sw[i][e] = sb[i][e] = 0.f;
            if (!p.weight) w[i][e] = 1.f;
        }
    for (int64_t n = first + own; n < last; n += RPW) {         // RPW == 1: all threads of the workgroup alike
        const int64_t r = g * p.group_rows + n;
        float x[NV][4], dy[NV][4], a = 0.f, b = 0.f;
        RowIO<TX, VEC, TPR, NV>::load(static_cast<const TX*>(p.x) + r * D, D, t, x);
        RowIO<TY, VEC, TPR, NV>::load(static_cast<const TY*>(p.dy) + r * D, D, t, dy);
        const float mean = p.mean[r], rstd = p.rstd[r];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[i][e] = (x[i][e] - mean) * rstd;              // columns behind D: dy = 0 there
                sw[i][e] = __builtin_fmaf(dy[i][e], x[i][e], sw[i][e]);
                sb[i][e] += dy[i][e];
                dy[i][e] *= w[i][e];
                a += dy[i][e];
                b = __builtin_fmaf(dy[i][e], x[i][e], b);
            }
        if (p.y) {
            row_sum<TPR>(a, b, lds);
            a *= inv_d;
            b *= inv_d;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[i][e] = rstd * (dy[i][e] - a - x[i][e] * b);
            RowIO<TX, VEC, TPR, NV>::store(static_cast<TX*>(p.y) + r * D, D, t, x);
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

// dweight (blockIdx.z = 0) or dbias: 64 columns a workgroup, 16 threads a column, each a sixteenth of the chunks.
__global__ __launch_bounds__(1024) void layer_norm_join_kernel(const LayerNormParams p) {
    __shared__ float lds[16][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), w = threadIdx.x >> 6;
    const int64_t g = blockIdx.y;
    float* to = blockIdx.z == 0 ? p.dweight : p.dbias;
    if (!to) return;
    float s = 0.f;
    if (c < p.D) {
        const float* src = p.part + (g * p.chunks * 2 + blockIdx.z) * p.D + c;
        const int64_t i1 = p.chunks * (w + 1) / 16;
#pragma unroll 8
        for (int64_t i = p.chunks * w / 16; i < i1; ++i) s += src[i * 2 * p.D];
    }
    lds[w][threadIdx.x & 63] = s;
    __syncthreads();
    if (w == 0 && c < p.D) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += lds[i][threadIdx.x];
        to[g * p.D + c] = s;
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
        hipLaunchKernelGGL((layer_norm_fwd_kernel<TX, TY, VEC, TPR, NV>), dim3((unsigned)((p.rows + rpw - 1) / rpw)), dim3(ln_threads(TPR)), 0, st, p);
    }
    return hipGetLastError();
}

template <bool BWD, typename TX, typename TY, bool VEC>
static hipError_t launch_ln(const LayerNormParams& p, hipStream_t st) {
    if (p.D <= 256) return launch_ln<BWD, TX, TY, VEC, 64, 1>(p, st);
    if (p.D <= 512) return launch_ln<BWD, TX, TY, VEC, 64, 2>(p, st);
    if (p.D <= 1024) return launch_ln<BWD, TX, TY, VEC, 64, 4>(p, st);
    if (p.D <= 1536) return launch_ln<BWD, TX, TY, VEC, 64, 6>(p, st);
    if (p.D <= 2048) return launch_ln<BWD, TX, TY, VEC, 64, 8>(p, st);
    if (p.D <= 4096) return launch_ln<BWD, TX, TY, VEC, 256, 4>(p, st);
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
    hipLaunchKernelGGL(layer_norm_join_kernel, dim3((unsigned)((p.D + 63) / 64), (unsigned)p.groups, 2), dim3(1024), 0, st, p);
    return hipGetLastError();
}

}  // namespace pda

// Rows of a norm: access by groups of four elements of fp32 or bf16 at any alignment, and sums over the threads of a row.
#pragma once
#include <hip/hip_runtime.h>
#include <type_traits>
#include "train_device.h"

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

}  // namespace pda

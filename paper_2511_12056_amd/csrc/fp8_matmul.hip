// Product of two 8-bit matrices with a power-of-two scale per block of 128: out[m, n] = sum_k a[m, k] b[n, k] + bias[n].
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 bytes and each operand row's 128 values by 2^(byte - 127) of a lane's register, at the
// rate of the unscaled instruction: a block of 128 is one instruction's K, and scales cost no arithmetic.  The order of K inside a block is the same permutation
// for both operands and does not matter.  b's rows are the first operand, so a lane ends up with four consecutive n of one m.
#include <hip/hip_runtime.h>
#include "attn_device.h"
#include "attn_internal.h"
#include "proj_internal.h"

namespace pda {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

template <bool E5M2>
__device__ __forceinline__ f32x4 mfma(const i32x8& b, const i32x8& a, const f32x4& c, int sb, int sa) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, E5M2 ? 1 : 0, 0, sb, 0, sa);
}

__device__ __forceinline__ i32x8 join8(const i32x4& lo, const i32x4& hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }

// The compiler moves a matrix instruction into a branch that only some lanes take if nothing else uses its result; there the other lanes' operands would be missing.
template <int N>
__device__ __forceinline__ void keep(f32x4 (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(x[i]));
}
template <int N, int M>
__device__ __forceinline__ void keep(f32x4 (&x)[N][M]) {
#pragma unroll
    for (int i = 0; i < N; ++i) keep(x[i]);
}

__device__ __forceinline__ void lds_dma4(const void* sbase, unsigned voff, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 vcc, %2\n\tglobal_load_lds_dword %1, vcc"
                 :
                 : "s"(lds_addr), "v"(voff), "s"(sbase)
                 : "memory", "m0", "vcc");
}

// Four results of row m, columns n .. n + 3: rounded, or into the part's sums.
__device__ __forceinline__ void store4(const MatmulParams& p, float* part, int64_t m, int64_t n, f32x4 v) {
    if (part) {
        *reinterpret_cast<f32x4*>(part + m * ((p.N + 3) & ~(int64_t)3) + n) = v;       // (rows of the parts are padded to four)
        return;
    }
    __bf16* o = p.out + m * p.ldo + n;
    if (p.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += n + e < p.N ? p.bias[n + e] : 0.f;
    }
    if (n + 4 <= p.N && (reinterpret_cast<uintptr_t>(o) & 7) == 0) {
        *reinterpret_cast<u32x2*>(o) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) o[e] = (__bf16)v[e];
    }
}

// ---- tiles ------------------------------------------------------------------------------------------------------
// TM x TN results a workgroup of WM x WN wavefronts; tiles of 128 bytes a row in two LDS buffers.
template <int TM, int TN, int WM, int WN>
constexpr int matmul_smem() { return 2 * (TM + TN) * 132; }

template <int TM, int TN, int WM, int WN, bool E5M2>
__global__ __launch_bounds__(WM * WN * 64, 2) void fp8_matmul_kernel(const MatmulParams p) {
    constexpr int NW = WM * WN, MT = TM / WM / 16, NT = TN / WN / 16;
    static_assert(NT == 4, "a wavefront's 64 columns are dealt to four instructions");
    constexpr int STAGE = (TM + TN) * 132, B_AT = TM * 128, SA_AT = (TM + TN) * 128, SB_AT = SA_AT + TM * 4;
    extern __shared__ __attribute__((aligned(1024))) unsigned char matmul_smem_[];
    const unsigned lds0 = (unsigned)(uintptr_t)(LDS_PTR(unsigned char))matmul_smem_;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w / WN, wn = w % WN;
    const int r16 = lane & 15, g = lane >> 4;
    const int64_t tiles_n = (p.N + TN - 1) / TN;
    const int64_t tm = blockIdx.x / tiles_n, tn = blockIdx.x % tiles_n;
    const int part = blockIdx.y;
    const int64_t m0 = tm * TM, n0 = tn * TN;
    const int nk_all = (int)(p.K / 128), kb0 = part * p.part_steps, nk = nk_all - kb0 < p.part_steps ? nk_all - kb0 : p.part_steps;
    // what this wavefront fetches of each tile: chunks of eight rows
    unsigned va[TM / 8 / NW], vb[TN / 8 / NW];
    const int last_m = (int)(p.M - m0 < TM ? p.M - m0 : TM) - 1, last_n = (int)(p.N - n0 < TN ? p.N - n0 : TN) - 1;
#pragma unroll
    for (int i = 0; i < TM / 8 / NW; ++i) {
        const int r = (w + NW * i) * 8 + lane / 8, at = r < last_m ? r : last_m;
        va[i] = (unsigned)at * (unsigned)p.K + (unsigned)(((lane & 7) ^ ((r >> 1) & 7)) * 16);
    }
#pragma unroll
    for (int i = 0; i < TN / 8 / NW; ++i) {
        const int r = (w + NW * i) * 8 + lane / 8, at = r < last_n ? r : last_n;
        vb[i] = (unsigned)at * (unsigned)p.K + (unsigned)(((lane & 7) ^ (((r >> 1) & 1) | ((r >> 4) & 3) << 1)) * 16);
    }
    // scales: wavefronts 0 .. TM/64 - 1 those of a, the others those of b, 64 rows each
    const bool of_a = w < TM / 64;
    const unsigned char* sbase = of_a ? p.a_scales + m0 * p.scale_cols : p.b_scales + (n0 >> p.b_shift) * p.scale_cols;
    unsigned vs = 0;
    {
        const int r = (of_a ? w : w - TM / 64) * 64 + lane, lim = of_a ? last_m : last_n, at = r < lim ? r : lim;
        vs = (unsigned)(of_a ? at : at >> p.b_shift) * (unsigned)p.scale_cols;
    }
    const unsigned char* pa = p.a + m0 * p.K;
    const unsigned char* pb = p.b + n0 * p.K;
    const auto fetch = [&](int t) __attribute__((always_inline)) {
        const unsigned to = lds0 + (t & 1) * STAGE;
        const int kb = kb0 + t;
        const unsigned char* a = pa + (int64_t)kb * 128;
        const unsigned char* b = pb + (int64_t)kb * 128;
#pragma unroll
        for (int i = 0; i < TM / 8 / NW; ++i) lds_dma16(a, va[i], to + (w + NW * i) * 1024);
#pragma unroll
        for (int i = 0; i < TN / 8 / NW; ++i) lds_dma16(b, vb[i], to + B_AT + (w + NW * i) * 1024);
        if (w < (TM + TN) / 64) lds_dma4(sbase + (kb & ~3), vs, to + SA_AT + w * 256);
    };
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // operand addresses: granules 2g and 2g + 1 of a row, at their swizzled places
    const int nrow = wn * 64 + (r16 / 4) * 16 + (r16 & 3);      // + 4 j: the row of instruction j, so that a lane's results are 16 consecutive columns
    const int mrow = wm * (TM / WM) + r16;                      // + 16 i
    const unsigned sw_b = ((nrow >> 1) & 1) | ((nrow >> 4) & 3) << 1, sw_a = (mrow >> 1) & 7;
    const unsigned a_lo = mrow * 128 + (((2 * g) ^ sw_a) * 16), a_hi = mrow * 128 + (((2 * g + 1) ^ sw_a) * 16);
    const unsigned b_lo = B_AT + nrow * 128 + (((2 * g) ^ sw_b) * 16), b_hi = B_AT + nrow * 128 + (((2 * g + 1) ^ sw_b) * 16);
    if (nk > 0) fetch(0);
    for (int t = 0; t < nk; ++t) {
        wait_vmcnt<0>();
        __syncthreads();
        if (t + 1 < nk) fetch(t + 1);
        const unsigned char* s = matmul_smem_ + (t & 1) * STAGE;
        const int shift = 8 * ((kb0 + t) & 3);
        i32x8 fb[NT];
        int sb[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            // rows 4 j apart: bits 2 and 3, which the swizzle does not look at
            fb[j] = join8(*reinterpret_cast<const i32x4*>(s + b_lo + j * 512), *reinterpret_cast<const i32x4*>(s + b_hi + j * 512));
            sb[j] = *reinterpret_cast<const int*>(s + SB_AT + (nrow + 4 * j) * 4) >> shift;
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const i32x8 fa = join8(*reinterpret_cast<const i32x4*>(s + a_lo + i * 2048), *reinterpret_cast<const i32x4*>(s + a_hi + i * 2048));
            const int sa = *reinterpret_cast<const int*>(s + SA_AT + (mrow + 16 * i) * 4) >> shift;
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mfma<E5M2>(fb[j], fa, acc[i][j], sb[j], sa);
        }
    }
    keep(acc);
    float* to = p.parts > 1 ? p.part + (int64_t)part * p.M * ((p.N + 3) & ~(int64_t)3) : nullptr;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = m0 + mrow + 16 * i;
        if (m < p.M)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int64_t n = n0 + wn * 64 + 16 * g + 4 * j;
                if (n < p.N) store4(p, to, m, n, acc[i][j]);
            }
    }
}

// ---- few rows -----------------------------------------------------------------------------------------------------
// 16 columns a workgroup, 16 MT rows; its wavefronts share K and add their sums in LDS, in order.  Operands come straight from memory: a row of b is used once.
constexpr int kFewWaves = 4;
template <int MT, bool E5M2>
__global__ __launch_bounds__(kFewWaves * 64) void fp8_matmul_few_kernel(const MatmulParams p) {
    __shared__ f32x4 sums[kFewWaves][MT][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, r16 = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16, m0 = (int64_t)blockIdx.y * (16 * MT);
    const int64_t bn = n0 + r16 < p.N ? n0 + r16 : p.N - 1;
    const int nk = (int)(p.K / 128);
    f32x4 acc[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const unsigned char* b = p.b + bn * p.K + 32 * g;
    const uint8_t* sbp = p.b_scales + (bn >> p.b_shift) * p.scale_cols;
    const unsigned char* a[MT];
    const uint8_t* sap[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = m0 + 16 * i + r16 < p.M ? m0 + 16 * i + r16 : p.M - 1;
        a[i] = p.a + m * p.K + 32 * g;
        sap[i] = p.a_scales + m * p.scale_cols;
    }
    for (int kb = w; kb < nk; kb += kFewWaves) {
        const i32x8 fb = join8(*reinterpret_cast<const i32x4*>(b + (int64_t)kb * 128), *reinterpret_cast<const i32x4*>(b + (int64_t)kb * 128 + 16));
        const int sb = sbp[kb];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const i32x8 fa = join8(*reinterpret_cast<const i32x4*>(a[i] + (int64_t)kb * 128), *reinterpret_cast<const i32x4*>(a[i] + (int64_t)kb * 128 + 16));
            acc[i] = mfma<E5M2>(fb, fa, acc[i], sb, sap[i][kb]);
        }
    }
    keep(acc);
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[w][i][lane] = acc[i];
    __syncthreads();
    for (int i = w; i < MT; i += kFewWaves) {
        f32x4 v = sums[0][i][lane];
#pragma unroll
        for (int o = 1; o < kFewWaves; ++o) v += sums[o][i][lane];
        const int64_t m = m0 + 16 * i + r16, n = n0 + 4 * g;
        if (m < p.M && n < p.N) store4(p, nullptr, m, n, v);
    }
}

// ---- sums of the ranges of K --------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void fp8_matmul_join_kernel(const MatmulParams p) {
    const int64_t n4 = (p.N + 3) / 4, m = (int64_t)blockIdx.z * gridDim.y + blockIdx.y, c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (m >= p.M || c >= n4) return;
    const f32x4* src = reinterpret_cast<const f32x4*>(p.part) + m * n4 + c;
    f32x4 v = *src;
    for (int k = 1; k < p.parts; ++k) v += src[k * p.M * n4];
    store4(p, nullptr, m, c * 4, v);
}

// K == 0: the bias
__global__ __launch_bounds__(256) void fp8_matmul_bias_kernel(const MatmulParams p) {
    const int64_t n4 = (p.N + 3) / 4, m = (int64_t)blockIdx.z * gridDim.y + blockIdx.y, c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (m < p.M && c < n4) store4(p, nullptr, m, c * 4, f32x4{0.f, 0.f, 0.f, 0.f});
}

MatmulPlan plan_matmul(int64_t M, int64_t N, int64_t K, int n_cu) {
    const int nk = (int)(K / 128);
    if (M <= 64) return {MatmulPlan::FEW, 1, nk};
    const auto tiles = [&](int64_t t) { return (M + t - 1) / t * ((N + t - 1) / t); };
    const bool large = tiles(256) * (nk / 16 + 1) >= n_cu;
    const int64_t n = large ? tiles(256) : tiles(128), room = large ? n_cu : 2 * n_cu;
    const int least = large ? 16 : 4;                          // steps of a part
    int64_t parts = n >= room ? 1 : room / n;
    if (parts > nk / least) parts = nk / least > 1 ? nk / least : 1;
    const int steps = (int)((nk + parts - 1) / parts);
    return {large ? MatmulPlan::LARGE : MatmulPlan::SMALL, steps > 0 ? (nk + steps - 1) / steps : 1, steps};
}

int64_t matmul_workspace_bytes(const MatmulPlan& w, int64_t M, int64_t N) { return w.parts > 1 ? w.parts * M * ((N + 3) / 4 * 16) : 0; }

static dim3 row_grid(const MatmulParams& p) {
    const int64_t y = p.M < 65535 ? p.M : 65535;
    return dim3((unsigned)(((p.N + 3) / 4 + 255) / 256), (unsigned)y, (unsigned)((p.M + y - 1) / y));
}

template <int TM, int TN, int WM, int WN, bool E5M2>
static hipError_t launch_tiles(const MatmulParams& p, hipStream_t st) {
    static KernelSetup setup;
    const hipError_t e = setup.ensure(reinterpret_cast<const void*>(fp8_matmul_kernel<TM, TN, WM, WN, E5M2>), matmul_smem<TM, TN, WM, WN>(), nullptr);
    if (e != hipSuccess) return e;
    const int64_t tiles = (p.M + TM - 1) / TM * ((p.N + TN - 1) / TN);
    hipLaunchKernelGGL((fp8_matmul_kernel<TM, TN, WM, WN, E5M2>), dim3((unsigned)tiles, (unsigned)p.parts), dim3(WM * WN * 64), (matmul_smem<TM, TN, WM, WN>()), st, p);
    return hipGetLastError();
}

template <bool E5M2>
static hipError_t launch_form(const MatmulParams& p, const MatmulPlan& w, hipStream_t st) {
    if (w.form == MatmulPlan::LARGE) return launch_tiles<256, 256, 2, 4, E5M2>(p, st);
    if (w.form == MatmulPlan::SMALL) return launch_tiles<128, 128, 2, 2, E5M2>(p, st);
    const unsigned x = (unsigned)((p.N + 15) / 16);
    if (p.M <= 16) hipLaunchKernelGGL((fp8_matmul_few_kernel<1, E5M2>), dim3(x), dim3(kFewWaves * 64), 0, st, p);
    else if (p.M <= 32) hipLaunchKernelGGL((fp8_matmul_few_kernel<2, E5M2>), dim3(x), dim3(kFewWaves * 64), 0, st, p);
    else hipLaunchKernelGGL((fp8_matmul_few_kernel<4, E5M2>), dim3(x), dim3(kFewWaves * 64), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_fp8_matmul(MatmulParams p, const MatmulPlan& w, hipStream_t st) {
    p.parts = w.parts;
    p.part_steps = w.part_steps;
    if (p.K == 0) {
        hipLaunchKernelGGL(fp8_matmul_bias_kernel, row_grid(p), dim3(256), 0, st, p);
        return hipGetLastError();
    }
    const hipError_t e = p.e5m2 ? launch_form<true>(p, w, st) : launch_form<false>(p, w, st);
    if (e != hipSuccess || p.parts == 1) return e;
    hipLaunchKernelGGL(fp8_matmul_join_kernel, row_grid(p), dim3(256), 0, st, p);
    return hipGetLastError();
}

}  // namespace pda

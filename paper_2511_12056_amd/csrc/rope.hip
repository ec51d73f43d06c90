// The pack with rotary positions and its gradient, bound by HBM.  Work split of pack_heads_kernel (layout.hip): a d-vector belongs to LPV = d/4 lanes, four
// consecutive columns each; a workgroup takes 256 / LPV consecutive tokens, here with several heads one after the other, because all heads of a token
// turn by the same angles: cos and sin are computed once a token and pair, into LDS, and each lane keeps those of its four columns in registers.
//
// An angle is position * frequency in 64 bits, in turns; the whole turns are taken off before the rest is rounded to 32 bits, so far positions lose
// nothing.  A lane's columns turn as x cos + partner * (-sin or sin): the partner lies in the same lane (interleaved) or rot/8 lanes away (half), which
// takes four lane permutations through LDS.
//
// 119 056 x 12 x 128, unit RMS: 146 us (5.0 TB/s), 427 with a head a workgroup.  2 x 4 797 x 12 x 64, the gradient: 15.7 us with a workgroup for half of the heads, 18.7 for all
// of them, 19.5 for one.
#include <hip/hip_runtime.h>
#include "attn_internal.h"
#include "proj_internal.h"
#include "train_device.h"

namespace pda {

template <bool BF16>
__device__ __forceinline__ float4 load_cols(const void* p, int64_t at) {
    if constexpr (BF16) {
        const u32x2 v = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(static_cast<const __bf16*>(p) + at));
        return make_float4(bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y));
    } else {
        return nt_load4(reinterpret_cast<const float4*>(static_cast<const float*>(p) + at));
    }
}
template <bool BF16>
__device__ __forceinline__ void store_cols(void* p, int64_t at, const float4& a) {
    if constexpr (BF16) nt_store2(reinterpret_cast<uint2*>(static_cast<__bf16*>(p) + at), pack_bf16(a.x, a.y), pack_bf16(a.z, a.w));
    else nt_store4(reinterpret_cast<float4*>(static_cast<float*>(p) + at), a);
}

template <int LPV, bool BWD, bool XBF16, bool RMS>
__global__ __launch_bounds__(256) void rope_kernel(const RopeParams p) {
    constexpr int TOK = 256 / LPV, U = 4;                       // tokens of a workgroup; heads in flight
    __shared__ float2 turn[TOK * LPV * 2];
    const int t = threadIdx.x, lane = t % LPV, tok = t / LPV, half = p.rot / 2;
    const int64_t bb = (int64_t)blockIdx.z * gridDim.y + blockIdx.y;
    if (bb >= p.token_blocks * p.B) return;
    int64_t b = 0, blk = bb;
    if (p.B > 1) { b = bb / p.token_blocks; blk = bb - b * p.token_blocks; }
    const int64_t s0 = blk * TOK;
    for (int k = t; k < TOK * half; k += 256) {
        const int tk = k / half, i = k - tk * half;
        const int64_t s = s0 + tk;
        if (s < p.S) {
            int axis = 0;
            while (axis < p.axes - 1 && i >= p.axis_end[axis]) ++axis;
            const double pos = p.positions ? (double)p.positions[b * p.pos_batch + s * p.axes + axis] : (double)(p.first + s);
            const double a = pos * p.turns[i];
            const float f = 2.0f * (float)(a - __builtin_rint(a));
            turn[k] = make_float2(cospif(f), sinpif(f));
        }
    }
    __syncthreads();
    const int64_t s = s0 + tok;
    const bool live = s < p.S;
    const int c = 4 * lane;
    const bool turns = c < p.rot && live, apart = p.layout == PDA_ROPE_HALF;
    // partner's lane in the wavefront (apart), and this lane's cosines and signed sines
    const int me = t & 63, other = !turns || !apart ? me : c < half ? me + p.rot / 8 : me - p.rot / 8;
    float co[4] = {1.f, 1.f, 1.f, 1.f}, si[4] = {0.f, 0.f, 0.f, 0.f};
    if (turns) {
        const float2* row = turn + tok * half;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 v = apart ? row[(c < half ? c : c - half) + e] : row[(c + e) / 2];
            const bool minus = (apart ? c < half : e % 2 == 0) != BWD;       // the gradient turns back
            co[e] = v.x;
            si[e] = minus ? -v.y : v.y;
        }
    }
    const auto rotate = [&](float4 a) __attribute__((always_inline)) {
        float4 o;
        if (apart) {
            const auto from = [&](float v) __attribute__((always_inline)) { return __uint_as_float(__builtin_amdgcn_ds_bpermute(other * 4, __float_as_uint(v))); };
            o = make_float4(from(a.x), from(a.y), from(a.z), from(a.w));
        } else {
            o = make_float4(a.y, a.x, a.w, a.z);
        }
        if (!turns) return a;                                   // also what is not finite stays as it is
        return make_float4(__builtin_fmaf(o.x, si[0], a.x * co[0]), __builtin_fmaf(o.y, si[1], a.y * co[1]),
                           __builtin_fmaf(o.z, si[2], a.z * co[2]), __builtin_fmaf(o.w, si[3], a.w * co[3]));
    };
    const int h0 = blockIdx.x * p.heads, h1 = h0 + p.heads < p.H ? h0 + p.heads : p.H;
    const int64_t xt = b * p.x_batch + s * p.x_token + c, yt = b * p.y_batch + s * (4 * LPV) + c, dt = b * p.dx_batch + s * p.dx_token + c;
    for (int h = h0; h < h1; h += U) {
        float4 x[U], g[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = g[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (live && h + u < h1) {
                if constexpr (!BWD || RMS) x[u] = load_cols<XBF16>(p.x, xt + (h + u) * (4 * LPV));
                if constexpr (BWD) g[u] = load_cols<true>(p.y, yt + (h + u) * p.y_head);
            }
        }
        bool again = false;
        // the hardware's 1/sqrt (1 ulp, of a normal number): far inside the bf16 rounding that follows
        const auto unit = [&](float ss) __attribute__((always_inline)) { return ss == 0.f ? 0.f : p.premul * __builtin_amdgcn_rsqf(ss * (1.0f / (4 * LPV))); };      // (NaN goes into the whole vector)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float4 a = x[u];
            float4 r;
            if constexpr (!BWD) {
                float f = p.premul;
                if constexpr (RMS) {
                    const float ss = sum_of_squares<LPV>(a);
                    again = again || into_range(ss) != 1.f;
                    f = unit(ss);
                }
                r = rotate(make_float4(a.x * f, a.y * f, a.z * f, a.w * f));
            } else {
                r = rotate(g[u]);
                if constexpr (RMS) {
                    const float ss = lane_sum<LPV>(a.x * a.x + a.y * a.y + a.z * a.z + a.w * a.w);
                    const float dot = lane_sum<LPV>(a.x * r.x + a.y * r.y + a.z * r.z + a.w * r.w);
                    // pack_heads_bwd_kernel's formula
                    const float f = ss == 0.f ? 0.f : ss < 0x1p-100f ? p.premul * sqrtf(4 * LPV) / sqrtf(ss) : p.premul / sqrtf(ss * (1.0f / (4 * LPV)));
                    const float m = ss == 0.f ? 0.f : -dot / ss;
                    r.x = f * __builtin_fmaf(a.x, m, r.x);
                    r.y = f * __builtin_fmaf(a.y, m, r.y);
                    r.z = f * __builtin_fmaf(a.z, m, r.z);
                    r.w = f * __builtin_fmaf(a.w, m, r.w);
                } else {
                    r.x *= p.premul; r.y *= p.premul; r.z *= p.premul; r.w *= p.premul;
                }
            }
            if (live && h + u < h1) {
                if constexpr (!BWD) store_cols<true>(p.y, yt + (h + u) * p.y_head, r);
                else store_cols<XBF16>(p.dx, dt + (h + u) * (4 * LPV), r);
            }
        }
        if constexpr (!BWD && RMS) {                            // written again: in front of the stores the branch would keep the heads' sums apart, 119 056 x 12 x 128: 146 us instead of 145 (144 without it)
            if (__any(again)) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float by = into_range(sum_of_squares<LPV>(x[u]));
                    float4 a = make_float4(x[u].x * by, x[u].y * by, x[u].z * by, x[u].w * by);
                    const float f = unit(sum_of_squares<LPV>(a));
                    a = rotate(make_float4(a.x * f, a.y * f, a.z * f, a.w * f));
                    if (by != 1.f && live && h + u < h1) store_cols<true>(p.y, yt + (h + u) * p.y_head, a);
                }
            }
        }
    }
}

template <int LPV, bool BWD, bool XBF16>
static hipError_t launch(RopeParams& p, int n_cu, hipStream_t st) {
    constexpr int TOK = 256 / LPV;
    p.token_blocks = (p.S + TOK - 1) / TOK;
    const int64_t rows = p.token_blocks * p.B, y = rows < 65535 ? rows : 65535;
    // all heads of its tokens for a workgroup, fewer where that leaves compute units with less than four of them
    const int64_t chunks = rows >= 4 * (int64_t)n_cu ? 1 : (4 * (int64_t)n_cu + rows - 1) / rows;
    p.heads = chunks >= p.H ? 1 : (int)((p.H + chunks - 1) / chunks);
    const dim3 grid((unsigned)((p.H + p.heads - 1) / p.heads), (unsigned)y, (unsigned)((rows + y - 1) / y));
    if (p.unit_rms) hipLaunchKernelGGL((rope_kernel<LPV, BWD, XBF16, true>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((rope_kernel<LPV, BWD, XBF16, false>), grid, dim3(256), 0, st, p);
    return hipGetLastError();
}

template <int LPV>
static hipError_t launch(RopeParams& p, bool backward, int n_cu, hipStream_t st) {
    if (backward) return p.x_bf16 ? launch<LPV, true, true>(p, n_cu, st) : launch<LPV, true, false>(p, n_cu, st);
    return p.x_bf16 ? launch<LPV, false, true>(p, n_cu, st) : launch<LPV, false, false>(p, n_cu, st);
}

hipError_t launch_rope(RopeParams& p, int d, bool backward, int n_cu, hipStream_t st) {
    return d == 128 ? launch<32>(p, backward, n_cu, st) : launch<16>(p, backward, n_cu, st);
}

}  // namespace pda

// Attention backward, gfx950, d = 128 and 64: dq, dk, dv from dout and the forward call's log-sum-exp.
//
// Two kinds of work items in one launch, both of which compute the probabilities again:
//   * keys:    128 keys of a head stay (k and v rows as MFMA operands in registers), its query rows stream by:
//              S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS                        4 products
//   * queries: 128 query rows stay (q and dout), the head's keys stream by:
//              S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T                                   3 products
// Seven products where five are the least: one item kind that also summed dq would have to add to the same dq rows
// from every block of keys, in an order that changes from run to run (atomics), or keep dq partials of every block.
//
// As in the forward kernels the products are taken so that one resident row lies in each lane pair (l, l + 32) of a wavefront, and
// the exponentiated scores in their accumulator registers are the operand of the next product as they stand, because the
// contraction index is permuted identically on both sides (the transposing LDS reads).
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "attn_internal.h"
#include "train_device.h"
#include "train_internal.h"

namespace pda {

constexpr float kLog2e = 1.4426950408889634f;

// Row-dependent XOR on the 16-byte granules of a tile's rows.  The tiles here are read both ways: 16 rows, one
// granule each (ds_read_b128), and four consecutive rows, four granules each (transposing reads); see swz_k and swz_v for either alone.  The row's two
// low bits choose the group of four granules, the next two the place in it, so both touch every bank once.
template <int D>
__device__ __forceinline__ constexpr int swz_kv(int row) {
    return D == 128 ? ((row & 3) << 2 | ((row >> 2) & 3)) : (((row >> 1) & 1) << 2 | ((row >> 2) & 3));
}

// ---- delta and the log-sum-exp in units of log2, 16 or 8 lanes a row -----------------------------------------
template <int D, bool OUT16>
__global__ __launch_bounds__(256) void attn_bwd_stats_kernel(const AttnBwdParams p) {
    constexpr int LPR = D / 8;
    const int lane = threadIdx.x % LPR;
    const int64_t row = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int bh = blockIdx.y, b = bh / p.H, h = bh - b * p.H;
    if (row >= p.stat_rows) return;
    float sum = 0.f;
    if (row < p.Sq) {
        const u32x4 g = *reinterpret_cast<const u32x4*>(p.dout + (int64_t)b * p.do_bs + (int64_t)h * p.do_hs + row * D + lane * 8);
        const int64_t at = (int64_t)b * p.o_bs + (int64_t)h * p.o_hs + row * D + lane * 8;
        float o[8];
        if constexpr (OUT16) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(static_cast<const __bf16*>(p.out) + at);
#pragma unroll
            for (int i = 0; i < 4; ++i) { o[2 * i] = bf16_lo(x[i]); o[2 * i + 1] = bf16_hi(x[i]); }
        } else {
            const f32x4 x = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.out) + at);
            const f32x4 y = *reinterpret_cast<const f32x4*>(static_cast<const float*>(p.out) + at + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { o[i] = x[i]; o[4 + i] = y[i]; }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sum = __builtin_fmaf(bf16_hi(g[i]), o[2 * i + 1], __builtin_fmaf(bf16_lo(g[i]), o[2 * i], sum));
    }
    sum = lane_sum<LPR>(sum);
    if (lane == 0) {
        float l = -INFINITY;
        if (row < p.Sq) {
            const float x = p.lse[(int64_t)b * p.l_bs + (int64_t)h * p.l_hs + row];
            l = x == -INFINITY ? -INFINITY : -x * kLog2e;
        }
        p.nlse2[bh * p.stat_rows + row] = l;
        p.ndelta[bh * p.stat_rows + row] = -sum;
    }
}

// ---- the products ---------------------------------------------------------------------------------------------
constexpr int kBwdTile = 32;            // streamed rows of a step
constexpr int kBwdRows = 128;           // resident rows of a workgroup: 32 a wavefront
constexpr int bwd_smem(int d) { return 2 * 2 * kBwdTile * d * 2; }

template <int D, bool KEYS>
__device__ __forceinline__ void attn_bwd_item(const AttnBwdParams& p, int bh, int64_t row0) {
    extern __shared__ __attribute__((aligned(256))) unsigned char bwd_smem_[];
    constexpr int G = D / 8, NKK = D / 16, NDB = D / 32;
    constexpr int TILE = kBwdTile * D * 2, CPT = TILE / 1024, RPC = 1024 / (D * 2);
    const int lane = threadIdx.x & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int b = bh / p.H, h = bh - b * p.H;
    const __bf16* qp = p.q + (int64_t)b * p.q_bs + (int64_t)h * p.q_hs;
    const __bf16* dop = p.dout + (int64_t)b * p.do_bs + (int64_t)h * p.do_hs;
    const __bf16* kp = p.k + (int64_t)b * p.kv_bs + (int64_t)h * p.kv_hs;
    const __bf16* vp = p.v + (int64_t)b * p.kv_bs + (int64_t)h * p.kv_hs;
    const float* nlse2 = p.nlse2 + bh * p.stat_rows;
    const float* ndelta = p.ndelta + bh * p.stat_rows;
    const int64_t n_res = KEYS ? p.n_v : p.Sq, n_str = KEYS ? p.Sq : p.n_v;
    const int64_t row = row0 + wave * 32 + li;                 // this lane's resident row
    const int nt = row0 < n_res ? (int)((n_str + kBwdTile - 1) / kBwdTile) : 0;

    f32x16 acc1[NDB], acc2[KEYS ? NDB : 1];                    // dK^T or dQ^T; dV^T
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            acc1[db][r] = 0.f;
            if constexpr (KEYS) acc2[db][r] = 0.f;
        }
    if (nt > 0) {
        const __bf16* s1 = KEYS ? qp : kp;
        const __bf16* s2 = KEYS ? dop : vp;
        LDS_PTR(unsigned char) smem = (LDS_PTR(unsigned char))bwd_smem_;
        const unsigned lds0 = (unsigned)(uintptr_t)smem;
        // chunk j of a tile holds rows j RPC ..; wavefront w fetches chunks w, w + 4 of both tensors
        auto issue = [&](int t) __attribute__((always_inline)) {
            const int last = (int)(n_str - 1 - (int64_t)t * kBwdTile < kBwdTile - 1 ? n_str - 1 - (int64_t)t * kBwdTile : kBwdTile - 1);
            const unsigned to = lds0 + (t & 1) * 2 * TILE;
#pragma unroll
            for (int i = 0; i < CPT / 4; ++i) {
                const int j = wave + 4 * i;
                const int r = j * RPC + lane / G, c = r < last ? r : last;      // rows behind the last: that row again
                const unsigned off = c * (D * 2) + (((lane % G) ^ swz_kv<D>(r)) * 16);
                lds_dma16(s1 + (int64_t)t * (kBwdTile * D), off, to + j * 1024);
                lds_dma16(s2 + (int64_t)t * (kBwdTile * D), off, to + TILE + j * 1024);
            }
        };
        issue(0);
        bf16x8 r1[NKK], r2[NKK];
        {
            const int64_t c = row < n_res ? row : n_res - 1;
            const __bf16* a1 = (KEYS ? kp : qp) + c * D + lh * 8;
            const __bf16* a2 = (KEYS ? vp : dop) + c * D + lh * 8;
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) {
                r1[kk] = *reinterpret_cast<const bf16x8*>(a1 + kk * 16);
                r2[kk] = *reinterpret_cast<const bf16x8*>(a2 + kk * 16);
            }
        }
        float l_res = 0.f, d_res = 0.f;
        if constexpr (!KEYS) {
            l_res = row < n_res ? nlse2[row] : -INFINITY;
            d_res = row < n_res ? ndelta[row] : 0.f;
        }
        wait_vmcnt<0>();
        __syncthreads();
        const int t16 = lane & 15, tr_row = 4 * lh + (t16 >> 2);
        auto rows_frag = [&](LDS_PTR(const unsigned char) tile, int kk) __attribute__((always_inline)) {
            return *(LDS_PTR(const bf16x8))(tile + li * (D * 2) + (((2 * kk + lh) ^ swz_kv<D>(li)) * 16));
        };
        auto tr_frag = [&](LDS_PTR(const unsigned char) tile, int db, int u) __attribute__((always_inline)) {
            const int g = db * 4 + 2 * (li >> 4) + ((t16 & 3) >> 1);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(tile + (u * 16 + tr_row) * (D * 2) + ((g ^ swz_kv<D>(tr_row)) * 16) + (t16 & 1) * 8));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(tile + (u * 16 + tr_row + 8) * (D * 2) + ((g ^ swz_kv<D>(tr_row + 8)) * 16) + (t16 & 1) * 8));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        const float c = p.scale_log2e;
        for (int t = 0; t < nt; ++t) {
            if (t + 1 < nt) issue(t + 1);
            LDS_PTR(const unsigned char) t1 = (LDS_PTR(const unsigned char))smem + (t & 1) * 2 * TILE;
            LDS_PTR(const unsigned char) t2 = t1 + TILE;
            f32x16 s, dp;
            f32x4 l[4];
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                f32x4 dl = {d_res, d_res, d_res, d_res};
                l[a] = f32x4{l_res, l_res, l_res, l_res};
                if constexpr (KEYS) {
                    l[a] = *reinterpret_cast<const f32x4*>(nlse2 + t * kBwdTile + 8 * a + 4 * lh);
                    dl = *reinterpret_cast<const f32x4*>(ndelta + t * kBwdTile + 8 * a + 4 * lh);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) { s[4 * a + e] = 0.f; dp[4 * a + e] = dl[e]; }
            }
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows_frag(t1, kk), r1[kk], s, 0, 0, 0);
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rows_frag(t2, kk), r2[kk], dp, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, l[r / 4][r % 4]));
            if (!KEYS && (int64_t)(t + 1) * kBwdTile > n_str) {
                const int hidden = (int)(n_str - (int64_t)t * kBwdTile) - 4 * lh;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if ((r >> 2) * 8 + (r & 3) >= hidden) s[r] = 0.f;
            }
            u32x4 pk[2], ds[2];
#pragma unroll
            for (int r = 0; r < 16; r += 2) {
                pk[r / 8][(r % 8) / 2] = pack_bf16(s[r], s[r + 1]);
                ds[r / 8][(r % 8) / 2] = pack_bf16(s[r] * dp[r], s[r + 1] * dp[r + 1]);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int db = 0; db < NDB; ++db) {
                    if constexpr (KEYS) acc2[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr_frag(t2, db, u), __builtin_bit_cast(bf16x8, pk[u]), acc2[db], 0, 0, 0);
                    acc1[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tr_frag(t1, db, u), __builtin_bit_cast(bf16x8, ds[u]), acc1[db], 0, 0, 0);
                }
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __syncthreads();
        }
    }
    // ---- results: 16 bytes a lane (the lane pair's halves of eight columns trade places)
    const int64_t n_out = KEYS ? p.Skv : p.Sq;
    auto store = [&](const f32x16* acc, __bf16* base, float factor) __attribute__((always_inline)) {
        const bool hidden = KEYS && row >= n_res;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int a = 0; a < 4; a += 2) {
                unsigned x[2][2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        x[i][e] = hidden ? 0u : pack_bf16(acc[db][4 * (a + i) + 2 * e] * factor, acc[db][4 * (a + i) + 2 * e + 1] * factor);
                const auto lo = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
                const auto hi = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
                if (row < n_out) *reinterpret_cast<u32x4*>(base + row * D + db * 32 + a * 8 + lh * 8) = u32x4{lo[0], hi[0], lo[1], hi[1]};
            }
    };
    if constexpr (KEYS) {
        store(acc1, p.dk + (int64_t)b * p.dkv_bs + (int64_t)h * p.dkv_hs, p.scale);
        store(acc2, p.dv + (int64_t)b * p.dkv_bs + (int64_t)h * p.dkv_hs, 1.0f);
    } else {
        store(acc1, p.dq + (int64_t)b * p.dq_bs + (int64_t)h * p.dq_hs, p.scale);
    }
}

template <int D>
__global__ __launch_bounds__(256, 1) void attn_bwd_kernel(const AttnBwdParams p) {
    const int key_blocks = (int)((p.Skv + kBwdRows - 1) / kBwdRows), query_blocks = (int)((p.Sq + kBwdRows - 1) / kBwdRows);
    int i = (int)blockIdx.x;
    const int key_items = key_blocks * p.B * p.H;
    if (i < key_items) {
        attn_bwd_item<D, true>(p, i / key_blocks, (int64_t)(i % key_blocks) * kBwdRows);
    } else {
        i -= key_items;
        attn_bwd_item<D, false>(p, i / query_blocks, (int64_t)(i % query_blocks) * kBwdRows);
    }
}

template <int D>
static hipError_t launch_bwd(const AttnBwdParams& p, hipStream_t st) {
    const int BH = p.B * p.H;
    if (p.Sq > 0) {
        constexpr int rows = 256 / (D / 8);
        const dim3 grid((unsigned)((p.stat_rows + rows - 1) / rows), (unsigned)BH);
        if (p.out_bf16) hipLaunchKernelGGL((attn_bwd_stats_kernel<D, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((attn_bwd_stats_kernel<D, false>), grid, dim3(256), 0, st, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int64_t items = ((p.Skv + kBwdRows - 1) / kBwdRows + (p.Sq + kBwdRows - 1) / kBwdRows) * BH;
    if (items > 0x7fffffff) return hipErrorInvalidValue;
    hipLaunchKernelGGL(attn_bwd_kernel<D>, dim3((unsigned)items), dim3(256), bwd_smem(D), st, p);
    return hipGetLastError();
}

hipError_t launch_attn_bwd(const AttnBwdParams& p, int d, hipStream_t st) {
    return d == 128 ? launch_bwd<128>(p, st) : launch_bwd<64>(p, st);
}

}  // namespace pda

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
        float* to = p.stats + (bh * p.stat_rows + row / 32 * 32) * 2 + row % 32;
        to[0] = l;
        to[32] = -sum;
    }
}

// ---- the products ---------------------------------------------------------------------------------------------
constexpr int kBwdTile = 32;            // streamed rows of a step
constexpr int kBwdRows = 256;           // resident rows of a workgroup: 64 for each of four pairs of wavefronts
constexpr int kBwdRing = 4;             // tile buffers per streamed tensor
constexpr int kBwdExchange = 64 * kBwdTile * 4;          // bytes of the probabilities of a pair and step
constexpr int bwd_tile_bytes(int d) { return kBwdTile * d * 2; }
constexpr int bwd_stat_base(int d) { return kBwdRing * 2 * bwd_tile_bytes(d); }
constexpr int bwd_p_base(int d) { return bwd_stat_base(d) + kBwdRing * 256; }
constexpr int bwd_smem(int d) { return bwd_p_base(d) + 2 * 4 * kBwdExchange; }

// 4 bytes per lane from global memory straight into LDS (see lds_dma16).
__device__ __forceinline__ void lds_dma4(const void* sbase, unsigned voff, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 vcc, %2\n\tglobal_load_lds_dword %1, vcc"
                 :
                 : "s"(lds_addr), "v"(voff), "s"(sbase)
                 : "memory", "m0", "vcc");
}

template <int D, bool KEYS>
__device__ __forceinline__ void attn_bwd_item(const AttnBwdParams& p, int bh, int64_t row0) {
    constexpr int G = D / 8, NKK = D / 16, NDB = D / 32;
    constexpr int TILE = bwd_tile_bytes(D), RPC = 1024 / (D * 2);
    constexpr int LPI = D == 128 ? 2 : 1;                      // loads of a wavefront per step: a chunk of both tensors, or of one
    constexpr int PF = 3;                                      // operand fragments read ahead
    extern __shared__ __attribute__((aligned(256))) unsigned char bwd_smem_[];
    const unsigned lds0 = (unsigned)(uintptr_t)(LDS_PTR(unsigned char))bwd_smem_;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), pair = wave & 3;
    const int lane = opaque_lane(), li = lane & 31, lh = lane >> 5;
    const bool second = wave >= 4;
    const int b = bh / p.H, h = bh - b * p.H;
    const __bf16* qp = p.q + (int64_t)b * p.q_bs + (int64_t)h * p.q_hs;
    const __bf16* dop = p.dout + (int64_t)b * p.do_bs + (int64_t)h * p.do_hs;
    const __bf16* kp = p.k + (int64_t)b * p.kv_bs + (int64_t)h * p.kv_hs;
    const __bf16* vp = p.v + (int64_t)b * p.kv_bs + (int64_t)h * p.kv_hs;
    const float* stats = p.stats + bh * p.stat_rows * 2;
    const int64_t n_res = KEYS ? p.n_v : p.Sq;
    const int n_str = (int)(KEYS ? p.Sq : p.n_v);
    const int64_t first = row0 + pair * 64;                    // this lane's resident rows: first + li and first + 32 + li
    const int nt = row0 < n_res ? (n_str + kBwdTile - 1) / kBwdTile : 0;

    // ---- loads of the streamed tiles
    const __bf16* s1 = KEYS ? qp : kp;
    const __bf16* s2 = KEYS ? dop : vp;
    auto issue = [&](int t) __attribute__((always_inline)) {
        const int slot = t % kBwdRing;
        const int last = n_str - 1 - t * kBwdTile;
        const int j = D == 128 ? wave : pair, r = j * RPC + lane / G;
        const int c = r < last ? r : last;                     // rows behind the last: that row again
        const unsigned off = c * (D * 2) + (((lane % G) ^ swz_kv<D>(r)) * 16);
        const unsigned to = lds0 + slot * 2 * TILE + j * 1024;
        if (D == 128 || !second) lds_dma16(s1 + (int64_t)t * (kBwdTile * D), off, to);
        if (D == 128 || second) lds_dma16(s2 + (int64_t)t * (kBwdTile * D), off, to + TILE);
        if (KEYS && wave == 4) lds_dma4(stats + (int64_t)t * (2 * kBwdTile), lane * 4, lds0 + bwd_stat_base(D) + slot * 256);
    };
    // the end of step t: what step t + 1 needs is there, what was fetched in this step may be under way
    auto step_end = [&](int t) __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        if (t + 2 < nt) {
            if (KEYS && wave == 4) wait_vmcnt<LPI + 1>();
            else wait_vmcnt<LPI>();
        } else {
            wait_vmcnt<0>();
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

    // ---- operand addresses in slot 0; blocks are XORed in
    const int t16 = lane & 15, tr_row = 4 * lh + (t16 >> 2), tr_g = 2 * (li >> 4) + ((t16 & 3) >> 1);
    const unsigned rows_at = lds0 + li * (D * 2) + ((lh ^ swz_kv<D>(li)) * 16);
    const unsigned tr_lo = lds0 + tr_row * (D * 2) + ((tr_g ^ swz_kv<D>(tr_row)) * 16) + (t16 & 1) * 8;
    const unsigned tr_hi = lds0 + (tr_row + 8) * (D * 2) + ((tr_g ^ swz_kv<D>(tr_row + 8)) * 16) + (t16 & 1) * 8;
    auto block = [](unsigned at, auto n) __attribute__((always_inline)) {
        unsigned r = at;
        if constexpr (decltype(n)::value != 0) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(r) : "n"(decltype(n)::value), "v"(at));
        return r;
    };
    auto rows_frag = [&](unsigned at, auto kk) __attribute__((always_inline)) {
        return *(LDS_PTR(const bf16x8))(LDS_PTR(const unsigned char))(uintptr_t)block(at, std::integral_constant<int, decltype(kk)::value * 32>{});
    };
    auto tr_frag = [&](unsigned lo_at, unsigned hi_at, auto idx) __attribute__((always_inline)) {      // idx = u * NDB + db
        constexpr int db = decltype(idx)::value % NDB, u = decltype(idx)::value / NDB;
        LDS_PTR(const unsigned char) x = (LDS_PTR(const unsigned char))(uintptr_t)block(lo_at, std::integral_constant<int, db * 64>{});
        LDS_PTR(const unsigned char) y = (LDS_PTR(const unsigned char))(uintptr_t)block(hi_at, std::integral_constant<int, db * 64>{});
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(x + u * 16 * (D * 2)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(y + u * 16 * (D * 2)));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const unsigned p_at = lds0 + bwd_p_base(D) + pair * kBwdExchange + lane * 16;
    auto exchange = [&](int t, int i, int a) __attribute__((always_inline)) {
        return (LDS_PTR(f32x4))(LDS_PTR(unsigned char))(uintptr_t)(p_at + (t & 1) * (4 * kBwdExchange) + (i * 4 + a) * 1024);
    };
    auto stat_at = [&](int t, int which, int a) __attribute__((always_inline)) {
        return *(LDS_PTR(const f32x4))(LDS_PTR(const unsigned char))(uintptr_t)(lds0 + bwd_stat_base(D) + (t % kBwdRing) * 256 + which * 128 + 32 * a + 16 * lh);
    };

    // ---- resident rows
    bf16x8 res[2][NKK];
    float res_stat[2] = {0.f, 0.f};
    f32x16 acc[2][NDB];                                        // first wavefront of a pair: dV^T; second: dK^T or dQ^T
    if (nt > 0) {
        issue(0);
        if (nt > 1) issue(1);
        const __bf16* src = second ? (KEYS ? vp : dop) : (KEYS ? kp : qp);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t c = first + li + 32 * i < n_res ? first + li + 32 * i : n_res - 1;
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) res[i][kk] = *reinterpret_cast<const bf16x8*>(src + c * D + lh * 8 + kk * 16);
            if constexpr (!KEYS) res_stat[i] = stats[(c / kBwdTile) * (2 * kBwdTile) + (second ? kBwdTile : 0) + c % kBwdTile];
        }
        wait_vmcnt<0>();
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][db][r] = 0.f;
    const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    bf16x8 frag[PF + 1];
    auto step = []() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };

    if (!second) {
        const float c = p.scale_log2e;
        for (int t = 0; t < nt; ++t) {
            if (t + 2 < nt) issue(t + 2);
            const unsigned slot = (t % kBwdRing) * 2 * TILE;
            f32x16 s[2];
            {
                const unsigned at = rows_at + slot;
                static_for<0, PF>([&](auto j) { frag[decltype(j)::value] = rows_frag(at, j); });
                static_for<0, NKK>([&](auto j) {
                    constexpr int n = decltype(j)::value;
                    if constexpr (n + PF < NKK) frag[(n + PF) % (PF + 1)] = rows_frag(at, std::integral_constant<int, n + PF>{});
#pragma unroll
                    for (int i = 0; i < 2; ++i) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % (PF + 1)], res[i][n], n == 0 ? zero : s[i], 0, 0, 0);
                    step();
                });
            }
            const unsigned lo = tr_lo + slot + TILE, hi = tr_hi + slot + TILE;
            if constexpr (KEYS) static_for<0, PF>([&](auto j) { frag[decltype(j)::value] = tr_frag(lo, hi, j); });
            u32x4 pk[2][2];
            const bool tail = !KEYS && (t + 1) * kBwdTile > n_str;
            const int hidden = n_str - t * kBwdTile - 4 * lh;
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                f32x4 l;
                if constexpr (KEYS) l = stat_at(t, 0, a);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (!KEYS) l = f32x4{res_stat[i], res_stat[i], res_stat[i], res_stat[i]};
                    f32x4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][4 * a + e], c, l[e]));
                    if (tail)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[e] = 8 * a + e >= hidden ? 0.f : x[e];
                    *exchange(t, i, a) = x;
                    if constexpr (KEYS) {
                        pk[i][a / 2][(a % 2) * 2] = pack_bf16(x[0], x[1]);
                        pk[i][a / 2][(a % 2) * 2 + 1] = pack_bf16(x[2], x[3]);
                    }
                }
                step();
            }
            if constexpr (KEYS) {
                static_for<0, 2 * NDB>([&](auto j) {
                    constexpr int n = decltype(j)::value;
                    if constexpr (n + PF < 2 * NDB) frag[(n + PF) % (PF + 1)] = tr_frag(lo, hi, std::integral_constant<int, n + PF>{});
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        acc[i][n % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % (PF + 1)], __builtin_bit_cast(bf16x8, pk[i][n / NDB]), acc[i][n % NDB], 0, 0, 0);
                    step();
                });
            }
            step_end(t);
        }
    } else {
        f32x16 dp[2];
        // ds of step t - 1 (its p is there), its products, then dp of step t
        auto sums = [&](int t) __attribute__((always_inline)) {
            const unsigned slot = (t % kBwdRing) * 2 * TILE;
            const unsigned lo = tr_lo + slot, hi = tr_hi + slot;
            u32x4 ds[2][2];
            static_for<0, PF>([&](auto j) { frag[decltype(j)::value] = tr_frag(lo, hi, j); });
#pragma unroll
            for (int a = 0; a < 4; ++a) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const f32x4 x = *exchange(t, i, a);
                    float y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = x[e] * (KEYS ? dp[i][4 * a + e] : dp[i][4 * a + e] + res_stat[i]);
                    ds[i][a / 2][(a % 2) * 2] = pack_bf16(y[0], y[1]);
                    ds[i][a / 2][(a % 2) * 2 + 1] = pack_bf16(y[2], y[3]);
                }
            }
            step();
            static_for<0, 2 * NDB>([&](auto j) {
                constexpr int n = decltype(j)::value;
                if constexpr (n + PF < 2 * NDB) frag[(n + PF) % (PF + 1)] = tr_frag(lo, hi, std::integral_constant<int, n + PF>{});
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    acc[i][n % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % (PF + 1)], __builtin_bit_cast(bf16x8, ds[i][n / NDB]), acc[i][n % NDB], 0, 0, 0);
                step();
            });
        };
        auto products = [&](int t) __attribute__((always_inline)) {
            const unsigned at = rows_at + (t % kBwdRing) * 2 * TILE + TILE;
            if constexpr (KEYS) {
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const f32x4 x = stat_at(t, 1, a);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dp[0][4 * a + e] = dp[1][4 * a + e] = x[e];
                }
            }
            static_for<0, PF>([&](auto j) { frag[decltype(j)::value] = rows_frag(at, j); });
            static_for<0, NKK>([&](auto j) {
                constexpr int n = decltype(j)::value;
                if constexpr (n + PF < NKK) frag[(n + PF) % (PF + 1)] = rows_frag(at, std::integral_constant<int, n + PF>{});
#pragma unroll
                for (int i = 0; i < 2; ++i) dp[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % (PF + 1)], res[i][n], !KEYS && n == 0 ? zero : dp[i], 0, 0, 0);
                step();
            });
        };
        for (int t = 0; t < nt; ++t) {
            if (t + 2 < nt) issue(t + 2);
            if (t > 0) sums(t - 1);
            products(t);
            step_end(t);
        }
        if (nt > 0) sums(nt - 1);
    }

    // ---- results: 16 bytes a lane (the lane pair's halves of eight columns trade places)
    const int64_t n_out = KEYS ? p.Skv : p.Sq;
    if (KEYS || second) {
        const int end_lane = opaque_lane(), col = (end_lane >> 5) * 8;      // formed here, not kept through the steps
        const float factor = second ? p.scale : 1.0f;
        __bf16* base = p.dq + (int64_t)b * p.dq_bs + (int64_t)h * p.dq_hs;
        if constexpr (KEYS) {
            base = p.dv + (int64_t)b * p.dkv_bs + (int64_t)h * p.dkv_hs;
            if (second) base += p.dk - p.dv;                   // (a choice of one of two arguments would put both into scratch memory)
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t r = first + (end_lane & 31) + 32 * i;
            const bool hidden = KEYS && r >= n_res;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int a = 0; a < 4; a += 2) {
                    unsigned x[2][2];
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            x[j][e] = hidden ? 0u : pack_bf16(acc[i][db][4 * (a + j) + 2 * e] * factor, acc[i][db][4 * (a + j) + 2 * e + 1] * factor);
                    const auto l = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
                    const auto u = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
                    if (r < n_out) *reinterpret_cast<u32x4*>(base + r * D + db * 32 + a * 8 + col) = u32x4{l[0], u[0], l[1], u[1]};
                }
        }
    }
}

template <int D>
__global__ __launch_bounds__(512, 2) void attn_bwd_kernel(const AttnBwdParams p) {
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
    static KernelSetup setup;
    const hipError_t e = setup.ensure(reinterpret_cast<const void*>(attn_bwd_kernel<D>), bwd_smem(D), nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(attn_bwd_kernel<D>, dim3((unsigned)items), dim3(512), bwd_smem(D), st, p);
    return hipGetLastError();
}

hipError_t launch_attn_bwd(const AttnBwdParams& p, int d, hipStream_t st) {
    return d == 128 ? launch_bwd<128>(p, st) : launch_bwd<64>(p, st);
}

}  // namespace pda

// Attention backward, gfx950, d = 128 and 64: dq, dk, dv from dout and the forward call's log-sum-exp.
//
//   P = exp(scale Q K^T - lse),  delta_i = <dout_i, out_i>,  dS = P (dO V^T - delta),
//   dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K
//
// Two kinds of work items in one launch, both of which compute the probabilities again:
//   * keys:    256 keys of a head stay (k and v rows as MFMA operands in registers), its query rows stream by, 32 a step:
//              S = Q K^T, dP = dO V^T, dV^T += dO^T P, dK^T += Q^T dS                        4 products
//   * queries: 256 query rows stay (q and dout), the head's valid keys stream by:
//              S^T = K Q^T, dP^T = V dO^T, dQ^T += K^T dS^T                                   3 products
// Seven products where five are the least: one kind of item that also summed dq would have to add to the same dq rows from every block of keys, in an
// order that changes from run to run (atomics), or keep dq partials of every block (256 rows' worth of reads and writes for a step's work).
// The same call gives the same bits.
//
// As in the forward kernels the products are taken so that one resident row lies in each lane pair (l, l + 32) of a wavefront, and
// the exponentiated scores in their accumulator registers are the operand of the next product as they stand, because the
// contraction index is permuted identically on both sides (the transposing LDS reads).
//
// What bounds it: the matrix cores and, beside them, the arithmetic of the softmax, which both kinds of items do.  On a SIMD that is full of matrix
// instructions a vector instruction costs 6 cycles and an exponential 11, a 32x32x16 product 33.  So each SIMD has two wavefronts, of which one is in matrix
// instructions while the other computes, held in step by barriers: the split differs by d.
//   * d = 128: a step has twice the products for the same exponentials, and the sums of 64 rows and two gradients do not fit one wavefront's registers.  Two
//     wavefronts share 64 resident rows (attn_bwd_pair_item): one has the scores, the probabilities and dV, the other dP, dS and dK or dQ.
//     Without the phases, both wavefronts through their steps as they come, 24 x 9 600 3.80 instead of 3.40 ms.
//   * d = 64: a wavefront has 32 resident rows to itself (attn_bwd_lone_item), so that the probabilities stay in its registers.  Pairs instead:
//     24 x 9 600 2 146 us and then 2 058, 6 x 33 000 6 457 and 6 020, 24 x 4 797 on 4 701 559 and 545, 2 x 1 024 23.5 and 22.2.  (At d = 128 such wavefronts spill.)
// Rounding to bf16: P as the operand of dV and dS as the operand of dK and dQ, as in the forward call; the P in dS stays fp32 (rounded there too,
// dq and dk are off by 0.0029 instead of 0.0024 of the largest value).
// Measured, whole call (floating-point operations of the five products that are the least, 10 Sq n_v d, per second): d = 128: 3 x 67 576 on 67 476 18.3 ms
// = 954 TFLOP/s (the seven products run at 1 340, as fast as a large library product), 24 x 9 600 3.04 ms = 930, 1 x 9 600 160 us = 736, 24 x 16 384 on 570
// 484 us = 593 (a sixth of its products are of rows behind the last key); d = 64: 6 x 33 000 5.29 ms = 791, 24 x 4 797 on 4 701 492 us = 704, 2 x 1 024 18.6 us = 72
// (three launches, parts of four steps).  Cards differ by up to 5 %.  The matrix cores are busy 72 % of the time in 24 x 9 600, 61 % in 24 x 16 384 on 570 and 53 % in 24 x 4 797, d = 64; no bank conflicts.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "attn_internal.h"
#include "train_device.h"
#include "train_internal.h"

namespace pda {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaitLoads = 0x0f70;      // s_waitcnt vmcnt(0), the other counters not waited for

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
    const int64_t row = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * (256 / LPR) + threadIdx.x / LPR;
    const int bh = blockIdx.y, b = bh / p.H, h = bh - b * p.H;
    if (row >= p.stat_rows) return;
    if (row == 0 && bh == 0 && lane == 0) *p.counter = 0;      // for the kernel that follows
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
        const float delta = l == -INFINITY ? 0.f : -sum;       // a row without keys: whatever stands in its out
        if constexpr (D == 64) {
            // each as a sum of three bf16 (24 bits, nothing is lost), 8 bytes that are the operand of a product with ones (attn_bwd_lone_item).  l in units of
            // the scores, finite in a row without keys: no score comes near 2^100.
            l /= p.scale_log2e;                                // may pass fp32's range
            l = l < -0x1p100f ? -0x1p100f : l;                 // (NaN stays)
            auto rest = [](float x) { return x - __uint_as_float(pack_bf16(x, 0.f) << 16); };
            const float l1 = rest(l), l2 = rest(l1), d1 = rest(delta), d2 = rest(d1);
            *reinterpret_cast<u32x4*>(p.stats + (bh * p.stat_rows + row) * 4) = u32x4{pack_bf16(l, l1), pack_bf16(l2, 0.f), pack_bf16(delta, d1), pack_bf16(d2, 0.f)};
        } else {
            float* to = p.stats + (bh * p.stat_rows + row / 32 * 32) * 2 + row % 32;
            to[0] = l;
            to[32] = delta;
        }
    }
}

// ---- the products ---------------------------------------------------------------------------------------------
constexpr int kBwdRing = 5;             // tile buffers per streamed tensor
constexpr int kBwdAhead = 3;            // tile t + kBwdAhead is fetched in step t, into the buffer of tile t - 2
constexpr int kBwdExchange = 64 * kBwdTile * 4;          // bytes of the probabilities of a pair and step
constexpr int bwd_tile_bytes(int d) { return kBwdTile * d * 2; }
constexpr int bwd_stat_base(int d) { return kBwdRing * 2 * bwd_tile_bytes(d); }
constexpr int bwd_p_base(int d) { return bwd_stat_base(d) + kBwdRing * 256; }
constexpr int bwd_next_base(int d) { return bwd_p_base(d) + 4 * kBwdExchange; }      // two places for the next item's number
constexpr int bwd_smem(int d) { return bwd_next_base(d) + 16; }

// 4 bytes per lane from global memory straight into LDS (see lds_dma16).
__device__ __forceinline__ void lds_dma4(const void* sbase, unsigned voff, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 vcc, %2\n\tglobal_load_lds_dword %1, vcc"
                 :
                 : "s"(lds_addr), "v"(voff), "s"(sbase)
                 : "memory", "m0", "vcc");
}

// Results of 32 resident rows and NDB blocks of 32 columns from f(db, e), element e of the accumulator of block db: 16 bytes a lane (the lane pair's halves of
// eight columns trade places).  Rows from n_live on get zeros, rows from n_out on are not written.
template <int D, int NDB, typename F>
__device__ __forceinline__ void store_rows(__bf16* base, int64_t first, int64_t n_live, int64_t n_out, float factor, F&& f) {
    const int lane = opaque_lane(), col = (lane >> 5) * 8;     // formed here, not kept through the steps
    const int64_t r = first + (lane & 31);
    const bool hidden = r >= n_live;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int a = 0; a < 4; a += 2) {
            unsigned x[2][2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    x[j][e] = hidden ? 0u : pack_bf16(f(db, 4 * (a + j) + 2 * e) * factor, f(db, 4 * (a + j) + 2 * e + 1) * factor);
            const auto l = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
            const auto u = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
            if (r < n_out) *reinterpret_cast<u32x4*>(base + r * D + db * 32 + a * 8 + col) = u32x4{l[0], u[0], l[1], u[1]};
        }
}

// Operand fragments of a streamed tile in LDS.  rows: 16 columns from 16 * KK on of 32 rows; tr: 16 rows from 16 * (IDX / (D / 32)) on, transposed, of the columns of
// block IDX % (D / 32) = db.  `at` is the lane's address in the tile (frag_rows_at, frag_tr_at); frag_block moves it by granules.
template <int D>
__device__ __forceinline__ unsigned frag_rows_at(int lane) { return (lane & 31) * (D * 2) + (((lane >> 5) ^ swz_kv<D>(lane & 31)) * 16); }
template <int D>
__device__ __forceinline__ unsigned frag_tr_at(int lane) {
    const int li = lane & 31, t16 = lane & 15, row = 4 * (lane >> 5) + (t16 >> 2), g = 2 * (li >> 4) + ((t16 & 3) >> 1);
    return row * (D * 2) + ((g ^ swz_kv<D>(row)) * 16) + (t16 & 1) * 8;
}
template <int N>
__device__ __forceinline__ LDS_PTR(const unsigned char) frag_block(unsigned at) {
    unsigned r = at;
    if constexpr (N != 0) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(r) : "n"(N), "v"(at));
    return (LDS_PTR(const unsigned char))(uintptr_t)r;
}
template <int KK>
__device__ __forceinline__ bf16x8 read_rows(unsigned at) { return *(LDS_PTR(const bf16x8))frag_block<KK * 32>(at); }
template <int D, int IDX>
__device__ __forceinline__ bf16x8 read_tr(LDS_PTR(const unsigned char) x, LDS_PTR(const unsigned char) y) {      // frag_block<db * 64>, frag_block<(db * 64) ^ 32>
    constexpr int u = IDX / (D / 32);
    static_assert(swz_kv<D>(8) == 2 && swz_kv<D>(0) == 0, "eight rows on, the granule differs in one bit");
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(x + u * 16 * (D * 2)));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(y + (u * 16 + 8) * (D * 2)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// ---- d = 128: two wavefronts for 64 resident rows ----------------------------------------------------------------
// A step is two phases with a barrier behind each:
//   1  first: sums of dV of step t - 1, scores of step t (matrix)     second: dS of step t - 1 (vector)
//   2  first: probabilities of step t, into LDS for the other (vector)   second: sums of dK or dQ of step t - 1, dP of step t (matrix)
// Phase 2 is the longer one: 64 multiply-adds and exponentials take 540 cycles beside matrix instructions, packing them 80, and writing them to LDS, four
// wavefronts at once, 320.  (A single barrier a step and two buffers for the probabilities, each wavefront at its own pace: 24 x 9 600 3 043 us and 3 101, 12 x 3 000
// 183 and 194.  Query items' tiles fetched by the first wavefronts, which wait in phase 1: no change.)  All launches run below the full clock: on zeros, which need
// less power, 24 x 9 600 takes 2 362 us, 1 x 9 600 133 instead of 159.
// One block of resident rows against the streamed tiles [t0, t1).  part: where the sums go in fp32 if other work items have the
// block's other tiles (dQ, or dK and behind it dV: kBwdRows * D floats each, in the order of the accumulator registers), else null.
// claim: called once by all wavefronts when none reads the tiles any more.
template <int D, bool KEYS, typename F>
__device__ __forceinline__ void attn_bwd_pair_item(const AttnBwdParams& p, int wave, int bh, int64_t row0, int t0, int t1, float* part, F&& claim) {
    constexpr int G = D / 8, NKK = D / 16, NDB = D / 32;
    constexpr int TILE = bwd_tile_bytes(D), RPC = 1024 / (D * 2);
    constexpr int CPW = TILE / 4096;                           // chunks of 1 KB of a tile that a fetching wavefront brings
    constexpr int PF = 3;                                      // operand fragments read ahead
    extern __shared__ __attribute__((aligned(256))) unsigned char bwd_smem_[];
    const unsigned lds0 = (unsigned)(uintptr_t)(LDS_PTR(unsigned char))bwd_smem_;
    const int pair = wave & 3;
    const int lane = opaque_lane(), li = lane & 31, lh = lane >> 5;
    const bool second = wave >= 4;
    const int b = bh / p.H, h = bh - b * p.H;
    const __bf16* qp = p.q + (int64_t)b * p.q_bs + (int64_t)h * p.q_hs;
    const __bf16* dop = p.dout + (int64_t)b * p.do_bs + (int64_t)h * p.do_hs;
    const __bf16* kp = p.k + (int64_t)b * p.kv_bs + (int64_t)h * p.kv_hs;
    const __bf16* vp = p.v + (int64_t)b * p.kv_bs + (int64_t)h * p.kv_hs;
    const float* stats = p.stats + bh * p.stat_rows * 2 + (KEYS ? (int64_t)t0 * (2 * kBwdTile) : 0);
    const int64_t n_res = KEYS ? p.n_v : p.Sq;
    const int n_all = (int)(KEYS ? p.Sq : p.n_v);
    const int n_str = (n_all < (int64_t)t1 * kBwdTile ? n_all : t1 * kBwdTile) - t0 * kBwdTile;        // streamed rows, counted from tile t0 on
    const int64_t first = row0 + pair * 64;                    // this lane's resident rows: first + li and first + 32 + li
    const int nt = row0 < n_res ? t1 - t0 : 0;

    auto step = []() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };
    auto barrier = [&]() __attribute__((always_inline)) {      // keeps the phases apart
        step();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        step();
    };

    // ---- loads of the streamed tiles, by the second wavefronts: 1 KB chunks pair, pair + 4 of a tile; chunk j holds rows j RPC ..,
    // lane -> row lane / G of them, granule lane % G.  Sixteen rows on, the lane's offset in its row is the same.
    const __bf16* s1 = (KEYS ? qp : kp) + (int64_t)t0 * (kBwdTile * D);
    const __bf16* s2 = (KEYS ? dop : vp) + (int64_t)t0 * (kBwdTile * D);
    constexpr int LOADS = 2 * CPW;                             // of a wavefront per step, and in pair 0 one for the statistics
    const unsigned whole = (pair * RPC + lane / G) * (D * 2) + (((lane % G) ^ swz_kv<D>(pair * RPC + lane / G)) * 16);
    auto issue = [&](int t) __attribute__((always_inline)) {
        const unsigned to = lds0 + t % kBwdRing * 2 * TILE + pair * 1024;
        const __bf16* from1 = s1 + (int64_t)t * (kBwdTile * D);
        const __bf16* from2 = s2 + (int64_t)t * (kBwdTile * D);
        const int last = n_str - 1 - t * kBwdTile;
        if (last >= kBwdTile - 1) {
#pragma unroll
            for (int i = 0; i < CPW; ++i) {
                lds_dma16(from1 + i * 16 * D, whole, to + i * 4096);
                lds_dma16(from2 + i * 16 * D, whole, to + TILE + i * 4096);
            }
        } else {                                               // rows behind the last: that row again
#pragma unroll
            for (int i = 0; i < CPW; ++i) {
                const int l = opaque_lane(), r = (pair + 4 * i) * RPC + l / G;
                const unsigned off = (r < last ? r : last) * (D * 2) + (((l % G) ^ swz_kv<D>(r)) * 16);
                lds_dma16(from1, off, to + i * 4096);
                lds_dma16(from2, off, to + TILE + i * 4096);
            }
        }
        if (KEYS && pair == 0) lds_dma4(stats + (int64_t)t * (2 * kBwdTile), opaque_lane() * 4, lds0 + bwd_stat_base(D) + t % kBwdRing * 256);
    };

    // ---- operand fragments, in buffer 0 from these addresses on
    unsigned rows_at = lds0 + frag_rows_at<D>(lane), tr_at = lds0 + frag_tr_at<D>(lane);
    bf16x8 frag[PF + 1];
    auto rows_frag = [&](int t, int tensor, auto kk) __attribute__((always_inline)) {
        frag[decltype(kk)::value % (PF + 1)] = read_rows<decltype(kk)::value>(rows_at + t % kBwdRing * 2 * TILE + tensor * TILE);
    };
    auto tr_frag = [&](int t, int tensor, auto idx) __attribute__((always_inline)) {
        constexpr int db = decltype(idx)::value % NDB;
        const unsigned at = tr_at + t % kBwdRing * 2 * TILE + tensor * TILE;
        frag[decltype(idx)::value % (PF + 1)] = read_tr<D, decltype(idx)::value>(frag_block<db * 64>(at), frag_block<(db * 64) ^ 32>(at));
    };
    // A pair's probabilities of a step: group a of block i, 16 bytes a lane.  Statistics of a tile's rows: four rows of group a.
    // (Addresses from a fresh lane index: they are not kept over the products.)
    auto exchange_at = [&]() __attribute__((always_inline)) { return lds0 + bwd_p_base(D) + pair * kBwdExchange + opaque_lane() * 16; };
    auto exchange = [](unsigned at, int i, int a) __attribute__((always_inline)) {
        return (LDS_PTR(f32x4))(LDS_PTR(unsigned char))(uintptr_t)(at + (i * 4 + a) * 1024);
    };
    auto stat_at = [&](int t) __attribute__((always_inline)) { return lds0 + bwd_stat_base(D) + t % kBwdRing * 256 + (opaque_lane() >> 5) * 16; };
    auto stat = [](unsigned at, int which, int a) __attribute__((always_inline)) {
        return *(LDS_PTR(const f32x4))(LDS_PTR(const unsigned char))(uintptr_t)(at + which * 128 + 32 * a);
    };

    // ---- resident rows
    bf16x8 res[2][NKK];
    float res_stat[2] = {0.f, 0.f};
    f32x16 acc[2][NDB];                                        // first wavefront of a pair: dV^T; second: dK^T or dQ^T
    if (nt > 0) {
        if (second)
            for (int t = 0; t < kBwdAhead && t < nt; ++t) issue(t);
        const __bf16* src = second ? (KEYS ? vp : dop) : (KEYS ? kp : qp);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t c = first + li + 32 * i < n_res ? first + li + 32 * i : n_res - 1;
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) res[i][kk] = *reinterpret_cast<const bf16x8*>(src + c * D + lh * 8 + kk * 16);
            if constexpr (!KEYS) res_stat[i] = stats[(c / kBwdTile) * (2 * kBwdTile) + (second ? kBwdTile : 0) + c % kBwdTile];
        }
        // The compiler's own count of loads under way starts from here: it knows this wait, and would otherwise wait inside the loops for
        // loads of the resident rows, and so for the tiles that have just been requested.
        __builtin_amdgcn_s_waitcnt(kWaitLoads);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            asm volatile("" : "+v"(res_stat[i]));
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) asm volatile("" : "+v"(res[i][kk]));
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][db][r] = 0.f;
    const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    f32x16 s[2];                                               // scores or <dout, v>; then p or ds, as operands in groups 0 and 2
    // Four values (group a) as half an operand of bf16.
    auto put = [&](int i, int a, const float (&x)[4]) __attribute__((always_inline)) {
        s[i][a / 2 * 8 + a % 2 * 2] = __uint_as_float(pack_bf16(x[0], x[1]));
        s[i][a / 2 * 8 + a % 2 * 2 + 1] = __uint_as_float(pack_bf16(x[2], x[3]));
    };
    // acc += (tile, transposed) operand: the first PF fragments are there; `next` reads those of what comes next.
    auto nothing = [](auto) __attribute__((always_inline)) {};
    auto sums = [&](int t, int tensor, auto next) __attribute__((always_inline)) {
        static_for<0, 2 * NDB>([&](auto j) {
            constexpr int n = decltype(j)::value, u = n / NDB * 8;
            if constexpr (n + PF < 2 * NDB) tr_frag(t, tensor, std::integral_constant<int, n + PF>{});
            else next(std::integral_constant<int, n + PF - 2 * NDB>{});
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const bf16x8 x = __builtin_bit_cast(bf16x8, __builtin_shufflevector(s[i], s[i], u, u + 1, u + 2, u + 3));
                acc[i][n % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % (PF + 1)], x, acc[i][n % NDB], 0, 0, 0);
            }
            step();
        });
    };
    // s = tile * resident rows; the first PF fragments are there
    auto products = [&](int t, int tensor, auto next) __attribute__((always_inline)) {
        static_for<0, NKK>([&](auto j) {
            constexpr int n = decltype(j)::value;
            if constexpr (n + PF < NKK) rows_frag(t, tensor, std::integral_constant<int, n + PF>{});
            else next(std::integral_constant<int, n + PF - NKK>{});
#pragma unroll
            for (int i = 0; i < 2; ++i) s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % (PF + 1)], res[i][n], n == 0 ? zero : s[i], 0, 0, 0);
            step();
        });
    };

    if (!second) {
        const float c = p.scale_log2e;
        // -lse * log2 e of a step's rows, four at a time, into two fragments' registers as the last fragments go into products
        auto read_l = [&](unsigned at, int a) __attribute__((always_inline)) { if constexpr (KEYS) frag[a % 2] = __builtin_bit_cast(bf16x8, stat(at, 0, a)); };
        auto scores = [&](int t) __attribute__((always_inline)) {
            const unsigned l_at = KEYS ? stat_at(t) : 0;
            products(t, 0, [&](auto n) __attribute__((always_inline)) { if constexpr (decltype(n)::value < 2) read_l(l_at, decltype(n)::value); });
            barrier();
        };
        auto softmax = [&](int t) __attribute__((always_inline)) {
            const unsigned to = exchange_at(), l_at = KEYS ? stat_at(t) : 0;
            const bool tail = !KEYS && (t + 1) * kBwdTile > n_str;
            // Eight groups of four values in place, each written and packed while the next one's exponentials are under way.
            static_for<0, 9>([&](auto j) {
                constexpr int n = decltype(j)::value;
                if constexpr (n < 8) {
                    constexpr int a = n / 2, i = n % 2;
                    const f32x4 l = __builtin_bit_cast(f32x4, frag[a % 2]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[i][4 * a + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i][4 * a + e], c, KEYS ? l[e] : res_stat[i]));
                    if (tail) {
                        const int hidden = n_str - t * kBwdTile - (opaque_lane() >> 5) * 4;
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i][4 * a + e] = 8 * a + e >= hidden ? 0.f : s[i][4 * a + e];
                    }
                    if constexpr (i == 1 && a < 2) read_l(l_at, a + 2);
                }
                if constexpr (n > 0) {
                    constexpr int a = (n - 1) / 2, i = (n - 1) % 2;
                    const float x[4] = {s[i][4 * a], s[i][4 * a + 1], s[i][4 * a + 2], s[i][4 * a + 3]};
                    *exchange(to, i, a) = f32x4{x[0], x[1], x[2], x[3]};
                    if constexpr (KEYS) put(i, a, x);
                }
                step();
            });
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            // first fragments of what follows: dV of this step, or the scores of the next one, whose tile is there
            if constexpr (KEYS) static_for<0, PF>([&](auto n) { tr_frag(t, 1, n); });
            else static_for<0, PF>([&](auto n) { rows_frag(t + 1, 0, n); });
            barrier();
        };
        if (nt > 0) {
            static_for<0, PF>([&](auto n) { rows_frag(0, 0, n); });
            scores(0);
            softmax(0);
        }
        for (int t = 1; t < nt; ++t) {
            asm volatile("" : "+v"(rows_at), "+v"(tr_at));     // nothing formed from them is kept across steps
            __builtin_amdgcn_s_setprio(1);                     // matrix instructions ahead of the other wavefront's arithmetic
            if constexpr (KEYS) sums(t - 1, 1, [&](auto n) __attribute__((always_inline)) { rows_frag(t, 0, n); });
            scores(t);
            __builtin_amdgcn_s_setprio(0);
            softmax(t);
        }
        if (KEYS && nt > 0) sums(nt - 1, 1, nothing);
    } else {
        // ds from the probabilities that the other wavefront has left there.  They and -delta, four values of each at a time, are read into the
        // registers of the fragments, which follow them, and one more.
        auto differences = [&](int t) __attribute__((always_inline)) {
            const unsigned p_at = exchange_at(), d_at = KEYS ? stat_at(t) : 0;
            f32x4 odd = {0.f, 0.f, 0.f, 0.f};
            auto read_p = [&](int n) __attribute__((always_inline)) { frag[n % 3] = __builtin_bit_cast(bf16x8, *exchange(p_at, n % 2, n / 2)); };
            auto read_d = [&](int a) __attribute__((always_inline)) {
                if constexpr (KEYS) {
                    if (a % 2) odd = stat(d_at, 1, a);
                    else frag[3] = __builtin_bit_cast(bf16x8, stat(d_at, 1, a));
                }
            };
            read_d(0);
            read_p(0);
            read_p(1);
            read_d(1);
            read_p(2);
            step();
            static_for<0, 8>([&](auto j) {
                constexpr int n = decltype(j)::value, a = n / 2, i = n % 2;
                const f32x4 x = __builtin_bit_cast(f32x4, frag[n % 3]), d = a % 2 ? odd : __builtin_bit_cast(f32x4, frag[3]);
                float y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = x[e] * (s[i][4 * a + e] + (KEYS ? d[e] : res_stat[i]));
                asm volatile("" : "+v"(y[0]), "+v"(y[1]), "+v"(y[2]), "+v"(y[3]));      // in this order: no registers for another
                put(i, a, y);
                if constexpr (n + 3 < 8) read_p(n + 3);
                else tr_frag(t, 0, std::integral_constant<int, n % 3>{});
                if constexpr (n % 2 == 1 && a < 2) read_d(a + 2);
                step();
            });
        };
        // the end of step t: tile t + 2 is there, tile t + 3 may be under way
        auto step_end = [&](int t) __attribute__((always_inline)) {
            step();
            if (t + kBwdAhead < nt) {
                if (KEYS && pair == 0) wait_vmcnt<LOADS + 1>();
                else wait_vmcnt<LOADS>();
            } else {
                wait_vmcnt<0>();
            }
            barrier();
        };
        if (nt > 0) {
            if (nt > kBwdAhead) issue(kBwdAhead);
            static_for<0, PF>([&](auto n) { rows_frag(0, 1, n); });
            barrier();
            products(0, 1, nothing);
            step_end(0);
        }
        for (int t = 1; t < nt; ++t) {
            asm volatile("" : "+v"(rows_at), "+v"(tr_at));
            if (t + kBwdAhead < nt) issue(t + kBwdAhead);
            differences(t - 1);
            barrier();
            __builtin_amdgcn_s_setprio(1);
            sums(t - 1, 0, [&](auto n) __attribute__((always_inline)) { rows_frag(t, 1, n); });
            products(t, 1, nothing);
            __builtin_amdgcn_s_setprio(0);
            step_end(t);
        }
        if (nt > 0) {
            differences(nt - 1);
            sums(nt - 1, 0, nothing);
        }
    }

    // ---- results
    claim();
    if (!KEYS && !second) return;
    if (part) {
        f32x4* to = reinterpret_cast<f32x4*>(part + (KEYS && !second ? kBwdRows * D : 0)) + pair * (2 * NDB * 4 * 64) + opaque_lane();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int a = 0; a < 4; ++a)
                    to[((i * NDB + db) * 4 + a) * 64] = f32x4{acc[i][db][4 * a], acc[i][db][4 * a + 1], acc[i][db][4 * a + 2], acc[i][db][4 * a + 3]};
        return;
    }
    __bf16* base = p.dq + (int64_t)b * p.dq_bs + (int64_t)h * p.dq_hs;
    if constexpr (KEYS) {
        base = p.dv + (int64_t)b * p.dkv_bs + (int64_t)h * p.dkv_hs;
        if (second) base += p.dk - p.dv;                       // (a choice of one of two arguments would put both into scratch memory)
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        store_rows<D, NDB>(base, first + 32 * i, n_res, KEYS ? p.Skv : p.Sq, second ? p.scale : 1.0f, [&](int db, int e) __attribute__((always_inline)) { return acc[i][db][e]; });
}

// A pointer that is the same in all lanes, in scalar registers (the compiler may choose one of two by vector instructions).
template <typename T>
__device__ __forceinline__ T* uniform(T* p) {
    const uint64_t x = reinterpret_cast<uint64_t>(p);
    return reinterpret_cast<T*>((uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)x));
}

// ---- d = 64: a wavefront for 32 resident rows -------------------------------------------------------------------
// A wavefront alternates between a matrix phase (sums of step t - 1, products of step t) and a vector phase (probabilities and dS of step t); of the two
// on a SIMD the second is half a step behind the first.  (Matrix instructions at a higher priority: 24 x 9 600 1 873 instead of 1 855 us.)
constexpr int kLoneRing = 4;            // tile buffers per streamed tensor
constexpr int lone_stat_base(int d) { return kLoneRing * 2 * bwd_tile_bytes(d); }
constexpr int lone_next_base(int d) { return lone_stat_base(d) + kLoneRing * 512; }
constexpr int lone_smem(int d) { return lone_next_base(d) + 16; }

template <int D, bool KEYS, typename F>
__device__ __forceinline__ void attn_bwd_lone_item(const AttnBwdParams& p, int wave, int bh, int64_t row0, int t0, int t1, float* part, F&& claim) {
    constexpr int G = D / 8, NKK = D / 16, NDB = D / 32, R = kLoneRing;
    constexpr int TILE = bwd_tile_bytes(D), RPC = 1024 / (D * 2), CPW = TILE / 4096;
    constexpr int NF = 8;                                      // operand fragments under way (24 x 9 600: 1 855 us; 3: 1 859, 4: 1 873, 2: 2 224, 10: 1 949)
    extern __shared__ __attribute__((aligned(256))) unsigned char bwd_smem_[];
    const unsigned lds0 = (unsigned)(uintptr_t)(LDS_PTR(unsigned char))bwd_smem_;
    const int quarter = wave & 3;
    const int lane = opaque_lane(), li = lane & 31, lh = lane >> 5;
    const bool second = wave >= 4;                             // the wavefronts that run a phase behind
    const int b = bh / p.H, h = bh - b * p.H;
    const __bf16* qp = p.q + (int64_t)b * p.q_bs + (int64_t)h * p.q_hs;
    const __bf16* dop = p.dout + (int64_t)b * p.do_bs + (int64_t)h * p.do_hs;
    const __bf16* kp = p.k + (int64_t)b * p.kv_bs + (int64_t)h * p.kv_hs;
    const __bf16* vp = p.v + (int64_t)b * p.kv_bs + (int64_t)h * p.kv_hs;
    const float* stats = p.stats + bh * p.stat_rows * 4 + (KEYS ? (int64_t)t0 * (4 * kBwdTile) : 0);
    const int64_t n_res = KEYS ? p.n_v : p.Sq;
    const int n_all = (int)(KEYS ? p.Sq : p.n_v);
    const int n_str = (n_all < (int64_t)t1 * kBwdTile ? n_all : t1 * kBwdTile) - t0 * kBwdTile;        // streamed rows, counted from tile t0 on
    const int64_t first = row0 + wave * 32;                    // this lane's resident row: first + li
    const int nt = row0 < n_res ? t1 - t0 : 0;

    auto step = []() __attribute__((always_inline)) { __builtin_amdgcn_sched_barrier(0); };
    auto barrier = [&]() __attribute__((always_inline)) {      // keeps the phases apart
        step();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        step();
    };

    // ---- loads of the streamed tiles: one tensor by either group, 1 KB chunks quarter, quarter + 4 .. of a tile (see attn_bwd_pair_item)
    const __bf16* from = (second ? (KEYS ? dop : vp) : (KEYS ? qp : kp)) + (int64_t)t0 * (kBwdTile * D);
    const unsigned whole = (quarter * RPC + lane / G) * (D * 2) + (((lane % G) ^ swz_kv<D>(quarter * RPC + lane / G)) * 16);
    const bool with_stats = KEYS && (wave & 6) == 4;           // half of a tile's
    auto issue = [&](int t) __attribute__((always_inline)) {
        const unsigned to = __builtin_amdgcn_readfirstlane(lds0 + t % R * 2 * TILE + (second ? TILE : 0) + quarter * 1024);
        const __bf16* src = uniform(from + (int64_t)t * (kBwdTile * D));
        const int last = n_str - 1 - t * kBwdTile;
#pragma unroll
        for (int i = 0; i < CPW; ++i) {
            if (last >= kBwdTile - 1) {
                lds_dma16(src + i * 16 * D, whole, to + i * 4096);
            } else {                                           // rows behind the last: that row again
                const int l = opaque_lane(), r = (quarter + 4 * i) * RPC + l / G;
                lds_dma16(src, (r < last ? r : last) * (D * 2) + (((l % G) ^ swz_kv<D>(r)) * 16), to + i * 4096);
            }
        }
        if (with_stats) {
            lds_dma4(uniform(stats + (int64_t)t * (4 * kBwdTile) + quarter * 64), opaque_lane() * 4, __builtin_amdgcn_readfirstlane(lds0 + lone_stat_base(D) + t % R * 512 + quarter * 256));
        }
    };
    // what was fetched before tile t is there, tile t may be under way
    auto arrived = [&](int t) __attribute__((always_inline)) {
        step();
        if (t < nt) {
            if (with_stats) wait_vmcnt<CPW + 1>();
            else wait_vmcnt<CPW>();
        } else {
            wait_vmcnt<0>();
        }
    };

    // ---- operand fragments, number n of a matrix phase into frag[n % NF].  Their addresses in buffer 0 stay in registers, a phase adds its buffer to each: what a
    // vector instruction costs here is seen in the time (a XOR for every read instead: 24 x 9 600 2 145 us and now 2 009).
    bf16x8 frag[NF];
    const unsigned stat_0 = lds0 + lone_stat_base(D) + li * 16;
    unsigned rows_0[NKK], tr_0[NDB * 2], rows_at[NKK], tr_at[NDB * 2];
    static_for<0, NKK>([&](auto k) { rows_0[decltype(k)::value] = (unsigned)(uintptr_t)frag_block<decltype(k)::value * 32>(lds0 + frag_rows_at<D>(lane)); });
    static_for<0, NDB * 2>([&](auto k) { tr_0[decltype(k)::value] = (unsigned)(uintptr_t)frag_block<decltype(k)::value * 32>(lds0 + frag_tr_at<D>(lane)); });
    auto rows_frag = [&](int tensor, auto kk, auto n) __attribute__((always_inline)) {
        frag[decltype(n)::value % NF] = *(LDS_PTR(const bf16x8))((LDS_PTR(const unsigned char))(uintptr_t)rows_at[decltype(kk)::value] + tensor * TILE);
    };
    auto tr_frag = [&](int tensor, auto idx, auto n) __attribute__((always_inline)) {
        constexpr int db = decltype(idx)::value % NDB;
        frag[decltype(n)::value % NF] = read_tr<D, decltype(idx)::value>((LDS_PTR(const unsigned char))(uintptr_t)tr_at[db * 2] + tensor * TILE,
                                                                         (LDS_PTR(const unsigned char))(uintptr_t)tr_at[db * 2 + 1] + tensor * TILE);
    };

    // ---- resident rows
    bf16x8 res[2][NKK];                                        // k and v rows, or q and dout rows
    float l_res = 0.f, d_res = 0.f;
    if (nt > 0) {
        for (int t = 0; t < 2 && t < nt; ++t) issue(t);
        const int64_t c = first + li < n_res ? first + li : n_res - 1;
#pragma unroll
        for (int kk = 0; kk < NKK; ++kk) {
            res[0][kk] = *reinterpret_cast<const bf16x8*>((KEYS ? kp : qp) + c * D + lh * 8 + kk * 16);
            res[1][kk] = *reinterpret_cast<const bf16x8*>((KEYS ? vp : dop) + c * D + lh * 8 + kk * 16);
        }
        if constexpr (!KEYS) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(stats + c * 4);
            l_res = (bf16_lo(x[0]) + bf16_hi(x[0]) + bf16_lo(x[1])) * p.scale_log2e;
            d_res = bf16_lo(x[2]) + bf16_hi(x[2]) + bf16_lo(x[3]);
        }
        __builtin_amdgcn_s_waitcnt(kWaitLoads);
        asm volatile("" : "+v"(l_res), "+v"(d_res));
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int kk = 0; kk < NKK; ++kk) asm volatile("" : "+v"(res[i][kk]));
        __syncthreads();
    }
    f32x16 acc[2][NDB];                                        // dK^T or dQ^T; dV^T
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][db][r] = 0.f;
    const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    f32x16 s, dp;                                              // scores, then p; <dout, v>, then ds: as operands in groups 0 and 2
    // What the accumulators of the products start with.  Query items: <dout, v> with -delta of the lane's row.  Key items, where rows are the accumulators'
    // rows: a product of the three parts of l, and one of those of -delta, with ones; read as fp32 values, four rows a lane and read, they took as much of the LDS as
    // a tile does (24 x 9 600 1 869 us and now 1 838, 1 x 9 600 104.5 and 98.1).  Over k = 8, so that neither is in the other's product: a delta that is not
    // finite would otherwise reach the scores, zero times NaN, and with them dv.
    f32x16 delta = zero;
    s16x4 ones, stat_l, stat_d;
    if constexpr (KEYS) {
        const unsigned one = lh == 0 ? 0x3f80u : 0u;
        ones = __builtin_bit_cast(s16x4, u32x2{one << 16 | one, one});
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) delta[e] = d_res;
    }

    // Matrix phase: the sums of step t - 1 (SUMS), then the products of step t (PRODS).  Product n of the phase:
    constexpr int N_SUM = (KEYS ? 2 : 1) * 2 * NDB, N_PROD = 2 * NKK + (KEYS ? 2 : 0), STAT = KEYS ? 2 : 0;
    auto matrix = [&](int t, auto has_sums, auto has_prods) __attribute__((always_inline)) {
        constexpr int N0 = decltype(has_sums)::value ? 0 : N_SUM, N1 = N_SUM + (decltype(has_prods)::value ? N_PROD : 0);
        auto load = [&](auto j) __attribute__((always_inline)) {
            constexpr int n = decltype(j)::value;
            if constexpr (n < N_SUM) {
                if constexpr (KEYS) tr_frag(1 - n % 2, std::integral_constant<int, n / 2>{}, j);       // dout for dV, q for dK
                else tr_frag(0, j, j);
            } else if constexpr (n < N_SUM + STAT && n < N1) {
                if constexpr (n == N_SUM) {
                    const u32x4 x = *(LDS_PTR(const u32x4))(LDS_PTR(const unsigned char))(uintptr_t)(stat_0 + t % R * 512);
                    stat_l = __builtin_bit_cast(s16x4, u32x2{x[0], x[1]});
                    stat_d = __builtin_bit_cast(s16x4, u32x2{x[2], x[3]});
                }
            } else if constexpr (n < N1) {
                rows_frag((n - N_SUM) % 2, std::integral_constant<int, (n - N_SUM - STAT) / 2>{}, j);
            }
        };
        static_for<0, NKK>([&](auto k) { rows_at[decltype(k)::value] = rows_0[decltype(k)::value] + t % R * 2 * TILE; });
        static_for<0, NDB * 2>([&](auto k) { tr_at[decltype(k)::value] = tr_0[decltype(k)::value] + (t + R - 1) % R * 2 * TILE; });
        static_for<N0, N0 + NF - 1>([&](auto j) { load(j); });
        step();
        static_for<N0, N1>([&](auto j) {
            constexpr int n = decltype(j)::value;
            load(std::integral_constant<int, n + NF - 1>{});
            if constexpr (n < N_SUM) {
                constexpr bool dv = KEYS && n % 2 == 0;
                constexpr int idx = KEYS ? n / 2 : n, u = idx / NDB * 8;
                const f32x16& v = dv ? s : dp;
                const bf16x8 x = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v, v, u, u + 1, u + 2, u + 3));
                acc[dv][idx % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % NF], x, acc[dv][idx % NDB], 0, 0, 0);
            } else {
                constexpr int kk = (n - N_SUM - STAT) / 2;
                if constexpr (n < N_SUM + STAT) {
                    f32x16& x = n == N_SUM ? s : dp;
                    x = __builtin_amdgcn_mfma_f32_32x32x8bf16_1k(n == N_SUM ? stat_l : stat_d, ones, zero, 0, 0, 0);
                } else if constexpr ((n - N_SUM) % 2 == 0) {
                    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % NF], res[0][kk], !KEYS && kk == 0 ? zero : s, 0, 0, 0);
                } else {
                    dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[n % NF], res[1][kk], !KEYS && kk == 0 ? delta : dp, 0, 0, 0);
                }
            }
            step();
        });
    };
    const float c = p.scale_log2e;
    auto vector = [&](int t) __attribute__((always_inline)) {
        const bool tail = !KEYS && (t + 1) * kBwdTile > n_str;
        // groups of four values in place, the exponentials of one beside the products of the one before
        static_for<0, 5>([&](auto j) {
            constexpr int n = decltype(j)::value;
            if constexpr (n < 4) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[4 * n + e] = __builtin_amdgcn_exp2f(KEYS ? s[4 * n + e] * c : __builtin_fmaf(s[4 * n + e], c, l_res));
                if (tail) {
                    const int hidden = n_str - t * kBwdTile - (opaque_lane() >> 5) * 4;
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[4 * n + e] = 8 * n + e >= hidden ? 0.f : s[4 * n + e];
                }
            }
            if constexpr (n > 0) {
                constexpr int a = n - 1, at = a / 2 * 8 + a % 2 * 2;
                float x[4], y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = s[4 * a + e];
                    y[e] = x[e] * dp[4 * a + e];
                }
                if constexpr (KEYS) {
                    s[at] = __uint_as_float(pack_bf16(x[0], x[1]));
                    s[at + 1] = __uint_as_float(pack_bf16(x[2], x[3]));
                }
                dp[at] = __uint_as_float(pack_bf16(y[0], y[1]));
                dp[at + 1] = __uint_as_float(pack_bf16(y[2], y[3]));
            }
            step();
        });
        asm volatile("" : "+v"(s), "+v"(dp));                  // here, not where they are used
    };
    constexpr std::false_type no{};
    constexpr std::true_type yes{};
    // Half a step each, a barrier behind it: the first group's matrix phase of step t is half step 2 t, the second's 2 t + 1; a vector phase follows.  Tile
    // u goes into the buffer of tile u - 4, which is last read in half step 2 u - 5 (sums of the second group), and is first read in 2 u.
    // Key items, whose matrix phase is the longer one, request it in the vector phase (half step 2 u - 3 of the first group, 2 u - 4 of the second),
    // query items in the matrix phase (2 u - 4 and 2 u - 3); each group waits for it at the end of half step 2 u - 1.
    // (Query items' requests in the vector phase too: 24 x 9 600 2 094 instead of 2 032 us; key items' in the matrix phase: 2 083.)
    if (nt > 0) {
        if (second) {
            if (KEYS && nt > 2) issue(2);
            barrier();
        }
        if (!KEYS && nt > 2) issue(2);
        matrix(0, no, yes);
        if (second) arrived(2);
        barrier();
        for (int t = 1; t < nt; ++t) {
#pragma unroll
            for (int k = 0; k < NKK; ++k) asm volatile("" : "+v"(rows_0[k]));      // what is formed from them is not kept across steps
#pragma unroll
            for (int k = 0; k < 2 * NDB; ++k) asm volatile("" : "+v"(tr_0[k]));
            const int next = t + 1 + (second ? 1 : 0);
            if (KEYS && next < nt) issue(next);
            vector(t - 1);
            if (!second) arrived(t + 1);
            barrier();
            if (!KEYS && t + 2 < nt) issue(t + 2);
            matrix(t, yes, yes);
            if (second) arrived(t + 2);
            barrier();
        }
        vector(nt - 1);
        barrier();
        matrix(nt, yes, no);
        if (!second) barrier();                                // the second group's half step
    }

    // ---- results
    claim();
    static_for<0, KEYS ? 2 : 1>([&](auto k) {
        constexpr int i = decltype(k)::value;
        if (part) {
            f32x4* to = reinterpret_cast<f32x4*>(part + i * kBwdRows * D) + wave * (NDB * 4 * 64) + opaque_lane();
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
                for (int a = 0; a < 4; ++a) to[(db * 4 + a) * 64] = f32x4{acc[i][db][4 * a], acc[i][db][4 * a + 1], acc[i][db][4 * a + 2], acc[i][db][4 * a + 3]};
        } else {
            __bf16* base = i == 1 ? p.dv + (int64_t)b * p.dkv_bs + (int64_t)h * p.dkv_hs
                          : KEYS ? p.dk + (int64_t)b * p.dkv_bs + (int64_t)h * p.dkv_hs : p.dq + (int64_t)b * p.dq_bs + (int64_t)h * p.dq_hs;
            store_rows<D, NDB>(base, first, n_res, KEYS ? p.Skv : p.Sq, i == 1 ? 1.0f : p.scale, [&](int db, int e) __attribute__((always_inline)) { return acc[i][db][e]; });
        }
    });
}

template <int D>
constexpr int item_smem() { return D == 128 ? bwd_smem(D) : lone_smem(D); }
template <int D, bool KEYS, typename F>
__device__ __forceinline__ void attn_bwd_item(const AttnBwdParams& p, int wave, int bh, int64_t row0, int t0, int t1, float* part, F&& claim) {
    if constexpr (D == 128) attn_bwd_pair_item<D, KEYS>(p, wave, bh, row0, t0, t1, part, claim);
    else attn_bwd_lone_item<D, KEYS>(p, wave, bh, row0, t0, t1, part, claim);
}

// A workgroup per compute unit takes items in order: item blockIdx.x, then what a counter gives it.  XCDs run at different speeds, the hardware deals a grid's
// workgroups to them round robin, and a workgroup that goes on needs no new launch and starts on its next block while others still store.  A grid
// of one workgroup an item instead, us: 3 x 67 576 18 896 and now 18 309, 24 x 9 600 3 139 and 3 066, 24 x 16 384 on 570 465 and 449; d = 64: 6 x 33 000
// 6 050 and 5 913, 24 x 4 797 548 and 538.  (Each XCD with its own eighth of the items first, for its L2: 18 496, 3 084, 446, 5 892, 547.)
// A launch with no more items than compute units has a workgroup for each and does not touch the counter.
template <int D>
__global__ __launch_bounds__(512, 2) void attn_bwd_kernel(const AttnBwdParams args) {
    extern __shared__ __attribute__((aligned(256))) unsigned char bwd_smem_[];
    using Args = const __attribute__((address_space(4))) AttnBwdParams*;
    Args at = (Args)__builtin_amdgcn_kernarg_segment_ptr();
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int item = (int)blockIdx.x, turn = 0;
    for (;;) {
        asm volatile("" : "+s"(at));                           // arguments are read where they are used, not carried through the items in registers
        const AttnBwdParams& p = *(const AttnBwdParams*)at;
        const BwdPlan& w = p.plan;
        if (item >= p.items) break;
        const int nk = w.key_blocks * w.key_parts, whole = w.query_blocks - w.query_cut, nq = whole + w.query_cut * w.query_parts;
        int next = 0x7fffffff;
        auto claim = [&]() __attribute__((always_inline)) {    // the next item: asked for by one lane, between two barriers of the items at the most
            if (p.grid >= p.items) return;
            volatile int* to = reinterpret_cast<int*>(bwd_smem_ + (D == 128 ? bwd_next_base(D) : lone_next_base(D))) + turn;
            turn ^= 1;                                         // (a wavefront may still be reading the one before)
            if (wave == 0 && opaque_lane() == 0) *to = p.grid + __hip_atomic_fetch_add(p.counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            next = __builtin_amdgcn_readfirstlane(*to);
        };
        int i = item;
        if (i < nk) {
            const int j = i / w.key_blocks, blk = i - j * w.key_blocks, bh = blk / w.key_per_head;
            const int nt = (int)((p.Sq + kBwdTile - 1) / kBwdTile);
            attn_bwd_item<D, true>(p, wave, bh, (int64_t)(blk - bh * w.key_per_head) * kBwdRows, (int)((int64_t)nt * j / w.key_parts), (int)((int64_t)nt * (j + 1) / w.key_parts),
                                   w.key_parts > 1 ? p.parts + (int64_t)(blk * w.key_parts + j) * (2 * kBwdRows * D) : nullptr, claim);
        } else if ((i -= nk) < nq) {
            const int j = i < whole ? 0 : (i - whole) / w.query_cut, c = i - whole - j * w.query_cut;  // part j of cut block c
            const int blk = i < whole ? i : whole + c, bh = blk / w.query_per_head, parts = i < whole ? 1 : w.query_parts;
            const int nt = (int)((p.n_v + kBwdTile - 1) / kBwdTile);
            attn_bwd_item<D, false>(p, wave, bh, (int64_t)(blk - bh * w.query_per_head) * kBwdRows, (int)((int64_t)nt * j / parts), (int)((int64_t)nt * (j + 1) / parts),
                                    i < whole ? nullptr : p.parts + bwd_key_floats(w, D) + (int64_t)(c * w.query_parts + j) * (kBwdRows * D), claim);
        } else {
            // keys that nobody sees: zeros from the first row behind the last block of valid ones
            claim();
            i -= nq;
            const int64_t from = (int64_t)w.key_per_head * kBwdRows, rows = p.Skv - from;
            const int per_head = (int)((rows + kBwdRows - 1) / kBwdRows), bh = i / per_head, b = bh / p.H, h = bh - b * p.H;
            const int64_t first = from + (int64_t)(i - bh * per_head) * kBwdRows, at = (int64_t)b * p.dkv_bs + (int64_t)h * p.dkv_hs + first * D;
            const int n = (int)(p.Skv - first < kBwdRows ? p.Skv - first : kBwdRows) * (D / 8);
            for (int x = wave * 64 + opaque_lane(); x < n; x += 512) {
                reinterpret_cast<u32x4*>(p.dk + at)[x] = u32x4{0, 0, 0, 0};
                reinterpret_cast<u32x4*>(p.dv + at)[x] = u32x4{0, 0, 0, 0};
            }
        }
        item = next;
    }
}

// Sums of the parts of cut blocks, part after part: a wavefront for 32 rows and 32 columns of dq, dk or dv, a workgroup for 128 rows.
template <int D>
__global__ __launch_bounds__(256) void attn_bwd_join_kernel(const AttnBwdParams p) {
    constexpr int NDB = D / 32;
    const BwdPlan& w = p.plan;
    const int db = blockIdx.x % NDB;
    const int sub = (blockIdx.x / NDB & 1) * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);       // 32 of the 256 rows
    int i = (int)blockIdx.x / (2 * NDB);
    const int nk = w.key_parts > 1 ? w.key_blocks * 2 : 0;
    const bool keys = i < nk;
    const float* src;
    int blk, parts;
    int64_t stride;
    bool is_dv = false;
    if (keys) {
        blk = i >> 1;
        is_dv = i & 1;
        parts = w.key_parts;
        stride = 2 * kBwdRows * D;
        src = p.parts + (int64_t)blk * parts * stride + (is_dv ? kBwdRows * D : 0);
    } else {
        i -= nk;
        blk = w.query_blocks - w.query_cut + i;
        parts = w.query_parts;
        stride = kBwdRows * D;
        src = p.parts + bwd_key_floats(w, D) + (int64_t)i * parts * stride;
    }
    const int per_head = keys ? w.key_per_head : w.query_per_head, bh = blk / per_head, b = bh / p.H, h = bh - b * p.H;
    const int64_t first = (int64_t)(blk - bh * per_head) * kBwdRows + sub * 32;
    const int64_t n_live = keys ? p.n_v : p.Sq, n_out = keys ? p.Skv : p.Sq;
    if (first >= n_out) return;
    const f32x4* from = reinterpret_cast<const f32x4*>(src) + (sub * NDB + db) * (4 * 64) + (threadIdx.x & 63);
    f32x4 acc[4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (int j = 0; j < parts; j += 4) {                       // loads of four parts in flight together
        f32x4 x[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (j + k < parts)
#pragma unroll
                for (int a = 0; a < 4; ++a) x[k][a] = from[(j + k) * (stride / 4) + a * 64];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (j + k < parts)
#pragma unroll
                for (int a = 0; a < 4; ++a) acc[a] += x[k][a];
    }
    __bf16* base = p.dq + (int64_t)b * p.dq_bs + (int64_t)h * p.dq_hs;
    if (keys) {
        base = p.dk + (int64_t)b * p.dkv_bs + (int64_t)h * p.dkv_hs;
        if (is_dv) base += p.dv - p.dk;
    }
    store_rows<D, 1>(base + db * 32, first, n_live, n_out, is_dv ? 1.0f : p.scale, [&](int, int e) __attribute__((always_inline)) { return acc[e / 4][e % 4]; });
}

template <int D>
static hipError_t launch_bwd(AttnBwdParams& p, hipStream_t st) {
    const int BH = p.B * p.H;
    if (D == 64 && p.scale_log2e < 0x1p-64f) p.scale_log2e = 0x1p-64f;        // l is kept in units of the scores; below, every score counts for nothing
    if (p.Sq > 0) {
        constexpr int rows = 256 / (D / 8);
        const int64_t n = (p.stat_rows + rows - 1) / rows, x = n < 1 << 21 ? n : 1 << 21;       // a launch has fewer than 2^32 threads along x, and is cut short without an error beyond
        const dim3 grid((unsigned)x, (unsigned)BH, (unsigned)((n + x - 1) / x));
        if (p.out_bf16) hipLaunchKernelGGL((attn_bwd_stats_kernel<D, true>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((attn_bwd_stats_kernel<D, false>), grid, dim3(256), 0, st, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const BwdPlan& w = p.plan;
    const int64_t hidden = p.Skv > (int64_t)w.key_per_head * kBwdRows ? (p.Skv - (int64_t)w.key_per_head * kBwdRows + kBwdRows - 1) / kBwdRows * BH : 0;
    const int64_t items = (int64_t)w.key_blocks * w.key_parts + w.query_blocks + (int64_t)w.query_cut * (w.query_parts - 1) + hidden;
    if (items > 0x7fffffff - p.n_cu) return hipErrorInvalidValue;
    p.items = (int)items;
    p.grid = p.Sq > 0 && items > p.n_cu ? p.n_cu : p.items;
    static KernelSetup setup;
    hipError_t e = setup.ensure(reinterpret_cast<const void*>(attn_bwd_kernel<D>), item_smem<D>(), nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(attn_bwd_kernel<D>, dim3((unsigned)p.grid), dim3(512), item_smem<D>(), st, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int64_t joins = (w.key_parts > 1 ? (int64_t)w.key_blocks * 2 : 0) + w.query_cut;
    if (joins == 0) return hipSuccess;
    hipLaunchKernelGGL(attn_bwd_join_kernel<D>, dim3((unsigned)(joins * (2 * (D / 32)))), dim3(256), 0, st, p);
    return hipGetLastError();
}

hipError_t launch_attn_bwd(AttnBwdParams p, int d, hipStream_t st) {
    return d == 128 ? launch_bwd<128>(p, st) : launch_bwd<64>(p, st);
}

}  // namespace pda

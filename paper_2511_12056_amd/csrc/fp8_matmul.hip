// Product of two 8-bit matrices with a power-of-two scale per block of 128: out[m, n] = sum_k a[m, k] b[n, k] + bias[n].
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 bytes and each operand row's 128 values by 2^(byte - 127) of a lane's register, at the
// rate of the unscaled instruction: a block of 128 is one instruction's K, and scales cost no arithmetic.  The order of K inside a block is the same permutation
// for both operands and does not matter.  b's rows are the first operand, so a lane ends up with four consecutive n of one m.
#include <hip/hip_runtime.h>
#include "attn_device.h"
#include "attn_internal.h"
#include "proj_internal.h"
#include "train_device.h"

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

typedef u32x2 u32x2_loose __attribute__((aligned(2)));      // rows of any length start at any element
typedef u32x4 u32x4_loose __attribute__((aligned(2)));

// The first n (or all) of eight values.
__device__ __forceinline__ void store_row(__bf16* at, const u32x4& x, int64_t n) {
    typedef unsigned u32_loose __attribute__((aligned(2)));
    if (n >= 8) {
        *reinterpret_cast<u32x4_loose*>(at) = x;
        return;
    }
    if (n & 4) *reinterpret_cast<u32x2_loose*>(at) = u32x2{x[0], x[1]};
    if (n & 2) *reinterpret_cast<u32_loose*>(at + (n & 4)) = n & 4 ? x[2] : x[0];
    if (n & 1) at[n & 6] = __builtin_bit_cast(__bf16, (unsigned short)(n & 4 ? n & 2 ? x[3] : x[2] : n & 2 ? x[1] : x[0]));
}

// Four results of row m, columns n .. n + 3: the bias added, rounded.
__device__ __forceinline__ void store4(const MatmulParams& p, int64_t m, int64_t n, f32x4 v) {
    __bf16* o = p.out + m * p.ldo + n;
    if (p.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += n + e < p.N ? p.bias[n + e] : 0.f;
    }
    if (n + 4 <= p.N) {
        *reinterpret_cast<u32x2_loose*>(o) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) o[e] = (__bf16)v[e];
    }
}

// Eight results of row m, columns n .. n + 7.
__device__ __forceinline__ void store8(const MatmulParams& p, int64_t m, int64_t n, f32x4 v0, f32x4 v1) {
    float bias[8] = {};
    if (p.bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[e] = n + e < p.N ? p.bias[n + e] : 0.f;
    }
    store_row(p.out + m * p.ldo + n, u32x4{pack_bf16(v0[0] + bias[0], v0[1] + bias[1]), pack_bf16(v0[2] + bias[2], v0[3] + bias[3]),
                                           pack_bf16(v1[0] + bias[4], v1[1] + bias[5]), pack_bf16(v1[2] + bias[6], v1[3] + bias[7])}, p.N - n);
}

// ---- large products -----------------------------------------------------------------------------------------------
// 256 x 256 results a workgroup of four wavefronts, 128 x 128 each, one workgroup a compute unit and one wavefront a SIMD, with all of its registers: 256
// accumulators, 128 of operands.  A step is a block of 128: 64 matrix instructions in 64 slots, each with the LDS read or fetch that is
// due between two of them.  The first 32 take rows 0 to 3 (of 16) with all columns, the others column by column rows 4 to 7, so that every operand register is free
// some time before its next content is needed: rows 4 to 7 are read in the first half, and the next step's columns and rows 0 to 3 in the second.
// Two barriers a step.  Behind the first (slot 7) all have read the block but its rows 4 to 7, which have arrived: what has been read is fetched for the block
// after the next.  Behind the second (slot 31) all have read those rows and their scales too, which are fetched, and the rest of the next block has arrived.  A fetch has 54 slots
// (1 730 cycles) at least, and a wavefront asks for 1 KB every third slot: faster, requests wait in line and matrix instructions behind them.
// A workgroup goes through its items (tiles, or ranges of K of a tile) without a break; blocks are fetched across the border of an item too.
// 119 056 x 4 608 x 1 536: 680 to 735 us (2.3 to 2.5 PFLOP/s; cards differ), of which 65 are stores and 70 conversion and LDS; 8 192^3: 2.9 PFLOP/s.  The matrix units are 64 to 71 %
// busy at 1.9 to 2.0 of 2.4 GHz.
constexpr int kLargeA = 0, kLargeB = kLargeA + 32768, kLargeStage = kLargeB + 32768, kLargeScales = 2 * kLargeStage, kLargeSa = 0, kLargeSb = 1024, kLargeBias = kLargeScales + 2 * 2048, kLargeEdge = kLargeBias + 4 * 1024, kLargeSmem = kLargeEdge + 4 * 4096;

// Place of tile t of tm x tn, in an order in which neighbours share operands: strips of `strip` tiles of n, tile of m by tile of m.
__device__ __forceinline__ void tile_place(int t, int tm, int tn, int strip, int& m, int& n) {
    const int before = t / (strip * tm), rem = t - before * (strip * tm);
    const int left = tn - before * strip, width = left < strip ? left : strip;
    m = rem / width;
    n = before * strip + rem - m * width;
}

// An accumulator's values where they are wanted: left to itself the compiler copies all 256 out of their registers first, into memory.
__device__ __forceinline__ f32x4 taken(const f32x4& a) {
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float x;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(a[e]));
        v[e] = x;
    }
    return v;
}

// lds_dma16 and lds_dma4 (above) to lds_base + OFF.
template <int OFF>
__device__ __forceinline__ void lds_dma16_to(const void* sbase, unsigned voff, unsigned lds_base) {
    asm volatile("s_add_u32 m0, %0, %1\n\ts_mov_b64 vcc, %3\n\tglobal_load_lds_dwordx4 %2, vcc" : : "s"(lds_base), "n"(OFF), "v"(voff), "s"(sbase) : "memory", "m0", "vcc", "scc");
}

// The piece of a block that is fetched in slot k, or -1: every third slot, twelve behind the step's first barrier, four behind the second.
constexpr int large_piece(int k) { return k >= 8 && k <= 41 && (k - 8) % 3 == 0 ? (k - 8) / 3 : k >= 44 && k <= 53 && (k - 44) % 3 == 0 ? 12 + (k - 44) / 3 : -1; }

struct LargeItem {
    int64_t m0, n0;
    int kb0, nk;
};
__device__ __forceinline__ LargeItem large_item(const MatmulParams& p, int i) {
    const int tm = (int)((p.M + 255) / 256), tn = (int)((p.N + 255) / 256), tiles = tm * tn, part = i / tiles;
    int m, n;
    tile_place(i - part * tiles, tm, tn, p.strip, m, n);
    const int nk_all = (int)(p.K / 128), kb0 = part * p.part_steps, nk = nk_all - kb0 < p.part_steps ? nk_all - kb0 : p.part_steps;
    return {(int64_t)m * 256, (int64_t)n * 256, kb0, nk};
}

template <bool E5M2>
__global__ __launch_bounds__(256, 1) void fp8_matmul_large_kernel(const MatmulParams p, int items) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char matmul_smem_[];
    const unsigned lds0 = (unsigned)(uintptr_t)(LDS_PTR(unsigned char))matmul_smem_;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w >> 1, wn = w & 1;
    // this workgroup's items: XCD x (every eighth workgroup) has a consecutive eighth of them
    const int x = blockIdx.x % 8, per = gridDim.x / 8;
    const int end = (int)((int64_t)items * (x + 1) / 8);
    int next = (int)((int64_t)items * x / 8) + blockIdx.x / 8;  // the item that is fetched
    if (next >= end) return;

    // ---- fetching: a cursor that runs up to two blocks ahead
    const unsigned char *pa = nullptr, *pb = nullptr, *psa = nullptr, *psb = nullptr;
    int f_left = 0, f_kb = 0, f_items = 0;                      // blocks left of the item, its block, items begun
    unsigned f_to = lds0 + w * 1024;                            // stage, this wavefront's place in its chunks
    const int r0 = w * 8 + lane / 8;                            // row of chunk 0, + 32 i
    unsigned f_scales = lds0 + kLargeScales + w * 256;
    unsigned va[8], vb[8], vsa = 0, vsb = 0;                    // byte offsets of the lane's pieces
    const auto fetch_begin = [&]() __attribute__((always_inline)) {
        if (f_left > 0 || next >= end) return;                  // (behind the last item its last block is fetched again, for nobody)
        const LargeItem it = large_item(p, next);
        next += per;
        const int last_m = (int)(p.M - it.m0 < 256 ? p.M - it.m0 : 256) - 1, last_n = (int)(p.N - it.n0 < 256 ? p.N - it.n0 : 256) - 1;
        const unsigned ga = ((lane & 7) ^ ((r0 >> 1) & 7)) * 16, gb = ((lane & 7) ^ (((r0 >> 1) & 1) | ((r0 >> 3) & 3) << 1)) * 16;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = r0 + 32 * i;
            va[i] = __umul24(r < last_m ? r : last_m, (unsigned)p.K) + ga;
            vb[i] = __umul24(r < last_n ? r : last_n, (unsigned)p.K) + gb;
        }
        const int sr = w * 64 + lane, sm = sr < last_m ? sr : last_m, sn = sr < last_n ? sr : last_n;
        vsa = (unsigned)sm * (unsigned)p.scale_cols;
        vsb = (unsigned)(sn >> p.b_shift) * (unsigned)p.scale_cols;
        psa = p.a_scales + it.m0 * p.scale_cols;
        psb = p.b_scales + (it.n0 >> p.b_shift) * p.scale_cols;
        pa = p.a + it.m0 * p.K + (int64_t)it.kb0 * 128;
        pb = p.b + it.n0 * p.K + (int64_t)it.kb0 * 128;
        f_left = it.nk;
        f_kb = it.kb0;
        if (p.bias && p.parts == 1) {                           // 64 values a wavefront; four places, because an item of one block lets the fetch run two items ahead
            lds_dma4(p.bias + it.n0, (unsigned)sn * 4, lds0 + kLargeBias + (f_items & 3) * 1024 + w * 256);
        }
        ++f_items;
    };
    // piece q of a block: rows of b, 0 to 7; rows 0 to 3 (of 16) of a's wavefronts, 8 to 11; rows 4 to 7, 12 to 15
    const auto fetch = [&](auto piece) __attribute__((always_inline)) {
        constexpr int q = decltype(piece)::value;
        if constexpr (q < 8) {
            lds_dma16_to<kLargeB + q * 4096>(pb, vb[q], f_to);
        } else {
            constexpr int i = q < 12 ? (q - 8) / 2 * 4 + q % 2 : (q - 12) / 2 * 4 + 2 + q % 2;      // chunk of 32 rows
            lds_dma16_to<kLargeA + i * 4096>(pa, va[i], f_to);
        }
    };
    // Words of four blocks' scales, with the first of them: a word a row may be a line a row, as many as the block itself has.
    const auto fetch_scales = [&]() __attribute__((always_inline)) {
        if ((f_kb & 3) != 0) return;
        lds_dma4(psa + f_kb, vsa, f_scales + kLargeSa);
        lds_dma4(psb + f_kb, vsb, f_scales + kLargeSb);
        f_scales = 2 * (lds0 + kLargeScales + w * 256) + 2048 - f_scales;
    };
    const auto fetch_end = [&]() __attribute__((always_inline)) {
        --f_left;
        const int more = f_left > 0 ? 1 : 0;
        pa += 128 * more;
        pb += 128 * more;
        f_kb += more;
        f_to = 2 * (lds0 + w * 1024) + kLargeStage - f_to;      // the other stage
    };

    // ---- operands.  Granules g and g + 4 of a row, at their swizzled places (LDS serves 16-byte reads of 16 lanes at a time, from two neighbouring g: with 2g and
    // 2g + 1 half of its time went into bank conflicts).  nrow + 32 (j / 2) + 4 (j % 2) is the row of b of column block j, so that a lane's results of two blocks are
    // eight consecutive columns and those of four lanes 64 bytes (bits 2, 5 and 6, which b's swizzle does not look at)
    const int r16 = lane & 15, g = lane >> 4;
    const int mrow = wm * 128 + r16, nrow = wn * 128 + (r16 / 4) * 8 + (r16 & 3);
    const unsigned ra = kLargeA + mrow * 128 + ((g ^ (r16 >> 1)) * 16), rb = kLargeB + nrow * 128 + ((g ^ (r16 >> 1)) * 16);
    const unsigned ra2 = kLargeA + ((ra - kLargeA) ^ 64), rb2 = kLargeB + ((rb - kLargeB) ^ 64);
    i32x8 fa[8], fb[8];
    int sa[8], sb[8];
    f32x4 acc[8][8];
    const unsigned char* s = matmul_smem_;                      // the stage that is read
    const unsigned char* s_scales = matmul_smem_ + kLargeScales;        // its words of scales, and its byte in them
    const unsigned char* s_byte = s_scales;
    const auto read_a = [&](auto i) __attribute__((always_inline)) {
        constexpr int I = decltype(i)::value;
        fa[I] = join8(*reinterpret_cast<const i32x4*>(s + ra + I * 2048), *reinterpret_cast<const i32x4*>(s + ra2 + I * 2048));
        sa[I] = s_byte[kLargeSa + mrow * 4 + I * 64];
    };
    const auto read_b = [&](auto j) __attribute__((always_inline)) {
        constexpr int J = decltype(j)::value, at = (J / 2) * 4096 + (J % 2) * 512;
        fb[J] = join8(*reinterpret_cast<const i32x4*>(s + rb + at), *reinterpret_cast<const i32x4*>(s + rb2 + at));
        sb[J] = s_byte[kLargeSb + nrow * 4 + at / 32];
    };
    const auto next_stage = [&](int kb) __attribute__((always_inline)) {
        s = s == matmul_smem_ ? matmul_smem_ + kLargeStage : matmul_smem_;
        if ((kb & 3) == 0) s_scales = s_scales == matmul_smem_ + kLargeScales ? matmul_smem_ + kLargeScales + 2048 : matmul_smem_ + kLargeScales;
        s_byte = s_scales + (kb & 3);
    };

    static_for<0, 2>([&](auto) __attribute__((always_inline)) {
        fetch_begin();
        static_for<0, 16>([&](auto q) __attribute__((always_inline)) { fetch(q); });
        fetch_scales();
        fetch_end();
    });
    int item = (int)((int64_t)items * x / 8) + blockIdx.x / 8, items_read = 0;
    LargeItem it = large_item(p, item);
    wait_vmcnt<0>();
    asm volatile("s_barrier" ::: "memory");
    static_for<0, 8>([&](auto j) __attribute__((always_inline)) { read_b(j); });
    static_for<0, 4>([&](auto i) __attribute__((always_inline)) { read_a(i); });
    bool stored = false;                                        // this wavefront has stored a whole tile's part just now: 32 stores behind the last fetch
    for (;;) {
        const int item_n = item + per;
        const bool more = item_n < end;
        const LargeItem it_n = large_item(p, more ? item_n : item);
        const auto run = [&](auto first, int kb_next) __attribute__((always_inline)) {
            static_for<0, 64>([&](auto slot) __attribute__((always_inline)) {
                constexpr int k = decltype(slot)::value, k2 = k - 32;
                constexpr int i = k < 32 ? k / 8 : 4 + k2 % 4, j = k < 32 ? k % 8 : k2 / 4;
                acc[i][j] = mfma<E5M2>(fb[j], fa[i], decltype(first)::value ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[i][j], sb[j], sa[i]);
                asm volatile("" : "+a"(acc[i][j]));             // in its slot: nothing else keeps it there
                if constexpr (k == 7) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (decltype(first)::value && stored) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(16 + 32) : "memory");     // the stores of the tile ahead may still be on their way
                    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(16) : "memory");
                    asm volatile("s_barrier" ::: "memory");
                    fetch_begin();
                }
                if constexpr (k >= 8 && k < 16 && k % 2 == 0) read_a(std::integral_constant<int, 4 + (k >= 8 && k < 16 ? (k - 8) / 2 : 0)>{});
                if constexpr (large_piece(k) >= 0) fetch(std::integral_constant<int, large_piece(k) >= 0 ? large_piece(k) : 0>{});
                if constexpr (k == 31) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (decltype(first)::value && stored) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(4 + 8 + 32) : "memory");
                    else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(4 + 8) : "memory");
                    asm volatile("s_barrier" ::: "memory");
                    next_stage(kb_next);
                }
                if constexpr (k == 32) fetch_scales();
                if constexpr (k == 54) fetch_end();
                if constexpr (k2 >= 0 && k2 < 16 && k2 % 4 == 1) read_a(std::integral_constant<int, k2 >= 0 ? k2 / 4 : 0>{});
                if constexpr (k2 >= 0 && k2 % 4 == 3) read_b(std::integral_constant<int, k2 >= 0 ? k2 / 4 : 0>{});
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        run(std::true_type{}, it.nk > 1 ? it.kb0 + 1 : it_n.kb0);
        for (int t = 1; t < it.nk; ++t) run(std::false_type{}, t + 1 < it.nk ? it.kb0 + t + 1 : it_n.kb0);
        // (the accumulators come out of the loop or of the step ahead of it, so no instruction can be moved down here: see keep)
        asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");       // behind the last matrix instruction, for what reads its result in inline assembly
        const int l = opaque_lane();
        stored = false;
        if (p.parts > 1) {
            float* to = p.part + ((int64_t)item << 16) + w * 16384 + l * 4;      // as they lie in the registers: 1 KB a store
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) *reinterpret_cast<f32x4*>(to + (i * 8 + j) * 256) = taken(acc[i][j]);
        } else {
            // 16 rows at a time through LDS (granules of 16 bytes at granule ^ row), so that a store is 256 bytes of four rows: with 64 bytes of 16 rows, straight from the
            // registers, 119 056 x 4 608 x 1 536 took 746 us instead of 723 (both without the stores' hint).  Under the
            // matrix instructions of the last step's second half and the next tile's first, one accumulator a slot, it took 705 instead of 695: the card's power is the same
            const int rows = (int)(p.M - it.m0 < 256 ? p.M - it.m0 : 256), cols = (int)(p.N - it.n0 < 256 ? p.N - it.n0 : 256);
            stored = rows == 256 && cols == 256 && p.vec_out;
            f32x4 bias[8];
            const float* b = reinterpret_cast<const float*>(matmul_smem_ + kLargeBias + (items_read & 3) * 1024) + wn * 128 + 8 * (l >> 4);
#pragma unroll
            for (int j = 0; j < 8; ++j) bias[j] = p.bias ? *reinterpret_cast<const f32x4*>(b + (j / 2) * 32 + (j % 2) * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
            const auto rounded = [&](const f32x4& a, const f32x4& c) __attribute__((always_inline)) {
                const f32x4 v = taken(a);
                return u32x2{pack_bf16(v[0] + c[0], v[1] + c[1]), pack_bf16(v[2] + c[2], v[3] + c[3])};
            };
            unsigned char* mine = matmul_smem_ + kLargeEdge + w * 4096;
            const int r1 = l >> 4, c1 = l & 15, row = wm * 128 + r1, col = wn * 128 + c1 * 8;     // row (+ 16 i + 4 k) and columns that this lane stores
            unsigned char* to = reinterpret_cast<unsigned char*>(p.out + it.m0 * p.ldo + it.n0);
            u32x4 v[4];                                         // read back while the next 16 rows are rounded
            const auto through = [&](auto&& store) __attribute__((always_inline)) {
                static_for<0, 9>([&](auto ic) __attribute__((always_inline)) {
                    constexpr int i = decltype(ic)::value;
                    if constexpr (i < 8) {
#pragma unroll
                        for (int j = 0; j < 8; j += 2) {
                            const u32x2 lo = rounded(acc[i][j], bias[j]), hi = rounded(acc[i][j + 1], bias[j + 1]);
                            *reinterpret_cast<u32x4*>(mine + (l & 15) * 256 + ((2 * j + (l >> 4)) ^ (l & 15)) * 16) = u32x4{lo[0], lo[1], hi[0], hi[1]};
                        }
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {               // (LDS serves a wavefront in order)
                        if constexpr (i > 0) store(16 * (i - 1) + 4 * k, v[k]);
                        if constexpr (i < 8) v[k] = *reinterpret_cast<const u32x4*>(mine + (4 * k + r1) * 256 + (c1 ^ (4 * k + r1)) * 16);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                });
            };
            if (stored) {
                const unsigned pitch = (unsigned)p.ldo * 8;     // bytes of four rows
                unsigned at = ((unsigned)row * (unsigned)p.ldo + col) * 2;
                through([&](int, const u32x4& x) __attribute__((always_inline)) {
                    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(to + at));      // operands stay in L2: 698 us instead of 705, and what reads out next
                    at += pitch;                                                            // takes as long (9 600 x 4 608 x 1 536) or less (119 056 x 4 608 x 1 536)
                });
            } else {
                through([&](int k, const u32x4& x) __attribute__((always_inline)) {
                    if (row + k < rows && col < cols) store_row(reinterpret_cast<__bf16*>(to) + (int64_t)(row + k) * p.ldo + col, x, cols - col);
                });
            }
        }
        ++items_read;
        if (!more) break;
        item = item_n;
        it = it_n;
    }
    wait_vmcnt<0>();                                            // no fetch outlives the workgroup's LDS
}

// ---- middle tiles -------------------------------------------------------------------------------------------------
// TM x TN results a workgroup of 2 x 2 wavefronts, for products that would leave most compute units without a large tile: there time is the latency of
// memory, so six blocks of 128 are on their way at once, in a ring of eight LDS buffers with a barrier every two blocks.  A block takes 0.28 us (32 x 64) or 0.35 us (64 x 64).
// 256 x 1 536 x 4 096 is 11.1 us with the call (32 x 64: 192 workgroups; 64 x 64: 96 workgroups, 14.1), 13.2 with a barrier every block, 16.2 with operands straight
// from memory into registers.
constexpr int kMidRing = 8, kMidChunks = 4;             // words of scales: of four blocks each
template <int TM, int TN> constexpr int mid_stage() { return (TM + TN) * 128; }
template <int TM, int TN> constexpr int mid_smem() { return kMidRing * mid_stage<TM, TN>() + kMidChunks * 512; }

template <int TM, int TN, bool E5M2>
__global__ __launch_bounds__(256) void fp8_matmul_mid_kernel(const MatmulParams p) {
    constexpr int MT = TM / 32, NT = TN / 32, PA = TM / 32, PB = TN / 32, STAGE = mid_stage<TM, TN>(), B_AT = TM * 128, SCALES = kMidRing * STAGE;
    static_assert(NT == 2, "a lane's results of two instructions are eight consecutive columns");
    extern __shared__ __attribute__((aligned(1024))) unsigned char matmul_smem_[];
    const unsigned lds0 = (unsigned)(uintptr_t)(LDS_PTR(unsigned char))matmul_smem_;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = w >> 1, wn = w & 1, r16 = lane & 15, g = lane >> 4;
    const int tn = (int)((p.N + TN - 1) / TN), tile_m = blockIdx.x / tn, tile_n = blockIdx.x - tile_m * tn;
    const int64_t m0 = (int64_t)tile_m * TM, n0 = (int64_t)tile_n * TN;
    const int nk_all = (int)(p.K / 128), kb0 = blockIdx.y * p.part_steps, nk = nk_all - kb0 < p.part_steps ? nk_all - kb0 : p.part_steps;
    const int last_m = (int)(p.M - m0 < TM ? p.M - m0 : TM) - 1, last_n = (int)(p.N - n0 < TN ? p.N - n0 : TN) - 1;
    // fetching: eight rows a request, the granules of 16 bytes swizzled as in large tiles
    unsigned va[PA], vb[PB];
#pragma unroll
    for (int i = 0; i < PA; ++i) {
        const int r = (w + 4 * i) * 8 + lane / 8;
        va[i] = __umul24(r < last_m ? r : last_m, (unsigned)p.K) + ((lane & 7) ^ ((r >> 1) & 7)) * 16;
    }
#pragma unroll
    for (int i = 0; i < PB; ++i) {
        const int r = (w + 4 * i) * 8 + lane / 8;
        vb[i] = __umul24(r < last_n ? r : last_n, (unsigned)p.K) + ((lane & 7) ^ (((r >> 1) & 1) | ((r >> 3) & 3) << 1)) * 16;
    }
    const int slim = wm == 0 ? last_m : last_n, sr = lane < slim ? lane : slim;
    const unsigned vs = (unsigned)(wm == 0 ? sr : sr >> p.b_shift) * (unsigned)p.scale_cols;
    const unsigned char* pa = p.a + m0 * p.K + (int64_t)kb0 * 128;
    const unsigned char* pb = p.b + n0 * p.K + (int64_t)kb0 * 128;
    const unsigned char* ps = wm == 0 ? p.a_scales + m0 * p.scale_cols : p.b_scales + (n0 >> p.b_shift) * p.scale_cols;
    const auto fetch = [&](int t) __attribute__((always_inline)) {
        const int kb = kb0 + t;
        if (wn == 0 && (t == 0 || (kb & 3) == 0)) lds_dma4(ps + (kb & ~3), vs, lds0 + SCALES + (kb >> 2) % kMidChunks * 512 + wm * 256);     // wavefront 0 those of a, 2 those of b
        const unsigned to = lds0 + t % kMidRing * STAGE + w * 1024;
        const int64_t at = (int64_t)t * 128;
#pragma unroll
        for (int i = 0; i < PA; ++i) lds_dma16(pa + at, va[i], to + i * 4096);
#pragma unroll
        for (int i = 0; i < PB; ++i) lds_dma16(pb + at, vb[i], to + B_AT + i * 4096);
    };
    const int mrow = wm * (TM / 2) + r16, nrow = wn * 32 + (r16 / 4) * 8 + (r16 & 3);
    const unsigned ra = mrow * 128 + ((g ^ (r16 >> 1)) * 16), rb = B_AT + nrow * 128 + ((g ^ (r16 >> 1)) * 16);
    f32x4 acc[MT][NT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < kMidRing - 2; ++t)
        if (t < nk) fetch(t);
    for (int t = 0; t < nk; t += 2) {
        // blocks t and t + 1 have arrived when no more are on their way than belong to the blocks behind them (scales apart: then for a little longer)
        switch (nk - 2 - t) {
            case -1:
            case 0: wait_vmcnt<0>(); break;
            case 1: wait_vmcnt<PA + PB>(); break;
            case 2: wait_vmcnt<2 * (PA + PB)>(); break;
            case 3: wait_vmcnt<3 * (PA + PB)>(); break;
            default: wait_vmcnt<4 * (PA + PB)>();
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");    // and all have read blocks t - 2 and t - 1
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (t + kMidRing - 2 + u < nk) fetch(t + kMidRing - 2 + u);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (u == 1 && t + 1 >= nk) break;
            const unsigned char* s = matmul_smem_ + (t + u) % kMidRing * STAGE;
            const int kb = kb0 + t + u;
            const unsigned char* sc = matmul_smem_ + SCALES + (kb >> 2) % kMidChunks * 512 + (kb & 3);
            i32x8 fb[NT];
            int sb[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                fb[j] = join8(*reinterpret_cast<const i32x4*>(s + rb + j * 512), *reinterpret_cast<const i32x4*>(s + (rb ^ 64) + j * 512));
                sb[j] = sc[256 + (nrow + 4 * j) * 4];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const i32x8 fa = join8(*reinterpret_cast<const i32x4*>(s + ra + i * 2048), *reinterpret_cast<const i32x4*>(s + (ra ^ 64) + i * 2048));
                const int sa = sc[(mrow + 16 * i) * 4];
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[i][j] = mfma<E5M2>(fb[j], fa, acc[i][j], sb[j], sa);
            }
        }
    }
    keep(acc);
    const int col = wn * 32 + 8 * g;
    if (p.parts > 1) {
        float* to = p.part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (TM * TN) + mrow * TN + col;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4*>(to + i * 16 * TN + 4 * j) = acc[i][j];
        return;
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t m = m0 + mrow + 16 * i, n = n0 + col;
        if (m < p.M && n < p.N) store8(p, m, n, acc[i][0], acc[i][1]);
    }
}

// ---- few rows -----------------------------------------------------------------------------------------------------
// 16 x 16 results a workgroup, whose four wavefronts each take a range of K, straight from memory into registers without a barrier, and add their sums in LDS, in
// order: for up to 16 rows, where every row of b is read once and that is all the time there is.  1 x 4 608 x 1 536 is 9.8 us with the call, 4.9 us without; 1 x 8 192 x
// 8 192 is 14.3 (32 x 64 tiles: 19.5).
constexpr int kFewWaves = 4, kFewAhead = 4;             // blocks in registers
template <bool E5M2>
__global__ __launch_bounds__(kFewWaves * 64) void fp8_matmul_few_kernel(const MatmulParams p) {
    __shared__ f32x4 sums[kFewWaves][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
    const int tn = (int)((p.N + 15) / 16), tile_m = blockIdx.x / tn, tile_n = blockIdx.x - tile_m * tn;
    const int64_t m0 = (int64_t)tile_m * 16, n0 = (int64_t)tile_n * 16;
    const int nk_all = (int)(p.K / 128), first = blockIdx.y * p.part_steps, nk = nk_all - first < p.part_steps ? nk_all - first : p.part_steps;
    const int kb0 = first + nk * w / kFewWaves, kb1 = first + nk * (w + 1) / kFewWaves;
    const int64_t m = m0 + r16 < p.M ? m0 + r16 : p.M - 1, n = n0 + r16 < p.N ? n0 + r16 : p.N - 1;      // rows behind the last are the last one's again
    const unsigned char *a = p.a + m * p.K + 16 * g, *b = p.b + n * p.K + 16 * g;
    const uint8_t *sap = p.a_scales + m * p.scale_cols, *sbp = p.b_scales + (n >> p.b_shift) * p.scale_cols;
    struct Block {
        i32x8 a, b;
        int sa, sb;
    };
    const auto load = [&](Block& x, int kb) __attribute__((always_inline)) {
        const int64_t at = (int64_t)kb * 128;
        x.b = join8(*reinterpret_cast<const i32x4*>(b + at), *reinterpret_cast<const i32x4*>(b + at + 64));
        x.sb = sbp[kb];
        x.a = join8(*reinterpret_cast<const i32x4*>(a + at), *reinterpret_cast<const i32x4*>(a + at + 64));
        x.sa = sap[kb];
    };
    f32x4 acc[1] = {f32x4{0.f, 0.f, 0.f, 0.f}};
    Block x[kFewAhead];
#pragma unroll
    for (int u = 0; u < kFewAhead; ++u)
        if (kb0 + u < kb1) load(x[u], kb0 + u);
    for (int kb = kb0; kb < kb1; kb += kFewAhead) {
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u)
            if (kb + u < kb1) {
                acc[0] = mfma<E5M2>(x[u].b, x[u].a, acc[0], x[u].sb, x[u].sa);
                if (kb + u + kFewAhead < kb1) load(x[u], kb + u + kFewAhead);
            }
    }
    keep(acc);
    sums[w][lane] = acc[0];
    __syncthreads();
    if (w != 0) return;
    f32x4 v = sums[0][lane];
#pragma unroll
    for (int o = 1; o < kFewWaves; ++o) v += sums[o][lane];
    if (p.parts > 1) *reinterpret_cast<f32x4*>(p.part + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + r16 * 16 + 4 * g) = v;
    else if (m0 + r16 < p.M && n0 + 4 * g < p.N) store4(p, m0 + r16, n0 + 4 * g, v);
}

// ---- sums of the ranges of K --------------------------------------------------------------------------------------
// Parts hold whole tiles: large ones (TM = 256) as they lay in the registers, others by rows.  Eight columns a thread, or four.
template <int TM, int TN>
__global__ __launch_bounds__(256) void fp8_matmul_join_kernel(const MatmulParams p, int tiles, int tm, int tn) {
    constexpr int C = TN >= 32 ? 8 : 4;
    const int tile = blockIdx.x, e = blockIdx.y * 256 + threadIdx.x;
    if (e >= TM * TN / C) return;
    int im, in, r, c, at, second = 4;                           // row and column in the tile, place of its first four sums, of the others behind them
    if constexpr (TM == 256) {
        tile_place(tile, tm, tn, p.strip, im, in);
        const int lane = e & 63, jj = e >> 6 & 3, i = e >> 8 & 7, w = e >> 11;
        r = (w >> 1) * 128 + i * 16 + (lane & 15);
        c = (w & 1) * 128 + jj * 32 + (lane >> 4) * 8;
        at = ((w * 64 + i * 8 + jj * 2) * 64 + lane) * 4;
        second = 256;
    } else {
        im = tile / tn;
        in = tile - im * tn;
        r = e / (TN / C);
        c = e % (TN / C) * C;
        at = r * TN + c;
    }
    const int64_t m = (int64_t)im * TM + r, n = (int64_t)in * TN + c;
    if (m >= p.M || n >= p.N) return;
    const float* src = p.part + (int64_t)tile * (TM * TN) + at;
    f32x4 v0 = *reinterpret_cast<const f32x4*>(src), v1 = C == 8 ? *reinterpret_cast<const f32x4*>(src + second) : v0;
#pragma unroll 4
    for (int k = 1; k < p.parts; ++k) {
        src += (int64_t)tiles * (TM * TN);
        v0 += *reinterpret_cast<const f32x4*>(src);
        if constexpr (C == 8) v1 += *reinterpret_cast<const f32x4*>(src + second);
    }
    if constexpr (C == 8) store8(p, m, n, v0, v1);
    else store4(p, m, n, v0);
}

// K == 0: the bias
__global__ __launch_bounds__(256) void fp8_matmul_bias_kernel(const MatmulParams p) {
    const int64_t n4 = (p.N + 3) / 4, m = (int64_t)blockIdx.z * gridDim.y + blockIdx.y, c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (m < p.M && c < n4) store4(p, m, c * 4, f32x4{0.f, 0.f, 0.f, 0.f});
}

template <bool E5M2>
static hipError_t launch_large(const MatmulParams& p, hipStream_t st) {
    static KernelSetup setup;
    int n_cu = 0;
    const hipError_t e = setup.ensure(reinterpret_cast<const void*>(fp8_matmul_large_kernel<E5M2>), kLargeSmem, &n_cu);
    if (e != hipSuccess) return e;
    const int64_t items = (p.M + 255) / 256 * ((p.N + 255) / 256) * p.parts;
    if (items > 0x7fffff00) return hipErrorInvalidValue;
    const int grid = n_cu < 8 ? 8 : n_cu / 8 * 8;
    hipLaunchKernelGGL(fp8_matmul_large_kernel<E5M2>, dim3((unsigned)grid), dim3(256), kLargeSmem, st, p, (int)items);
    return hipGetLastError();
}

template <int TM, int TN>
static hipError_t launch_join(const MatmulParams& p, hipStream_t st) {
    if (p.parts == 1) return hipSuccess;
    const int tm = (int)((p.M + TM - 1) / TM), tn = (int)((p.N + TN - 1) / TN), threads = TM * TN / (TN >= 32 ? 8 : 4);
    hipLaunchKernelGGL((fp8_matmul_join_kernel<TM, TN>), dim3((unsigned)(tm * tn), (unsigned)((threads + 255) / 256)), dim3(256), 0, st, p, tm * tn, tm, tn);
    return hipGetLastError();
}

template <int TM, int TN, bool E5M2>
static hipError_t launch_mid(const MatmulParams& p, dim3 grid, hipStream_t st) {
    static KernelSetup setup;
    const hipError_t e = setup.ensure(reinterpret_cast<const void*>(fp8_matmul_mid_kernel<TM, TN, E5M2>), mid_smem<TM, TN>(), nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((fp8_matmul_mid_kernel<TM, TN, E5M2>), grid, dim3(256), (mid_smem<TM, TN>()), st, p);
    return hipGetLastError();
}

template <int F>
static hipError_t launch_form(const MatmulParams& p, hipStream_t st) {
    constexpr FormSize s = kForms[F];
    const dim3 grid((unsigned)((p.M + s.m - 1) / s.m * ((p.N + s.n - 1) / s.n)), (unsigned)p.parts);
    hipError_t e = hipSuccess;
    if constexpr (F == MatmulPlan::LARGE) {
        e = p.e5m2 ? launch_large<true>(p, st) : launch_large<false>(p, st);
    } else if constexpr (F == MatmulPlan::FEW) {
        if (p.e5m2) hipLaunchKernelGGL(fp8_matmul_few_kernel<true>, grid, dim3(kFewWaves * 64), 0, st, p);
        else hipLaunchKernelGGL(fp8_matmul_few_kernel<false>, grid, dim3(kFewWaves * 64), 0, st, p);
        e = hipGetLastError();
    } else {
        e = p.e5m2 ? launch_mid<s.m, s.n, true>(p, grid, st) : launch_mid<s.m, s.n, false>(p, grid, st);
    }
    return e == hipSuccess ? launch_join<s.m, s.n>(p, st) : e;
}

hipError_t launch_fp8_matmul(MatmulParams p, const MatmulPlan& w, hipStream_t st) {
    p.parts = w.parts;
    p.part_steps = w.part_steps;
    // strips of b of which an XCD's L2 (4 MB) keeps 2.5 MB while a runs past, six tiles at least: 32 compute units' tiles side by side are then about a square.
    // Blocks of eight tiles of m, tile of n by tile of n, took 768 us instead of 725 at 4 608 x 119 056 x 1 536, 664 instead of 653 at 4 608 x 1 536 x 119 056 and as long elsewhere
    const int tn = (int)((p.N + 255) / 256), width = (int)(2500000 / (256 * 128 * (int64_t)(w.part_steps > 0 ? w.part_steps : 1))), strip = width > 6 ? width : 6, strips = (tn + strip - 1) / strip;
    p.strip = strips > 0 ? (tn + strips - 1) / strips : 1;
    p.vec_out = p.ldo % 8 == 0 && p.ldo < (int64_t)1 << 22 && reinterpret_cast<uintptr_t>(p.out) % 16 == 0;      // 256 rows within 2^32 bytes
    if (p.K == 0) {
        const int64_t y = p.M < 65535 ? p.M : 65535;
        hipLaunchKernelGGL(fp8_matmul_bias_kernel, dim3((unsigned)(((p.N + 3) / 4 + 255) / 256), (unsigned)y, (unsigned)((p.M + y - 1) / y)), dim3(256), 0, st, p);
        return hipGetLastError();
    }
    switch (w.form) {
        case MatmulPlan::FEW: return launch_form<MatmulPlan::FEW>(p, st);
        case MatmulPlan::MID: return launch_form<MatmulPlan::MID>(p, st);
        case MatmulPlan::MID_WIDE: return launch_form<MatmulPlan::MID_WIDE>(p, st);
    }
    return launch_form<MatmulPlan::LARGE>(p, st);
}

}  // namespace pda

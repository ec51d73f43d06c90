// Internal declarations of the projection side (not part of the ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/pipedit_proj.h"
#include "train_internal.h"

namespace pda {

// ---- 8-bit matrices (fp8_quant.hip) -------------------------------------------------------------
constexpr int64_t fp8_cols(int64_t cols) { return (cols + 127) / 128 * 128; }             // bytes of a row
constexpr int64_t fp8_scale_cols(int64_t cols) { return ((cols + 127) / 128 + 3) / 4 * 4; }     // bytes of a row of scales
struct QuantParams {
    const void* x;
    void* q;                 // nullable
    uint8_t* q_scales;
    void* qt;                // nullable
    uint8_t* qt_scales;
    int64_t rows, cols, ldx;
    int x_bf16, e5m2, square;
};
hipError_t launch_fp8_quant(const QuantParams& p, hipStream_t st);

// ---- their product (fp8_matmul.hip) -------------------------------------------------------------
struct MatmulParams {
    const unsigned char* a;
    const unsigned char* b;
    const uint8_t* a_scales;
    const uint8_t* b_scales;
    const float* bias;       // nullable
    __bf16* out;
    float* part;             // [parts][tiles][tile] partial sums
    int64_t M, N, K, ldo;
    int64_t scale_cols;      // bytes between rows of scales
    int b_shift;             // 0 or 7: rows of b that share a scale
    int e5m2;                // of a
    int parts;               // ranges of K, each of part_steps blocks of 128 (the last may have fewer)
    int part_steps;
    int strip;               // large tiles: tiles of n in a row
    int vec_out;             // rows of out lie at multiples of 16 bytes
};
constexpr int kMatmulMaxParts = 32;
// How a product is split over workgroups: the form of its tiles and the ranges of K.
struct MatmulPlan {
    static constexpr int FEW = 0, MID = 1, MID_WIDE = 2, LARGE = 3, FORMS = 4;
    int form;
    int parts, part_steps;
};
// Tiles of the forms, in rows and columns.
struct FormSize { int m, n; };
inline constexpr FormSize kForms[MatmulPlan::FORMS] = {{16, 16}, {32, 64}, {64, 64}, {256, 256}};

// An estimate of a launch's time in us, for choosing among the forms and numbers of parts.  Its rates are fits to every form's times at 14 products, from 1 x 8 192 x 8 192
// to 119 056 x 4 608 x 1 536 (256 compute units; us, the least of each row is what the rule takes or within 10 % of it):
//                             few    32 x 64    64 x 64    large    large, 4 parts
//       1 x 8 192 x 8 192      14         20         24       74          33
//     256 x 1 536 x 4 096      29         11         14       40          19
//   1 000 x 1 536 x 1 536      37         15         14       21          18
//   2 000 x 1 536 x 6 144     281         85         56       59          35
//   2 048 x 4 608 x 1 536     207         80         54       20          56
inline double form_time(int f, int64_t tiles, int parts, int steps, int n_cu) {
    const FormSize& s = kForms[f];
    const int64_t items = tiles * parts, rounds = (items + n_cu - 1) / n_cu;
    const double load = (double)items / n_cu;
    double t;
    if (f == MatmulPlan::LARGE) t = 6.0 + (double)rounds * (steps * (1.07 + 0.4 * (load < 1.0 ? load : 1.0)) + 4.0);
    else if (f == MatmulPlan::FEW) t = 3.0 + steps * (load > 1.1 ? 0.11 * load : 0.12);
    else t = 3.0 + (double)rounds * (1.0 + steps * (s.m == 64 ? 0.345 : 0.28));
    if (parts > 1) {                                            // parts written and read, more than 128 MB of them from memory: 4 608 x 1 536 x 119 056 took 678 us in
        const double bytes = (double)items * s.m * s.n * 8;     // 2 parts on 216 compute units (now 666), 717 in 7 on 252 (three times)
        t += 5.0 + (bytes < 128e6 ? bytes / 10e6 : 12.8 + (bytes - 128e6) / 4e6);
    }
    return t;
}

inline MatmulPlan plan_matmul(int64_t M, int64_t N, int64_t K, int n_cu) {
    const int nk = (int)(K / 128);
    MatmulPlan best{0, 1, nk};
    double best_time = 1e300;
    if (nk == 0) return best;                                              // the bias alone
    for (int f = 0; f < MatmulPlan::FORMS; ++f) {
        const FormSize& s = kForms[f];
        const int64_t tiles = (M + s.m - 1) / s.m * ((N + s.n - 1) / s.n);
        if (tiles > 0x3fffff && f != MatmulPlan::LARGE) continue;          // a launch has fewer than 2^32 threads along x
        for (int parts = 1; parts <= kMatmulMaxParts; ++parts) {
            const int steps = ((nk + parts - 1) / parts + 3) / 4 * 4;      // (words of four scales in the large form)
            if (parts > 1 && (nk + steps - 1) / steps != parts) continue;
            const double t = form_time(f, tiles, parts, steps < nk ? steps : nk, n_cu);
            if (t < best_time) {
                best_time = t;
                best = {f, parts, steps};
            }
        }
    }
    return best;
}

inline int64_t matmul_workspace_bytes(const MatmulPlan& w, int64_t M, int64_t N) {
    const FormSize& s = kForms[w.form];
    return w.parts > 1 ? w.parts * ((M + s.m - 1) / s.m) * ((N + s.n - 1) / s.n) * s.m * s.n * 4 : 0;
}
hipError_t launch_fp8_matmul(MatmulParams p, const MatmulPlan& w, hipStream_t st);

// ---- root-mean-square norm (rms_norm.hip) -------------------------------------------------------
struct RmsNormParams {
    const void* x;           // forward: x; backward: dy
    const void* res;         // nullable; backward: dres
    const float* weight;     // nullable
    void* h;                 // forward: nullable
    void* y;                 // backward: dh (nullable)
    uint8_t* y_scales;
    float* rstd;             // forward: nullable
    float* dweight;          // nullable
    float* part;             // [groups][chunks][D] partial sums of dweight
    int64_t rows, group_rows, groups;
    int64_t chunks;          // backward: workgroups of a group
    int D;
    int x_type, h_type, y_type;
    float eps;
};
hipError_t launch_rms_norm_fwd(const RmsNormParams& p, hipStream_t st);
hipError_t launch_rms_norm_bwd(const RmsNormParams& p, hipStream_t st);
// (workgroups of a group as layer norm has them)
inline int64_t rms_workspace_bytes(int64_t rows, int64_t groups, int D, int n_cu) {
    if (rows == 0 || groups == 0) return 0;
    const int64_t c = ln_chunks(rows / groups, groups, D, n_cu);
    return c <= 1 ? 0 : groups * c * D * 4;
}

// ---- pack with rotary positions (rope.hip) ------------------------------------------------------
struct RopeParams {
    const void* x;           // token-major; backward: the pack's input (nullable)
    void* dx;                // backward
    __bf16* y;               // head-major; backward: dy, read
    const int32_t* positions;
    int64_t x_batch, x_token, dx_batch, dx_token, y_batch, y_head, pos_batch, first;
    int64_t S, token_blocks;
    int B, H, heads;         // heads: of a workgroup
    int rot, layout, axes;
    int axis_end[PDA_ROPE_MAX_AXES];       // the pairs' running sums
    int x_bf16, unit_rms;
    float premul;
    double turns[64];        // frequencies over 2 pi
};
hipError_t launch_rope(RopeParams& p, int d, bool backward, int n_cu, hipStream_t st);

}  // namespace pda

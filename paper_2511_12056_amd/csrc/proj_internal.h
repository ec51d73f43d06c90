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
MatmulPlan plan_matmul(int64_t M, int64_t N, int64_t K, int n_cu);
int64_t matmul_workspace_bytes(const MatmulPlan& w, int64_t M, int64_t N);
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

// Internal declarations of the training operators (not part of the ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pda {

// Sets the calling thread's error message and returns `code` (api.hip).
int report(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// ---- attention, backward (attn_bwd.hip) ---------------------------------------------------------
struct AttnBwdParams {
    const __bf16* dout;
    const __bf16* q;
    const __bf16* k;
    const __bf16* v;
    const void* out;
    const float* lse;
    __bf16* dq;
    __bf16* dk;
    __bf16* dv;
    float* stats;            // [B*H][stat_rows / 32][2][32]: -lse * log2(e) of 32 rows (-inf where a row has no keys and behind the last row),
                             // -<dout, out> of the same rows (0 behind the last row)
    int64_t Sq, Skv, n_v;    // query rows, key rows, valid keys
    int64_t stat_rows;       // bwd_stat_rows(Sq)
    int64_t do_bs, do_hs, q_bs, q_hs, kv_bs, kv_hs, o_bs, o_hs, l_bs, l_hs, dq_bs, dq_hs, dkv_bs, dkv_hs;
    int B, H;
    int out_bf16;
    float scale, scale_log2e;
};
inline int64_t bwd_stat_rows(int64_t Sq) { return (Sq + 63) / 64 * 64; }
inline int64_t bwd_workspace_bytes(int64_t BH, int64_t Sq) { return (BH * bwd_stat_rows(Sq) * 8 + 255) / 256 * 256; }
hipError_t launch_attn_bwd(const AttnBwdParams& p, int d, hipStream_t st);

// ---- layer norm (layer_norm.hip) ----------------------------------------------------------------
struct LayerNormParams {
    const void* x;
    const void* dy;          // backward
    const float* weight;     // nullable
    const float* bias;       // nullable, forward
    void* y;                 // forward: y; backward: dx (nullable)
    float* mean;
    float* rstd;
    float* dweight;          // nullable
    float* dbias;            // nullable
    float* part;             // [groups][chunks][2][D] partial sums of dweight and dbias
    int64_t rows, group_rows;
    int64_t groups;
    int64_t chunk_rows;      // backward: rows of a workgroup
    int64_t chunks;          // backward: workgroups of a group
    int D;
    float eps;
};
hipError_t launch_layer_norm_fwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, hipStream_t st);
hipError_t launch_layer_norm_bwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, hipStream_t st);

// Rows of a workgroup of the backward kernel: about four workgroups per CU, four rows at least (a row per wavefront).
inline int64_t ln_chunk_rows(int64_t group_rows, int64_t groups, int n_cu) {
    const int64_t want = 4 * (int64_t)n_cu / groups > 0 ? 4 * (int64_t)n_cu / groups : 1;
    const int64_t rows = (group_rows + want - 1) / want;
    return rows < 4 ? 4 : rows;
}
inline int64_t ln_chunks(int64_t group_rows, int64_t groups, int n_cu) {
    const int64_t r = ln_chunk_rows(group_rows, groups, n_cu);
    return (group_rows + r - 1) / r;
}
// One workgroup per group writes its sums itself.
inline int64_t ln_workspace_bytes(int64_t rows, int64_t groups, int D, int n_cu) {
    if (rows == 0 || groups == 0) return 0;
    const int64_t c = ln_chunks(rows / groups, groups, n_cu);
    return c <= 1 ? 0 : groups * c * 2 * D * 4;
}

// ---- pack, backward (layout.hip) ----------------------------------------------------------------
hipError_t launch_pack_bwd(const void* dy, const float* x, float* dx, int B, int64_t S, int H, int d, int unit_rms, float premul, hipStream_t st);

}  // namespace pda

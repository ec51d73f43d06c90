/*
 * libpipedit_attn, projection side: the way from the residual stream to the attention call and back.  Root-mean-square norm with
 * the residual's addition, 8-bit matrices with a scale per block of 128 and their product (projections and their gradients), and
 * the pack with rotary positions.  Conventions of pipedit_train.h: device pointers, caller-owned tensors, workspaces
 * from the caller, pda_status and pda_last_error(), kernels enqueued on the given stream, arguments validated before any device
 * work, nothing allocates, frees or synchronises (every call may be captured into a HIP graph from the start), equal calls give
 * equal bits.  A workspace holds nothing between calls; calls whose execution may overlap need workspaces of their own.
 */
#ifndef PIPEDIT_PROJ_H
#define PIPEDIT_PROJ_H

#include "pipedit_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit element types, beside PDA_F32 and PDA_BF16: largest values 448 and 57 344, the first without infinities. */
#define PDA_E4M3 2
#define PDA_E5M2 3

/*
 * An 8-bit matrix [rows, cols] is two tensors:
 *
 *     q       [rows, cols rounded up to 128], one byte an element; the columns behind cols hold zeros
 *     scales  [rows or ceil(rows / 128), S], one byte a block of 128 columns of 1 or 128 rows; S = ceil(cols / 128) rounded up to
 *             4; the bytes behind the last block are not used and not written
 *
 * and stands for q * 2^(scale - 127).  The scale of a block is the smallest of these powers (from 2^-127 on) with which its largest finite
 * magnitude does not pass the type's largest value: 2^0 for a block without any but zeros.  Values are multiplied by the inverse power, exactly, and
 * rounded to nearest even.  An infinity becomes NaN in PDA_E4M3 and stays in PDA_E5M2.  The byte 255 is never written; the
 * product takes it as NaN.  A range of rows (of 128-row blocks) of such a matrix is one itself.
 */

/*
 * x [rows, cols] fp32 or bf16, rows ldx >= cols elements apart -> q, its 8-bit matrix, and qt, that of the transposed
 * matrix (rows and columns exchanged: [cols, rows rounded up to 128]); either pair may be NULL.  block_rows = 1: blocks lie along
 * the rows of what is written, so q and qt have scales of their own (activations and gradients: q for x W^T and dy W, qt for dy^T x).
 * block_rows = 128: blocks of 128 x 128, whose scales and values agree in both (weights: q for x W^T, qt for dy W).
 * fp8_type: PDA_E4M3 or PDA_E5M2.  q and qt 16-byte aligned, scales 4-byte, x its element; nothing that is written may overlap anything else.
 * rows == 0 or cols == 0 is a no-op.
 */
int pda_fp8_quant(const void* x, int x_type, int64_t rows, int64_t cols, int64_t ldx, int fp8_type, int block_rows,
                  void* q, uint8_t* q_scales, void* qt, uint8_t* qt_scales, void* stream);

/*
 * out[m, n] = sum_k a[m, k] b[n, k] + bias[n]: a [M, K] in blocks of one row, b [N, K] in blocks of b_block_rows = 1 or 128, out
 * [M, N] bf16, rows ldo >= N elements apart, bias [N] fp32 or NULL.  K is a multiple of 128 (the padded length of the rows); K == 0 gives the bias.
 *
 *     x W^T     a = x, b = W (blocks of 128)        a projection
 *     dy W      a = dy, b = W's qt (blocks of 128)  the gradient of its input
 *     dy^T x    a = dy's qt, b = x's qt             the gradient of its weight
 *
 * a_type: PDA_E4M3 or PDA_E5M2; b is PDA_E4M3.  Sums are fp32.  The matrix instructions for 8-bit operands align the products of eight consecutive k to the largest of
 * them and drop what lies 2^-13 below it, before they add them: 1.5e-5 of the result on Gaussian values, at any K.  The result is rounded to bf16 once.  A NaN, or an
 * infinity, of either matrix goes into the results that it is part of.
 * a, b and out 16-byte aligned, scales and bias 4-byte; out must not overlap anything else.  workspace: 256-byte aligned, of
 * at least what pda_fp8_matmul_workspace gives for M, N and K (NULL if that is 0).
 */
int pda_fp8_matmul(const void* a, int a_type, const uint8_t* a_scales, const void* b, const uint8_t* b_scales, int b_block_rows,
                   const float* bias, void* out, int64_t M, int64_t N, int64_t K, int64_t ldo,
                   void* workspace, int64_t workspace_bytes, void* stream);
int pda_fp8_matmul_workspace(int64_t M, int64_t N, int64_t K, int n_cu, int64_t* bytes);

/*
 * Root-mean-square norm over the last axis, with the addition that stands in front of it in a transformer block:
 *
 *     h[r,c] = res[r,c] + x[r,c]                                  the residual stream, rounded to its type
 *     rstd_r = 1 / sqrt(sum_c h[r,c]^2 / D + eps)
 *     y[r,c] = h[r,c] * rstd_r * weight[g,c]
 *
 * x [rows, D] and res, h [rows, D] (res_type, both) are PDA_F32 or PDA_BF16; what is normalised is h as it is stored.  res == NULL: no addition, h must be
 * NULL too and stands for x.  weight [groups, D] fp32, group g holding the rows / groups consecutive rows from g * rows / groups on
 * (pda_layer_norm_fwd), or NULL (1).  y_type PDA_F32 or PDA_BF16: y [rows, D], rounded once.  y_type PDA_E4M3: y and y_scales are
 * the 8-bit matrix, in blocks of one row, of the fp32 values, as pda_fp8_quant makes it; where these are too near to a scale's border, 64 bits decide on its side.  rstd [rows] fp32, for the backward call, may be NULL.
 * h may be res or x itself (if the types agree), otherwise nothing that is written may overlap anything else.  Sums are fp32 (rstd is 0 where
 * the squares of a row pass its range).
 * 1 <= D <= PDA_LAYER_NORM_MAX; eps finite and >= 0; tensors 16-byte aligned, y_scales and rstd 4-byte; rows == 0 is a no-op.
 */
int pda_rms_norm_fwd(const void* x, int x_type, const void* res, int res_type, const float* weight, void* h, void* y, int y_type,
                     uint8_t* y_scales, float* rstd, int64_t rows, int64_t groups, int D, float eps, void* stream);

/*
 * Gradient of pda_rms_norm_fwd, with hh = h * rstd and g = dy * weight:
 *
 *     dh[r,c]      = dres[r,c] + rstd_r * (g[r,c] - hh[r,c] * sum_c (g * hh)[r,:] / D)
 *     dweight[g,c] = sum over the rows r of group g of dy[r,c] * hh[r,c]
 *
 * dh is the gradient of res and of x; dres, the gradient that reaches h past the norm, may be NULL (0).  dy PDA_F32 or PDA_BF16 (of an 8-bit y as well); h, dres
 * and dh of one type, h_type; dh is rounded once.  dh or dweight [groups, D] fp32, which is written, not added to, may be NULL, not both.
 * dh may be h, dres or dy itself if the types agree, otherwise nothing that is written may overlap anything else.  rows == 0 writes
 * dweight = 0.  workspace: 16-byte aligned, at least what pda_rms_norm_bwd_workspace gives (NULL if that is 0 or dweight not wanted).
 */
int pda_rms_norm_bwd(const void* dy, int dy_type, const void* h, int h_type, const float* weight, const float* rstd, const void* dres,
                     void* dh, float* dweight, int64_t rows, int64_t groups, int D, void* workspace, int64_t workspace_bytes, void* stream);
int pda_rms_norm_bwd_workspace(int64_t rows, int64_t groups, int D, int n_cu, int64_t* bytes);

/*
 * Rotary positions: columns (2i, 2i+1) (PDA_ROPE_INTERLEAVED) or (i, i + rot/2) (PDA_ROPE_HALF) of the first rot columns of a head
 * are pair i = 0 .. rot/2 - 1, which turns by the angle position * freqs[i]:
 *
 *     (u, v) -> (u cos - v sin, u sin + v cos)
 *
 * The position has 1 to PDA_ROPE_MAX_AXES axes (frame, row and column of a video token): the first axis_pairs[0] pairs turn with the
 * first, the next axis_pairs[1] with the second, and so on; they sum to rot/2.  positions: DEVICE int32 [S, axes], a batch
 * pos_batch entries behind the one before (0: shared), or NULL: token s is at first + s on the one axis.  rot is a
 * multiple of 8, at most d; 0: nothing turns (and the rest is not used).  freqs, axis_pairs: HOST, read during the call.  Angles are formed in 64 bits.
 */
#define PDA_ROPE_INTERLEAVED 0
#define PDA_ROPE_HALF 1
#define PDA_ROPE_MAX_AXES 4
typedef struct {
    int rot, layout, axes;
    int axis_pairs[PDA_ROPE_MAX_AXES];
    const double* freqs;
    const int32_t* positions;
    int64_t pos_batch, first;
} pda_rope;

/*
 * pda_pack_heads with rotary positions: token-major x (fp32 or bf16), token s of batch b at x + b * x_batch + s * x_token, its heads
 * compact [H, d] (a third of a fused projection: x_token = 3 H d) -> head-major y bf16, head h of batch b at y + b * y_batch + h * y_head, its tokens compact
 * (a part of a longer sequence, a cache's next places): unit_rms and premul as there, then the rotation, then one rounding.
 * Strides in ELEMENTS, none negative, those of x multiples of 4 (fp32) or 8 (bf16), those of y of 8; heads and batches of y must not overlap.  x and y
 * 16-byte aligned, apart from each other; H < 2^24.
 */
int pda_pack_heads_rope(const void* x, int x_type, int64_t x_batch, int64_t x_token, void* y, int64_t y_batch, int64_t y_head,
                        int B, int64_t S, int H, int d, const pda_rope* rope, int unit_rms, float premul, void* stream);

/*
 * Its gradient: dy bf16 (strides as y) -> dx of x_type (strides as x, rounded once): turned back, then pda_pack_heads_bwd's formula.
 * x is the pack's input and is read with unit_rms only (NULL without); tokens of dx must not overlap; dx may be x itself with equal strides.
 */
int pda_pack_heads_rope_bwd(const void* dy, int64_t dy_batch, int64_t dy_head, const void* x, int x_type, int64_t x_batch, int64_t x_token,
                            void* dx, int64_t dx_batch, int64_t dx_token, int B, int64_t S, int H, int d,
                            const pda_rope* rope, int unit_rms, float premul, void* stream);

/*
 * Frequencies of n pairs (host only; freqs, magnitude: HOST): base^(-i/n), scaled for a context `factor` (>= 1) times the original
 * one of `original` positions:
 *     PDA_ROPE_PLAIN    not at all
 *     PDA_ROPE_LINEAR   divided by factor (positions interpolated)
 *     PDA_ROPE_BASE     base * factor^(n/(n-1)) as the base: the fastest pair keeps its frequency, the slowest is divided by factor
 *     PDA_ROPE_BLEND    pairs of at most slow_turns turns in the original context are divided by factor, those of fast_turns and more kept, those
 *                       between take a share of both in proportion to their turns; magnitude = 0.1 ln(factor) + 1 (Peng et al. 2023, arXiv 2309.00071)
 * magnitude (may be NULL) is what queries and keys are to be multiplied by, as part of premul; 1 for the others.
 */
#define PDA_ROPE_PLAIN 0
#define PDA_ROPE_LINEAR 1
#define PDA_ROPE_BASE 2
#define PDA_ROPE_BLEND 3
int pda_rope_frequencies(int n, double base, int scaling, double factor, double original, double slow_turns, double fast_turns,
                         double* freqs, double* magnitude);

#ifdef __cplusplus
}
#endif
#endif /* PIPEDIT_PROJ_H */

/*
 * libpipedit_attn, training side: gradients of the attention call and of the pack in front of it, and layer
 * norm forward and backward.  Same library, conventions and error reporting as pipedit_attn.h (device pointers,
 * caller-owned tensors, pda_status, pda_last_error(), kernels enqueued on the given stream, arguments validated
 * before any device work, deterministic results: no atomics in any reduction), with one difference: a call that
 * needs device memory of its own takes it from the caller as `workspace`, of at least the size that the
 * matching *_workspace function gives.  Nothing here allocates, frees or synchronises, so every call may be
 * captured into a HIP graph from the start.  A workspace holds nothing between calls; calls whose execution may
 * overlap (different streams, graphs replayed side by side) need workspaces of their own.
 */
#ifndef PIPEDIT_TRAIN_H
#define PIPEDIT_TRAIN_H

#include "pipedit_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of arguments that come in two. */
#define PDA_F32 0
#define PDA_BF16 1

/*
 * Gradient of pda_attn_fwd / pda_attn_fwd_bf16out: dq, dk, dv from dout.  The probabilities are computed again
 * from the log-sum-exp that the forward call has written; no score matrix is stored.  For every (b, h), with keys
 * j < kv_valid_len:
 *
 *     p_ij    = exp(scale * <q_i, k_j> - lse_i)                 0 in a row with lse_i = -inf (a row without keys;
 *                                                     its out is not used, its q and dout must be finite)
 *     delta_i = <dout_i, out_i>
 *     ds_ij   = p_ij * (<dout_i, v_j> - delta_i)
 *     dq_i = scale * sum_j ds_ij k_j,    dk_j = scale * sum_i ds_ij q_i,    dv_j = sum_i p_ij dout_i
 *
 * dk and dv of keys j >= kv_valid_len are written as 0, and their k and v rows are never read.  Sq == 0 writes
 * dk = dv = 0, kv_valid_len == 0 writes zeros everywhere.
 *
 *     q, dout, dq [B, H, Sq, d]  bf16     k, v, dk, dv [B, H, Skv, d]  bf16     lse [B, H, Sq]  fp32 (natural log)
 *     out [B, H, Sq, d]  out_type: PDA_F32 (what pda_attn_fwd writes) or PDA_BF16 (pda_attn_fwd_bf16out)
 *
 * The gradient of pda_attn_fwd_base2 is this call with scale = ln 2 (0.69314718f; the scores are then used as
 * they are).  Shares of the keys (key chunks whose partial results went through pda_attn_merge): each share's call
 * with the MERGED out and lse gives its exact dk and dv, and the sum of the shares' dq is dq.  Shares of the
 * queries: dq per share, and dk and dv are the sums.  Each share's gradients are rounded to bf16, so a sum over shares, which the
 * caller makes (in fp32), holds a rounding of every share where one call holds one.
 *
 * Arithmetic: products of bf16 accumulated in fp32 on the matrix cores; probabilities, delta and ds in fp32, p and
 * ds rounded to bf16 only as operands of the products that sum them; gradients rounded once to bf16.
 * d must be 64 or 128, scale finite and >= 0; every tensor 16-byte aligned (lse 4).  dq, dk, dv and the workspace must not
 * overlap each other or any input (inputs may share memory).  workspace: 256-byte aligned, workspace_bytes >= what pda_attn_bwd_workspace gives for the
 * same sizes and kv_valid_len, or for larger ones with PDA_ANY_LEN, on this device (with B*H == 0 or Sq == Skv == 0 nothing is done and nothing needed).
 */
int pda_attn_bwd(const void* dout, const void* q, const void* k, const void* v, const void* out, int out_type,
                 const float* lse, void* dq, void* dk, void* dv,
                 int B, int H, int64_t Sq, int64_t Skv, int d, float scale, int64_t kv_valid_len,
                 void* workspace, int64_t workspace_bytes, void* stream);

/*
 * pda_attn_bwd on views, as pda_attn_fwd_strided: batch and head strides in ELEMENTS, rows compact (d elements
 * apart): head groups of larger tensors, query ranges, key chunks.  k and v share their strides, dk and dv theirs.
 * Strides of bf16 tensors must be multiples of 8, of an fp32 out multiples of 4, none negative; heads and
 * batches of dq, dk and dv, which are written, must not overlap (either axis may be the outer one).
 */
typedef struct {
    int64_t dout_batch, dout_head, q_batch, q_head, kv_batch, kv_head, out_batch, out_head, lse_batch, lse_head;
    int64_t dq_batch, dq_head, dkv_batch, dkv_head;
} pda_attn_bwd_strides;
int pda_attn_bwd_strided(const void* dout, const void* q, const void* k, const void* v, const void* out, int out_type,
                         const float* lse, void* dq, void* dk, void* dv,
                         int B, int H, int64_t Sq, int64_t Skv, int d, const pda_attn_bwd_strides* strides, float scale,
                         int64_t kv_valid_len, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Bytes of workspace of a pda_attn_bwd or pda_attn_bwd_strided call (host only; bytes is a HOST pointer): 256 bytes for a
 * counter; for every query row, rounded up to 64 a head, 8 bytes of statistics (d = 128) or 16 (d = 64); and where the launch does not
 * fill the device evenly the partial gradients of its shares.
 * n_cu: compute units of the device (0 = ask the current device).
 *
 * The need does not grow with the lengths: a shorter launch may be cut where a longer one is not.  kv_valid_len = PDA_ANY_LEN gives
 * a size, of at most n_cu * d * 4 KB beside the statistics, that serves every call of the same d and of at most this B * H, Sq and
 * Skv, with any kv_valid_len: for programs that keep one workspace for sequences or batches of several lengths.
 */
#define PDA_ANY_LEN (-1)
int pda_attn_bwd_workspace(int B, int H, int64_t Sq, int64_t Skv, int d, int64_t kv_valid_len, int n_cu, int64_t* bytes);

/*
 * Layer norm over the last axis of x [rows, D], the step in front of the projections:
 *
 *     mean_r = sum_c x[r,c] / D,   rstd_r = 1 / sqrt(sum_c (x[r,c] - mean_r)^2 / D + eps)
 *     y[r,c] = (x[r,c] - mean_r) * rstd_r * weight[g,c] + bias[g,c]
 *
 * weight and bias are [groups, D] fp32, group g holding the rows / groups consecutive rows from g * rows / groups on:
 * groups = 1 is the usual layer norm, groups = B with rows = B * S the modulation of a diffusion transformer (a scale
 * and a shift per sample).  Either may be NULL (1 and 0).  rows must be a multiple of groups.
 * x_type, y_type: PDA_F32 or PDA_BF16, any of the four pairs; y is rounded once.  mean and rstd [rows] fp32, for the backward
 * call; both may be NULL, not one alone.  y may be x itself if their types agree (the statistics then
 * describe what was overwritten); otherwise nothing that is written may overlap anything else.  Sums are fp32, the variance from the centred values.
 * 1 <= D <= PDA_LAYER_NORM_MAX; eps finite and >= 0; x, y, weight and bias 16-byte aligned; rows == 0 is a no-op.
 */
#define PDA_LAYER_NORM_MAX 8192
int pda_layer_norm_fwd(const void* x, int x_type, const float* weight, const float* bias, void* y, int y_type,
                       float* mean, float* rstd, int64_t rows, int64_t groups, int D, float eps, void* stream);

/*
 * Gradient of pda_layer_norm_fwd, with xh = (x - mean) * rstd and g = dy * weight:
 *
 *     dx[r,c]      = rstd_r * (g[r,c] - sum_c g[r,:] / D - xh[r,c] * sum_c (g * xh)[r,:] / D)
 *     dweight[g,c] = sum over the rows r of group g of dy[r,c] * xh[r,c],    dbias[g,c] = sum of dy[r,c]
 *
 * dy has the type y_type, dx the type x_type (rounded once); mean and rstd are the forward call's.  dweight and dbias
 * [groups, D] fp32 are written, not added to; either may be NULL.  dx may be NULL (only the sums are wanted) and may be
 * x or dy itself if the types agree; otherwise nothing that is written may overlap anything else.  rows == 0 writes dweight = dbias = 0.  The sums over the rows are made in a fixed order: equal calls give equal bits.
 * workspace: 16-byte aligned, at least what pda_layer_norm_bwd_workspace gives (NULL if that is 0, or if neither
 * dweight nor dbias is wanted).
 */
int pda_layer_norm_bwd(const void* dy, int y_type, const void* x, int x_type, const float* weight, const float* mean,
                       const float* rstd, void* dx, float* dweight, float* dbias, int64_t rows, int64_t groups, int D,
                       void* workspace, int64_t workspace_bytes, void* stream);
int pda_layer_norm_bwd_workspace(int64_t rows, int64_t groups, int D, int n_cu, int64_t* bytes);

/*
 * Gradient of pda_pack_heads: head-major bf16 dy [B,H,S,d] (what pda_attn_bwd writes) -> token-major fp32 dx
 * [B,S,H,d].  Without unit_rms dx = premul * dy.  With unit_rms, r = 1 / sqrt(mean(x^2)) of the d-vector and xh = x r,
 *
 *     dx = premul * r * (dy - xh * mean(dy * xh)),        0 for a zero vector
 *
 * mean(x^2) is taken in fp32: a vector of elements so small that their squares are 0 (below some 1e-23) counts as
 * a zero vector, as in the pack (the squares lose bits below some 1e-19), one whose squares pass fp32's range (some 1e19) has the gradient 0.  A NaN in the vector or its dy makes all of its dx NaN.
 *
 * x is the pack's input and is read with unit_rms only (NULL without).  dx may be x itself.  The rounding of the pack
 * counts as the identity.  d, alignment and sizes as pda_pack_heads, H < 2^24.
 */
int pda_pack_heads_bwd(const void* dy, const float* x, float* dx, int B, int64_t S, int H, int d, int unit_rms,
                       float premul, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PIPEDIT_TRAIN_H */

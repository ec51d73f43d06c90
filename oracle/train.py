"""fp64 oracle of the training operators: the gradients of attention and of the pack, and layer norm forward and backward.
TEST INFRASTRUCTURE ONLY (see the package docstring).

Every function also returns how far the library's results may be off, element by element, from its number formats alone:

  * a rounding to bf16 is off by at most U16 = 2^-8 of the value, one to fp32 by U32 = 2^-24;
  * attention: p and ds are rounded to bf16 as operands of the products that sum them, so those sums are off by at most
    U16 sum |terms|; p itself is exp2 of an fp32 argument, off relatively by ln 2 times the argument's absolute error
    (fp32 sums of d products in the scores, one multiply-add, the rounding of lse * log2 e) plus 2^-22 for the exponential;
    <dout, v> - delta are fp32 sums of d products each; a sum of n fp32 terms is off by at most n U32 sum |terms|;
  * layer norm and the pack: sums of D terms in fp32 over chains of at most DEPTH additions, a few more operations an element.
"""
from __future__ import annotations

import numpy as np

U16, U32 = 2.0 ** -8, 2.0 ** -24
LOG2E = 1.4426950408889634
DEPTH = 64          # additions one after the other, and the operations around them, in a sum over a row


def attention_bwd(dout, q, k, v, out, lse, scale, n_v):
    """All [B,H,S,*] fp64 values of the bf16/fp32 inputs -> ((dq, dk, dv), their bounds)."""
    B, H, Sq, d = q.shape
    Skv = k.shape[2]
    res = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    tol = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    if Sq == 0 or n_v == 0:
        return res, tol
    for b in range(B):
        for h in range(H):
            Q, DO, O, L = (x[b, h] for x in (q, dout, out, lse))
            K, V = k[b, h, :n_v], v[b, h, :n_v]
            live = L > -np.inf
            Ls = np.where(live, L, 0.0)[:, None]
            s = Q @ K.T
            p = np.where(live[:, None], np.exp(scale * s - Ls), 0.0)
            dp = DO @ V.T - (DO * O).sum(-1, keepdims=True)
            ds = p * dp
            res[0][b, h] = scale * ds @ K
            res[1][b, h, :n_v] = scale * ds.T @ Q
            res[2][b, h, :n_v] = p.T @ DO
            aq, ak, ado, av = np.abs(Q), np.abs(K), np.abs(DO), np.abs(V)
            arg = U32 * LOG2E * ((d + 2) * scale * (aq @ ak.T) + 3 * np.abs(Ls) + 2 * scale * np.abs(s))
            rel_p = np.log(2) * arg + 2.0 ** -22
            err_dp = (d + 2) * U32 * (ado @ av.T + (ado * np.abs(O)).sum(-1, keepdims=True))
            e_p = p * rel_p
            e_ds = np.abs(ds) * (rel_p + 2 * U32) + p * err_dp
            op_ds = e_ds + U16 * (np.abs(ds) + e_ds)              # what a ds is off as an operand
            op_p = e_p + U16 * (p + e_p)
            sums = [scale * op_ds @ ak, scale * op_ds.T @ aq, op_p.T @ ado]
            big = [scale * np.abs(ds) @ ak, scale * np.abs(ds).T @ aq, p.T @ ado]
            n = [n_v, Sq, Sq]
            for i, at in enumerate((slice(None), slice(0, n_v), slice(0, n_v))):
                e = sums[i] + (n[i] + 2) * U32 * (big[i] + sums[i])
                tol[i][b, h, at] = e + U16 * (np.abs(res[i][b, h, at]) + e) + 1e-38
    return res, tol


def layer_norm(x, weight, bias, groups, eps, y_bf16):
    """x [rows, D], weight and bias [groups, D] or None -> (y, mean, rstd), their bounds."""
    rows, D = x.shape
    per = rows // groups
    w = np.ones((groups, D)) if weight is None else weight
    b = np.zeros((groups, D)) if bias is None else bias
    w, b = np.repeat(w, per, axis=0), np.repeat(b, per, axis=0)
    mean = x.mean(-1, keepdims=True)
    var = ((x - mean) ** 2).mean(-1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    e_mean = DEPTH * U32 * np.abs(x).mean(-1, keepdims=True)
    e_c = e_mean + U32 * np.abs(x - mean)                      # a centred value
    e_var = DEPTH * U32 * var + 2 * np.sqrt(var) * e_c.max(-1, keepdims=True) + e_c.max(-1, keepdims=True) ** 2
    e_rstd = rstd * (0.5 * e_var / (var + eps) + 8 * U32)
    xh = (x - mean) * rstd
    y = xh * w + b
    e = np.abs(w) * (e_c * rstd + np.abs(x - mean) * e_rstd + 4 * U32 * np.abs(xh)) + U32 * np.abs(y)
    return (y, mean[:, 0], rstd[:, 0]), (e + (U16 if y_bf16 else U32) * (np.abs(y) + e), e_mean[:, 0] + U32 * np.abs(mean[:, 0]), e_rstd[:, 0])


def layer_norm_bwd(dy, x, weight, mean, rstd, groups, dx_bf16):
    """-> (dx, dweight, dbias), their bounds; mean and rstd are taken as given."""
    rows, D = x.shape
    per = rows // groups if groups else 0
    w = np.repeat(np.ones((groups, D)) if weight is None else weight, per, axis=0)
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * w
    c1, c2 = (g * xh).mean(-1, keepdims=True), g.mean(-1, keepdims=True)
    dx = rstd[:, None] * (g - c2 - xh * c1)
    m1, m2 = np.abs(g * xh).mean(-1, keepdims=True), np.abs(g).mean(-1, keepdims=True)
    e_xh = 2 * U32 * (np.abs(xh) + (np.abs(x) + np.abs(mean[:, None])) * rstd[:, None])
    e1 = DEPTH * U32 * m1 + (np.abs(g) * e_xh).mean(-1, keepdims=True)
    e = rstd[:, None] * (4 * U32 * np.abs(g) + DEPTH * U32 * m2 + np.abs(xh) * e1 + e_xh * np.abs(c1) + 4 * U32 * (np.abs(c2) + np.abs(xh * c1)))
    fold = lambda t: t.reshape(groups, per, D).sum(1)  # noqa: E731
    n = per + DEPTH
    return ((dx, fold(dy * xh), fold(dy)),
            (e + (U16 if dx_bf16 else U32) * (np.abs(dx) + e), n * U32 * fold(np.abs(dy * xh)) + fold(np.abs(dy) * e_xh), n * U32 * fold(np.abs(dy))))


def pack_heads_bwd(dy, x, unit_rms, premul):
    """dy [B,H,S,d], x [B,S,H,d] -> dx [B,S,H,d], its bound."""
    g = dy.transpose(0, 2, 1, 3)
    if not unit_rms:
        dx = premul * g
        return dx, U32 * np.abs(dx)
    ms = (x * x).mean(-1, keepdims=True)
    r = np.divide(1.0, np.sqrt(ms), out=np.zeros_like(ms), where=ms > 0)
    xh = x * r
    dx = premul * r * (g - xh * (g * xh).mean(-1, keepdims=True))
    tol = DEPTH * U32 * np.abs(premul) * r * (np.abs(g) + np.abs(xh) * np.abs(g * xh).mean(-1, keepdims=True))
    return dx, tol

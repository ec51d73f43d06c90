"""fp64 oracle of the projection side: 8-bit matrices with power-of-two scales and their product, root-mean-square norm forward and backward,
and the pack with rotary positions and its gradient.  TEST INFRASTRUCTURE ONLY (see the package docstring).

Quantisation is exact.  The other functions also return how far the library's results may be off, element by element, from its number formats alone:

  * a rounding to bf16 is off by at most U16 = 2^-8 of the value, one to fp32 by U32 = 2^-24;
  * the product: the matrix instruction aligns the products of eight consecutive k to the largest of them and drops what lies 2^-13 below it (seven of them can
    lose something); the sums of eight and the accumulator are added in fp32, and the result is rounded to bf16 once;
  * the norm and the pack: sums of D terms in fp32 over chains of at most DEPTH additions, a few more operations an element.
"""
from __future__ import annotations

import numpy as np

U16, U32 = 2.0 ** -8, 2.0 ** -24
DEPTH = 64          # additions one after the other, and the operations around them, in a sum over a row
FP8 = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}        # largest value, bits behind the point, exponent of the smallest normal number


def up(n, m):
    return (n + m - 1) // m * m


def round_fp8(v, kind):
    """Finite values to the type, ties to even."""
    _, m, least = FP8[kind]
    step = np.ldexp(1.0, np.maximum(np.frexp(v)[1] - 1, least) - m)
    return np.round(v / step) * step


def quantise(x, kind, block_rows):
    """x [rows, cols] -> values [rows, cols padded to 128] before the scale, scale bytes [blocks of rows, blocks of columns]."""
    top_value = FP8[kind][0]
    rows, cols = x.shape
    r, c = up(rows, block_rows), up(cols, 128)
    full = np.zeros((r, c))
    full[:rows, :cols] = x
    finite = np.isfinite(full)
    mag = np.where(finite, np.abs(np.where(finite, full, 0.0)), 0.0).reshape(r // block_rows, block_rows, c // 128, 128).max(axis=(1, 3))
    f, p = np.frexp(mag / top_value)                    # f 2^p, 1/2 <= f < 1: a power of two itself is enough for 1/2
    e = np.where(mag > 0, np.maximum(np.where(f == 0.5, p - 1, p), -127), 0)
    scale = np.ldexp(1.0, e)
    q = full / np.repeat(np.repeat(scale, block_rows, axis=0), 128, axis=1)
    q = np.where(finite, round_fp8(np.where(finite, q, 0.0), kind), q if kind == "e5m2" else np.nan)
    return q[:rows], (e + 127).astype(np.uint8)


def values(q, scale_bytes, block_rows):
    """What an 8-bit matrix stands for."""
    s = np.where(scale_bytes == 255, np.nan, np.ldexp(1.0, scale_bytes.astype(int) - 127))
    return q * np.repeat(np.repeat(s, block_rows, axis=0), 128, axis=1)[:q.shape[0]]


def matmul(a, b, bias):
    """a [M, K], b [N, K] values, both with rows padded to 128 -> a b^T + bias, its bound."""
    out = a @ b.T
    size = np.abs(a) @ np.abs(b).T
    lost = np.zeros(out.shape)
    for k in range(0, a.shape[1], 8):
        lost += (np.abs(a[:, None, k:k + 8]) * np.abs(b[None, :, k:k + 8])).max(axis=-1)
    if bias is not None:
        out = out + bias
        size = size + np.abs(bias)
    e = 7 * 2.0 ** -13 * lost + (a.shape[1] // 8 + 64) * U32 * size
    return out, e + U16 * (np.abs(out) + e) + 1e-38


def rms_norm(x, res, weight, groups, eps, round_h, y_bf16):
    """round_h: the rounding of the stream to its type, as a function.  -> (h, y, rstd), bounds of (y, rstd)."""
    rows, D = x.shape
    h = x if res is None else round_h(x + res)
    w = np.repeat(np.ones((groups, D)) if weight is None else weight, rows // groups, axis=0)
    rstd = 1 / np.sqrt((h * h).mean(axis=-1) + eps)
    y = h * rstd[:, None] * w
    rel = (DEPTH + 8) * U32                             # the mean is off by DEPTH U32 at most, its root by half of that
    e = np.abs(y) * rel
    return (h, y, rstd), (e + ((U16 if y_bf16 else U32) * (np.abs(y) + e)) + 1e-38, rstd * rel)


def rms_norm_bwd(dy, h, weight, rstd, dres, groups, h_bf16):
    """-> (dh, dweight), their bounds."""
    rows, D = h.shape
    per = rows // groups
    w = np.repeat(np.ones((groups, D)) if weight is None else weight, per, axis=0)
    r = rstd[:, None]
    hh, g = h * r, dy * w
    dot = (g * hh).mean(axis=-1, keepdims=True)
    add = 0.0 if dres is None else dres
    dh = add + r * (g - hh * dot)
    e_dot = (DEPTH + 4) * U32 * np.abs(g * hh).mean(axis=-1, keepdims=True)
    e = r * (4 * U32 * np.abs(g) + np.abs(hh) * (e_dot + 6 * U32 * np.abs(dot))) + 2 * U32 * (np.abs(add) + np.abs(r * g) + np.abs(r * hh * dot))
    dw = (dy * hh).reshape(groups, per, D).sum(axis=1)
    chain = per + 64                                    # rows of a workgroup one after the other, then workgroups; no more than all of them
    e_w = (chain + 3) * U32 * np.abs(dy * hh).reshape(groups, per, D).sum(axis=1) + 1e-38
    return (dh, dw), (e + (U16 if h_bf16 else U32) * (np.abs(dh) + e) + 1e-38, e_w)


def angles(positions, freqs, axis_pairs):
    """positions [..., axes] -> radians [..., pairs], in extended precision where numpy has it."""
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    return np.asarray(positions, dtype=np.longdouble)[..., axis] * np.asarray(freqs, dtype=np.longdouble)


def turn(x, angle, layout, back=False):
    """x [..., d] with the pairs of its first columns turned by angle [..., pairs]."""
    n = angle.shape[-1]
    cos, sin = np.cos(angle).astype(np.float64), np.sin(angle).astype(np.float64) * (-1 if back else 1)
    out = x.copy()
    u, v = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    out[..., u] = x[..., u] * cos - x[..., v] * sin
    out[..., v] = x[..., u] * sin + x[..., v] * cos
    return out


def _pair_size(x, n, layout):
    """An upper bound of each column's size after any turn of its pair."""
    a = np.abs(x)
    out = a.copy()
    u, v = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    out[..., u] = out[..., v] = a[..., u] + a[..., v]
    return out


# a turn: the angle is off by 2 pi 2^-25 of a turn's half after its whole turns are gone, some 3 U32 of cos and sin, two products and a sum
TURN = 16 * U32


def pack_rope(x, angle, layout, unit_rms, premul):
    """x [B,S,H,d], angle [B,S,1,pairs] -> y [B,H,S,d], its bound."""
    r = 1.0
    if unit_rms:
        ms = (x * x).mean(axis=-1, keepdims=True)
        r = np.where(ms > 0, 1 / np.sqrt(np.where(ms > 0, ms, 1.0)), 0.0)
    x = x * r * premul
    y = turn(x, angle, layout)
    e = (TURN + (DEPTH * U32 if unit_rms else 2 * U32)) * _pair_size(x, angle.shape[-1], layout)
    return np.moveaxis(y, 2, 1), np.moveaxis(e + U16 * (np.abs(y) + e) + 1e-38, 2, 1)


def pack_rope_bwd(dy, x, angle, layout, unit_rms, premul, x_bf16):
    """dy [B,H,S,d] -> dx [B,S,H,d], its bound."""
    g = np.moveaxis(dy, 1, 2)
    out = turn(g, angle, layout, back=True)
    e = TURN * _pair_size(g, angle.shape[-1], layout)
    if unit_rms:
        ms = (x * x).mean(axis=-1, keepdims=True)
        live = ms > 0
        r = np.where(live, 1 / np.sqrt(np.where(live, ms, 1.0)), 0.0)
        xh = x * r
        dot = (out * xh).mean(axis=-1, keepdims=True)
        e_dot = (DEPTH * U32 * np.abs(out * xh) + e * np.abs(xh)).mean(axis=-1, keepdims=True)
        e = r * (e + np.abs(xh) * e_dot) + 8 * U32 * r * (np.abs(out) + np.abs(xh * dot)) + (DEPTH + 8) * U32 * r * np.abs(out - xh * dot)
        out = r * (out - xh * dot)
    out = out * premul
    e = e * abs(premul) + 2 * U32 * np.abs(out)
    return out, e + (U16 if x_bf16 else U32) * (np.abs(out) + e) + 1e-38

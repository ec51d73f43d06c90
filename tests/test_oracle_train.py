"""Pins of the fp64 oracle of the training operators: gradients against central differences of the forward definitions."""
import numpy as np
import pytest

from oracle import attention, widen_bf16
from oracle import train


def _differences(f, x, dy, h=1e-5):
    g = np.zeros_like(x)
    it = np.nditer(x, flags=["multi_index"])
    for _ in it:
        i = it.multi_index
        old = x[i]
        x[i] = old + h
        up = f()
        x[i] = old - h
        down = f()
        x[i] = old
        g[i] = ((up - down) * dy).sum() / (2 * h)
    return g


def _attn(q, k, v, scale, n_v):
    s = scale * np.einsum("bhid,bhjd->bhij", q, k[:, :, :n_v])
    top = s.max(-1, keepdims=True)
    e = np.exp(s - top)
    lse = (top + np.log(e.sum(-1, keepdims=True)))[..., 0]
    return np.einsum("bhij,bhjd->bhid", np.exp(s - lse[..., None]), v[:, :, :n_v]), lse


@pytest.mark.parametrize("Sq,Skv,n_v", [(1, 1, 1), (5, 7, 6), (6, 4, 4)])
def test_attention_gradient_against_differences(Sq, Skv, n_v):
    rng = np.random.default_rng(Sq)
    q, k, v = rng.standard_normal((1, 2, Sq, 8)), rng.standard_normal((1, 2, Skv, 8)), rng.standard_normal((1, 2, Skv, 8))
    dout = rng.standard_normal((1, 2, Sq, 8))
    out, lse = _attn(q, k, v, 0.4, n_v)
    (dq, dk, dv), tol = train.attention_bwd(dout, q, k, v, out, lse, 0.4, n_v)
    f = lambda: _attn(q, k, v, 0.4, n_v)[0]  # noqa: E731
    for got, x in ((dq, q), (dk, k), (dv, v)):
        assert np.abs(got - _differences(f, x, dout)).max() < 1e-8
    assert (dk[:, :, n_v:] == 0).all() and (dv[:, :, n_v:] == 0).all()
    assert all(np.isfinite(t).all() for t in tol)


def test_attention_gradient_of_empty_rows():
    z = np.zeros((1, 1, 3, 8))
    (dq, dk, dv), _ = train.attention_bwd(z + 1, z + 1, z + 1, z + 1, z, np.full((1, 1, 3), -np.inf), 1.0, 0)
    assert (dq == 0).all() and (dk == 0).all() and (dv == 0).all()
    (dq, dk, dv), _ = train.attention_bwd(z + 1, z + 1, z + 1, z + 1, z, np.full((1, 1, 3), -np.inf), 1.0, 3)
    assert (dq == 0).all() and (dk == 0).all() and (dv == 0).all()


def test_attention_oracle_agrees_with_the_forward_oracle():
    rng = np.random.default_rng(3)
    bits = [(rng.standard_normal((1, 1, 9, 64)).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16) for _ in range(3)]
    out, lse = attention(*bits, 0.125, 8)
    out2, lse2 = _attn(*(widen_bf16(b).astype(np.float64) for b in bits), 0.125, 8)
    assert np.allclose(out, out2, atol=1e-12) and np.allclose(lse, lse2, atol=1e-12)


@pytest.mark.parametrize("rows,groups,D", [(1, 1, 5), (6, 1, 7), (6, 3, 4)])
def test_layer_norm_gradient_against_differences(rows, groups, D):
    rng = np.random.default_rng(rows + D)
    x, dy = rng.standard_normal((rows, D)), rng.standard_normal((rows, D))
    w, b = rng.standard_normal((groups, D)), rng.standard_normal((groups, D))
    (y, mean, rstd), _ = train.layer_norm(x, w, b, groups, 1e-3, False)
    f = lambda: train.layer_norm(x, w, b, groups, 1e-3, False)[0][0]  # noqa: E731
    (dx, dw, db), _ = train.layer_norm_bwd(dy, x, w, mean, rstd, groups, False)
    for got, t in ((dx, x), (dw, w), (db, b)):
        assert np.abs(got - _differences(f, t, dy)).max() < 1e-8
    xh = (x - x.mean(-1, keepdims=True)) / np.sqrt(x.var(-1, keepdims=True) + 1e-3)
    assert np.allclose(y, xh * np.repeat(w, rows // groups, 0) + np.repeat(b, rows // groups, 0))


@pytest.mark.parametrize("unit_rms", [False, True])
def test_pack_gradient_against_differences(unit_rms):
    rng = np.random.default_rng(8)
    x, dy = rng.standard_normal((1, 2, 3, 4)), rng.standard_normal((1, 3, 2, 4))

    def pack():
        r = 1 / np.sqrt((x * x).mean(-1, keepdims=True)) if unit_rms else 1.0
        return (0.7 * x * r).transpose(0, 2, 1, 3)

    dx, tol = train.pack_heads_bwd(dy, x, unit_rms, 0.7)
    assert np.abs(dx - _differences(pack, x, dy)).max() < 1e-8 and np.isfinite(tol).all()
    x[0, 0, 0] = 0
    assert unit_rms is False or (train.pack_heads_bwd(dy, x, True, 0.7)[0][0, 0, 0] == 0).all()

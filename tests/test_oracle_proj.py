"""The fp64 oracle of the projection side against independent statements: torch's 8-bit types on the CPU, differences, rotations as complex numbers."""
import numpy as np
import pytest

from oracle import proj


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_rounding_is_the_types(kind):
    import torch
    dt = torch.float8_e4m3fn if kind == "e4m3" else torch.float8_e5m2
    every = torch.arange(256, dtype=torch.uint8).view(dt).double().numpy()
    every = np.unique(every[np.isfinite(every)])
    between = (every[1:] + every[:-1]) / 2                       # ties
    for v in (every, between, np.nextafter(between, -np.inf), np.nextafter(between, np.inf), every * 0.99, every * 0.97):
        v = v[np.abs(v) <= proj.FP8[kind][0]].astype(np.float32).astype(np.float64)
        assert np.array_equal(proj.round_fp8(v, kind), torch.from_numpy(v).float().to(dt).double().numpy())


@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
@pytest.mark.parametrize("block", [1, 128])
def test_scales_are_the_smallest_that_hold(kind, block):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((140, 300)) * np.exp(3 * rng.standard_normal((140, 1)))
    x[7] = 0
    x[9, 128:256] = proj.FP8[kind][0] * 2.0 ** 5                  # the border itself
    q, s = proj.quantise(x, kind, block)
    assert q.shape == (140, 384) and s.shape == (proj.up(140, block) // block, 3) and not q[:, 300:].any()
    assert np.abs(q).max() <= proj.FP8[kind][0]
    scale = np.repeat(np.repeat(np.ldexp(1.0, s.astype(int) - 127), block, axis=0), 128, axis=1)[:140]
    full = np.zeros((140, 384))
    full[:, :300] = x
    half = scale * np.maximum(np.ldexp(1.0, np.frexp(q)[1] - 1), 2.0 ** proj.FP8[kind][2]) * 2.0 ** -proj.FP8[kind][1] / 2
    assert (np.abs(proj.values(q, s, block) - full) <= half).all()
    if block == 1:
        assert s[7].tolist() == [127] * 3 and s[9, 1] == 127 + 5
        live = np.ones(s.shape, bool)
        live[7] = False
        top = np.abs(full).reshape(140, 3, 128).max(axis=-1)
        assert (top[live] > proj.FP8[kind][0] * np.ldexp(1.0, s[live].astype(int) - 128)).all()


def test_quantise_what_is_not_finite():
    x = np.array([[1.0, np.inf, -np.inf, np.nan] + [0.0] * 124])
    q, s = proj.quantise(x, "e4m3", 1)
    assert s[0, 0] == 127 - 8 and q[0, 0] == 256 and np.isnan(q[0, 1:4]).all()
    q, _ = proj.quantise(x, "e5m2", 1)
    assert q[0, 1] == np.inf and q[0, 2] == -np.inf and np.isnan(q[0, 3])


def test_rms_norm_gradient_by_differences():
    rng = np.random.default_rng(1)
    x, res, dy, w = (rng.standard_normal((6, 37)) for _ in range(4))
    w, eps, same = rng.standard_normal((2, 37)), 1e-3, lambda v: v
    f = lambda r, ww: float((proj.rms_norm(x, r, ww, 2, eps, same, False)[0][1] * dy).sum())  # noqa: E731
    (h, _, rstd), _ = proj.rms_norm(x, res, w, 2, eps, same, False)
    (dh, dw), _ = proj.rms_norm_bwd(dy, h, w, rstd, None, 2, False)
    d = 1e-6
    for i, j in ((0, 0), (3, 17), (5, 36)):
        e = np.zeros((6, 37))
        e[i, j] = d
        assert abs((f(res + e, w) - f(res - e, w)) / (2 * d) - dh[i, j]) < 1e-7
    for g, j in ((0, 4), (1, 30)):
        e = np.zeros((2, 37))
        e[g, j] = d
        assert abs((f(res, w + e) - f(res, w - e)) / (2 * d) - dw[g, j]) < 1e-7
    assert np.allclose(proj.rms_norm_bwd(dy, h, w, rstd, x, 2, False)[0][0], dh + x)


@pytest.mark.parametrize("layout", ["interleaved", "half"])
@pytest.mark.parametrize("rms", [False, True])
def test_rope_is_a_rotation_and_its_gradient_by_differences(layout, rms):
    rng = np.random.default_rng(2)
    B, S, H, d, n = 2, 5, 3, 64, 20
    x, dy = rng.standard_normal((B, S, H, d)), rng.standard_normal((B, H, S, d))
    angle = proj.angles(rng.integers(0, 1000, (B, S, 1, 2)), rng.uniform(0, 1, n), [8, 12])
    y, _ = proj.pack_rope(x, angle, layout, rms, 0.7)
    u = x / np.sqrt((x * x).mean(-1, keepdims=True)) if rms else x
    z = u[..., :n] + 1j * u[..., n:2 * n] if layout == "half" else u[..., 0:2 * n:2] + 1j * u[..., 1:2 * n:2]
    z = z * np.exp(1j * angle.astype(np.float64)) * 0.7
    want = np.moveaxis(y, 1, 2)
    got = want[..., :n] + 1j * want[..., n:2 * n] if layout == "half" else want[..., 0:2 * n:2] + 1j * want[..., 1:2 * n:2]
    assert np.allclose(got, z) and np.allclose(want[..., 2 * n:], u[..., 2 * n:] * 0.7)
    dx, _ = proj.pack_rope_bwd(dy, x, angle, layout, rms, 0.7, False)
    f = lambda v: float((proj.pack_rope(v, angle, layout, rms, 0.7)[0] * dy).sum())  # noqa: E731
    for at in ((0, 0, 0, 0), (1, 4, 2, 39), (1, 2, 1, 63), (0, 3, 0, 21)):
        e = np.zeros_like(x)
        e[at] = 1e-6
        assert abs((f(x + e) - f(x - e)) / 2e-6 - dx[at]) < 1e-6


def test_matmul_bound_covers_dropped_products():
    """The bound's share of the matrix instruction: with one large product, seven that lie just under 2^-13 of it may be gone."""
    a = np.zeros((1, 128))
    a[0, :8] = [256] + [1.9375 * 2 ** -2] * 7
    b = np.zeros((1, 128))
    b[0, :8] = [256] + [15.5] * 7
    out, tol = proj.matmul(a, b, None)
    assert tol[0, 0] >= 7 * 1.9375 * 2 ** -2 * 15.5 and tol[0, 0] <= out[0, 0] * (2 ** -8 + 2 ** -9)

"""Unit RMS in the pack where it can go wrong, against the fp64 oracle: vectors that are not finite, and vectors whose squares leave fp32's range."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _pack(x, premul=0.5):
    import torch
    import paper_2511_12056_amd as pda
    B, S, H, d = x.shape
    return pda.pack_heads(x, torch.full((B, H, S, d), 7.0, device="cuda", dtype=torch.bfloat16), True, premul)


@pytest.mark.parametrize("d", [64, 128])
def test_a_nan_is_in_all_of_its_vector(d):
    """<x, x> has it, and every element is divided by its root; the other vectors of its wavefront keep their bits, and one of zeros stays zero."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(2, 37, 3, d, generator=g, device="cuda")
    x[0, 0, 0] = 0.0
    want = _pack(x)
    at = [(0, 3, 1, 0), (1, 36, 2, d - 1), (1, 0, 0, d // 2 + 1)]
    for i in at:
        x[i] = float("nan")
    got = _pack(x)
    hit = torch.zeros(2, 3, 37, dtype=torch.bool, device="cuda")
    for b, s, h, _ in at:
        hit[b, h, s] = True
    assert got[hit].isnan().all() and torch.equal(got[~hit], want[~hit]) and (got[0, 0, 0] == 0).all()


@pytest.mark.parametrize("d", [64, 128])
def test_an_infinite_element(d):
    """x / rms(x) of a vector with an infinity: NaN in its place, 0 elsewhere."""
    import torch
    x = torch.ones(1, 4, 2, d, device="cuda")
    x[0, 2, 1, 9] = float("-inf")
    got = _pack(x)
    assert got[0, 1, 2, 9].isnan() and not got[0, 1, 2, :9].any() and not got[0, 1, 2, 10:].any()
    assert (got[0, 0] == 0.5).all() and (got[0, 1, :2] == 0.5).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", [1e-15, 1e-18, 1e-19, 3e-20, 1e-20, 1e-21, 1e-22, 3e-22, 1e18, 2e18, 1e19, 1e20, 1e30, 3e37])
def test_vectors_whose_squares_leave_the_range(size, d):
    """Small and large vectors, whole and with few columns, beside ordinary ones in a wavefront: the definition, within the bound of any other vector.  (One element
    of 2^-75, 2.6e-23, or less has a square of 0.)"""
    import torch
    from oracle import proj
    g = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn(2, 21, 3, d, generator=g, device="cuda")
    x[:, ::2] *= size
    x[:, 4, :, 1:] = 0.0
    x[:, 4, :, 0] = size
    x[:, 6, :, : d // 2] = 0.0
    x[:, 8, :, d - 1] = 3 * size
    x[:, 10, :, 1::2] *= 1e-3                                      # columns whose own squares vanish beside the others'
    x[:, 12] = x[:, 12].abs().clamp(min=size)
    x[:, 14] = size
    x[0, 16, 1] = 0.0
    y = _pack(x)
    want, tol = proj.pack_rope(x.double().cpu().numpy(), np.zeros((1, 1, 1, 0)), "half", True, 0.5)
    got = y.double().cpu().numpy()
    assert np.isfinite(got).all()
    over = np.abs(got - want) - tol
    assert over.max() <= 0, (float(over.max()), np.unravel_index(over.argmax(), over.shape))
    assert (y[0, 1, 16] == 0).all()


def test_squares_that_are_all_zero():
    """Elements below 2^-75: the vector counts as one of zeros, as in the gradient."""
    import torch
    x = torch.randn(1, 9, 2, 64, device="cuda")
    want = _pack(x)
    x[0, ::2] = torch.where(x[0, ::2] > 0, 1e-23, -1e-38)
    got = _pack(x)
    assert not got[0, :, ::2].any() and torch.equal(got[0, :, 1::2], want[0, :, 1::2])

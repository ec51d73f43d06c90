"""Unit RMS in the pack where it can go wrong: vectors that are not finite."""
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

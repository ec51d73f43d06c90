"""Root-mean-square norm of rows whose squares lie below fp32's range, against the fp64 oracle with the bounds of any other row.  (Those above it give zeros.)"""
import numpy as np
import pytest

from tests.test_gpu_rms_norm import _check, _check_fp8, _dt, _f64

pytestmark = pytest.mark.gpu


def _forward(x, w, yt, eps, res=None):
    import torch
    import paper_2511_12056_amd as pda
    rows, D = x.shape
    y, s = pda.fp8_empty(rows, D) if yt == "e4m3" else (torch.full(x.shape, 7.0, device="cuda", dtype=_dt(yt)), None)
    h = None if res is None else torch.empty_like(res)
    return pda.rms_norm_fwd(x, w, y, res=res, h=h, y_scales=s, rstd=torch.empty(rows, device="cuda"), eps=eps)


@pytest.mark.parametrize("D", [1, 3, 30, 64, 100, 128, 256, 300, 384, 512, 1001, 1024, 1536, 1537, 2048, 3001, 4096, 8192])
@pytest.mark.parametrize("yt", ["fp32", "bf16", "e4m3"])
@pytest.mark.parametrize("xt,rt", [("fp32", "none"), ("bf16", "none"), ("bf16", "bf16")])
@pytest.mark.parametrize("size,eps", [(1e-15, 0.0), (1e-18, 0.0), (1e-20, 0.0), (1e-22, 0.0), (1e-30, 0.0), (1e-36, 0.0), (1e-20, 1e-40), (1e-20, 1e-38), (1e-17, 1e-34), (1e-14, 1e-28), (1e-20, 1e-6),
                                      (1e17, 1e-6)])
def test_rows_whose_squares_nearly_vanish(size, eps, xt, rt, yt, D):
    """Whole and with one element, beside ordinary rows, which may share a wavefront."""
    import torch
    from oracle import proj
    g = torch.Generator(device="cuda").manual_seed(D)
    rows = 21
    x = torch.randn(rows, D, generator=g, device="cuda")
    x = x.sign() * x.abs().clamp(min=1e-3)                          # (no row of zeros, for which eps = 0 has no result)
    x[::2] *= size
    x[4] = 0.0
    x[4, D // 2] = 2 * size
    x[6, : D // 2] = 0.0
    x[8, : D // 2] *= 1e-3
    res = None
    x = x.to(_dt(xt))
    if rt != "none":
        res, x = x, torch.zeros_like(x)
    w = 1 + 0.3 * torch.rand(1, D, generator=g, device="cuda")
    _, y, s, rstd = _forward(x, w, yt, eps, res)
    stored = _f64(x if res is None else res)
    (_, wy, wr), (ty, tr) = proj.rms_norm(stored, None, _f64(w), 1, float(np.float32(eps)), None, yt == "bf16")
    _check("rstd", rstd, wr, tr)
    if yt == "e4m3":
        _check_fp8(y, s, wy, np.where(wy == 0, 0.0, ty))            # zeros come out as they are, so the scale of a block of them is the definition's
    else:
        _check("y", y, wy, ty)


@pytest.mark.parametrize("D", [64, 1001, 1536, 8192])
def test_rows_of_zeros_and_of_what_is_not_finite(D):
    """Without an eps a row of zeros has none; an infinity is NaN in its place and makes the others 0, a NaN is in the whole row; other rows keep their bits."""
    import torch
    x = torch.randn(40, D, device="cuda")
    want = _forward(x, None, "fp32", 0.0)[1].clone()
    x[3] = 0.0
    x[10, 5] = float("inf")
    x[20, D - 1] = float("nan")
    _, y, _, rstd = _forward(x, None, "fp32", 0.0)
    assert y[3].isnan().all() and rstd[3].isinf() and y[20].isnan().all() and y[10, 5].isnan() and not y[10, :5].any() and not y[10, 6:].any() and rstd[10] == 0
    others = [r for r in range(40) if r not in (3, 10, 20)]
    assert torch.equal(y[others], want[others])
    assert not _forward(x, None, "fp32", 1e-6)[1][3].any()

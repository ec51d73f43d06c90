"""GPU parity of the root-mean-square norm with the fp64 oracle, element by element, and of its 8-bit results with the quantiser's rule."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
EPS = 1e-6
TYPES = ("fp32", "bf16")


def _dt(name):
    import torch
    return torch.float32 if name == "fp32" else torch.bfloat16


def _f64(t):
    return t.double().cpu().numpy()


def _round_h(name):
    import torch
    return lambda v: torch.from_numpy(v).float().to(_dt(name)).double().numpy()


def _inputs(seed, rows, D, groups, xt, rt):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, D, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))).to(_dt(xt))
    res = None if rt == "none" else (3 * torch.randn(rows, D, generator=g, device="cuda")).to(_dt(rt))
    return x, res, 1 + 0.3 * torch.randn(groups, D, generator=g, device="cuda")


def _check(what, got, want, tol):
    x = _f64(got)
    assert np.isfinite(x).all(), what
    over = np.abs(x - want) - tol
    assert over.max() <= 0, (what, float(over.max()), np.unravel_index(over.argmax(), over.shape))


def _check_fp8(y, scales, want, tol):
    """want: the fp64 results [rows, D], tol: how far the fp32 ones may be off.  The scale is the rule's for a largest value within tol, the values are within
    half a step of the type."""
    import torch
    from oracle import proj
    rows, D = want.shape
    cols = proj.up(D, 128)
    q, s = _f64(y), scales.view(torch.uint8).cpu().numpy()[:, :cols // 128]
    assert q.shape == (rows, cols) and not q[:, D:].any()
    lo, hi = (proj.quantise(np.maximum(np.abs(want) + d, 0), "e4m3", 1)[1] for d in (-tol, tol))
    assert ((s >= lo) & (s <= hi)).all() and (lo != hi).sum() <= 1 + lo.size // 1000
    scale = np.repeat(np.ldexp(1.0, s.astype(int) - 127), 128, axis=1)[:, :D]
    v = np.abs(want) / scale
    step = np.ldexp(1.0, np.maximum(np.frexp(np.maximum(v + tol / scale, 1e-30))[1] - 1, -6) - 3)
    assert (np.abs(q[:, :D] * scale - want) <= scale * step / 2 + tol).all()


def _forward(x, res, w, yt, rstd=True, h=None):
    import torch
    import paper_2511_12056_amd as pda
    rows, D = x.shape
    if yt == "e4m3":
        y, s = pda.fp8_empty(rows, D)
        y.view(torch.uint8).fill_(0x7F)
        s.view(torch.uint8).fill_(7)
    else:
        y, s = torch.full(x.shape, float("nan"), device="cuda", dtype=_dt(yt)), None
    r = torch.full((rows,), float("nan"), device="cuda") if rstd else None
    if res is not None and h is None:
        h = torch.full_like(res, float("nan"))
    return pda.rms_norm_fwd(x, w, y, res=res, h=h, y_scales=s, rstd=r, eps=EPS)


SHAPES = [(1, 1, 1), (3, 8, 1), (5, 63, 1), (2, 64, 2), (7, 65, 1), (9, 127, 3), (4, 128, 1), (6, 129, 2), (33, 256, 3), (4, 257, 2), (130, 512, 1), (9, 516, 3), (66, 1023, 2),
          (40, 1152, 4), (37, 1536, 1), (12, 1540, 2), (21, 2048, 3), (6, 2049, 2), (10, 2052, 1), (19, 4096, 1), (5, 4100, 1), (4, 5001, 2), (9, 8192, 3), (2, 8191, 1), (4111, 200, 1), (11, 384, 1), (8, 300, 2)]


@pytest.mark.parametrize("yt", ["fp32", "bf16", "e4m3"])
@pytest.mark.parametrize("xt,rt", [("fp32", "none"), ("bf16", "none"), ("bf16", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("fp32", "fp32")])
@pytest.mark.parametrize("rows,D,groups", SHAPES)
def test_forward(rows, D, groups, xt, rt, yt):
    from oracle import proj
    rows -= rows % groups
    x, res, w = _inputs(rows * D, rows, D, groups, xt, rt)
    h, y, s, rstd = _forward(x, res, w, yt)
    (wh, wy, wr), (ty, tr) = proj.rms_norm(_f64(x), None if res is None else _f64(res), _f64(w), groups, float(np.float32(EPS)), _round_h(rt if rt != "none" else xt), yt == "bf16")
    if res is not None:
        assert np.array_equal(_f64(h), wh)                         # one addition and one rounding
    _check("rstd", rstd, wr, tr)
    if yt == "e4m3":
        _check_fp8(y, s, wy, ty)
    else:
        _check("y", y, wy, ty)


@pytest.mark.parametrize("yt", TYPES)
@pytest.mark.parametrize("ht", TYPES)
@pytest.mark.parametrize("dres", [False, True])
@pytest.mark.parametrize("rows,D,groups", SHAPES)
def test_backward(rows, D, groups, ht, yt, dres):
    import torch
    import paper_2511_12056_amd as pda
    from oracle import proj
    rows -= rows % groups
    h, dr, w = _inputs(rows * D + 1, rows, D, groups, ht, ht)
    dr = dr if dres else None
    g = torch.Generator(device="cuda").manual_seed(5)
    dy = torch.randn(rows, D, generator=g, device="cuda").to(_dt(yt))
    rstd = (h.double().square().mean(dim=-1) + EPS).rsqrt().float()
    dh, dw = torch.full_like(h, float("nan")), torch.full((groups, D), float("nan"), device="cuda")
    pda.rms_norm_bwd(dy, h, w, rstd, dh, dw, dres=dr)
    (wh, ww), (th, tw) = proj.rms_norm_bwd(_f64(dy), _f64(h), _f64(w), _f64(rstd), None if dr is None else _f64(dr), groups, ht == "bf16")
    _check("dh", dh, wh, th)
    _check("dweight", dw, ww, tw)
    # parts alone, and twice: the same bits
    one, two = torch.empty_like(dh), torch.empty_like(dw)
    pda.rms_norm_bwd(dy, h, w, rstd, one, None, dres=dr)
    pda.rms_norm_bwd(dy, h, w, rstd, None, two, dres=dr)
    assert torch.equal(one, dh) and torch.equal(two, dw)


def test_eight_bit_results_are_the_quantisers():
    """The norm's 8-bit results are those of pda_fp8_quant on its fp32 results, bit for bit."""
    import torch
    import paper_2511_12056_amd as pda
    for rows, D in ((7, 100), (33, 1536), (5, 2500), (3, 8192)):
        x, res, w = _inputs(D, rows, D, 1, "bf16", "fp32")
        _, y, _, _ = _forward(x, res, w, "fp32")
        _, q, s, _ = _forward(x, res, w, "e4m3")
        wq, ws = pda.fp8_empty(rows, D)
        pda.fp8_quant(y, wq, ws)
        n = (D + 127) // 128
        assert torch.equal(q.view(torch.uint8), wq.view(torch.uint8)) and torch.equal(s.view(torch.uint8)[:, :n], ws.view(torch.uint8)[:, :n])
        assert (s.view(torch.uint8)[:, n:] == 7).all()             # bytes behind the last block are left as they were


@pytest.mark.parametrize("yt", ["fp32", "bf16", "e4m3"])
def test_without_weight_or_rstd_and_in_place(yt):
    import torch
    x, res, w = _inputs(3, 19, 1100, 1, "fp32", "fp32")
    one = torch.ones_like(w)
    ref = _forward(x, res, one, yt)
    got = _forward(x, res, None, yt, rstd=False)
    assert got[3] is None and torch.equal(got[0], ref[0])
    assert torch.equal(got[1].view(torch.uint8), ref[1].view(torch.uint8))
    for target in (x, res):
        a, b = x.clone(), res.clone()
        h = a if target is x else b
        out = _forward(a, b, None, yt, h=h)
        assert torch.equal(h, ref[0]) and torch.equal(out[1].view(torch.uint8), ref[1].view(torch.uint8))


@pytest.mark.parametrize("xt,rt", [("bf16", "fp32"), ("fp32", "none"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,D", [(3000, 128), (1500, 203), (900, 1536), (700, 2176), (300, 5000)])
def test_scales_at_their_borders(rows, D, xt, rt):
    """A weight a row that puts the largest value of one of its blocks within some 2^-22 of 1.75 times a power of two, where the scale doubles: the bytes of those blocks are what the
    definition gives in 64 bits, on either side."""
    import torch
    x, res, _ = _inputs(rows + D, rows, D, 1, xt, rt)
    h = (x.float() if res is None else (x.float() + res.float()).to(res.dtype).float()).double()
    y = h / torch.sqrt(h.square().mean(dim=-1, keepdim=True) + float(np.float32(EPS)))
    pad = torch.nn.functional.pad(y.abs(), (0, -D % 128)).view(rows, -1, 128).amax(dim=-1)
    r = torch.arange(rows, device="cuda")
    block = r % pad.shape[1]
    step = torch.linspace(-2.0 ** -22, 2.0 ** -22, rows, device="cuda", dtype=torch.float64)
    w = (1.75 * (1 << r % 20).double() * (1 + step) / pad[r, block]).float()
    out = _forward(x, res, w[:, None].expand(rows, D).contiguous(), "e4m3")
    top = pad[r, block] * w.double()
    got = out[2].view(torch.uint8)[r, block].double()
    mantissa, e = torch.frexp(top)                          # top = mantissa 2^e, 1/2 <= mantissa < 1: 2^(e - 1 - 8) is enough up to 0.875
    assert torch.equal(got, (e - 9 + (mantissa > 0.875).int() + 127).double())
    assert (mantissa > 0.875).any() and (mantissa <= 0.875).any()
    if res is not None:                                     # and in place
        again = _forward(x, res, w[:, None].expand(rows, D).contiguous(), "e4m3", h=res)
        assert torch.equal(again[2].view(torch.uint8)[r, block], out[2].view(torch.uint8)[r, block]) and torch.equal(again[1].view(torch.uint8), out[1].view(torch.uint8))


@pytest.mark.parametrize("ht", TYPES)
def test_backward_in_place(ht):
    import torch
    import paper_2511_12056_amd as pda
    h, dr, w = _inputs(9, 300, 700, 2, ht, ht)
    dy = torch.randn_like(h.float()).to(h.dtype)
    rstd = (h.double().square().mean(dim=-1) + EPS).rsqrt().float()
    ref, dw = torch.empty_like(h), torch.empty(2, 700, device="cuda")
    pda.rms_norm_bwd(dy, h, w, rstd, ref, dw, dres=dr)
    for which in range(3):
        a = [dy.clone(), h.clone(), dr.clone()]
        dw2 = torch.empty_like(dw)
        pda.rms_norm_bwd(a[0], a[1], w, rstd, a[which], dw2, dres=a[2])
        assert torch.equal(a[which], ref) and torch.equal(dw2, dw)


def test_rows_that_are_zero_or_not_finite():
    """A row touches its own results only; zeros give zeros (scale 1 for 8 bits), a NaN its whole row, what overflows the sum of squares zeros."""
    import torch
    x = torch.randn(6, 300, device="cuda")
    x[1] = 0
    x[2, 17] = float("nan")
    x[3, 5] = float("inf")
    x[4] *= 1e25
    for yt in ("fp32", "e4m3"):
        _, y, s, rstd = _forward(x, None, None, yt)
        _, clean, sc, _ = _forward(x[[0, 5]].contiguous(), None, None, yt)
        y = y.float()
        assert torch.equal(y[[0, 5]], clean.float()) and not y[1].any() and y[2, :300].isnan().all()
        assert rstd[3] == 0 and rstd[4] == 0 and y[3, 5].isnan() and not y[3, :5].any() and not y[4].any()
        if yt == "e4m3":
            b = s.view(torch.uint8)[:, :3]
            assert torch.equal(b[[0, 5]], sc.view(torch.uint8)[:, :3]) and (b[[1, 2, 3, 4]] == 127).all() and not y[:, 300:].any()


def test_no_rows():
    import torch
    import paper_2511_12056_amd as pda
    dw = torch.full((3, 70), 5.0, device="cuda")
    e = torch.empty(0, 70, device="cuda")
    pda.rms_norm_bwd(e, e, None, torch.empty(0, device="cuda"), e.clone(), dw)
    assert not dw.any()
    pda.rms_norm_fwd(e, None, e.clone())


def test_rows_beyond_one_axis_of_a_launch():
    """More workgroups than fit along x, and offsets past 2^31 elements."""
    import torch
    import paper_2511_12056_amd as pda
    rows, D = (1 << 24) + 5, 130
    x = torch.zeros(rows, D, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1 << 23, (1 << 24) - 1, rows - 1], device="cuda")
    x[at] = torch.randn(4, D, device="cuda").to(torch.bfloat16)
    y, s = pda.fp8_empty(rows, D)
    pda.rms_norm_fwd(x, None, y, y_scales=s)
    want, ws = pda.fp8_empty(4, D)
    pda.rms_norm_fwd(x[at].contiguous(), None, want, y_scales=ws)
    assert torch.equal(y[at].view(torch.uint8), want.view(torch.uint8)) and torch.equal(s.view(torch.uint8)[at, :2], ws.view(torch.uint8)[:, :2])
    assert (s.view(torch.uint8)[2, :2] == 127).all()
    del x, y, s
    torch.cuda.empty_cache()


def test_refusals_of_the_wrappers():
    import torch
    import paper_2511_12056_amd as pda
    x, w = torch.randn(4, 96, device="cuda"), torch.ones(96, device="cuda")
    y, s = pda.fp8_empty(4, 96)
    rstd = torch.empty(4, device="cuda")
    bad = [lambda: pda.rms_norm_fwd(x, w, y), lambda: pda.rms_norm_fwd(x, w, y, y_scales=s[:, :2]), lambda: pda.rms_norm_fwd(x, w, x.clone(), y_scales=s),
           lambda: pda.rms_norm_fwd(x, w, y[:, :96], y_scales=s), lambda: pda.rms_norm_fwd(x, w, y.view(torch.float8_e5m2), y_scales=s),
           lambda: pda.rms_norm_fwd(x, w, x.clone(), res=x.clone()), lambda: pda.rms_norm_fwd(x, w, x.clone(), res=x.clone(), h=x.to(torch.bfloat16)),
           lambda: pda.rms_norm_fwd(x, w[:95], x.clone()), lambda: pda.rms_norm_fwd(x, w, x.clone(), rstd=rstd[:3]), lambda: pda.rms_norm_fwd(x.half(), w, x.clone()),
           lambda: pda.rms_norm_bwd(x.clone(), x, w, rstd, x.to(torch.bfloat16), None), lambda: pda.rms_norm_bwd(x[:3], x, w, rstd, x.clone(), None),
           lambda: pda.rms_norm_bwd(x.clone(), x, w, rstd, x.clone(), torch.empty(2, 96, device="cuda"))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(pda.PdaError):
        pda.rms_norm_bwd(x.clone(), x, w, rstd, None, None)
    with pytest.raises(pda.PdaError):
        big = torch.randn(4096, 96, device="cuda")
        pda.rms_norm_bwd(big.clone(), big, w, torch.ones(4096, device="cuda"), None, torch.empty(96, device="cuda"), workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))

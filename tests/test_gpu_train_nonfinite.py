"""NaN and infinities in the training operators: they reach what the formulas put them in, all of it and nothing else."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _attention(d, H, S, n_v, seed):
    import torch
    import paper_2511_12056_amd as pda
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v, dout = (torch.randn(1, H, S, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(4))
    out, lse = torch.empty(1, H, S, d, device="cuda"), torch.empty(1, H, S, device="cuda")
    pda.attn_fwd(q, k, v, out, lse, d ** -0.5, n_v)
    return dout, q, k, v, out, lse


def _gradients(x, d, n_v):
    import torch
    import paper_2511_12056_amd as pda
    got = pda.attn_bwd(*x, *(torch.full_like(t, 7.0) for t in x[1:4]), d ** -0.5, n_v)
    torch.cuda.synchronize()
    return got


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,S,n_v", [(2, 700, 690), (30, 2500, 2410), (1, 40, 40)])      # cut blocks, whole ones, a tile and a part
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_delta_that_is_not_finite(value, H, S, n_v, d):
    """An entry of out makes one row's delta NaN or infinite: dk of its head and the row's dq are lost, dv has no delta in it."""
    import torch
    x = _attention(d, H, S, n_v, S)
    want = [t.clone() for t in _gradients(x, d, n_v)]
    row = S // 3
    x[4][0, -1, row, 5] = value
    x[0][0, -1, row, 5] = 1.0
    x[0][0, -1, row, 6] = -2.0
    dv = _gradients((x[0], *x[1:4], torch.nan_to_num(x[4], 0.0, 0.0, 0.0), x[5]), d, n_v)[2].clone()
    got = _gradients(x, d, n_v)
    assert torch.equal(got[2], dv)                                         # dv: the bits of a call with another out
    assert not torch.isfinite(got[0][0, -1, row]).any() and not torch.isfinite(got[1][0, -1, :n_v]).any()
    rest = [r for r in range(S) if r != row]
    assert torch.equal(got[0][0, -1, rest], want[0][0, -1, rest])
    assert all(torch.equal(a[0, :-1], b[0, :-1]) for a, b in zip(got, want)) and (got[1][0, -1, n_v:] == 0).all()


@pytest.mark.parametrize("d", [128, 64])
def test_log_sum_exp_that_is_nan(d):
    """The row's probabilities are NaN: its dq, and dk and dv of its head."""
    import torch
    x = _attention(d, 2, 300, 280, 1)
    want = [t.clone() for t in _gradients(x, d, 280)]
    x[5][0, 1, 77] = float("nan")
    got = _gradients(x, d, 280)
    assert torch.isnan(got[0][0, 1, 77]).all() and all(torch.isnan(t[0, 1, :280]).all() for t in got[1:])
    assert all(torch.equal(a[0, 0], b[0, 0]) for a, b in zip(got, want)) and torch.equal(got[0][0, 1, :77], want[0][0, 1, :77])


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("scale", [0.125, 1e-6])
def test_log_sum_exps_near_the_largest_float(scale, d):
    """Rows whose log-sum-exp leaves no probability give nothing, however large it is (-lse log2 e, and it over the scale, pass fp32's range)."""
    import torch
    import paper_2511_12056_amd as pda
    x = _attention(d, 2, 300, 280, 2)
    call = lambda: [t.clone() for t in pda.attn_bwd(*x, *(torch.full_like(t, 7.0) for t in x[1:4]), scale, 280)]  # noqa: E731
    x[5][0, :, 3::8] = float("inf")
    want = call()
    for value in (3.4e38, 2.3e38, 1e38, 1e33, 1e31, 1e7):
        x[5][0, :, 3::8] = value
        got = call()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), value
        assert (got[0][0, :, 3::8] == 0).all()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("where", ["x", "dy"])
def test_pack_gradient_of_a_vector_with_nan(where, d):
    """With unit_rms every element of the vector's gradient has <x, x> and <x, dy> in it; the other vectors keep their bits."""
    import torch
    import paper_2511_12056_amd as pda
    g = torch.Generator(device="cuda").manual_seed(d)
    B, S, H = 2, 37, 3
    x, dy = torch.randn(B, S, H, d, generator=g, device="cuda"), torch.randn(B, H, S, d, generator=g, device="cuda").to(torch.bfloat16)
    x[0, 0, 0] = 0.0
    want = pda.pack_heads_bwd(dy, x, torch.empty_like(x), True, 0.5).clone()
    at = [(0, 3, 1), (1, 36, 2), (1, 0, 0)]
    for i, (b, s, h) in enumerate(at):
        if where == "x":
            x[b, s, h, 7 * i] = float("nan")
        else:
            dy[b, h, s, 7 * i] = float("nan")
    got = pda.pack_heads_bwd(dy, x, torch.full_like(x, 7.0), True, 0.5)
    hit = np.zeros((B, S, H), dtype=bool)
    for i in at:
        hit[i] = True
        assert torch.isnan(got[i]).all(), i
    hit = torch.from_numpy(hit).cuda()
    assert torch.equal(got[~hit], want[~hit]) and (got[0, 0, 0] == 0).all()


def test_pack_gradient_of_an_infinite_element():
    """An infinite element: x / rms(x) is NaN there, and so is the gradient."""
    import torch
    import paper_2511_12056_amd as pda
    x, dy = torch.ones(1, 4, 2, 64, device="cuda"), torch.ones(1, 2, 4, 64, device="cuda", dtype=torch.bfloat16)
    x[0, 2, 1, 9] = float("inf")
    got = pda.pack_heads_bwd(dy, x, torch.empty_like(x), True)
    assert torch.isnan(got[0, 2, 1, 9]) and torch.isfinite(got[0, :2]).all()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("value", [1e-21, 3e-22, 2e-22, 1.5e-22, 1e-22, 5e-23, 1e-23, 1e-30])
def test_pack_gradient_of_a_vector_whose_squares_nearly_vanish(value, d):
    """One element whose square, or its mean over the vector, is at the end of fp32's range: the gradient is that of the formula, or 0 where the square is."""
    import torch
    import paper_2511_12056_amd as pda
    x, dy = torch.zeros(1, 3, 1, d, device="cuda"), torch.ones(1, 1, 3, d, device="cuda", dtype=torch.bfloat16)
    x[0, :, 0, 5] = value
    dy[..., 9] = -2.0
    got = pda.pack_heads_bwd(dy, x, torch.full_like(x, 7.0), True)
    assert torch.isfinite(got).all()
    x2 = float(x[0, 0, 0, 5].double()) ** 2
    if x2 < 2.0 ** -150:
        assert (got == 0).all()
        return
    # the square is rounded to whole units of 2^-149: off by e = 2^-150 / x^2 < 1 relatively, to half and twice its value at the most.  r = 1 / sqrt(..) is off by
    # less than 1.5 e (1 / sqrt(1 - e) - 1 <= e up to e = 0.6, 0.42 beyond it), the element itself, r (1 - x^2 / square), by r times 2 e; 2^-20 for the other roundings
    r, e = d ** 0.5 / x2 ** 0.5, 2.0 ** -150 / x2
    want = r * dy.double().transpose(1, 2)
    want[..., 5] = 0
    assert ((got.double() - want).abs() <= 2 * r * (1.5 * e + 2.0 ** -20)).all(), (got[0, 0, 0, :10], want[0, 0, 0, :10])


@pytest.mark.parametrize("D", [3, 30, 64, 100, 128, 300, 640, 1001, 1536, 3001])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_layer_norm_of_a_row_that_is_not_finite(value, D):
    """It loses its own results, and in the backward pass its group's sums; rows beside it, which may share a wavefront, keep their bits."""
    import torch
    import paper_2511_12056_amd as pda
    g = torch.Generator(device="cuda").manual_seed(D)
    rows, groups, bad = 66, 2, 13
    x, dy = (torch.randn(rows, D, generator=g, device="cuda") for _ in range(2))
    w, b = 1 + torch.randn(groups, D, generator=g, device="cuda"), torch.randn(groups, D, generator=g, device="cuda")

    def both():
        y, mean, rstd = pda.layer_norm_fwd(x, w, b, torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"))
        dx, dw, db = pda.layer_norm_bwd(dy, x, w, mean, rstd, torch.empty_like(x), torch.empty_like(w), torch.empty_like(b))
        return y, mean, rstd, dx, dw, db
    want = [t.clone() for t in both()]
    x[bad, D // 2] = value
    y, mean, rstd, dx, dw, db = both()
    others = [r for r in range(rows) if r != bad]
    for a, c in zip((y, mean, rstd, dx), want):
        assert torch.equal(a[others], c[others])
    assert torch.isnan(y[bad]).all() and torch.isnan(dx[bad]).all() and not torch.isfinite(mean[bad]) and torch.isnan(dw[0]).all()
    assert torch.equal(dw[1], want[4][1]) and torch.equal(db, want[5])

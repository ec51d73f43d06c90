"""GPU parity of layer norm forward and backward, and of the gradient of the pack, with the fp64 oracle, element by element."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
TYPES = ("fp32", "bf16")


def _dt(name):
    import torch
    return torch.float32 if name == "fp32" else torch.bfloat16


def _f64(t):
    return t.double().cpu().numpy()


def _inputs(seed, rows, D, groups, xt, yt, offset=0.5):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (torch.randn(rows, D, generator=g, device="cuda") * 1.5 + offset).to(_dt(xt))
    dy = torch.randn(rows, D, generator=g, device="cuda").to(_dt(yt))
    w = 1 + 0.3 * torch.randn(groups, D, generator=g, device="cuda")
    b = 0.3 * torch.randn(groups, D, generator=g, device="cuda")
    return x, dy, w, b


def _check(what, got, want, tol):
    x = _f64(got)
    assert np.isfinite(x).all(), what
    over = np.abs(x - want) - tol
    assert over.max() <= 0, (what, float(over.max()), np.unravel_index(over.argmax(), over.shape))


def _forward(x, w, b, yt, eps=1e-6):
    import torch
    import paper_2511_12056_amd as pda
    rows = x.shape[0]
    y = torch.full(x.shape, float("nan"), device="cuda", dtype=_dt(yt))
    mean, rstd = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    return pda.layer_norm_fwd(x, w, b, y, mean, rstd, eps)


SHAPES = [(1, 1, 1), (3, 8, 1), (5, 63, 1), (2, 64, 2), (7, 65, 1), (33, 256, 3), (4, 257, 2), (130, 512, 1), (9, 516, 3), (66, 1023, 2), (40, 1152, 4),
          (37, 1536, 1), (12, 1540, 2), (21, 2048, 3), (6, 2049, 2), (10, 2052, 1), (19, 4096, 1), (5, 4100, 1), (4, 5001, 2), (9, 8192, 3), (2, 8191, 1), (4111, 200, 1)]


@pytest.mark.parametrize("xt", TYPES)
@pytest.mark.parametrize("yt", TYPES)
@pytest.mark.parametrize("rows,D,groups", SHAPES)
def test_against_the_oracle(rows, D, groups, xt, yt):
    import torch
    import paper_2511_12056_amd as pda
    from oracle import train
    rows -= rows % groups
    x, dy, w, b = _inputs(rows * D, rows, D, groups, xt, yt)
    y, mean, rstd = _forward(x, w, b, yt)
    want, tol = train.layer_norm(_f64(x), _f64(w), _f64(b), groups, float(np.float32(1e-6)), yt == "bf16")
    for n, g, e, t in zip(("y", "mean", "rstd"), (y, mean, rstd), want, tol):
        if D == 1 and n == "rstd":
            continue                                     # a variance of zero: rstd = 1 / sqrt(eps), nothing to bound by
        _check(n, g, e, t)
    dx, dw, db = torch.full_like(x, float("nan")), torch.full_like(w, float("nan")), torch.full_like(b, float("nan"))
    pda.layer_norm_bwd(dy, x, w, mean, rstd, dx, dw, db)
    want, tol = train.layer_norm_bwd(_f64(dy), _f64(x), _f64(w), _f64(mean), _f64(rstd), groups, xt == "bf16")
    for n, g, e, t in zip(("dx", "dweight", "dbias"), (dx, dw, db), want, tol):
        _check(n, g, e, t)


@pytest.mark.parametrize("rows,D", [(50, 96), (300, 2100)])
def test_optional_arguments(rows, D):
    """Without weight or bias; results that are not wanted; the others keep their bits."""
    import torch
    import paper_2511_12056_amd as pda
    from oracle import train
    x, dy, w, b = _inputs(1, rows, D, 1, "fp32", "fp32")
    for weight, bias in ((None, None), (w[0], None), (None, b[0])):
        y, mean, rstd = _forward(x, weight, bias, "fp32")
        want, tol = train.layer_norm(_f64(x), None if weight is None else _f64(w), None if bias is None else _f64(b), 1, float(np.float32(1e-6)), False)
        _check("y", y, want[0], tol[0])
        again = torch.empty_like(y)
        pda.layer_norm_fwd(x, weight, bias, again)
        assert torch.equal(again, y)
        new = lambda: (torch.full_like(x, float("nan")), torch.full((D,), float("nan"), device="cuda"), torch.full((D,), float("nan"), device="cuda"))  # noqa: E731
        dx, dw, db = new()
        pda.layer_norm_bwd(dy, x, weight, mean, rstd, dx, dw, db)
        want, tol = train.layer_norm_bwd(_f64(dy), _f64(x), None if weight is None else _f64(w), _f64(mean), _f64(rstd), 1, False)
        _check("dx", dx, want[0], tol[0])
        _check("dweight", dw, want[1][0], tol[1][0])
        _check("dbias", db, want[2][0], tol[2][0])
        for wanted in ((0,), (1,), (2,), (0, 2), (1, 2)):
            some = [t if i in wanted else None for i, t in enumerate(new())]
            pda.layer_norm_bwd(dy, x, weight, mean, rstd, *some)
            assert all(t is None or torch.equal(t, r) for t, r in zip(some, (dx, dw, db))), wanted


def test_in_place():
    import torch
    import paper_2511_12056_amd as pda
    for D in (96, 3000, 101):
        x, dy, w, b = _inputs(2, 64, D, 2, "bf16", "bf16")
        y, mean, rstd = _forward(x, w, b, "bf16")
        z = x.clone()
        pda.layer_norm_fwd(z, w, b, z)
        assert torch.equal(z, y)
        dx = torch.empty_like(x)
        pda.layer_norm_bwd(dy, x, w, mean, rstd, dx, None, None)
        for over_dy in (True, False):
            a, g = x.clone(), dy.clone()
            pda.layer_norm_bwd(g, a, w, mean, rstd, g if over_dy else a, None, None)
            assert torch.equal(g if over_dy else a, dx)


def test_constant_rows_and_large_offsets():
    """A variance of zero is held up by eps; values far from zero lose nothing to a difference of squares."""
    import torch
    import paper_2511_12056_amd as pda
    from oracle import train
    x = torch.full((4, 300), 3.0, device="cuda")
    y, mean, rstd = _forward(x, None, None, "fp32", eps=1e-4)
    assert (y == 0).all() and (mean == 3).all() and torch.allclose(rstd, torch.full_like(rstd, 100.0), rtol=1e-6)
    dx = torch.empty_like(x)
    pda.layer_norm_bwd(torch.ones_like(x), x, None, mean, rstd, dx, None, None)
    assert dx.abs().max() <= 100 * 64 * 2.0 ** -24
    x = (torch.randn(16, 1000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) + 1000.0)
    y, mean, rstd = _forward(x, None, None, "fp32")
    want, tol = train.layer_norm(_f64(x), None, None, 1, float(np.float32(1e-6)), False)
    for n, g, e, t in zip(("y", "mean", "rstd"), (y, mean, rstd), want, tol):
        _check(n, g, e, t)
    assert (y.double().cpu().numpy() - want[0]).__abs__().max() < 2e-3


def test_no_rows():
    import torch
    import paper_2511_12056_amd as pda
    x = torch.empty(0, 64, device="cuda")
    dw, db = torch.full((3, 64), float("nan"), device="cuda"), torch.full((3, 64), float("nan"), device="cuda")
    e = torch.empty(0, device="cuda")
    pda.layer_norm_fwd(x, None, None, torch.empty_like(x), e, e.clone())
    pda.layer_norm_bwd(x, x, None, e, e, torch.empty_like(x), dw, db)
    assert (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("D", [192, 1001, 2304])
def test_other_memory_is_left_alone_and_equal_calls_give_equal_bits(D):
    import torch
    import paper_2511_12056_amd as pda
    rows, pad = 5000, 64
    x, dy, w, b = _inputs(4, rows, D, 1, "fp32", "bf16")
    y = torch.full((rows * D + pad,), 7.0, device="cuda", dtype=torch.bfloat16)
    dx = torch.full((rows * D + pad,), 7.0, device="cuda")
    stats, sums = torch.full((2, rows + pad), 7.0, device="cuda"), torch.full((2, D + pad + (-D) % 4), 7.0, device="cuda")
    n = pda.layer_norm_bwd_workspace_bytes(rows, D)
    ws = torch.full((n + pad,), 0xA5, device="cuda", dtype=torch.uint8)
    kept = None
    for _ in range(2):
        pda.layer_norm_fwd(x, w, b, y[:rows * D].view(rows, D), stats[0, :rows], stats[1, :rows])
        pda.layer_norm_bwd(dy, x, w, stats[0, :rows], stats[1, :rows], dx[:rows * D].view(rows, D), sums[0, :D], sums[1, :D], workspace=ws[:n])
        assert (y[rows * D:] == 7).all() and (dx[rows * D:] == 7).all() and (stats[:, rows:] == 7).all() and (sums[:, D:] == 7).all()
        assert (ws[n:] == 0xA5).all()
        now = [t.clone() for t in (y, dx, stats, sums)]
        assert kept is None or all(torch.equal(a, c) for a, c in zip(kept, now))
        kept = now
    with pytest.raises(pda.PdaError) as e:
        pda.layer_norm_bwd(dy, x, w, stats[0, :rows], stats[1, :rows], None, sums[0, :D], None, workspace=ws[:n - 16])
    assert e.value.code == 1


def test_graph_capture_and_another_stream():
    import torch
    import paper_2511_12056_amd as pda
    rows, D, groups = 6000, 640, 2
    x, dy, w, b = _inputs(5, rows, D, groups, "fp32", "bf16")
    y, mean, rstd = _forward(x, w, b, "bf16")
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    pda.layer_norm_bwd(dy, x, w, mean, rstd, dx, dw, db)
    want = [t.clone() for t in (y, mean, rstd, dx, dw, db)]
    got = [torch.empty_like(t) for t in want]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    ws = pda.layer_norm_bwd_workspace(rows, D, groups)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        pda.layer_norm_fwd(x, w, b, *got[:3], stream=side)
        pda.layer_norm_bwd(dy, x, w, got[1], got[2], *got[3:], workspace=ws, stream=side)
    for rep in range(3):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want)), rep
        pda.layer_norm_bwd(dy, x, w, mean, rstd, dx, dw, db)
        torch.cuda.synchronize()


@pytest.mark.parametrize("unit_rms", [False, True])
@pytest.mark.parametrize("B,S,H,d", [(1, 1, 1, 64), (1, 7, 3, 128), (2, 33, 5, 64), (3, 9, 24, 128), (1, 2051, 2, 64), (2, 1000, 3, 128)])
def test_pack_gradient(B, S, H, d, unit_rms):
    import torch
    import paper_2511_12056_amd as pda
    from oracle import train
    g = torch.Generator(device="cuda").manual_seed(B + S)
    x, dy = torch.randn(B, S, H, d, generator=g, device="cuda"), torch.randn(B, H, S, d, generator=g, device="cuda").to(torch.bfloat16)
    x[0, 0, 0] = 0.0                                      # a zero vector has no direction: its gradient is 0 with unit_rms
    x[-1, -1, -1] *= 1e-12
    x[-1, 0, -1] *= 1e12
    dx = torch.full((B * S * H * d + 64,), 7.0, device="cuda")
    to = dx[:-64].view(B, S, H, d)
    pda.pack_heads_bwd(dy, x if unit_rms else None, to, unit_rms, 0.3)
    want, tol = train.pack_heads_bwd(_f64(dy), _f64(x), unit_rms, float(np.float32(0.3)))
    _check("dx", to, want, tol + 1e-38)
    assert (dx[-64:] == 7).all() and (not unit_rms or (to[0, 0, 0] == 0).all() or B * S * H == 1)
    if unit_rms:
        again = x.clone()
        pda.pack_heads_bwd(dy, again, again, True, 0.3)
        assert torch.equal(again, to)


@pytest.mark.parametrize("D", [8, 132])
def test_more_rows_than_a_launch_has_threads_for(D):
    """2^23 rows of more than 128 elements are as many as one axis of a launch takes."""
    import torch
    import paper_2511_12056_amd as pda
    rows = (1 << 23) + 4099
    x = torch.randn(rows, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    y, mean, rstd = torch.full_like(x, float("nan")), *(torch.full((rows,), float("nan"), device="cuda") for _ in range(2))
    pda.layer_norm_fwd(x, None, None, y, mean, rstd, 1e-6)
    m = x.mean(-1)
    assert (mean - m).abs().max() <= D * 2.0 ** -23 * x.abs().max()      # D - 1 additions and a division, in fp32, on either side
    at = [0, 1, (1 << 23) - 1, 1 << 23, rows - 4097, rows - 1]
    part, pm, pr = x[at].contiguous(), torch.empty(len(at), device="cuda"), torch.empty(len(at), device="cuda")
    py = torch.empty_like(part)
    pda.layer_norm_fwd(part, None, None, py, pm, pr, 1e-6)
    assert torch.equal(y[at], py) and torch.equal(mean[at], pm) and torch.equal(rstd[at], pr)
    assert torch.isfinite(y).all() and torch.isfinite(rstd).all()
    dx, dw = torch.full_like(x, float("nan")), torch.empty(D, device="cuda")
    pda.layer_norm_bwd(y, x, None, mean, rstd, dx, dw, None)
    pdx = torch.empty_like(part)
    pda.layer_norm_bwd(py, part, None, pm, pr, pdx, None, None)
    assert torch.equal(dx[at], pdx) and torch.isfinite(dx).all()
    want = y.double().square().sum(0)                # dy = xh: squares, in chains of fewer than rows / 4 096 + 4 096 additions
    assert ((dw.double() - want).abs() <= 2.0 ** -24 * (rows / 4096 + 4096) * want).all()


def test_elements_beyond_32_bits():
    """2^31 elements and more, of rows that end beside a group of four."""
    import torch
    import paper_2511_12056_amd as pda
    rows, D = 2 * 697_300, 1541
    assert rows * D > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty(rows, D, device="cuda", dtype=torch.bfloat16)
    for r in range(0, rows, 139_460):
        x[r:r + 139_460].normal_(generator=g)
    w = 1 + torch.randn(2, D, generator=g, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    pda.layer_norm_fwd(x, w, None, y, mean, rstd, 1e-6)
    dx, dw = torch.empty_like(x), torch.empty(2, D, device="cuda")
    pda.layer_norm_bwd(y, x, w, mean, rstd, dx, dw, None)
    for a, b in ((0, 3), (rows - 1000, rows)):
        part, pw = x[a:b].clone(), w[0 if a == 0 else 1].clone()
        py, pm, pr, pdx = torch.empty_like(part), torch.empty(b - a, device="cuda"), torch.empty(b - a, device="cuda"), torch.empty_like(part)
        pda.layer_norm_fwd(part, pw, None, py, pm, pr, 1e-6)
        pda.layer_norm_bwd(py, part, pw, pm, pr, pdx, None, None)
        assert torch.equal(y[a:b], py) and torch.equal(mean[a:b], pm) and torch.equal(rstd[a:b], pr) and torch.equal(dx[a:b], pdx)
    del dx
    # dweight = sum of dy xh with dy = y: terms of one sign, each off by 3 * 2^-24 at most, in chains of fewer than rows / 512 + 512 additions
    for i in (0, 1):
        want = torch.zeros(D, device="cuda", dtype=torch.float64)
        for r in range(i * rows // 2, (i + 1) * rows // 2, 69_730):
            s = slice(r, r + 69_730)
            want += (y[s].double() * (x[s].double() - mean[s, None].double()) * rstd[s, None].double()).sum(0)
        assert ((dw[i].double() - want).abs() <= 2.0 ** -24 * (rows / 512 + 512) * want.abs()).all()


def test_pack_gradient_beyond_32_bits():
    import torch
    import paper_2511_12056_amd as pda
    S, H, d = 700_001, 24, 128
    assert S * H * d > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(1, S, H, d, generator=g, device="cuda")
    dy = torch.empty(1, H, S, d, device="cuda", dtype=torch.bfloat16)
    for h in range(H):
        dy[:, h].normal_(generator=g)
    dx = torch.full_like(x, float("nan"))
    pda.pack_heads_bwd(dy, x, dx, True, 0.25)
    for a, b in ((0, 9), (S // 2, S // 2 + 17), (S - 13, S)):
        want = torch.empty(1, b - a, H, d, device="cuda")
        pda.pack_heads_bwd(dy[:, :, a:b].contiguous(), x[:, a:b].contiguous(), want, True, 0.25)
        assert torch.equal(dx[:, a:b], want)
    assert not torch.isnan(dx).any()


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    import torch
    import paper_2511_12056_amd as pda
    g = torch.Generator(device="cuda").manual_seed(4)
    data, want = [], []
    for rows, D in ((30_000, 640), (20_001, 1001)):
        x, dy, w = (torch.randn(*s, generator=g, device="cuda") for s in ((rows, D), (rows, D), (D,)))
        y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        pda.layer_norm_fwd(x, w, None, y, mean, rstd)
        data.append((dy, x, w, mean, rstd, pda.layer_norm_bwd_workspace(rows, D)))
        want.append(pda.layer_norm_bwd(*data[-1][:5], torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)))
    res = [[[torch.empty_like(t) for t in w] for _ in range(5)] for w in want]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(5):
        for i in (0, 1):
            pda.layer_norm_bwd(*data[i][:5], *res[i][rep], workspace=data[i][5], stream=streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in (0, 1) for r in res[i] for a, b in zip(r, want[i]))


@pytest.mark.parametrize("xt", TYPES)
@pytest.mark.parametrize("yt", TYPES)
@pytest.mark.parametrize("rows,D,groups", [(4, 2, 1), (5, 3, 1), (9, 4, 3), (6, 5, 2), (8, 6, 1), (8, 7, 2), (40, 259, 2), (66, 510, 1), (35, 778, 1), (40, 1101, 2),
                                           (23, 1541, 1), (30, 1903, 2), (14, 3001, 2), (9, 4999, 1), (5, 8190, 1)])
def test_lengths_beside_a_group_of_four(rows, D, groups, xt, yt):
    test_against_the_oracle(rows, D, groups, xt, yt)


def test_in_place_beside_a_group_of_four():
    """A row's last elements are read together with the ones before them."""
    import torch
    import paper_2511_12056_amd as pda
    for D in (2, 3, 5, 6, 250, 511, 778, 1541, 3001, 4999, 8191):
        for t in TYPES:
            x, dy, w, b = _inputs(5, 600, D, 2, t, t)
            y, mean, rstd = _forward(x, w, b, t)
            z = x.clone()
            pda.layer_norm_fwd(z, w, b, z)
            assert torch.equal(z, y), (D, t)
            dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
            pda.layer_norm_bwd(dy, x, w, mean, rstd, dx, dw, db)
            for over_dy in (True, False):
                a, g, dw2, db2 = x.clone(), dy.clone(), torch.empty_like(w), torch.empty_like(b)
                pda.layer_norm_bwd(g, a, w, mean, rstd, g if over_dy else a, dw2, db2)
                assert torch.equal(g if over_dy else a, dx) and torch.equal(dw2, dw) and torch.equal(db2, db), (D, t, over_dy)


def test_lengths_beside_a_group_of_four_leave_their_surroundings():
    """NaN in front of and behind the tensors is not read, what stands there is kept."""
    import torch
    import paper_2511_12056_amd as pda

    def inside(x, fill):
        big = torch.full((x.numel() + 256,), fill, device="cuda", dtype=x.dtype)
        view = big[128:128 + x.numel()].view(x.shape)
        view.copy_(x)
        return big, view
    for D in (3, 6, 509, 1541, 3001):
        for t in TYPES:
            x, dy, w, b = _inputs(6, 37, D, 1, t, t)
            y, mean, rstd = _forward(x, w, b, t)
            dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
            pda.layer_norm_bwd(dy, x, w, mean, rstd, dx, dw, db)
            nan = [inside(v, float("nan"))[1] for v in (x, dy, w, b, mean, rstd)]
            res = [inside(torch.zeros_like(v), 7.0) for v in (y, dx, dw, db)]
            pda.layer_norm_fwd(nan[0], nan[2], nan[3], res[0][1])
            pda.layer_norm_bwd(nan[1], nan[0], nan[2], nan[4], nan[5], *(v for _, v in res[1:]))
            for (big, view), want in zip(res, (y, dx, dw, db)):
                assert torch.equal(view, want), (D, t)
                view.fill_(7.0)
                assert (big == 7.0).all(), (D, t)

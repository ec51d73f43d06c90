"""GPU parity of 8-bit quantisation (exact) and of the product of 8-bit matrices (element by element) with the fp64 oracle."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
KINDS = ("e4m3", "e5m2")


def _type(kind):
    import torch
    return torch.float8_e4m3fn if kind == "e4m3" else torch.float8_e5m2


def _bytes(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def _f64(t):
    return t.double().cpu().numpy()


def _empty(rows, cols, block, kind, fill=0x55):
    import torch
    import paper_2511_12056_amd as pda
    q, s = pda.fp8_empty(rows, cols, block, _type(kind))
    q.view(torch.uint8).fill_(fill)
    s.view(torch.uint8).fill_(fill)
    return q, s


def _check_quant(x, kind, block, order):
    """x: a torch matrix.  Values and scales are the oracle's, to the bit but for the payload of a NaN; padding as documented."""
    import paper_2511_12056_amd as pda
    from oracle import proj
    rows, cols = x.shape
    q = _empty(rows, cols, block, kind) if order != "cols" else (None, None)
    qt = _empty(cols, rows, block, kind) if order != "rows" else (None, None)
    pda.fp8_quant(x, *q, *qt, block_rows=block)
    a = _f64(x)
    for (got, scales), want in ((q, a), (qt, a.T)):
        if got is None:
            continue
        wq, ws = proj.quantise(want, kind, block)
        assert np.array_equal(_f64(got), wq, equal_nan=True)
        s = _bytes(scales)
        assert np.array_equal(s[:, :ws.shape[1]], ws) and (s[:, ws.shape[1]:] == 0x55).all()
    return q, qt


SHAPES = [(1, 1), (1, 128), (128, 1), (3, 129), (128, 128), (130, 257), (127, 512), (500, 1000), (513, 640), (700, 77), (2, 2000), (2051, 4)]


@pytest.mark.parametrize("order", ["rows", "cols", "both"])
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("xt", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quant(rows, cols, xt, kind, block, order):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows * cols)
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=g, device="cuda"))
    _check_quant((x * torch.exp(torch.randn(1, cols, generator=g, device="cuda"))).to(getattr(torch, xt)), kind, block, order)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("xt", ["float32", "bfloat16"])
def test_quant_of_views(xt, kind, block):
    """Rows that lie apart, at any element."""
    import torch
    big = torch.randn(300, 777, device="cuda").to(getattr(torch, xt))
    for r, c in ((slice(0, 300), slice(0, 400)), (slice(3, 291), slice(4, 308)), (slice(1, 200), slice(5, 261)), (slice(0, 300, 2), slice(8, 136)), (slice(7, 8), slice(3, 6))):
        _check_quant(big[r, c], kind, block, "both")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block", [1, 128])
def test_quant_of_extreme_values(kind, block):
    """Blocks of zeros, of one value, at the border between two scales, below fp32's normal numbers, near its largest, and with what is not finite."""
    import torch
    from oracle import proj
    top = proj.FP8[kind][0]
    x = torch.randn(300, 384, device="cuda")
    x[0] = 0
    x[1, 128:256] = 0
    x[2] = -0.0
    x[3] *= 1e-38
    x[4] *= 1e-43
    x[5] *= 1e37
    x[6] = 3.4e38
    x[7, :128] = torch.clamp(x[7, :128], -1, 1)
    x[7, 3] = top / 128
    x[8, :128] = torch.clamp(x[8, :128], -1, 1)
    x[8, 3] = np.nextafter(np.float32(top / 128), np.float32(1e9)).item()
    x[9, 5] = float("nan")
    x[10, 7] = float("inf")
    x[10, 200] = -float("inf")
    x[11] = float("nan")
    x[12, 0] = float("-inf")
    x[13] = 2.0 ** -149
    if block == 128:
        x[128:256, 128:256] = 0
    _check_quant(x, kind, block, "both")


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("xt", ["bfloat16", "float32"])
def test_quant_of_every_exponent(kind, block, xt):
    """Every bf16 value: a row of 128 for each sign and exponent, so that rows have scales of their own and columns one for 128 exponents; then each row beside
    values of 2^-24 .. 2^8 times as much, which end in every place of the 8-bit type, below its normal numbers too."""
    import torch
    bits = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.uint16).view(torch.bfloat16).view(512, 128)
    x = torch.cat([bits, bits.float().mul(2.0 ** -9).bfloat16(), bits.roll(7, 0), bits.roll(3, 0)], 1)
    x[:, 128:256:5] = (bits.float() * 2.0 ** -24).bfloat16()[:, ::5]
    x[:, 384:] = torch.where(x[:, 384:].isfinite(), x[:, 384:], torch.ones_like(x[:, 384:]))
    _check_quant(x.to(getattr(torch, xt)), kind, block, "both")


def test_square_blocks_agree_in_both_orders():
    import torch
    x = torch.randn(515, 900, device="cuda")
    (q, s), (qt, st) = _check_quant(x, "e4m3", 128, "both")
    assert np.array_equal(_f64(q)[:, :900], _f64(qt)[:, :515].T) and np.array_equal(_bytes(s)[:5, :8], _bytes(st)[:8, :5].T)


def test_quant_writes_nothing_else():
    """Bytes around the results stay."""
    import torch
    import paper_2511_12056_amd as pda
    rows, cols, x = 200, 300, torch.randn(200, 300, device="cuda")
    room = torch.full((4, 400 * 512), 9, dtype=torch.uint8, device="cuda")
    q, qt = (room[i, 512:512 + r * c].view(r, c).view(torch.float8_e4m3fn) for i, (r, c) in enumerate(((200, 384), (300, 256))))
    s, st = (room[i, 512:512 + r * 4].view(r, 4).view(torch.float8_e8m0fnu) for i, r in ((2, 200), (3, 300)))
    pda.fp8_quant(x, q, s, qt, st)
    for i, n in enumerate((200 * 384, 300 * 256, 200 * 4, 300 * 4)):
        assert (room[i, :512] == 9).all() and (room[i, 512 + n:] == 9).all()


@pytest.mark.parametrize("rows,cols", [(5_000_000, 500), (400, 5_500_000)])
def test_quant_past_2_to_the_31(rows, cols):
    import torch
    import paper_2511_12056_amd as pda
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-130:, -130:] = torch.randn(130, 130, device="cuda").to(torch.bfloat16)
    q, s = pda.fp8_empty(rows, cols)
    qt, st = pda.fp8_empty(cols, rows)
    pda.fp8_quant(x, q, s, qt, st)
    r0, c0 = (rows - 130) // 128 * 128, (cols - 130) // 128 * 128
    small = x[r0:, c0:].contiguous()
    wq, ws = pda.fp8_empty(*small.shape)
    wt, wst = pda.fp8_empty(small.shape[1], small.shape[0])
    pda.fp8_quant(small, wq, ws, wt, wst)
    assert torch.equal(q[r0:, c0:].view(torch.uint8), wq.view(torch.uint8)) and torch.equal(qt[c0:, r0:].view(torch.uint8), wt.view(torch.uint8))
    n, m = wq.shape[1] // 128, wt.shape[1] // 128
    assert torch.equal(s.view(torch.uint8)[r0:, c0 // 128:c0 // 128 + n], ws.view(torch.uint8)[:, :n])
    assert torch.equal(st.view(torch.uint8)[c0:, r0 // 128:r0 // 128 + m], wst.view(torch.uint8)[:, :m])
    del x, q, qt, s, st
    torch.cuda.empty_cache()


# ---- the product

def _matrix(seed, rows, cols, kind, block, spread=1.0):
    """A random 8-bit matrix and its values in 64 bits (from the oracle's quantiser, not the library's)."""
    import torch
    from oracle import proj
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(spread * rng.standard_normal((rows, 1)))
    q, s = proj.quantise(x, kind, block)
    b = np.full((s.shape[0], proj.up(s.shape[1], 4)), 255, np.uint8)               # bytes behind the last block are not used
    b[:, :s.shape[1]] = s
    return torch.from_numpy(q).float().to(_type(kind)).cuda(), torch.from_numpy(b).cuda().view(torch.float8_e8m0fnu), proj.values(q, s, block)


def _check_matmul(M, N, K, kind="e4m3", block=128, bias=True, seed=0):
    import torch
    import paper_2511_12056_amd as pda
    from oracle import proj
    a, sa, va = _matrix(seed + M, M, K, kind, 1)
    b, sb, vb = _matrix(seed + N + 1, N, K, "e4m3", block, 0.3)
    c = torch.randn(N, device="cuda") if bias else None
    out = torch.full((M, N), float("nan"), device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a, sa, b, sb, out, bias=c)
    want, tol = proj.matmul(va, vb, None if c is None else _f64(c))
    got = _f64(out)
    assert np.isfinite(got).all()
    over = np.abs(got - want) - tol
    assert over.max() <= 0, (float(over.max()), np.unravel_index(over.argmax(), over.shape))
    again = torch.empty_like(out)
    pda.fp8_matmul(a, sa, b, sb, again, bias=c)
    assert torch.equal(out, again)


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 4, 128), (1, 300, 640), (2, 17, 1536), (5, 130, 200), (16, 64, 256), (17, 100, 384), (31, 33, 1152), (33, 256, 128), (64, 129, 896),
                                   (65, 64, 128), (100, 255, 640), (127, 1, 512), (128, 128, 128), (129, 131, 256), (200, 64, 1664), (255, 300, 384), (256, 256, 512), (257, 513, 128),
                                   (300, 30, 2048), (511, 129, 640)])
@pytest.mark.parametrize("kind,block,bias", [("e4m3", 128, True), ("e5m2", 1, False), ("e4m3", 1, True)])
def test_matmul(M, N, K, kind, block, bias):
    _check_matmul(M, N, K, kind, block, bias)


@pytest.mark.parametrize("M,N,K", [(130, 140, 16384), (70, 66, 40000), (257, 256, 24576)])
def test_matmul_with_a_long_sum(M, N, K):
    _check_matmul(M, N, K, "e5m2", 1, False)


def _quantised(M, N, K, kind, block):
    import torch
    import paper_2511_12056_amd as pda
    g = torch.Generator(device="cuda").manual_seed(M + N)
    x, w = torch.randn(M, K, generator=g, device="cuda"), torch.randn(N, K, generator=g, device="cuda")
    a, sa = pda.fp8_empty(M, K, 1, _type(kind))
    b, sb = pda.fp8_empty(N, K, block)
    pda.fp8_quant(x, a, sa)
    pda.fp8_quant(w, b, sb, block_rows=block)
    return a, sa, b, sb


def _check_on_the_gpu(out, a, sa, b, sb, block, bias=None):
    """Every result within the matrix instruction's bound (summed magnitudes over 2^13, of which eight consecutive products cannot lose more than seven eighths) and a rounding."""
    import torch
    n, N, K = a.shape[1] // 128, b.shape[0], a.shape[1]
    va = a.double() * sa.double()[:, :n].repeat_interleave(128, dim=1)
    vb = b.double() * sb.double()[:, :n].repeat_interleave(128, dim=1).repeat_interleave(block, dim=0)[:N]
    want = torch.mm(va, vb.t().contiguous())
    # seven dropped shares of the largest of eight products: at most seven times their summed magnitude over 2^13
    tol = torch.mm(va.abs(), vb.abs().t().contiguous()) * (7 * 2.0 ** -13 + K * 2.0 ** -24)
    if bias is not None:
        want = want + bias.double()
        tol = tol + 2.0 ** -24 * want.abs()
    tol = tol + 2.0 ** -8 * (want.abs() + tol)
    assert ((out.double() - want).abs() <= tol).all()
    # and on the whole no further off than a rounding to bf16 (evenly spread: 2^-8 / sqrt(3) at most) and the instruction's share together
    assert (out.double() - want).norm() <= want.norm() * 2.0 ** -8


@pytest.mark.parametrize("M,N,K,kind,block", [(3000, 4608, 1536, "e4m3", 128), (9594, 1152, 1152, "e5m2", 128), (4608, 1536, 9594, "e5m2", 1), (40000, 130, 640, "e4m3", 128),
                                              (300, 20000, 300, "e4m3", 1), (1, 8192, 8192, "e4m3", 128), (64, 6144, 4096, "e4m3", 128)])
def test_larger_matmul_against_fp64_on_the_gpu(M, N, K, kind, block):
    """More tiles than compute units, ragged ends."""
    import torch
    import paper_2511_12056_amd as pda
    a, sa, b, sb = _quantised(M, N, K, kind, block)
    out = torch.full((M, N), float("nan"), device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a, sa, b, sb, out)
    _check_on_the_gpu(out, a, sa, b, sb, block)


# every tile, alone and in parts of K, with few and many blocks of it
MIDDLE = [(700, 700, 256), (257, 1500, 300), (150, 2050, 640), (1000, 300, 1000), (500, 517, 1152), (70, 3000, 2176), (150, 3000, 8192),
          (257, 3000, 100), (500, 1030, 256), (1000, 517, 900), (257, 2050, 1024), (500, 1030, 5120), (700, 300, 3008), (33, 700, 8192), (500, 66, 8192),
          (2500, 3000, 128), (2000, 2050, 640), (2500, 2050, 1100), (1500, 2050, 2176), (1000, 2050, 2944), (2000, 517, 5120), (500, 2050, 8192),
          (2000, 2049, 200), (2000, 2051, 128), (2000, 2052, 300), (2000, 2053, 128), (2000, 2054, 200), (2000, 2055, 128), (500, 1029, 256), (500, 1031, 256)]


@pytest.mark.parametrize("M,N,K", MIDDLE)
@pytest.mark.parametrize("kind,block,gap", [("e4m3", 128, 3), ("e5m2", 1, 8)])
def test_matmul_of_middle_sizes(M, N, K, kind, block, gap):
    """With a bias, into a view whose rows lie apart, with a NaN that reaches one row and one column, twice to the same bits."""
    import torch
    import paper_2511_12056_amd as pda
    a, sa, b, sb = _quantised(M, N, K, kind, block)
    bias = torch.randn(N, device="cuda")
    whole = torch.full((M, N + gap), 7.0, device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a, sa, b, sb, whole[:, :N], bias=bias)
    _check_on_the_gpu(whole[:, :N], a, sa, b, sb, block, bias)
    assert (whole[:, N:] == 7).all()
    again = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(pda.fp8_matmul(a, sa, b, sb, again, bias=bias), whole[:, :N])
    a.view(torch.uint8)[M - 1, K - 1] = 0x7f
    b.view(torch.uint8)[N - 2, 5] = 0x7f
    got = pda.fp8_matmul(a, sa, b, sb, torch.empty_like(again), bias=bias)
    nan = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    nan[M - 1] = nan[:, N - 2] = True
    assert torch.equal(got.isnan(), nan) and torch.equal(torch.where(nan, 0, got), torch.where(nan, 0, again))


@pytest.mark.parametrize("shapes", [[(500, 2050, 8192), (33, 700, 8192)], [(70, 66, 40000), (500, 517, 1152)], [(2500, 2050, 200), (3, 40, 256)]])
def test_captured_products_that_share_a_workspace(shapes):
    """Two products one after the other in a graph, in parts of K with one workspace or none; replayed with other operands, eager work between the replays."""
    import torch
    import paper_2511_12056_amd as pda
    sets = [_quantised(M, N, K, "e4m3", 128) for M, N, K in shapes]
    others = [_quantised(M, N, K, "e4m3", 128) for M, N, K in shapes]
    for o in others:
        o[0].view(torch.uint8)[:] = o[0].view(torch.uint8).flip(0)
        o[1].view(torch.uint8)[:] = o[1].view(torch.uint8).flip(0)
    outs = [torch.empty(M, N, device="cuda", dtype=torch.bfloat16) for M, N, _ in shapes]
    space = torch.empty(max(pda.fp8_matmul_workspace_bytes(*map(int, (M, N, s[0].shape[1]))) for (M, N, _), s in zip(shapes, sets)) or 256, device="cuda", dtype=torch.uint8)
    eager = [[pda.fp8_matmul(*s, torch.empty_like(o)) for s, o in zip(group, outs)] for group in (sets, others)]
    held = [[t.clone() for t in s] for s in sets]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for s, o in zip(held, outs):
            pda.fp8_matmul(*s, o, workspace=space)
    for turn in (0, 1, 1, 0):
        for h, s in zip(held, (sets, others)[turn]):
            for a, b in zip(h, s):
                a.view(torch.uint8).copy_(b.view(torch.uint8))
        space.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, e) for o, e in zip(outs, eager[turn]))


@pytest.mark.parametrize("M", [1, 40, 300])
def test_matmul_without_k_is_the_bias(M):
    import torch
    import paper_2511_12056_amd as pda
    a, sa = pda.fp8_empty(M, 0)
    b, sb = pda.fp8_empty(70, 0)
    c = torch.randn(70, device="cuda")
    out = torch.full((M, 70), 9.0, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(pda.fp8_matmul(a, sa, b, sb, out, bias=c), c.to(torch.bfloat16).expand(M, 70))
    assert not pda.fp8_matmul(a, sa, b, sb, out).any()


@pytest.mark.parametrize("M,N,K", [(1, 37, 256), (20, 100, 256), (90, 130, 1280), (300, 257, 128)])
@pytest.mark.parametrize("gap", [1, 3, 8])
def test_matmul_into_views(M, N, K, gap):
    """Rows of the result that lie apart, even or odd: what is between them stays."""
    import torch
    import paper_2511_12056_amd as pda
    a, sa, _ = _matrix(1, M, K, "e4m3", 1)
    b, sb, _ = _matrix(2, N, K, "e4m3", 128)
    whole = torch.full((M, N + gap), 7.0, device="cuda", dtype=torch.bfloat16)
    out = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a, sa, b, sb, out)
    pda.fp8_matmul(a, sa, b, sb, whole[:, :N])
    assert torch.equal(whole[:, :N], out) and (whole[:, N:] == 7).all()


@pytest.mark.parametrize("M", [1, 50, 140, 300])
def test_rows_of_a_and_blocks_of_b_are_matrices_themselves(M):
    import torch
    import paper_2511_12056_amd as pda
    a, sa, _ = _matrix(3, M, 640, "e4m3", 1)
    b, sb, _ = _matrix(4, 384, 640, "e4m3", 128)
    out = torch.empty(M, 384, device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a, sa, b, sb, out)
    part = torch.empty(M, 256, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(pda.fp8_matmul(a, sa, b[128:], sb[1:], part), out[:, 128:])
    one = torch.empty(1, 384, device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a[M - 1:], sa[M - 1:], b, sb, one)
    assert (one - out[M - 1:]).abs().max() <= 2 ** -7 * out[M - 1:].abs().max()


@pytest.mark.parametrize("M,N,K", [(3, 40, 256), (40, 200, 512), (150, 140, 1024), (300, 300, 384)])
def test_what_is_not_finite_and_extreme_scales(M, N, K):
    """A NaN (in a value or a scale) reaches the results that it is part of and no other; scales far apart cancel."""
    import torch
    import paper_2511_12056_amd as pda
    a, sa, va = _matrix(5, M, K, "e5m2", 1)
    b, sb, vb = _matrix(6, N, K, "e4m3", 1)
    clean = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a, sa, b, sb, clean)
    a.view(torch.uint8)[1, 77] = 0x7F                              # NaN
    a.view(torch.uint8)[2, K - 1] = 0x7C                           # infinity
    b.view(torch.uint8)[2, K - 1] = 0x38                           # times one
    sb.view(torch.uint8)[N - 1, 1] = 255
    out = torch.empty_like(clean)
    pda.fp8_matmul(a, sa, b, sb, out)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[1], bad[2], bad[:, N - 1], bad[:, 2] = True, True, True, True
    assert out[1].isnan().all() and out[:, N - 1].isnan().all() and out[2, 2].isinf() and not out[2, :N - 1].isfinite().any()
    assert torch.equal(out[~bad], clean[~bad])
    n = K // 128
    a, sa, _ = _matrix(5, M, K, "e5m2", 1)
    b, sb, _ = _matrix(6, N, K, "e4m3", 1)
    up, down = sa.view(torch.uint8).clone(), sb.view(torch.uint8).clone()
    up[:, :n] += 90
    down[:, :n] -= 90
    pda.fp8_matmul(a, up.view(torch.float8_e8m0fnu), b, down.view(torch.float8_e8m0fnu), out)
    assert torch.equal(out, clean)


def test_offsets_past_2_to_the_31():
    """Rows of a and of the result beyond 2^31 bytes and elements."""
    import torch
    import paper_2511_12056_amd as pda
    M, N, K = 1_500_000, 1536, 1536
    a, sa = pda.fp8_empty(M, K)
    a.view(torch.uint8).fill_(0)
    sa.view(torch.uint8).fill_(127)
    last = torch.randn(300, K, device="cuda")
    pda.fp8_quant(last, a[M - 300:], sa[M - 300:])
    b, sb = pda.fp8_empty(N, K, 128)
    pda.fp8_quant(torch.randn(N, K, device="cuda"), b, sb, block_rows=128)
    out = torch.full((M, N), 3.0, device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a, sa, b, sb, out)
    small = torch.empty(300, N, device="cuda", dtype=torch.bfloat16)
    pda.fp8_matmul(a[M - 300:], sa[M - 300:], b, sb, small)
    assert (out[M - 300:] - small).abs().max() <= 2 ** -7 * small.abs().max() and not out[:M - 300:997].any()
    del a, out
    torch.cuda.empty_cache()


def test_refusals_of_the_wrappers():
    import torch
    import paper_2511_12056_amd as pda
    a, sa, _ = _matrix(1, 70, 256, "e4m3", 1)
    b, sb, _ = _matrix(2, 130, 256, "e4m3", 128)
    out = torch.empty(70, 130, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(70, 256, device="cuda")
    bad = [lambda: pda.fp8_matmul(a, sa, b[:, :128].contiguous(), sb, out), lambda: pda.fp8_matmul(a, sa[:, :2], b, sb, out), lambda: pda.fp8_matmul(a, None, b, sb, out),
           lambda: pda.fp8_matmul(a, sa, b.view(torch.float8_e5m2), sb, out), lambda: pda.fp8_matmul(a, sa, b, sb, out.float()), lambda: pda.fp8_matmul(a, sa, b, sb, out.t()),
           lambda: pda.fp8_matmul(a, sa, b, sb, out, bias=torch.zeros(129, device="cuda")), lambda: pda.fp8_matmul(a, sa.view(torch.uint8), b, sb, out),
           lambda: pda.fp8_quant(x), lambda: pda.fp8_quant(x, a), lambda: pda.fp8_quant(x, a, sa, block_rows=64), lambda: pda.fp8_quant(x.t(), a, sa), lambda: pda.fp8_quant(x[:, :200], a[:, :200], sa),
           lambda: pda.fp8_quant(x.half(), a, sa), lambda: pda.fp8_quant(x, a, sa, *pda.fp8_empty(256, 70, 1, torch.float8_e5m2)), lambda: pda.fp8_quant(x, None, sa, *pda.fp8_empty(256, 70))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    M, N, K = 4608, 1536, 119056
    big = torch.empty(M, N, device="cuda", dtype=torch.bfloat16)
    (p, sp), (q, sq) = pda.fp8_empty(M, K), pda.fp8_empty(N, K)
    with pytest.raises(pda.PdaError, match="workspace"):
        pda.fp8_matmul(p, sp, q, sq, big, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))

"""GPU parity of pda_attn_bwd with the fp64 oracle, element by element within the bound that follows from the number formats
(oracle/train.py), and what a call may and may not touch."""
import numpy as np
import pytest

from synth import to_dev_bf16
from synth.inputs import bf16_bits_to_f32, f32_to_bf16_bits

pytestmark = pytest.mark.gpu


def _bf16(rng, *shape, scale=1.0):
    """bf16 payloads and their values."""
    bits = f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))
    return bits, bf16_bits_to_f32(bits).astype(np.float64)


def _forward(q, k, v, scale, n_v):
    B, H, Sq, d = q.shape
    out, lse = np.zeros((B, H, Sq, d)), np.full((B, H, Sq), -np.inf)
    if n_v and Sq:
        for b in range(B):
            for h in range(H):
                s = scale * q[b, h] @ k[b, h, :n_v].T
                top = s.max(-1, keepdims=True)
                e = np.exp(s - top)
                lse[b, h] = (top + np.log(e.sum(-1, keepdims=True)))[:, 0]
                out[b, h] = e @ v[b, h, :n_v] / e.sum(-1, keepdims=True)
    return out, lse


class Problem:
    def __init__(self, seed, B, H, Sq, Skv, d, n_v, out_type="fp32", scale=None, spread=1.0):
        import torch
        rng = np.random.default_rng(seed)
        self.scale = d ** -0.5 if scale is None else scale
        self.n_v, self.sizes = n_v, (B, H, Sq, Skv, d)
        qb, q = _bf16(rng, B, H, Sq, d, scale=spread)
        kb, k = _bf16(rng, B, H, Skv, d, scale=spread)
        vb, v = _bf16(rng, B, H, Skv, d)
        gb, g = _bf16(rng, B, H, Sq, d)
        if n_v < Skv:                                # hidden rows of k and v are never read
            kb, vb = kb.copy(), vb.copy()
            kb[:, :, n_v:], vb[:, :, n_v:] = 0x7FC0, 0x7F80
        out, lse = _forward(q, k, v, self.scale, n_v)
        lse = lse.astype(np.float32)
        ob = f32_to_bf16_bits(out.astype(np.float32))
        self.q, self.k, self.v, self.dout = (to_dev_bf16(x) for x in (qb, kb, vb, gb))
        self.out = torch.from_numpy(out.astype(np.float32)).cuda() if out_type == "fp32" else to_dev_bf16(ob)
        self.lse = torch.from_numpy(lse).cuda()
        self.host = (g, q, k, v, out.astype(np.float32).astype(np.float64) if out_type == "fp32" else bf16_bits_to_f32(ob).astype(np.float64),
                     lse.astype(np.float64))

    def grads(self):
        import torch
        return torch.full_like(self.q, float("nan")), torch.full_like(self.k, float("nan")), torch.full_like(self.v, float("nan"))

    def run(self, **kw):
        import torch
        import paper_2511_12056_amd as pda
        got = pda.attn_bwd(self.dout, self.q, self.k, self.v, self.out, self.lse, *self.grads(), self.scale, self.n_v, **kw)
        torch.cuda.synchronize()
        return got

    def check(self, got):
        from oracle.train import attention_bwd
        want, tol = attention_bwd(*self.host, self.scale, self.n_v)
        for name, x, w, t in zip(("dq", "dk", "dv"), got, want, tol):
            x = x.float().cpu().numpy().astype(np.float64)
            assert np.isfinite(x).all(), name
            over = np.abs(x - w) - t
            assert over.size == 0 or over.max() <= 0, (name, self.sizes, float(over.max()), np.unravel_index(over.argmax(), over.shape))
            if w.size and np.abs(w).max() > 0:       # the bound is for the worst case; as a whole the error is that of a few roundings
                assert np.linalg.norm(x - w) <= 8e-3 * np.linalg.norm(w), name


SIZES = [   # B, H, Sq, Skv, n_v
    (1, 1, 1, 1, 1), (1, 2, 1, 70, 70), (1, 2, 70, 1, 1), (2, 1, 31, 33, 33), (1, 1, 32, 32, 32), (1, 2, 33, 31, 30), (1, 1, 64, 64, 64),
    (1, 1, 65, 127, 127), (1, 3, 128, 128, 128), (2, 2, 129, 255, 250), (1, 1, 255, 257, 256), (1, 2, 256, 256, 193), (1, 1, 300, 513, 512),
    (2, 3, 257, 100, 97), (1, 1, 17, 1025, 1000), (1, 1, 1023, 40, 33), (1, 5, 640, 320, 320), (1, 1, 2049, 1100, 1090),
]


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(size, d):
    p = Problem(sum(size) + d, *size[:4], d, size[4], out_type="bf16" if sum(size) % 2 else "fp32")
    p.check(p.run())


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("Sq,Skv,n_v", [(5, 300, 0), (0, 300, 200), (0, 5, 0), (70, 0, 0)])
def test_empty(Sq, Skv, n_v, d):
    p = Problem(1, 1, 2, Sq, Skv, d, n_v)
    for x in p.run():
        assert (x == 0).all()


@pytest.mark.parametrize("d", [128, 64])
def test_rows_without_keys_give_nothing(d):
    """A row whose log-sum-exp is -inf has no probabilities, whatever its scores; the others keep theirs."""
    import torch
    p = Problem(2, 1, 2, 300, 200, d, 190)
    p.lse[0, 0, ::3] = -float("inf")
    p.lse[0, 1, :] = -float("inf")
    p.host = p.host[:5] + (p.lse.cpu().numpy().astype(np.float64),)
    got = p.run()
    p.check(got)
    assert (got[0][0, 0, ::3] == 0).all() and all((x[0, 1] == 0).all() for x in got)
    assert torch.isfinite(got[1]).all()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("scale,spread", [(0.0, 1.0), (0.125, 6.0), (1.0, 2.0), (0.6931471805599453, 0.4)])
def test_scales(scale, spread, d):
    """Flat, peaked (probabilities next to one and far below), and the scores of pda_attn_fwd_base2 (scale ln 2)."""
    p = Problem(3, 1, 2, 200, 300, d, 290, scale=scale, spread=spread)
    from oracle.train import attention_bwd
    got = p.run()
    want, tol = attention_bwd(*p.host, float(np.float32(scale)), p.n_v)
    for x, w, t in zip(got, want, tol):
        x = x.float().cpu().numpy()
        assert np.isfinite(x).all() and (np.abs(x - w) <= t).all()


@pytest.mark.parametrize("d", [128, 64])
def test_equal_calls_give_equal_bits(d):
    import torch
    p = Problem(4, 2, 3, 700, 900, d, 890)
    first = [x.clone() for x in p.run()]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, p.run()))


@pytest.mark.parametrize("d", [128, 64])
def test_memory_around_the_results_is_left_alone(d):
    """Views inside larger tensors: heads 1..2 of 4, rows 5.. of longer sequences, all surroundings kept."""
    import torch
    import paper_2511_12056_amd as pda
    B, H, Sq, Skv, n_v = 2, 2, 133, 90, 77
    p = Problem(5, B, H, Sq, Skv, d, n_v, out_type="bf16")
    want = p.run()

    def inside(x, rows, fill):
        big = torch.full((B, 4, x.shape[2] + rows, *x.shape[3:]), fill, device="cuda", dtype=x.dtype)
        view = big[:, 1:3, 5:5 + x.shape[2]]
        view.copy_(x)
        return big, view

    views = {n: inside(getattr(p, n), 9, float("nan"))[1] for n in ("q", "dout", "out", "lse")}
    views.update({n: inside(getattr(p, n), 13, float("nan"))[1] for n in ("k", "v")})
    big_q, dq = inside(p.q, 11, 7.0)
    (big_k, dk), (big_v, dv) = inside(p.k, 6, 7.0), inside(p.v, 6, 7.0)
    pda.attn_bwd_strided(views["dout"], views["q"], views["k"], views["v"], views["out"], views["lse"], dq, dk, dv, p.scale, n_v)
    torch.cuda.synchronize()
    for got, ref, big in zip((dq, dk, dv), want, (big_q, big_k, big_v)):
        assert torch.equal(got, ref)
        got.fill_(7.0)
        assert (big == 7.0).all()


def test_workspace_is_enough_and_not_exceeded():
    import torch
    import paper_2511_12056_amd as pda
    for d, size in ((64, (1, 2, 1000, 1030)), (128, (2, 2, 130, 700)), (128, (1, 1, 9000, 40))):
        p = Problem(6, *size, d, size[3])
        want = p.run()
        n = pda.attn_bwd_workspace_bytes(*size, d)
        ws = torch.full((n + 4096,), 0xA5, device="cuda", dtype=torch.uint8)
        got = p.run(workspace=ws[:n])
        assert (ws[n:] == 0xA5).all() and all(torch.equal(a, b) for a, b in zip(got, want))
        with pytest.raises(pda.PdaError) as e:
            p.run(workspace=ws[:n - 256])
        assert e.value.code == 1


def test_shares_of_the_keys_and_of_the_queries():
    """Key chunks with the merged out and lse: each has its exact dk and dv, their dq add up.  Query ranges: the other way round."""
    import torch
    import paper_2511_12056_amd as pda
    from oracle.train import attention_bwd
    p = Problem(7, 1, 2, 500, 600, 128, 600)
    want, tol = attention_bwd(*p.host, p.scale, 600)
    dq, dk, dv = p.grads()
    total = torch.zeros_like(dq, dtype=torch.float32)
    for a, b in ((0, 100), (100, 164), (164, 600)):
        part = torch.empty_like(dq)
        pda.attn_bwd_strided(p.dout, p.q, p.k[:, :, a:b], p.v[:, :, a:b], p.out, p.lse, part, dk[:, :, a:b], dv[:, :, a:b], p.scale)
        total += part.float()
    torch.cuda.synchronize()
    # dk and dv as in one call; the sum of dq holds a rounding of every share
    for x, w, t in zip((dk, dv), want[1:], tol[1:]):
        assert (np.abs(x.float().cpu().numpy() - w) <= t).all()
    x = total.cpu().numpy()
    assert np.linalg.norm(x - want[0]) <= 8e-3 * np.linalg.norm(want[0])
    tk, tv = torch.zeros_like(dk, dtype=torch.float32), torch.zeros_like(dv, dtype=torch.float32)
    for a, b in ((0, 33), (33, 500)):
        pk, pv = torch.empty_like(dk), torch.empty_like(dv)
        s = slice(a, b)
        pda.attn_bwd_strided(p.dout[:, :, s], p.q[:, :, s], p.k, p.v, p.out[:, :, s], p.lse[:, :, s], dq[:, :, s], pk, pv, p.scale)
        tk += pk.float()
        tv += pv.float()
    torch.cuda.synchronize()
    assert (np.abs(dq.float().cpu().numpy() - want[0]) <= tol[0]).all()
    for x, w in ((tk, want[1]), (tv, want[2])):
        assert np.linalg.norm(x.cpu().numpy() - w) <= 8e-3 * np.linalg.norm(w)


def test_another_stream_and_no_workspace_given():
    import torch
    import paper_2511_12056_amd as pda
    p = Problem(8, 1, 2, 400, 500, 64, 480)
    want = p.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    grads = p.grads()
    side.wait_stream(torch.cuda.current_stream())
    pda.attn_bwd(p.dout, p.q, p.k, p.v, p.out, p.lse, *grads, p.scale, p.n_v, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(grads, want))


@pytest.mark.parametrize("d,size", [(64, (1, 2, 1024, 1024)), (128, (1, 3, 300, 900))])
def test_graph_capture(d, size):
    """Captured without a call before it, replayed with other inputs in the same buffers and eager work in between."""
    import torch
    import paper_2511_12056_amd as pda
    a, b = Problem(9, *size, d, size[3] - 5), Problem(10, *size, d, size[3] - 5)
    want = [[x.clone() for x in p.run()] for p in (a, b)]
    ws = pda.attn_bwd_workspace(*size, d)
    grads = a.grads()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pda.attn_bwd(a.dout, a.q, a.k, a.v, a.out, a.lse, *grads, a.scale, a.n_v, workspace=ws)
    kept = {n: getattr(a, n).clone() for n in ("dout", "q", "k", "v", "out", "lse")}
    for rep in range(4):
        src = kept if rep % 2 == 0 else {n: getattr(b, n) for n in kept}
        for n, x in src.items():
            getattr(a, n).copy_(x)
        for x in grads:
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(grads, want[rep % 2])), rep
        b.run()                                     # eager work between the replays, on a workspace of its own


def test_long_sequence_against_64_bits_on_the_gpu():
    """Many tiles, more work items than compute units, a masked tail that ends inside a tile."""
    import torch
    import paper_2511_12056_amd as pda
    g = torch.Generator(device="cuda").manual_seed(11)
    for d, H, Sq, Skv, n_v in ((128, 2, 9600, 9001, 8977), (64, 3, 5003, 12100, 12033)):
        q, k, v, dout = (torch.randn(1, H, n, d, generator=g, device="cuda").to(torch.bfloat16) for n in (Sq, Skv, Skv, Sq))
        out, lse = torch.empty(1, H, Sq, d, device="cuda", dtype=torch.bfloat16), torch.empty(1, H, Sq, device="cuda")
        scale = d ** -0.5
        pda.attn_fwd_bf16out(q, k, v, out, lse, scale, n_v)
        got = pda.attn_bwd(dout, q, k, v, out, lse, torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), scale, n_v)
        for h in range(H):
            Q, K, V, G = (x[0, h].double() for x in (q, k[:, :, :n_v], v[:, :, :n_v], dout))
            p = torch.softmax(scale * torch.mm(Q, K.t()), dim=-1)
            dp = torch.mm(G, V.t())
            ds = p * (dp - (p * dp).sum(-1, keepdim=True))
            for x, w in zip(got, (scale * torch.mm(ds, K), scale * torch.mm(ds.t(), Q), torch.mm(p.t(), G))):
                x = x[0, h, :w.shape[0]].double()
                # three independent roundings of 2^-9 rms at most (operand, result, out in delta): below 2^-8 sqrt(3)
                assert (x - w).norm() <= 2.0 ** -8 * 3 ** 0.5 * w.norm()
            assert all((x[0, h, n_v:] == 0).all() for x in got[1:])


def _near_64_bits(got, dout, q, k, v, scale, n_v):
    """One head: the gradients of the formulas in 64 bits on the GPU, within the roundings that pass through whole rows."""
    import torch
    Q, K, V, G = (x.double() for x in (q, k[:n_v], v[:n_v], dout))
    p = torch.softmax(scale * torch.mm(Q, K.t()), dim=-1)
    dp = torch.mm(G, V.t())
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    for x, w in zip(got, (scale * torch.mm(ds, K), scale * torch.mm(ds.t(), Q), torch.mm(p.t(), G))):
        # three independent roundings of 2^-9 rms at most (operand, result, out in delta): below 2^-8 sqrt(3)
        assert (x[:w.shape[0]].double() - w).norm() <= 2.0 ** -8 * 3 ** 0.5 * w.norm()
    assert all((x[n_v:] == 0).all() for x in got[1:])


def _forward_call(B, H, Sq, Skv, d, n_v, seed):
    import torch
    import paper_2511_12056_amd as pda
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v, dout = (torch.randn(B, H, n, d, generator=g, device="cuda").to(torch.bfloat16) for n in (Sq, Skv, Skv, Sq))
    out, lse = torch.empty(B, H, Sq, d, device="cuda"), torch.empty(B, H, Sq, device="cuda")
    pda.attn_fwd(q, k, v, out, lse, d ** -0.5, n_v)
    return dout, q, k, v, out, lse


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("size", [
    (1, 10, 9000, 600, 570),         # key blocks cut, query blocks whole
    (1, 12, 3000, 3000, 2990),       # more blocks than compute units, the last query blocks cut
    (2, 3, 400, 1500, 100),          # blocks of hidden keys only
    (1, 1, 4100, 4100, 4033),        # one round, all blocks cut
    (1, 40, 2049, 1025, 1025),       # blocks with one live row
    (3, 30, 1600, 40, 33),           # many heads, two tiles of keys
], ids=str)
def test_forms_of_a_launch(size, d):
    import torch
    import paper_2511_12056_amd as pda
    B, H, Sq, Skv, n_v = size
    x = _forward_call(B, H, Sq, Skv, d, n_v, sum(size))
    got = pda.attn_bwd(*x, *(torch.full_like(t, float("nan")) for t in x[1:4]), d ** -0.5, n_v)
    for b, h in {(0, 0), (B - 1, H - 1), (B // 2, H // 3), (0, H // 2)}:
        _near_64_bits([t[b, h] for t in got], *(t[b, h] for t in x[:4]), d ** -0.5, n_v)
    assert all(torch.isfinite(t).all() for t in got)


@pytest.mark.parametrize("d", [128, 64])
def test_two_calls_at_once(d):
    """Two streams, a workspace each, several calls on both."""
    import torch
    import paper_2511_12056_amd as pda
    sizes = ((1, 4, 2500, 2500, d, 2400), (1, 2, 1111, 5000, d, 5000))
    xs = [_forward_call(*s, seed=i) for i, s in enumerate(sizes)]
    want = [[t.clone() for t in pda.attn_bwd(*x, *map(torch.empty_like, x[1:4]), d ** -0.5, s[5])] for x, s in zip(xs, sizes)]
    ws = [pda.attn_bwd_workspace(*s) for s in sizes]
    grads = [[[torch.empty_like(t) for t in x[1:4]] for _ in range(4)] for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for rep in range(4):
        for i in (0, 1):
            pda.attn_bwd(*xs[i], *grads[i][rep], d ** -0.5, sizes[i][5], workspace=ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in (0, 1):
        for rep in range(4):
            assert all(torch.equal(a, b) for a, b in zip(grads[i][rep], want[i])), (i, rep)


def test_two_graphs_share_a_workspace():
    """Replayed one after the other on one stream; the workspace keeps nothing from call to call."""
    import torch
    import paper_2511_12056_amd as pda
    sizes = ((1, 2, 1500, 1400, 64, 1390), (1, 3, 700, 900, 128, 900))
    xs = [_forward_call(*s, seed=i) for i, s in enumerate(sizes)]
    want = [[t.clone() for t in pda.attn_bwd(*x, *map(torch.empty_like, x[1:4]), s[4] ** -0.5, s[5])] for x, s in zip(xs, sizes)]
    ws = torch.empty(max(pda.attn_bwd_workspace_bytes(*s) for s in sizes), dtype=torch.uint8, device="cuda")
    grads = [[torch.empty_like(t) for t in x[1:4]] for x in xs]
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    torch.cuda.synchronize()
    for g, x, to, s in zip(graphs, xs, grads, sizes):
        with torch.cuda.graph(g):
            pda.attn_bwd(*x, *to, s[4] ** -0.5, s[5], workspace=ws)
    for rep in range(3):
        for to in grads:
            for t in to:
                t.fill_(float("nan"))
        ws.fill_(0xFF)                              # NaN in every float
        for i in (rep % 2, 1 - rep % 2):
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(a, b) for a, b in zip(grads[i], want[i])), (rep, i)


@pytest.mark.parametrize("d", [128, 64])
def test_heads_that_share_keys(d):
    """k and v of one head for all heads (stride 0): every head's own dk and dv, whose sums are the shared tensor's gradients."""
    import torch
    import paper_2511_12056_amd as pda
    dout, q, k, v, out, lse = _forward_call(2, 3, 333, 210, d, 200, 5)
    k, v = (t[:, :1].clone() for t in (k, v))
    kk, vv = (t.expand(2, 3, 210, d).contiguous() for t in (k, v))
    pda.attn_fwd(q, kk, vv, out, lse, d ** -0.5, 200)
    want = pda.attn_bwd(dout, q, kk, vv, out, lse, *map(torch.empty_like, (q, kk, vv)), d ** -0.5, 200)
    got = pda.attn_bwd_strided(dout, q, k.expand(2, 3, 210, d), v.expand(2, 3, 210, d), out, lse, *map(torch.empty_like, (q, kk, vv)), d ** -0.5, 200)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("d", [128, 64])
def test_offsets_beyond_32_bits(d):
    """Heads 2^32 bytes and more apart, in one allocation for all tensors."""
    import torch
    import paper_2511_12056_amd as pda
    S, n_v = 200, 190
    x = _forward_call(1, 2, S, S, d, n_v, 6)
    want = pda.attn_bwd(*x, *(torch.empty_like(t) for t in x[1:4]), d ** -0.5, n_v)
    far = (1 << 31) + 64 * d                                     # elements
    big = torch.empty(far + 16 * S * d, device="cuda", dtype=torch.bfloat16)

    def at(i):
        return torch.as_strided(big, (1, 2, S, d), (far, far, d, 1), i * S * d)
    views = []
    for i, t in enumerate(x[:4]):
        views.append(at(i).copy_(t))
    grads = [at(4 + i) for i in range(3)]
    bigf = torch.empty(far + 3 * S * d, device="cuda")
    out = torch.as_strided(bigf, (1, 2, S, d), (far, far, d, 1), 0).copy_(x[4])
    lse = torch.as_strided(bigf, (1, 2, S), (far, far, 1), S * d).copy_(x[5])
    pda.attn_bwd_strided(*views, out, lse, *grads, d ** -0.5, n_v)
    assert all(torch.equal(a, b) for a, b in zip(grads, want))


@pytest.mark.parametrize("d", [128, 64])
def test_out_of_rows_without_keys_is_not_used(d):
    import torch
    p = Problem(12, 1, 2, 130, 200, d, 190)
    p.lse[0, :, 5::7] = -float("inf")
    want = [x.clone() for x in p.run()]
    p.out[0, :, 5::14] = float("nan")
    p.out[0, :, 12::14] = float("inf")
    got = p.run()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (got[0][0, :, 5::7] == 0).all()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,Sq,Skv,n_v", [(2, 40_001, 40_100, 0), (2, 5, 80_001, 3), (1, 0, 70_000, 0), (20_000, 1, 2, 1)])
def test_more_items_than_compute_units_with_little_to_do(H, Sq, Skv, n_v, d):
    """No keys, hidden keys only, no rows, one row and key a head."""
    import torch
    import paper_2511_12056_amd as pda
    g = torch.Generator(device="cuda").manual_seed(H)
    q, k, v, dout = (torch.randn(1, H, n, d, generator=g, device="cuda").to(torch.bfloat16) for n in (Sq, Skv, Skv, Sq))
    out, lse = torch.zeros(1, H, Sq, d, device="cuda"), torch.full((1, H, Sq), -float("inf"), device="cuda")
    if n_v == 1:
        out.copy_(v[:, :, :1])
        lse.copy_((q.double() * k[:, :, :1].double()).sum(-1) * d ** -0.5)
    elif n_v and Sq:
        pda.attn_fwd(q, k, v, out, lse, d ** -0.5, n_v)
    dq, dk, dv = pda.attn_bwd(dout, q, k, v, out, lse, *(torch.full_like(t, float("nan")) for t in (q, k, v)), d ** -0.5, n_v)
    assert (dk[:, :, n_v:] == 0).all() and (dv[:, :, n_v:] == 0).all()
    if n_v == 0:
        assert (dq == 0).all()
    elif n_v == 1:                                   # one key: p = 1; ds = 0 up to the fp32 rounding of <dout, v> and <dout, out>, d additions each
        assert torch.equal(dv[:, :, :1], dout)
        mag = (dout.double() * v[:, :, :1].double()).abs().sum(-1, keepdim=True)
        for x, w in ((dq, k[:, :, :1]), (dk[:, :, :1], q)):
            assert (x.double().abs() <= 2.0 ** -21 * d * mag * w.double().abs() * d ** -0.5).all()
    else:
        for h in range(H):
            _near_64_bits([t[0, h] for t in (dq, dk, dv)], dout[0, h], q[0, h], k[0, h], v[0, h], d ** -0.5, n_v)


def test_inputs_may_be_one_tensor():
    import torch
    import paper_2511_12056_amd as pda
    for d in (64, 128):
        x = torch.randn(1, 3, 700, d, generator=torch.Generator(device="cuda").manual_seed(d), device="cuda").to(torch.bfloat16)
        out, lse = torch.empty_like(x), torch.empty(1, 3, 700, device="cuda")
        pda.attn_fwd_bf16out(x, x, x, out, lse, d ** -0.5)
        got = pda.attn_bwd(x, x, x, x, out, lse, *(torch.empty_like(x) for _ in range(3)), d ** -0.5)
        want = pda.attn_bwd(*(x.clone() for _ in range(4)), out, lse, *(torch.empty_like(x) for _ in range(3)), d ** -0.5)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("d", [128, 64])
def test_log_sum_exps_far_off(d):
    """Rows with lse = inf, or so large that no probability is left, give nothing; far from zero the probabilities keep their accuracy."""
    import torch
    p = Problem(13, 1, 2, 200, 260, d, 250)
    want = [x.clone() for x in p.run()]
    lse = p.lse.clone()
    p.lse[0, 0, 3::5] = float("inf")
    p.lse[0, 0, 4::5] = 1e6
    got = p.run()
    assert (got[0][0, 0, 3::5] == 0).all() and (got[0][0, 0, 4::5] == 0).all()
    assert torch.equal(got[0][0, 0, 0::5], want[0][0, 0, 0::5]) and all(torch.equal(a[0, 1], b[0, 1]) for a, b in zip(got, want))
    assert all(torch.isfinite(x).all() for x in got)
    # one more column in q and k that adds the same to every score of a row: lse moves by up to 500, the probabilities stay
    p.lse.copy_(lse)
    p.q[..., d - 1] = torch.linspace(-16, 16, 200, device="cuda").to(torch.bfloat16)
    p.k[..., d - 1] = 32.0 * (d ** 0.5 / 8)
    q, k, v = (x.double() for x in (p.q, p.k[:, :, :250], p.v[:, :, :250]))
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()) * p.scale
    p.lse.copy_(torch.logsumexp(s, -1))
    p.out.copy_(torch.matmul(torch.softmax(s, -1), v))
    assert p.lse.abs().max() > 50
    got = p.run()
    for h in (0, 1):
        Q, K, V, G = q[0, h], k[0, h], v[0, h], p.dout[0, h].double()
        pr = torch.softmax(s[0, h], -1)
        dp = torch.mm(G, V.t().contiguous())
        ds = pr * (dp - (pr * dp).sum(-1, keepdim=True))
        # the bound of _near_64_bits, and 2^-22 |lse| for the exponents' rounding, which is far below it
        for x, w in zip(got[1:], (p.scale * torch.mm(ds.t().contiguous(), Q), torch.mm(pr.t().contiguous(), G))):
            assert (x[0, h, :250].double() - w).norm() <= 2.0 ** -8 * 3 ** 0.5 * w.norm()

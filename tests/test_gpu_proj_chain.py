"""The operators between the residual stream and the attention call in a run, as one attention half of a transformer block uses them, forward and backward: against
the same chain in 64 bits, captured into a graph, and on another stream."""
import pytest

pytestmark = pytest.mark.gpu

B, S, H, d, D, EPS = 2, 300, 3, 64, 200, 1e-6
HD = H * d


class Block:
    """Weights, buffers and the calls of a step."""

    def __init__(self, seed):
        import torch
        import paper_2511_12056_amd as pda
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        rows = B * S
        self.res, self.x = 2 * n(rows, D), n(rows, D).to(torch.bfloat16)
        self.norm, self.W, self.bias = 1 + 0.2 * n(B, D), n(3 * HD, D) * D ** -0.5, 0.1 * n(3 * HD)
        self.dout, self.dres = n(B, H, S, d).to(torch.bfloat16), n(rows, D)
        self.rope, self.still = pda.Rope(pda.rope_frequencies(16)[0], "half", [6, 5, 5]), pda.Rope([])
        s = torch.arange(S, device="cuda")
        self.positions = torch.stack([s // 30, s // 6 % 5, s % 6], dim=-1).int()
        e = lambda *sh, t=torch.float32: torch.empty(*sh, device="cuda", dtype=t)  # noqa: E731
        b16 = torch.bfloat16
        self.h, self.rstd = e(rows, D), e(rows)
        self.y, self.ys = pda.fp8_empty(rows, D)
        (self.w, self.ws), (self.wt, self.wts) = pda.fp8_empty(3 * HD, D, 128), pda.fp8_empty(D, 3 * HD, 128)
        self.qkv = e(rows, 3 * HD, t=b16)
        self.q, self.k, self.v, self.dq, self.dk, self.dv = (e(B, H, S, d, t=b16) for _ in range(6))
        self.out, self.lse = e(B, H, S, d, t=b16), e(B, H, S)
        self.dqkv = e(rows, 3 * HD, t=b16)
        (self.g, self.gs), (self.gt, self.gts) = pda.fp8_empty(rows, 3 * HD), pda.fp8_empty(3 * HD, rows)
        self.yt, self.yts = pda.fp8_empty(D, rows)
        self.yf = e(rows, D, t=b16)
        self.dy, self.dW = e(rows, D, t=b16), e(3 * HD, D, t=b16)
        self.dh, self.dnorm = e(rows, D), e(B, D)
        self.space = [pda.fp8_matmul_workspace(rows, 3 * HD, D), pda.fp8_matmul_workspace(rows, D, 3 * HD), pda.fp8_matmul_workspace(3 * HD, D, rows),
                      pda.attn_bwd_workspace(B, H, S, S, d), pda.rms_norm_bwd_workspace(rows, D, B)]

    def step(self, stream=None):
        import paper_2511_12056_amd as pda
        at = {"stream": stream}
        thirds = lambda t: [t.view(B, S, 3, H, d)[:, :, i] for i in range(3)]  # noqa: E731
        pda.fp8_quant(self.W, self.w, self.ws, self.wt, self.wts, block_rows=128, **at)
        pda.rms_norm_fwd(self.x, self.norm, self.y, res=self.res, h=self.h, y_scales=self.ys, rstd=self.rstd, eps=EPS, **at)
        pda.fp8_matmul(self.y, self.ys, self.w, self.ws, self.qkv, bias=self.bias, workspace=self.space[0], **at)
        tq, tk, tv = thirds(self.qkv)
        pda.pack_heads_rope(tq, self.q, self.rope, positions=self.positions, unit_rms=True, **at)
        pda.pack_heads_rope(tk, self.k, self.rope, positions=self.positions, unit_rms=True, **at)
        pda.pack_heads_rope(tv, self.v, self.still, **at)
        pda.attn_fwd_bf16out(self.q, self.k, self.v, self.out, self.lse, d ** -0.5, **at)
        pda.attn_bwd(self.dout, self.q, self.k, self.v, self.out, self.lse, self.dq, self.dk, self.dv, d ** -0.5, workspace=self.space[3], **at)
        gq, gk, gv = thirds(self.dqkv)
        pda.pack_heads_rope_bwd(self.dq, tq, gq, self.rope, positions=self.positions, unit_rms=True, **at)
        pda.pack_heads_rope_bwd(self.dk, tk, gk, self.rope, positions=self.positions, unit_rms=True, **at)
        pda.pack_heads_rope_bwd(self.dv, None, gv, self.still, **at)
        pda.fp8_quant(self.dqkv, self.g, self.gs, self.gt, self.gts, **at)
        pda.fp8_matmul(self.g, self.gs, self.wt, self.wts, self.dy, workspace=self.space[1], **at)
        pda.rms_norm_fwd(self.h, self.norm, self.yf, eps=EPS, **at)          # the norm's result again, for its columns' blocks
        pda.fp8_quant(self.yf, None, None, self.yt, self.yts, **at)
        pda.fp8_matmul(self.gt, self.gts, self.yt, self.yts, self.dW, workspace=self.space[2], **at)
        pda.rms_norm_bwd(self.dy, self.h, self.norm, self.rstd, self.dh, self.dnorm, dres=self.dres, workspace=self.space[4], **at)
        return self.results()

    def results(self):
        return [self.h, self.rstd, self.qkv, self.q, self.k, self.v, self.out, self.dqkv, self.dy, self.dW, self.dh, self.dnorm]


def _reference(b):
    """The chain in 64 bits by automatic differentiation, with the forward pass's 8-bit values as constants of rounding (gradients pass through)."""
    import torch
    up = lambda t: t.detach().double().cpu()  # noqa: E731
    through = lambda v, to: v + (to - v).detach()  # noqa: E731
    x = (up(b.res) + up(b.x)).requires_grad_()
    w, norm = up(b.W).requires_grad_(), up(b.norm).requires_grad_()

    def values(q, s, block):
        n = q.shape[1] // 128
        return up(q) * up(s.float())[:, :n].repeat_interleave(128, dim=1).repeat_interleave(block, dim=0)[:q.shape[0]]

    y = x * (x.square().mean(dim=-1, keepdim=True) + EPS).rsqrt() * norm.repeat_interleave(S, dim=0)
    y8 = through(y, values(b.y, b.ys, 1)[:, :D])
    qkv = y8 @ through(w, values(b.w, b.ws, 128)[:, :D]).t() + up(b.bias)
    q, k, v = qkv.view(B, S, 3, H, d).unbind(2)
    freqs = torch.tensor([10000.0 ** (-i / 16) for i in range(16)], dtype=torch.float64)
    axis = torch.tensor([0] * 6 + [1] * 5 + [2] * 5)
    angle = up(b.positions)[:, axis] * freqs
    cos, sin = angle.cos()[None, :, None], angle.sin()[None, :, None]

    def pack(t, turns):
        if turns:
            t = t * t.square().mean(dim=-1, keepdim=True).rsqrt()
            u, z = t[..., :16], t[..., 16:32]
            t = torch.cat([u * cos - z * sin, u * sin + z * cos, t[..., 32:]], dim=-1)
        return t.transpose(1, 2)

    q, k, v = pack(q, True), pack(k, True), pack(v, False)
    out = torch.softmax(q @ k.transpose(2, 3) * d ** -0.5, dim=-1) @ v
    qkv.retain_grad(), y.retain_grad()
    (out * up(b.dout)).sum().backward()
    return {"qkv": qkv, "q": q, "v": v, "out": out, "dqkv": qkv.grad, "dy": y.grad, "dW": w.grad, "dh": x.grad + up(b.dres), "dnorm": norm.grad}


def _off(got, want):
    g = got.detach().double().cpu().reshape(want.shape)
    return float((g - want).norm() / want.norm())


def test_against_64_bits():
    """Relative 2-norms.  The forward pass takes the library's own 8-bit values, so bf16 roundings are left: 2^-8 each (qkv one, q two, out four with the probabilities').
    A gradient that has passed through 8-bit matrices is off by at most half a step of the type, 2^-4, for each of them (dy: gradients; dW: gradients and activations), and what
    follows from it by no more; before them the attention's gradient holds a few bf16 roundings."""
    import torch
    b = Block(1)
    b.step()
    torch.cuda.synchronize()
    ref = _reference(b)
    gates = {"qkv": 2.0 ** -8, "q": 2 * 2.0 ** -8, "v": 2.0 ** -8, "out": 4 * 2.0 ** -8, "dqkv": 6 * 2.0 ** -8, "dy": 2.0 ** -4, "dW": 2 * 2.0 ** -4, "dnorm": 2.0 ** -4}
    for name, gate in gates.items():
        assert _off(getattr(b, name), ref[name].detach()) <= gate, (name, _off(getattr(b, name), ref[name].detach()), gate)
    part = b.dh.double().cpu() - b.dres.double().cpu()
    assert _off(part, ref["dh"] - b.dres.double().cpu()) <= 2.0 ** -4


def _captured(b, stream):
    """A graph of the step, after one on the same stream (where the attention call takes the stream's workspace, which it keeps)."""
    import torch
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        b.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        b.step()
    return graph


def test_captured_and_replayed():
    """A graph of the whole step, replayed with other inputs and eager work between the replays: the bits of the eager step each time."""
    import torch
    b, e = Block(2), Block(2)
    graph = _captured(b, torch.cuda.Stream())
    for i in range(4):
        x = torch.randn_like(b.res) * (i + 1)
        b.res.copy_(x)
        e.res.copy_(x)
        for t in b.results():
            t.zero_()
        graph.replay()
        want = e.step()
        torch.cuda.synchronize()
        for g, w in zip(b.results(), want):
            assert torch.equal(g, w)


def test_two_graphs_side_by_side():
    """Two captured steps with workspaces of their own, replayed on two streams at once."""
    import torch
    blocks = [Block(3), Block(4)]
    want = []
    for b in blocks:
        b.step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in b.results()])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    graphs = [_captured(b, s) for b, s in zip(blocks, streams)]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        for x, y in zip(b.results(), w):
            assert torch.equal(x, y)


def test_on_another_stream():
    """Calls go to the given stream; a workspace that a call takes itself lives on it."""
    import torch
    import paper_2511_12056_amd as pda
    b = Block(5)
    want = [t.clone() for t in b.step()]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for t in b.results():
        t.zero_()
    torch.cuda.synchronize()
    b.step(stream=s)
    s.synchronize()
    for x, y in zip(b.results(), want):
        assert torch.equal(x, y)
    a, sa = pda.fp8_empty(1536, 40000)
    w, sw = pda.fp8_empty(640, 40000)
    pda.fp8_quant(torch.randn(1536, 40000, device="cuda"), a, sa)
    pda.fp8_quant(torch.randn(640, 40000, device="cuda"), w, sw)
    outs = [torch.empty(1536, 640, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
    torch.cuda.synchronize()
    pda.fp8_matmul(a, sa, w, sw, outs[0])
    with torch.cuda.stream(s):
        pda.fp8_matmul(a, sa, w, sw, outs[1])
    pda.fp8_matmul(a, sa, w, sw, outs[2], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])

"""The training operators together, as one attention block of a diffusion transformer's training step uses them: layer norm
with a modulation per sample, projections (library products), pack with unit-RMS queries and keys, attention, and all of it back."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _block(x, w, b, wq, wk, wv, H, d, eps, n_v):
    """The block in 64 bits, differentiable; roundings to bf16 between the steps count as the identity."""
    import torch
    B, S, D = x.shape
    mean = x.mean(-1, keepdim=True)
    xc = x - mean
    y = xc / torch.sqrt(xc.square().mean(-1, keepdim=True) + eps) * w[:, None] + b[:, None]
    q, k, v = ((y @ m).view(B, S, H, d).transpose(1, 2) for m in (wq, wk, wv))
    q, k = (t / torch.sqrt(t.square().mean(-1, keepdim=True)) for t in (q, k))
    s = (q @ k.transpose(-1, -2)) * d ** -0.5
    s = s[..., :n_v]
    return torch.softmax(s, dim=-1) @ v[:, :, :n_v]


@pytest.mark.parametrize("B,S,H,d,n_v", [(2, 333, 3, 64, 320), (1, 700, 2, 128, 700)])
def test_block_gradients(B, S, H, d, n_v):
    import torch
    import paper_2511_12056_amd as pda
    D, eps, bf16 = 160, 1e-6, torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(S)
    x = torch.randn(B, S, D, generator=g, device="cuda")
    w, b = 1 + 0.2 * torch.randn(B, D, generator=g, device="cuda"), 0.2 * torch.randn(B, D, generator=g, device="cuda")
    wq, wk, wv = ((torch.randn(D, H * d, generator=g, device="cuda") * D ** -0.5).to(bf16) for _ in range(3))
    dout = torch.randn(B, H, S, d, generator=g, device="cuda").to(bf16)

    # forward
    y, mean, rstd = torch.empty_like(x, dtype=bf16), torch.empty(B, S, device="cuda"), torch.empty(B, S, device="cuda")
    pda.layer_norm_fwd(x, w, b, y, mean, rstd, eps)
    proj = [(y.float() @ m.float()).view(B, S, H, d).contiguous() for m in (wq, wk, wv)]
    q, k, v = (torch.empty(B, H, S, d, device="cuda", dtype=bf16) for _ in range(3))
    for t, to, rms in zip(proj, (q, k, v), (True, True, False)):
        pda.pack_heads(t, to, rms)
    out, lse = torch.empty_like(q), torch.empty(B, H, S, device="cuda")
    pda.attn_fwd_bf16out(q, k, v, out, lse, d ** -0.5, n_v)
    # backward
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    pda.attn_bwd(dout, q, k, v, out, lse, dq, dk, dv, d ** -0.5, n_v)
    dy, dm = torch.zeros_like(x), []
    for t, grad, m, rms in zip(proj, (dq, dk, dv), (wq, wk, wv), (True, True, False)):
        dt = torch.empty_like(t)
        pda.pack_heads_bwd(grad, t if rms else None, dt, rms)
        dt = dt.view(B, S, H * d)
        dm.append(y.float().view(-1, D).t() @ dt.view(-1, H * d))
        dy += dt @ m.float().t()
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    pda.layer_norm_bwd(dy.to(bf16), x, w, mean, rstd, dx, dw, db)

    leaves = [t.double().requires_grad_() for t in (x, w, b, wq, wk, wv)]
    ref = _block(*leaves, H, d, eps, n_v)
    ref.backward(dout.double())
    assert (out.double() - ref).norm() <= 1e-2 * ref.norm()
    # y, q/k/v, p, ds, the gradients and dy are each rounded to bf16 on the way (relative 2^-9 rms at most each, in the largest term of
    # what they enter); eight of them in quadrature, doubled for the cancellation in the two normalisations
    bound = 2 * 8 ** 0.5 * 2.0 ** -9
    for name, got, leaf in zip(("x", "weight", "bias", "wq", "wk", "wv"), (dx, dw, db, *dm), leaves):
        rel = float((got.double().view_as(leaf) - leaf.grad).norm() / leaf.grad.norm())
        assert rel <= bound, (name, rel, bound)
    assert np.isfinite(float(dx.double().norm()))

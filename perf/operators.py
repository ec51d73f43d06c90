"""The training operators around the attention call, as a video diffusion transformer's training step uses them: the
gradients of attention, of the pack that produces its inputs, and layer norm forward and backward.

A case is a dict with an "op" and the sizes of that operator:

    attn_bwd   B, H, Sq, Skv, valid (keys not masked), d, out ("fp32" or "bf16": which forward call wrote it)
    ln_fwd     rows, D, groups (rows that share a weight and a bias: one, or one per sample), x and y types
    ln_bwd     the same; dy has the type of y, dx that of x
    pack_bwd   B, S, H, d, unit_rms

Queries and keys are unit-RMS Gaussian vectors (what a normalised Q and K are), gradients Gaussian, the rows of layer norm
have offsets and scales of their own.  Everything is made on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

LARGEST = 10.0 * 3 * 67576 * 67476 * 128       # operations of the largest listed attention gradient
LARGEST_ROWS = 119056 * 1536                   # elements of the largest listed layer norm
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # the smallest attention: 2 heads of a 4 x 16 x 16 latent grid; latency and launches
        {"name": "attn_bwd_tiny_d64", "op": "attn_bwd", "B": 1, "H": 2, "Sq": 1024, "Skv": 1024, "valid": 1024, "d": 64, "out": "fp32"},
        # one head of a short clip (8 x 30 x 40 latent grid), what one GPU of a head-parallel step may hold
        {"name": "attn_bwd_one_head", "op": "attn_bwd", "B": 1, "H": 1, "Sq": 9600, "Skv": 9600, "valid": 9600, "d": 128, "out": "bf16"},
        # a batch of two, ragged length with a padded tail, head dimension 64
        {"name": "attn_bwd_batch_d64", "op": "attn_bwd", "B": 2, "H": 12, "Sq": 4797, "Skv": 4797, "valid": 4701, "d": 64, "out": "bf16"},
        # all 24 heads of the short clip
        {"name": "attn_bwd_lowres_clip", "op": "attn_bwd", "B": 1, "H": 24, "Sq": 9600, "Skv": 9600, "valid": 9600, "d": 128, "out": "bf16"},
        # many queries on few keys, a masked tail: attention to a short conditioning sequence
        {"name": "attn_bwd_few_keys", "op": "attn_bwd", "B": 1, "H": 24, "Sq": 16384, "Skv": 600, "valid": 570, "d": 128, "out": "fp32"},
        # three heads at 544 x 960 x 129 frames with 256 text tokens, 100 of them padding
        {"name": "attn_bwd_544x960", "op": "attn_bwd", "B": 1, "H": 3, "Sq": 67576, "Skv": 67576, "valid": 67476, "d": 128, "out": "fp32"},
        # one token: a conditioning vector, latency only
        {"name": "ln_fwd_one_token", "op": "ln_fwd", "rows": 1, "D": 1536, "groups": 1, "x": "fp32", "y": "bf16"},
        # the fp32 residual stream of a 720p clip on its way to a bf16 projection
        {"name": "ln_fwd_720p", "op": "ln_fwd", "rows": 119056, "D": 1536, "groups": 1, "x": "fp32", "y": "bf16"},
        # two samples of ragged length, each with a modulation of its own, everything in bf16
        {"name": "ln_bwd_batch", "op": "ln_bwd", "rows": 9594, "D": 1152, "groups": 2, "x": "bf16", "y": "bf16"},
        # back from the projections into the fp32 residual stream
        {"name": "ln_bwd_720p", "op": "ln_bwd", "rows": 119056, "D": 1536, "groups": 1, "x": "fp32", "y": "bf16"},
        # the values of a short batch: no normalisation, a transposition with a change of type
        {"name": "pack_bwd_batch_d64", "op": "pack_bwd", "B": 2, "S": 4797, "H": 12, "d": 64, "unit_rms": False},
        # the normalised queries of a 720p clip
        {"name": "pack_bwd_720p", "op": "pack_bwd", "B": 1, "S": 119056, "H": 24, "d": 128, "unit_rms": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn_bwd", "attn_bwd", "attn_bwd", "ln_fwd", "ln_bwd", "ln_bwd", "pack_bwd"])
    while True:
        if op == "attn_bwd":
            s = _log_int(rng, 200, 67576)
            skv = rng.choice([s, s, s, _log_int(rng, 50, 67576)])
            case = {"op": op, "B": rng.choice([1, 1, 2]), "H": rng.randint(1, 24), "Sq": s, "Skv": skv,
                    "valid": skv - rng.choice([0, rng.randint(0, 49)]), "d": rng.choice([128, 128, 64]), "out": rng.choice(["fp32", "bf16"])}
            if work(case)["flops"] <= LARGEST / 3:
                return case
        elif op == "pack_bwd":
            case = {"op": op, "B": rng.choice([1, 2]), "S": _log_int(rng, 100, 119056), "H": rng.randint(1, 24), "d": rng.choice([128, 64]),
                    "unit_rms": rng.random() < 0.6}
            if case["B"] * case["S"] * case["H"] * case["d"] <= LARGEST_ROWS:
                return case
        else:
            groups = rng.choice([1, 1, 2, 4])
            D = rng.choice([64 * rng.randint(4, 64), 64 * rng.randint(4, 64), _log_int(rng, 40, 5000)])
            case = {"op": op, "rows": groups * _log_int(rng, 1, 40000), "D": D, "groups": groups,
                    "x": rng.choice(["fp32", "bf16"]), "y": rng.choice(["fp32", "bf16", "bf16"])}
            if case["rows"] * D <= LARGEST_ROWS:
                return case


def _unit_rms(gen, *shape):
    """bf16 Gaussian tensor whose last-axis vectors have RMS one."""
    x = torch.randn(*shape, generator=gen, device="cuda")
    x *= x.square().mean(dim=-1, keepdim=True).rsqrt_()
    return x.to(torch.bfloat16)


def _heads_at_once(rows, keys):
    """Heads whose score matrices together stay within 2^32 elements."""
    return max(1, (1 << 32) // max(1, rows * keys))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    st = {"case": case}
    if op == "attn_bwd":
        B, H, Sq, Skv, d, n = case["B"], case["H"], case["Sq"], case["Skv"], case["d"], case["valid"]
        scale = d ** -0.5
        q, k, v = _unit_rms(gen, B, H, Sq, d), _unit_rms(gen, B, H, Skv, d), _unit_rms(gen, B, H, Skv, d)
        out, lse = torch.empty(B, H, Sq, d, device="cuda", dtype=TYPES[case["out"]]), torch.empty(B, H, Sq, device="cuda")
        qs, ks, vs = q.view(B * H, Sq, d), k.view(B * H, Skv, d)[:, :n], v.view(B * H, Skv, d)[:, :n]
        for h in torch.arange(B * H).split(_heads_at_once(Sq, n)):      # what the forward call has left: the result and its log-sum-exp
            a, b = int(h[0]), int(h[-1]) + 1
            s = torch.matmul(qs[a:b].float() * scale, ks[a:b].float().transpose(1, 2).contiguous())
            top = s.amax(dim=-1, keepdim=True)
            s.sub_(top).exp_()
            norm = s.sum(dim=-1, keepdim=True)
            out.view(B * H, Sq, d)[a:b] = torch.matmul(s, vs[a:b].float()) / norm
            lse.view(B * H, Sq)[a:b] = (top + norm.log()).squeeze(-1)
            del s
        st.update(q=q, k=k, v=v, out=out, lse=lse, scale=scale,
                  dout=torch.randn(B, H, Sq, d, generator=gen, device="cuda").to(torch.bfloat16),
                  dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v))
    elif op == "pack_bwd":
        B, S, H, d = case["B"], case["S"], case["H"], case["d"]
        st.update(x=torch.randn(B, S, H, d, generator=gen, device="cuda"),
                  dy=torch.randn(B, H, S, d, generator=gen, device="cuda").to(torch.bfloat16), premul=d ** -0.5 if case["unit_rms"] else 1.0,
                  dx=torch.empty(B, S, H, d, device="cuda"))
    else:
        rows, D, G = case["rows"], case["D"], case["groups"]
        x = torch.randn(rows, D, generator=gen, device="cuda")
        x = (x * (0.5 + torch.rand(rows, 1, generator=gen, device="cuda")) + 0.5 + 0.3 * torch.randn(rows, 1, generator=gen, device="cuda")).to(TYPES[case["x"]])
        st.update(x=x, weight=1 + 0.2 * torch.randn(G, D, generator=gen, device="cuda"), bias=0.2 * torch.randn(G, D, generator=gen, device="cuda"))
        if op == "ln_fwd":
            st.update(y=torch.empty(rows, D, device="cuda", dtype=TYPES[case["y"]]),
                      mean=torch.empty(rows, device="cuda"), rstd=torch.empty(rows, device="cuda"))
        else:                                           # the statistics as the forward call has left them
            mean = x.mean(dim=-1, dtype=torch.float64)
            st.update(mean=mean.float(), rstd=(x.double() - mean[:, None]).square_().mean(dim=-1).add_(EPS).rsqrt_().float(),
                      dy=torch.randn(rows, D, generator=gen, device="cuda").to(TYPES[case["y"]]),
                      dx=torch.empty_like(x), dweight=torch.empty(G, D, device="cuda"), dbias=torch.empty(G, D, device="cuda"))
    return st


def _own(st):
    import paper_2511_12056_amd as pda
    case, op = st["case"], st["case"]["op"]
    if op == "attn_bwd":
        if "workspace" not in st:                       # kept with the activations' buffers, as a training loop does
            st["workspace"] = pda.attn_bwd_workspace(case["B"], case["H"], case["Sq"], case["Skv"], case["d"], case["valid"])
        return pda.attn_bwd(st["dout"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["dq"], st["dk"], st["dv"], st["scale"],
                            case["valid"], workspace=st["workspace"])
    if op == "ln_fwd":
        return pda.layer_norm_fwd(st["x"], st["weight"], st["bias"], st["y"], st["mean"], st["rstd"], EPS)
    if op == "ln_bwd":
        if "workspace" not in st:
            st["workspace"] = pda.layer_norm_bwd_workspace(case["rows"], case["D"], case["groups"])
        return pda.layer_norm_bwd(st["dy"], st["x"], st["weight"], st["mean"], st["rstd"], st["dx"], st["dweight"], st["dbias"],
                                  workspace=st["workspace"])
    return pda.pack_heads_bwd(st["dy"], st["x"] if case["unit_rms"] else None, st["dx"], case["unit_rms"], st["premul"])


def _plain_attn_bwd(st):
    """Gradients of softmax(scale q k^T) v from the stored log-sum-exp, as many heads at a time as memory holds."""
    case, scale = st["case"], st["scale"]
    BH, Sq, Skv, d, n = case["B"] * case["H"], case["Sq"], case["Skv"], case["d"], case["valid"]
    q, dout, out, lse = (st[x].view(BH, Sq, -1) for x in ("q", "dout", "out", "lse"))
    k, v = (st[x].view(BH, Skv, d)[:, :n] for x in ("k", "v"))
    dq = torch.empty(BH, Sq, d, device=q.device, dtype=q.dtype)
    dk, dv = (torch.zeros(BH, Skv, d, device=q.device, dtype=q.dtype) for _ in range(2))
    step = _heads_at_once(Sq, n)
    for a in range(0, BH, step):
        h = slice(a, min(a + step, BH))
        qf, kf, vf, df = (t[h].float() for t in (q, k, v, dout))
        delta = (df * out[h].float()).sum(dim=-1, keepdim=True)
        p = torch.matmul(qf * scale, kf.transpose(1, 2).contiguous()).sub_(lse[h]).exp_()
        dv[h, :n] = torch.matmul(df.transpose(1, 2).contiguous(), p).transpose(1, 2)
        p *= torch.matmul(df, vf.transpose(1, 2).contiguous()).sub_(delta)
        dq[h] = torch.matmul(p, kf) * scale
        dk[h, :n] = torch.matmul(qf.transpose(1, 2).contiguous(), p).transpose(1, 2) * scale
        del p
    shape = st["q"].shape[:2]
    return tuple(t.view(*shape, *t.shape[1:]) for t in (dq, dk, dv))


def run(st):
    if own:
        return _own(st)
    case, op = st["case"], st["case"]["op"]
    if op == "attn_bwd":
        return _plain_attn_bwd(st)
    if op == "pack_bwd":
        dy = st["dy"].transpose(1, 2).to(torch.float32, memory_format=torch.contiguous_format)
        if not case["unit_rms"]:
            return dy * st["premul"]
        x = st["x"]
        r = x.square().mean(dim=-1, keepdim=True).rsqrt()
        xh = x * r
        return (dy - xh * (dy * xh).mean(dim=-1, keepdim=True)) * (r * st["premul"])
    G, D = case["groups"], case["D"]
    x, w = st["x"].float().view(G, -1, D), st["weight"].view(G, 1, D)
    if op == "ln_fwd":
        mean = x.mean(dim=-1, keepdim=True)
        xc = x - mean
        rstd = (xc.square().mean(dim=-1, keepdim=True) + EPS).rsqrt()
        y = xc * rstd * w + st["bias"].view(G, 1, D)
        return y.view(-1, D).to(TYPES[case["y"]]), mean.view(-1), rstd.view(-1)
    mean, rstd, dy = st["mean"].view(G, -1, 1), st["rstd"].view(G, -1, 1), st["dy"].float().view(G, -1, D)
    xh = (x - mean) * rstd
    g = dy * w
    dx = (g - g.mean(dim=-1, keepdim=True) - xh * (g * xh).mean(dim=-1, keepdim=True)) * rstd
    return dx.view(-1, D).to(TYPES[case["x"]]), (dy * xh).sum(dim=1), dy.sum(dim=1)


def exact(case, seed):
    """What `run` returns, in 64 bits from the definitions: rows of queries in blocks, each with all of its keys."""
    st = prepare(case, seed)
    op = case["op"]
    if op == "attn_bwd":
        B, H, Sq, n = case["B"], case["H"], case["Sq"], case["valid"]
        dq, dk, dv = (torch.zeros(st[x].shape, device="cuda", dtype=torch.float64) for x in ("q", "k", "v"))
        step = max(1, (1 << 28) // max(1, n))
        for b in range(B):
            for h in range(H):
                k, v = st["k"][b, h, :n].double(), st["v"][b, h, :n].double()
                kt, vt = k.t().contiguous(), v.t().contiguous()
                for r in range(0, Sq, step):
                    at = (b, h, slice(r, min(r + step, Sq)))
                    q, do = st["q"][at].double(), st["dout"][at].double()
                    prob = torch.exp(torch.mm(q, kt) * st["scale"] - st["lse"][at].double()[:, None])
                    dv[b, h, :n] += torch.mm(prob.t(), do)
                    ds = prob * (torch.mm(do, vt) - (do * st["out"][at].double()).sum(dim=-1, keepdim=True)) * st["scale"]
                    dq[at] = torch.mm(ds, k)
                    dk[b, h, :n] += torch.mm(ds.t(), q)
        return dq, dk, dv
    if op == "pack_bwd":
        x, dy = st["x"].double(), st["dy"].double().permute(0, 2, 1, 3)
        if not case["unit_rms"]:
            return dy * st["premul"]
        ss = torch.sum(x * x, dim=-1, keepdim=True)      # y = premul sqrt(d) x / |x|
        along = torch.sum(x * dy, dim=-1, keepdim=True) / ss
        return st["premul"] * math.sqrt(case["d"]) * (dy - x * along) / torch.sqrt(ss)
    D, per = case["D"], case["rows"] // case["groups"]
    x, w = st["x"].double(), st["weight"].double().repeat_interleave(per, dim=0)
    if op == "ln_fwd":
        var, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
        rstd = 1 / torch.sqrt(var + EPS)
        return (x - mean) * rstd * w + st["bias"].double().repeat_interleave(per, dim=0), mean[:, 0], rstd[:, 0]
    rstd, dy = st["rstd"].double()[:, None], st["dy"].double()
    xh = (x - st["mean"].double()[:, None]) * rstd
    g = dy * w
    dx = rstd / D * (D * g - g.sum(dim=-1, keepdim=True) - xh * (g * xh).sum(dim=-1, keepdim=True))
    groups = (case["groups"], per, D)
    return dx, (dy * xh).view(groups).sum(dim=1), dy.view(groups).sum(dim=1)


def work(case):
    """Each input read once, each output written once.  Attention: five products of 2 Sq valid d operations a head."""
    op = case["op"]
    if op == "attn_bwd":
        bh, Sq, Skv, n, d = case["B"] * case["H"], case["Sq"], case["Skv"], case["valid"], case["d"]
        out = 4 if case["out"] == "fp32" else 2
        return {"bytes": bh * (Sq * d * (2 + 2 + out + 2) + Sq * 4 + 2 * n * d * 2 + 2 * Skv * d * 2), "flops": 10.0 * bh * Sq * n * d}
    if op == "pack_bwd":
        n = case["B"] * case["S"] * case["H"] * case["d"]
        return {"bytes": n * (10 if case["unit_rms"] else 6), "flops": n * (8 if case["unit_rms"] else 1)}
    n, size = case["rows"] * case["D"], {"fp32": 4, "bf16": 2}
    if op == "ln_fwd":
        return {"bytes": n * (size[case["x"]] + size[case["y"]]) + case["rows"] * 8 + case["groups"] * case["D"] * 8, "flops": 8 * n}
    return {"bytes": n * (2 * size[case["x"]] + size[case["y"]]) + case["rows"] * 8 + case["groups"] * case["D"] * 12, "flops": 14 * n}
